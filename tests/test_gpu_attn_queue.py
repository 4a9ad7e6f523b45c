"""Long bf16 calls whose jobs are handed out whole, from a queue: prompts and pieces of several sequences, against the
float64 oracle on sampled rows, call after call on one workspace."""
import numpy as np
import pytest
import torch

from layer_util import Batch, f64
from paper_2404_01365_b200 import binding as G

pytestmark = pytest.mark.gpu
DEV, SMS = "cuda:0", 148


def jobs_of(b):
    """(jobs, whether the call is queued), from the rule as the kernels' comments state it: no sequence shares the reading of
    the prefix, three jobs per SM, and no job longer than a fair share of the tiles."""
    group = b.hq // b.hkv
    n = len(b.seq_len)
    keys, rows = (64, 128) if b.hd > 128 else (128, 256)
    block = (128 // group) * (rows // 128)
    if not (n == 1 or b.prefix == 0 or b.T * group > n * 128):
        return 0, False
    jobs, tiles = 0, []
    for s in range(n):
        nq, own = int(b.q_start[s + 1] - b.q_start[s]), int(b.seq_len[s])
        lens = [max(own - nq + min(nq, at + block), 0) for at in range(0, nq, block)]
        t = [-(-b.prefix // keys) + -(-x // keys) for x in lens]
        if t and t[-1] > 0:
            jobs += len(t) * b.hkv
            tiles += t
    return jobs, jobs >= 3 * SMS and max(tiles) * SMS <= sum(tiles) * b.hkv


def sampled(b, block):
    """Rows next to the edges of every sequence's first, second and last blocks, and of its first that sees something."""
    rows = set()
    for s in range(len(b.seq_len)):
        lo, hi = int(b.q_start[s]), int(b.q_start[s + 1])
        first = max(lo, hi - int(b.seq_len[s]))
        rows |= {t for a in (lo, lo + block, hi, first) for t in (a - 1, a) if lo <= t < hi}
    return rows


def check(b, rows, out):
    want, mass = b.reference(rows)
    at = sorted(rows)
    err = np.abs(f64(out)[at] - want[at])
    assert np.all(err <= b.bound(want, mass)[at]), np.nanmax(err / b.bound(want, mass)[at])
    assert torch.isfinite(out[:int(b.q_start[-1])]).all() and torch.all(out[int(b.q_start[-1]):] == 77.0)


CASES = {
    "one prompt": ([1800], [1800], 0, 64, 64, 64, 64),
    "one prompt, grouped heads": ([1100], [1100], 0, 128, 32, 128, 16),
    "a piece of a prompt": ([900], [1500], 0, 112, 112, 80, 32),
    "pieces of several sequences": ([700, 3, 0, 400, 256], [700, 40, 9, 1100, 256], 0, 96, 24, 64, 16),
    "blocks that see nothing": ([700, 3, 40, 400, 256, 129], [300, 40, 0, 400, 256, 1], 0, 96, 24, 64, 16),
    "rows that see the prefix only": ([600, 300, 5, 260], [100, 300, 5, 0], 200, 60, 60, 72, 16),
    "behind a prefix": ([500, 257, 300], [500, 300, 400], 130, 76, 76, 64, 128),
    "one accumulator": ([600, 0, 300, 77], [600, 4, 100, 500], 0, 50, 50, 256, 32),
    "one accumulator, grouped heads": ([400, 400, 20], [400, 700, 20], 90, 60, 30, 200, 64),
    "many short sequences": ([40] * 64, [40 + 3 * i for i in range(64)], 0, 32, 8, 64, 8),
}


@pytest.mark.parametrize("name", CASES)
def test_jobs_from_a_queue(name):
    q_lens, seq_lens, prefix, hq, hkv, hd, page = CASES[name]
    b = Batch(q_lens, seq_lens, prefix, hq, hkv, hd, page, "bf16", extra_rows=2)
    jobs, queued = jobs_of(b)
    assert queued, jobs
    block = (128 // (hq // hkv)) * (1 if hd > 128 else 2)
    rows = sampled(b, block)
    b.to_device()
    out = b.attend()
    assert G.griffin_check_device_status(b.ws) == G.OK
    check(b, rows, out)
    # on the same workspace: the same bits again, then a call that is not queued, then the queue from its beginning
    assert torch.equal(b.attend(), out)
    q_start, seq_len = b.dev[0].clone(), b.dev[1].clone()
    b.dev[0].copy_(torch.tensor([0] * len(q_lens) + [1], dtype=torch.int32))      # one row, of the last sequence
    b.dev[1][:-1] = 0
    b.dev[1][-1] = min(int(seq_len[-1]), page)
    few = b.attend()
    assert torch.all(few[1:] == 77.0) and torch.isfinite(few[:1]).all()
    b.dev[0].copy_(q_start)
    b.dev[1].copy_(seq_len)
    assert torch.equal(b.attend(), out) and G.griffin_check_device_status(b.ws) == G.OK


def test_queued_calls_in_a_graph_and_on_another_stream():
    b = Batch([500, 300, 513], [500, 310, 600], 0, 64, 64, 64, 16, "bf16")
    assert jobs_of(b)[1]
    b.to_device()
    plain, q = b.attend(), b.q.to(DEV)
    out = torch.zeros_like(plain)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(5):
            b.attend(q=q, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, plain)
    with torch.cuda.stream(side):
        again = b.attend()
    side.synchronize()
    assert torch.equal(again, plain) and G.griffin_check_device_status(b.ws) == G.OK

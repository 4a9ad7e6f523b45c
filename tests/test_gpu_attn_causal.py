"""A value that is not finite among a call's own tokens reaches the tokens that see it and no others."""
import numpy as np
import pytest
import torch

from layer_util import Batch, f64
from oracle import layer_oracle as L
from paper_2404_01365_b200 import binding as G

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN, INF = float("nan"), float("inf")


def put(b, seq, index, entry, value, head=0):
    b.v_host[int(b.page_table[seq, index // b.page]), head, index % b.page, entry] = value


def check(b, rows=None):
    with np.errstate(all="ignore"):
        want, mass = L.attention(f64(b.q), f64(b.k_host), f64(b.v_host), b.q_start.numpy(), b.seq_len.numpy(), b.page_table.numpy(),
                                 b.prefix_pages.numpy(), b.prefix, b.scale, rows)
        bound = b.bound(np.nan_to_num(want, posinf=0.0, neginf=0.0), np.nan_to_num(mass, nan=0.0, posinf=0.0))
    b.to_device()
    out = b.attend()
    got = f64(out)
    at = slice(0, int(b.q_start[-1])) if rows is None else sorted(rows)
    want, got, bound = want[at], got[at], bound[at]
    assert not np.all(np.isfinite(want)) and np.any(np.isfinite(want))
    assert np.array_equal(np.isnan(want), np.isnan(got)), np.argwhere(np.isnan(want) != np.isnan(got))[:5]
    assert np.array_equal(np.isinf(want), np.isinf(got)) and np.all(got[np.isinf(want)] == want[np.isinf(want)])
    fine = np.isfinite(want)
    assert np.all(np.abs(got[fine] - want[fine]) <= bound[fine])
    assert torch.equal(b.attend().view(torch.uint8), out.view(torch.uint8)) and G.griffin_check_device_status(b.ws) == G.OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", [(2, 2, 64), (4, 1, 128), (3, 1, 80), (2, 1, 256), (5, 1, 200)])
@pytest.mark.parametrize("n,own,prefix", [(2, 2, 0), (3, 50, 0), (8, 8, 0), (8, 301, 40), (40, 40, 0), (129, 200, 0), (300, 300, 0), (300, 290, 20)])
def test_one_value_of_the_calls_own_tokens(dtype, hq, hkv, hd, n, own, prefix):
    for value, back in ((NAN, 1), (INF, n // 2), (-INF, n - 1)):
        if own - back < 0:
            continue
        b = Batch([n], [own], prefix, hq, hkv, hd, 16, dtype, fill=0.0, seed=back)
        put(b, 0, own - back, hd - 3, value)
        check(b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 64), (3, 1, 128), (2, 1, 256)])
def test_values_of_several_sequences(dtype, hq, hkv, hd):
    # drafts behind a shared prefix, and pieces: every kind of value, also in one row and in one entry
    for q_lens, seq_lens, prefix in (([4, 1, 3], [4, 30, 140], 70), ([6, 0, 9, 7], [129, 3, 9, 70], 300), ([150, 40, 200], [150, 300, 180], 0),
                                     ([150, 40, 200], [150, 300, 180], 33)):
        b = Batch(q_lens, seq_lens, prefix, hq, hkv, hd, 16, dtype, fill=0.0)
        put(b, 0, seq_lens[0] - 2, 0, INF)
        put(b, 0, seq_lens[0] - 1, 0, -INF)
        put(b, 0, seq_lens[0] - 1, 1, INF)
        put(b, 2, seq_lens[2] - 1, 5, NAN, head=hkv - 1)
        put(b, 2, seq_lens[2] - 3, 9, -INF)
        for e in range(hd):
            put(b, 2, seq_lens[2] - 2, e, INF if e % 3 else NAN, head=0)
        check(b)


def test_values_of_tokens_whose_keys_are_cut_over_the_ctas():
    # long contexts: the last tiles are a segment of their own; and a prompt whose jobs come from a queue
    for n, own, hq, hkv, hd in ((5, 9000, 4, 1, 128), (20, 6000, 2, 1, 64), (30, 5000, 1, 1, 256)):
        b = Batch([n], [own], 0, hq, hkv, hd, 64, "bf16", fill=0.0)
        put(b, 0, own - n + n // 2, 7, NAN)
        put(b, 0, own - 1, 8, INF)
        check(b, {0, n // 2 - 1, n // 2, n - 2, n - 1})
    b = Batch([1000, 300], [1000, 450], 0, 76, 76, 64, 64, "bf16", fill=0.0)
    for seq, i in ((0, 999), (0, 500), (0, 3), (1, 449), (1, 200)):
        put(b, seq, i, 11, (NAN, INF, -INF)[i % 3], head=i % 76)
    check(b, {0, 2, 3, 4, 255, 256, 499, 500, 511, 512, 998, 999, 1000, 1049, 1050, 1051, 1298, 1299})

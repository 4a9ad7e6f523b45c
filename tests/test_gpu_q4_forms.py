"""Attention over the cache held in 4 bits, in the forms that its kernels divide calls into: more query heads under a key head than
a block of few rows has, tables that are narrow or wide (by what they could hold a bf16 call of many rows goes to the one kernel
or the other), calls whose jobs clusters of one to eight CTAs take whole, and calls that are cut."""
import numpy as np
import pytest
import torch

import q4_util as Q
from layer_util import f64
from paper_2404_01365_b200 import binding as G
from q4_util import BatchQ4
from test_gpu_attn_causal import check as check_not_finite, put
from test_gpu_layer import check_attention

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = float("nan")
TABLES = [1, 60000]     # keys that the tables could hold beyond the longest sequence: the second makes pieces of rows tcgen05 calls
WIDE = [(9, 1, 64), (12, 1, 80), (20, 2, 112), (16, 1, 128), (10, 1, 208), (48, 3, 256)]   # heads, key heads, width


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", WIDE)
@pytest.mark.parametrize("page", [8, 32, 256])
@pytest.mark.parametrize("room", TABLES)
def test_large_groups_of_steps_and_pieces(dtype, hq, hkv, hd, page, room):
    extra = -(-room // page)
    check_attention(BatchQ4([1, 1, 1, 1], [1, 40, 129, 77], 300, hq, hkv, hd, page, dtype, table_extra=extra))
    check_attention(BatchQ4([1], [260], 0, hq, hkv, hd, page, dtype, table_extra=extra))
    check_attention(BatchQ4([2, 0, 17, 1], [2, 5, 130, 0], 129, hq, hkv, hd, page, dtype, extra_rows=2, table_extra=extra))
    check_attention(BatchQ4([7, 1, 30], [7, 500, 300], 200, hq, hkv, hd, page, dtype, extra_rows=1, table_extra=extra))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", WIDE + [(11, 1, 128), (13, 1, 64), (64, 1, 256)])
@pytest.mark.parametrize("n", [1, 5, 33, 150])
@pytest.mark.parametrize("room", TABLES)
def test_large_groups_of_prompts(dtype, hq, hkv, hd, n, room):
    check_attention(BatchQ4([n], [n], 0, hq, hkv, hd, 16, dtype, table_extra=-(-room // 16)), rows={0, n // 2, n - 1})
    check_attention(BatchQ4([n, n], [n + 3, n], 65, hq, hkv, hd, 64, dtype, table_extra=-(-room // 64)), rows={0, n - 1, n, 2 * n - 1})


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix", [1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257])
@pytest.mark.parametrize("room", TABLES)
def test_large_groups_behind_prefixes(dtype, prefix, room):
    extra = -(-room // 32)
    for hd in (64, 128, 256):
        check_attention(BatchQ4([1, 2], [1, 33], prefix, 18, 2, hd, 32, dtype, table_extra=extra))
        check_attention(BatchQ4([6, 7], [6, 40], prefix, 18, 2, hd, 32, dtype, table_extra=extra))
        check_attention(BatchQ4([8], [9], prefix, 18, 2, hd, 32, dtype, table_extra=extra))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", WIDE)
@pytest.mark.parametrize("fill", [NAN, 12000.0])
@pytest.mark.parametrize("room", TABLES)
def test_large_groups_do_not_see_what_lies_behind_the_ends(dtype, hq, hkv, hd, fill, room):
    check_attention(BatchQ4([1, 2, 1], [5, 70, 129], 37, hq, hkv, hd, 64, dtype, fill=fill, table_extra=-(-room // 64)))
    check_attention(BatchQ4([9, 12, 1], [9, 70, 129], 37, hq, hkv, hd, 64, dtype, fill=fill, table_extra=-(-room // 64)))
    check_attention(BatchQ4([20], [23], 0, hq, hkv, hd, 8, dtype, fill=fill, table_extra=-(-room // 8)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", WIDE)
@pytest.mark.parametrize("n,own,prefix", [(2, 2, 0), (3, 50, 0), (8, 301, 40), (40, 40, 0), (150, 170, 20)])
@pytest.mark.parametrize("room", TABLES)
def test_large_groups_and_values_that_are_not_finite(dtype, hq, hkv, hd, n, own, prefix, room):
    for back in {1, n // 2, n - 1}:
        b = BatchQ4([n], [own], prefix, hq, hkv, hd, 16, dtype, fill=0.0, seed=back, table_extra=-(-room // 16))
        put(b, 0, own - back, hd - 3, NAN)
        put(b, 0, own - 1, 1, NAN, hkv - 1)
        b.requantise()
        check_not_finite(b, {0, n // 2, n - 1})


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 112, 256])
@pytest.mark.parametrize("room", TABLES)
def test_large_groups_report_bad_pages(dtype, hd, room):
    b = BatchQ4([9, 12], [300, 90], 40, 12, 1, hd, 8, dtype, fill=0.0, table_extra=-(-room // 8))
    b.page_table[0, 17], b.page_table[0, 30], b.prefix_pages[1] = 10 ** 6, -1, -5
    b.to_device()
    out = b.attend()
    assert G.griffin_check_device_status(b.ws) == G.ERR_INVALID_ARG
    b.k_host, b.v_host = (torch.cat((t, torch.zeros_like(t[:1]))) for t in (b.k_host, b.v_host))   # the pages read as zeros
    b.page_table[0, 17] = b.page_table[0, 30] = b.prefix_pages[1] = b.k_host.shape[0] - 1
    want, mass = b.reference()
    assert np.all(np.abs(f64(out) - want) <= b.bound(want, mass))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", [(16, 1, 128), (10, 1, 256), (4, 2, 64)])
@pytest.mark.parametrize("room", TABLES)
def test_in_place_captured_and_on_two_streams_at_once(dtype, hq, hkv, hd, room):
    bs = [BatchQ4(q, s, 90, hq, hkv, hd, 16, dtype, seed=i, table_extra=-(-room // 16)).to_device() for i, (q, s) in enumerate((([1, 9], [200, 60]), ([30], [400])))]
    plain = [b.attend() for b in bs]
    streams = [torch.cuda.Stream() for _ in bs]
    graphs, outs = [], []
    for b, stream in zip(bs, streams):
        stream.wait_stream(torch.cuda.current_stream())
        q = b.q.to(DEV)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            b.attend(q=q, out=q)
        graphs.append((graph, q))
    torch.cuda.synchronize()
    for _ in range(20):
        for b, (graph, q), stream in zip(bs, graphs, streams):
            with torch.cuda.stream(stream):
                q.copy_(b.q.to(DEV, non_blocking=True))
                graph.replay()
    torch.cuda.synchronize()
    for b, (_, q), want in zip(bs, graphs, plain):
        assert torch.equal(q, want) and G.griffin_check_device_status(b.ws) == G.OK


# (sequences, own keys, prefix, key heads): what clusters of 8, 4, 2 and 1 CTAs take, then what is cut
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,own,prefix,hkv", [(1, 33, 0, 1), (1, 4000, 0, 2), (8, 1000, 0, 1), (4, 600, 100, 2), (4, 500, 2000, 2), (20, 700, 0, 1),
                                              (32, 300, 0, 1), (5, 200, 0, 8), (18, 400, 0, 4), (73, 900, 0, 1), (24, 150, 0, 4), (148, 60, 0, 1),
                                              (149, 60, 0, 1), (50, 900, 0, 4), (1, 20000, 0, 9), (30, 700, 1000, 6)])
def test_jobs_whole_and_cut(dtype, n, own, prefix, hkv):
    lens = [own - (11 * i) % (own // 2) for i in range(n)]
    rows = {0, n // 2, n - 1}
    for group in (1, 4):
        b = BatchQ4([1] * n, lens, prefix, group * hkv, hkv, 64, 64, dtype)
        b.page_table = b.page_table[:, :-1].contiguous()
        check_attention(b, rows=rows)
    b = BatchQ4([1] * n, [0 if i % 3 == 1 else x // 20 for i, x in enumerate(lens)], prefix, hkv, hkv, 64, 64, dtype, table_extra=own // 64)
    check_attention(b, rows=rows | {1 % n})


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("extra", [0, 40, 2000])
def test_tables_wider_than_their_sequences(dtype, extra):
    # the table's width chooses the kernel and the way that the call is divided, and changes no more than roundings
    for q_lens, seq_lens, prefix, hq, hkv in [([1, 1], [70, 9], 300, 4, 2), ([4, 30], [5, 200], 50, 4, 4), ([200], [200], 0, 8, 1)]:
        check_attention(BatchQ4(q_lens, seq_lens, prefix, hq, hkv, 128, 32, dtype, table_extra=extra))


def test_lengths_around_tiles_and_shares():
    # every kernel: keys around 32, 64 and 128 (tiles), rows around 8, 128 and 256 (blocks)
    for own in (31, 32, 33, 63, 65, 95, 97, 127, 129, 255, 257):
        for hq, hkv, hd in ((2, 1, 128), (16, 1, 128), (16, 1, 256)):
            check_attention(BatchQ4([1, 1], [own, own - 1], 0, hq, hkv, hd, 16, "bf16"))
            check_attention(BatchQ4([10, 6], [own, own - 1], 0, hq, hkv, hd, 16, "bf16", table_extra=4000))
    for n in (7, 8, 9, 16, 17):
        check_attention(BatchQ4([n], [n + 40], 0, 16, 1, 128, 16, "bf16"), rows={0, n - 1})
        check_attention(BatchQ4([n], [n + 40], 0, 16, 1, 128, 16, "bf16", table_extra=4000), rows={0, n - 1})
        check_attention(BatchQ4([n, 3], [n + 40, 3], 200, 1, 1, 128, 16, "bf16"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128, 256])
def test_as_many_sequences_as_there_may_be(dtype, hd):
    n = 1024
    check_attention(BatchQ4([1] * n, [(13 * i) % 37 for i in range(n)], 130, 2, 1, hd, 8, dtype), rows={0, 1, 500, n - 2, n - 1})
    check_attention(BatchQ4([1 + i % 2 * 40 for i in range(n)], [50 + i % 7 for i in range(n)], 0, 4, 1, hd, 8, dtype, table_extra=20),
                    rows={0, 1, 30, 41, 42, 21 * n - 1})


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 1, 64), (2, 2, 128), (12, 1, 128), (10, 1, 256)])
@pytest.mark.parametrize("room", TABLES)
def test_queries_that_are_not_finite_spoil_their_own_row_only(dtype, hq, hkv, hd, room):
    for q_lens, seq_lens, prefix in (([1, 1], [40, 300], 200), ([9, 30], [9, 100], 60)):
        b = BatchQ4(q_lens, seq_lens, prefix, hq, hkv, hd, 16, dtype, table_extra=-(-room // 16))
        want, mass = b.reference()
        bound = b.bound(want, mass)
        b.q[0, 1, 3], b.q[b.T - 1, hq - 1, hd - 1] = NAN, float("inf")
        b.to_device()
        got = f64(b.attend())
        bad = np.zeros(got.shape[:2], bool)
        bad[0, 1] = bad[b.T - 1, hq - 1] = True
        assert np.all(np.isnan(got[bad])) and np.all(np.abs(got[~bad] - want[~bad]) <= bound[~bad])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("room", TABLES)
@pytest.mark.parametrize("starts", [[0, 5, 3, 40], [-3, 2, 20, 40], [0, 900, 30, 40], [7, 9, 30, 38]])
def test_rows_that_do_not_ascend(dtype, room, starts):
    # what they lead to is cut or left alone, and reported (the last ones are no mistake: rows in front and behind are no one's)
    for hq, hkv, hd in ((8, 2, 64), (9, 1, 128), (2, 1, 256)):
        b = BatchQ4([10, 20, 10], [60, 20, 300], 50, hq, hkv, hd, 16, dtype, table_extra=-(-room // 16)).to_device()
        b.dev[0].copy_(torch.tensor(starts, dtype=torch.int32))
        out = b.attend()
        st = G.griffin_check_device_status(b.ws)
        assert torch.isfinite(out).all() and st == (G.OK if starts[0] == 7 else G.ERR_INVALID_ARG)
        if starts[0] == 7:
            assert torch.all(out[:7] == 77.0) and torch.all(out[38:] == 77.0) and not torch.any(out[7:38] == 77.0)


def test_two_calls_share_a_captured_workspace():
    # append, attend, read of one layer behind the other in one graph, the workspace and the cache shared
    b = BatchQ4([1, 1, 1], [30, 140, 1], 70, 12, 1, 128, 16, "bf16").to_device()
    rope = G.make_rope(G.rope_table(512, 128, device=DEV))
    q, k, v = b.q.to(DEV), b.k.to(DEV), b.v.to(DEV)

    def run(out, kk, vv):
        for i in range(2):
            qr = torch.empty_like(q)
            G.griffin_kv_append_q4(b.desc, b.batch, b.cache, rope if i else None, q, k, v, qr, b.ws)
            G.griffin_attn_prefix_q4(b.desc, b.batch, b.cache, qr, out[i], b.ws)
            G.griffin_kv_read_q4(b.desc, b.batch, b.cache, kk[i], vv[i], b.ws)

    mk = lambda x: [torch.zeros_like(x) for _ in range(2)]
    eager, captured = [(mk(q), mk(k), mk(v)) for _ in range(2)]
    run(*eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(*captured)
    b.kb.fill_(0)
    graph.replay()
    torch.cuda.synchronize()
    assert G.griffin_check_device_status(b.ws) == G.OK
    for x, y in zip(eager[1:], captured[1:]):
        assert all(torch.equal(a, c) for a, c in zip(x, y))
    host = Q.values(*Q.quantise(b.v.float().numpy()))
    assert np.array_equal(f64(captured[2][1]), host)

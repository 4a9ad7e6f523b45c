"""The cache held in 4 bits on the GPU: written, read back and attended over, through the C ABI, against numpy.

Codes and scales are compared bit for bit (q4_util restates them in fp32, one rounding an operation); attention is held to the
float64 oracle over what the cache holds, with the bounds of the cache in the storage type."""
import numpy as np
import pytest
import torch

import q4_util as Q
from layer_util import DTYPES, f64
from oracle import layer_oracle as L
from paper_2404_01365_b200 import binding as G
from q4_util import BatchQ4
from test_gpu_attn_causal import check as check_not_finite, put
from test_gpu_layer import check_attention

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN, INF = float("nan"), float("inf")


# ---- written, and read back --------------------------------------------------------------------------------------
def check_append(b, rot, style, with_q=True, fused=False, in_place=False, gap=0):
    b.to_device(gap)
    b.kb.copy_(torch.randint(0, 256, b.kb.shape, dtype=torch.uint8, generator=torch.Generator().manual_seed(1)))
    b.vb.copy_(torch.randint(0, 256, b.vb.shape, dtype=torch.uint8, generator=torch.Generator().manual_seed(2)))
    n_pos = b.prefix + int(b.seq_len.max()) + 3
    table = G.rope_table(n_pos, rot) if rot else None
    rope = G.make_rope(table.to(DEV), style) if rot else None
    if fused:      # slices of one projection's output, whose rows are wider than they need be
        qkv = torch.cat((b.q.flatten(1), b.k.flatten(1), b.v.flatten(1), torch.zeros(b.T, 16, dtype=b.dt)), 1).to(DEV)
        nq, nk = b.hq * b.hd, b.hkv * b.hd
        q, k, v = qkv[:, :nq], qkv[:, nq:nq + nk].unflatten(1, (b.hkv, b.hd)), qkv[:, nq + nk:nq + 2 * nk]
    else:
        q, k, v = b.q.to(DEV), b.k.to(DEV), b.v.to(DEV)
    q_out = None if not with_q else q if in_place else torch.full((b.T, b.hq, b.hd), 33.0, dtype=b.dt, device=DEV)
    want = {"k": b.kb.cpu().numpy(), "v": b.vb.cpu().numpy()}
    G.griffin_kv_append_q4(b.desc, b.batch, b.cache, rope, q if with_q else None, k, v, q_out, b.ws)
    assert G.griffin_check_device_status(b.ws) == G.OK

    places = [(t, s, i) for t, s, i in L.places(b.q_start.numpy(), b.seq_len.numpy())]
    pos = np.zeros(b.T, np.int64)
    for t, s, i in places:
        pos[t] = max(b.prefix + i, 0)
    tab = None if table is None else table.numpy()
    rows = {"k": Q.rotate32(b.k.float().numpy(), tab, pos, style), "v": b.v.float().numpy()}
    held = {}
    codes_end, row = b.page * b.hd // 2, -(-b.hd // 64) * 4
    for name in ("k", "v"):
        c, s8 = Q.quantise(rows[name])
        held[name] = Q.values(c, s8)
        bytes_ = Q.pack(c[:, :, None], s8[:, :, None])               # [T, heads, one token's codes and padded scales]
        for t, s, i in places:
            if i >= 0:
                page, o = want[name][int(b.page_table[s, i // b.page])], i % b.page
                page[:, o * b.hd // 2:(o + 1) * b.hd // 2] = bytes_[t, :, :b.hd // 2]
                page[:, codes_end + o * row:codes_end + o * row + b.hd // 16] = s8[t]
    assert np.array_equal(b.kb.cpu().numpy(), want["k"]) and np.array_equal(b.vb.cpu().numpy(), want["v"])
    if gap:
        assert torch.all(b.kb._base[..., b.k_bytes.shape[-1]:] == 0xAB)

    n = int(b.q_start[-1])
    if with_q:
        _, _, want_q = L.kv_append(np.zeros((int(b.page_table.max()) + 1, b.hkv, b.page, b.hd)), np.zeros((int(b.page_table.max()) + 1, b.hkv, b.page, b.hd)),
                                   b.q_start.numpy(), b.seq_len.numpy(), b.page_table.numpy(), b.prefix, f64(b.q), f64(b.k), f64(b.v),
                                   None if table is None else f64(table), style)
        got_q = f64(q_out).reshape(b.T, b.hq, b.hd)
        # one rounding of the storage type, and two products and a sum in 32 bits
        ulp, size = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}[b.dtype], 2 * float(b.q.abs().max())
        assert np.all(np.abs(got_q[:n] - want_q[:n]) <= ulp * np.abs(want_q[:n]) + 4 * 2.0 ** -24 * size)
        assert np.all(got_q[n:] == (f64(b.q)[n:] if in_place else 33.0)), "rows behind the last sequence were written"
    # and back
    got = dict(zip("kv", b.read()))
    assert G.griffin_check_device_status(b.ws) == G.OK
    for name in ("k", "v"):
        out = f64(got[name])
        for t, s, i in places:
            assert np.array_equal(out[t], held[name][t] if i >= 0 else np.zeros_like(held[name][t]))
        assert np.all(out[n:] == 33.0), "rows behind the last sequence were written"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot,style", [(0, "half"), (16, "pairs"), (16, "half"), (48, "half"), (64, "half"), (64, "pairs")])
@pytest.mark.parametrize("gap", [0, 48])
def test_append_forms(dtype, rot, style, gap):
    check_append(BatchQ4([3, 1, 7], [19, 1, 40], 21, 4, 2, 80, 16, dtype), rot, style, gap=gap)


@pytest.mark.parametrize("hq,hkv,hd", [(1, 1, 64), (10, 2, 128), (40, 40, 128), (6, 3, 80), (3, 1, 256), (64, 1, 112), (2, 2, 208)])
def test_append_heads(hq, hkv, hd):
    check_append(BatchQ4([1, 4, 1], [1, 9, 130], 0, hq, hkv, hd, 32, "bf16"), hd, "half", fused=True)


@pytest.mark.parametrize("q_lens,seq_lens", [([1], [1]), ([0, 1, 0, 2, 0], [5, 1, 0, 9, 3]), ([4, 2], [2, 0]), ([700], [700]),
                                             ([1] * 300, list(range(1, 301)))])
def test_append_lengths_empty_sequences_and_padding(q_lens, seq_lens):
    check_append(BatchQ4(q_lens, seq_lens, 5, 2, 1, 64, 8, "bf16", extra_rows=3), 32, "half")


@pytest.mark.parametrize("dtype,style", [("bf16", "half"), ("f32", "pairs")])
def test_append_and_read_of_many_tokens(dtype, style):
    check_append(BatchQ4([1500, 1100], [1500, 1203], 7, 2, 1, 64, 64, dtype), 48, style)       # several tokens to a CTA


def test_append_in_place_without_queries_and_on_another_stream():
    mk = lambda: BatchQ4([2, 5], [9, 5], 17, 4, 2, 128, 64, "bf16")
    check_append(mk(), 128, "pairs", in_place=True)
    check_append(mk(), 128, "half", with_q=False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        check_append(mk(), 128, "half")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sizes_from_nothing_to_beyond_the_scales(dtype):
    # zeros, subnormal numbers, the smallest and the largest scales, saturation, and groups that are not finite
    b = BatchQ4([90], [90], 0, 1, 1, 64, 16, dtype)
    for t in range(90):
        b.k[t] = (b.k[t].float() * 2.0 ** (t - 45) if t < 85 else b.k[t].float() * 0).to(b.dt)
    b.k[86, 0, 3], b.k[87, 0, 20], b.k[88, 0, 63], b.v[5, 0, 40] = NAN, INF, -INF, NAN
    b.k[89, 0, 5] = torch.finfo(b.dt).max
    b.v[6] = torch.finfo(torch.float32).tiny / 4
    check_append_not_finite(b)


def check_append_not_finite(b):
    b.to_device()
    G.griffin_kv_append_q4(b.desc, b.batch, b.cache, None, None, b.k.to(DEV), b.v.to(DEV), None, b.ws)
    got = b.read()
    for x, out in ((b.k, got[0]), (b.v, got[1])):
        want = Q.values(*Q.quantise(x.float().numpy()))
        assert np.array_equal(f64(out), want, equal_nan=True)
        ok = np.isfinite(f64(x))
        groups = lambda a: a.reshape(-1, 16)
        fine = groups(ok).all(1)
        assert np.array_equal(~fine, np.isnan(groups(want)).all(1)) and np.array_equal(~fine, np.isnan(groups(want)).any(1))
        x, want = groups(f64(x))[fine], groups(want)[fine]
        s = np.array([L.q4_scale(g) for g in x])[:, None]
        held = np.abs(x) <= 12544.0
        assert np.all(np.abs(want - x)[held] <= np.broadcast_to(s / 2 * (1 + 2.0 ** -20), x.shape)[held])
        assert np.all(np.abs(want[~held]) == 12544.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_codes_next_to_their_borders(dtype):
    # (n + 1/2) s and its neighbours in the storage type, for every scale of an octave: ties and what is next to them
    n_tok, step = 2048, {"bf16": 2.0 ** -7, "f32": 2.0 ** -22}[dtype]
    b = BatchQ4([n_tok], [n_tok], 0, 4, 4, 64, 64, dtype)
    rng = np.random.default_rng(3)
    s = (8 + rng.integers(0, 8, (n_tok, 4, 4, 1))) * 2.0 ** rng.integers(-20, 6, (n_tok, 4, 4, 1))
    x = (rng.integers(-7, 7, (n_tok, 4, 4, 16)) + 0.5) * s * (1 + step * rng.integers(-4, 5, (n_tok, 4, 4, 16)) / 4)
    x[..., :1] = 7 * s
    b.k = torch.from_numpy(x.reshape(n_tok, 4, 64)).to(b.dt)
    b.v = (b.v.float() * 3.0).to(b.dt)
    b.to_device()
    G.griffin_kv_append_q4(b.desc, b.batch, b.cache, None, None, b.k.to(DEV), b.v.to(DEV), None, b.ws)
    for x, out in zip((b.k, b.v), b.read()):
        assert np.array_equal(f64(out), Q.values(*Q.quantise(x.float().numpy())))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hkv,hd,n", [(1, 64, 900), (1, 64, 12000), (3, 80, 9000), (16, 256, 700), (33, 64, 2500)])
def test_read_of_few_and_many_heads(dtype, hkv, hd, n):
    # units that a CTA's threads have several tokens of, or that several CTAs share; rows on 16-byte boundaries only
    b = BatchQ4([1, 1], [3, 5], 0, hkv, hkv, hd, 16, dtype)
    pages = torch.randint(0, b.k_bytes.shape[0], (2, -(-n // 16)), dtype=torch.int32, generator=torch.Generator().manual_seed(1))
    lens = [n, n // 3]
    b.to_device()
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
    batch = G.make_attn_batch(i32([0, n, n + n // 3]), i32(lens), pages.to(DEV), n + n // 3)
    pad = 16 // b.dt.itemsize
    k = torch.full((n + n // 3, hkv * hd + pad), 5.0, dtype=b.dt, device=DEV)
    v = torch.full((n + n // 3, hkv * hd), 5.0, dtype=b.dt, device=DEV)
    G.griffin_kv_read_q4(b.desc, batch, b.cache, k[:, :hkv * hd], v, b.ws)
    assert G.griffin_check_device_status(b.ws) == G.OK and torch.all(k[:, hkv * hd:] == 5.0)
    for out, host in ((k[:, :hkv * hd], b.k_host), (v, b.v_host)):
        want = torch.cat([host.transpose(1, 2)[pages[s].long()].flatten(0, 1)[:lens[s]] for s in range(2)]).flatten(1)
        assert torch.equal(torch.nan_to_num(out.cpu(), nan=77.0), torch.nan_to_num(want, nan=77.0))


def test_what_cannot_be_placed_is_reported():
    def run(b, table=None):
        b.to_device()
        q_out = torch.full((b.T, b.hq, b.hd), 3.0, dtype=b.dt, device=DEV)
        old = b.kb.clone()
        rope = None if table is None else G.make_rope(table)
        G.griffin_kv_append_q4(b.desc, b.batch, b.cache, rope, b.q.to(DEV), b.k.to(DEV), b.v.to(DEV), q_out, b.ws)
        return old, q_out, G.griffin_check_device_status(b.ws)

    b = BatchQ4([2, 1], [4, 3], 0, 2, 1, 64, 8, "bf16", fill=0.0)
    b.page_table[1, 0] = 999
    old, q_out, st = run(b, G.rope_table(16, 64, device=DEV))
    assert st == G.ERR_INVALID_ARG and torch.all(q_out[2] == 0) and not torch.all(q_out[0] == 0) and not torch.equal(b.kb, old)
    G.griffin_workspace_init(b.ws)
    k, v = b.read()
    assert G.griffin_check_device_status(b.ws) == G.ERR_INVALID_ARG and torch.all(k[2] == 0) and torch.all(v[2] == 0) and not torch.all(k[0] == 0)
    b = BatchQ4([2], [4], 10, 2, 1, 64, 8, "bf16", fill=0.0)
    old, q_out, st = run(b, G.rope_table(13, 64, device=DEV))            # positions 12 and 13: the second is beyond the table
    assert st == G.ERR_INVALID_ARG and not torch.all(q_out[0] == 0) and torch.all(q_out[1] == 0)
    b = BatchQ4([1], [8], 0, 2, 1, 64, 8, "bf16", fill=0.0, table_extra=0)
    b.seq_len[0] = 9                                                     # beyond the table's only page
    old, q_out, st = run(b)
    assert st == G.ERR_INVALID_ARG and torch.equal(b.kb, old)
    # q_start that does not begin at 0: the rows in front of it belong to no sequence
    b = BatchQ4([2, 3], [2, 3], 0, 2, 1, 64, 8, "bf16").to_device()
    b.dev[0][0] = 1
    k, v = b.read()
    assert torch.all(k[0] == 33.0) and torch.all(v[0] == 33.0) and not torch.any(k[1:] == 33.0)


def test_read_into_strided_rows_and_of_the_prefix():
    b = BatchQ4([1, 1], [5, 9], 45, 4, 2, 80, 16, "bf16").to_device()
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device=DEV)
    whole = G.make_attn_batch(i32(0, 45), i32(45), b.dev[3][None], 45)
    wide = torch.full((45, 2 * 160 + 24), 5.0, dtype=b.dt, device=DEV)
    G.griffin_kv_read_q4(b.desc, whole, b.cache, wide[:, :160], wide[:, 160:320], b.ws)
    assert G.griffin_check_device_status(b.ws) == G.OK and torch.all(wide[:, 320:] == 5.0)
    for at, host in ((slice(0, 160), b.k_host), (slice(160, 320), b.v_host)):
        want = L.gather(f64(host), b.prefix_pages.numpy(), 45)
        assert np.array_equal(f64(wide[:, at]).reshape(45, 2, 80), want)


# ---- attention ---------------------------------------------------------------------------------------------------
HEADS = [(1, 1, 64), (8, 8, 128), (8, 2, 128), (6, 2, 80), (5, 1, 112), (4, 4, 256), (8, 1, 208), (64, 1, 64)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hkv,hd", HEADS)
def test_attention_step_behind_a_shared_prefix(dtype, hq, hkv, hd):
    check_attention(BatchQ4([1, 1, 1, 1], [1, 40, 129, 77], 300, hq, hkv, hd, 16, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hkv,hd", [(2, 2, 64), (4, 1, 128), (3, 1, 80), (2, 1, 256)])
@pytest.mark.parametrize("n", [1, 7, 64, 128, 129, 300])
def test_attention_of_a_prompt(dtype, hq, hkv, hd, n):
    check_attention(BatchQ4([n], [n], 0, hq, hkv, hd, 32, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("prefix", [0, 1, 31, 32, 127, 128, 129, 1000])
def test_attention_prefix_lengths(dtype, prefix):
    check_attention(BatchQ4([1, 2], [1, 33], prefix, 4, 2, 128, 32, dtype))
    check_attention(BatchQ4([1], [5], prefix, 4, 2, 128, 32, dtype))               # one sequence walks the prefix itself


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page", [8, 16, 64, 128, 256])
def test_attention_pages(dtype, page):
    check_attention(BatchQ4([1, 3, 1], [200, 131, 3], 150, 4, 2, 128, page, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fill", [NAN, 12000.0])
def test_attention_does_not_see_what_lies_behind_the_ends(dtype, fill):
    check_attention(BatchQ4([1, 2, 1], [5, 70, 129], 37, 4, 2, 64, 64, dtype, fill=fill))
    check_attention(BatchQ4([1, 2, 1], [5, 70, 129], 37, 2, 1, 256, 32, dtype, fill=fill))
    check_attention(BatchQ4([200], [203], 0, 2, 1, 128, 64, dtype, fill=fill))
    check_attention(BatchQ4([4, 2, 3], [5, 70, 129], 37, 4, 2, 64, 64, dtype, fill=fill))
    check_attention(BatchQ4([9], [40], 37, 2, 2, 128, 16, dtype, fill=fill))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q_lens,seq_lens,prefix", [
    ([1, 0, 3, 0], [4, 9, 7, 0], 20),          # sequences without new tokens
    ([2, 1], [0, 0], 0),                       # padding only: nothing is seen
    ([2, 1], [0, 0], 50),                      # padding behind a prefix: the prefix is seen
    ([5, 1], [3, 1], 0),                       # two rows of padding in front of three tokens
    ([400, 1], [398, 2], 0),                   # and with more rows than a tile
    ([150, 1, 90], [150, 300, 512], 70),       # pieces and steps in one call
    ([1] * 40, [(7 * i) % 50 + 1 for i in range(40)], 513),
    ([33] * 6, [33 + 20 * i for i in range(6)], 260),
])
def test_attention_ragged_batches(dtype, q_lens, seq_lens, prefix):
    check_attention(BatchQ4(q_lens, seq_lens, prefix, 4, 2, 64, 16, dtype, extra_rows=2))
    check_attention(BatchQ4(q_lens, seq_lens, prefix, 3, 1, 128, 16, dtype))


@pytest.mark.parametrize("hq,hkv,hd", [(2, 2, 64), (4, 2, 80), (8, 1, 128), (3, 1, 208), (2, 1, 256)])
@pytest.mark.parametrize("page", [8, 16, 128])
def test_attention_of_a_few_rows(hq, hkv, hd, page):
    group = hq // hkv
    most = 8 // group
    for q_lens, seq_lens, prefix in [([1], [1], 0), ([1], [700], 0), ([most], [333], 90), ([most + 1], [333], 90), ([most, 0], [130, 5], 0),
                                     ([most - most // 2, most // 2], [17, 129], 300), ([most, 1], [17, 129], 300), ([1, 1], [0, 3], 0),
                                     ([3 * most, 1, 1], [3 * most + 5, 40, 16], 0), ([most, 1], [most - 1, 64], 0)]:
        check_attention(BatchQ4(q_lens, seq_lens, prefix, hq, hkv, hd, page, "bf16"))


def test_attention_of_few_rows_and_many_blocks():
    for n in (74, 75):
        check_attention(BatchQ4([1] * n, [(31 * i) % 190 for i in range(n)], 0, 8, 4, 64, 16, "bf16"), rows={0, 1, 7, n - 2, n - 1})
    check_attention(BatchQ4([1] * 8, [(31 * i) % 190 + 1 for i in range(8)], 1100, 37, 37, 64, 16, "bf16"), rows={0, 7})
    check_attention(BatchQ4([1] * 8, [(31 * i) % 190 + 1 for i in range(8)], 1100, 38, 38, 64, 16, "bf16"), rows={0, 7})
    check_attention(BatchQ4([1] * 1000, [(13 * i) % 37 for i in range(1000)], 64, 2, 1, 64, 8, "bf16"), rows={0, 1, 2, 500, 998, 999})


def test_attention_of_two_blocks_of_few_rows():
    check_attention(BatchQ4([4], [1500], 0, 8, 2, 128, 16, "bf16"))
    check_attention(BatchQ4([13, 9, 2], [700, 9, 40], 0, 2, 2, 80, 32, "bf16"))
    check_attention(BatchQ4([2, 2], [200, 5], 333, 8, 2, 128, 16, "bf16"))
    check_attention(BatchQ4([1, 3, 0, 1], [20, 90, 4, 1], 1111, 3, 1, 256, 64, "bf16"))
    check_attention(BatchQ4([17, 1], [16, 30], 0, 1, 1, 64, 8, "bf16"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_over_a_long_context(dtype):
    check_attention(BatchQ4([1], [9000], 0, 4, 1, 128, 64, dtype))
    check_attention(BatchQ4([1, 1], [37, 900], 7000, 4, 1, 128, 64, dtype))


def test_attention_whose_jobs_come_from_a_queue():
    # three row blocks per CTA and more: a prompt, and pieces of several sequences
    check_attention(BatchQ4([1000], [1000], 0, 76, 76, 64, 64, "bf16"), rows={0, 1, 255, 256, 511, 512, 767, 768, 999})
    check_attention(BatchQ4([300] * 3, [300, 450, 310], 0, 78, 78, 128, 16, "bf16"), rows={0, 255, 256, 299, 300, 600, 899})


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q_scale", [0.0, 12.0])
def test_attention_flat_and_sharp(dtype, q_scale):
    check_attention(BatchQ4([1, 4], [300, 700], 200, 4, 2, 128, 64, dtype, q_scale=q_scale))
    check_attention(BatchQ4([60], [300], 0, 4, 2, 128, 64, dtype, q_scale=q_scale))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hkv,hd", [(2, 2, 64), (4, 1, 128), (3, 1, 80), (2, 1, 256), (5, 1, 208)])
@pytest.mark.parametrize("n,own,prefix", [(2, 2, 0), (3, 50, 0), (8, 8, 0), (8, 301, 40), (40, 40, 0), (129, 200, 0), (300, 300, 0), (300, 290, 20)])
def test_a_group_of_values_that_is_not_finite_reaches_those_that_see_it(dtype, hq, hkv, hd, n, own, prefix):
    for back in {1, n // 2, n - 1}:
        if own - back < 0:
            continue
        b = BatchQ4([n], [own], prefix, hq, hkv, hd, 16, dtype, fill=0.0, seed=back)
        put(b, 0, own - back, hd - 3, NAN)
        b.requantise()
        check_not_finite(b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq", [2, 10])
def test_a_group_of_a_key_that_is_not_finite(dtype, hq):
    for prefix, own, at in [(0, 1, 0), (0, 9, 3), (40, 200, 197), (40, 200, 2), (0, 300, 128)]:
        b = BatchQ4([1, 1], [own, 30], prefix, hq, 1, 128, 16, dtype, fill=0.0)
        b.k_host[int(b.page_table[0, at // 16]), 0, at % 16, 5] = NAN
        b.requantise()
        b.to_device()
        got = b.attend()
        assert torch.isnan(got[0]).all() and torch.isfinite(got[1]).all()


def test_attention_strided_rows_and_in_place():
    b = BatchQ4([2, 5], [9, 40], 17, 4, 2, 128, 64, "bf16")
    wide = torch.zeros(b.T, 4 * 128 + 24, dtype=b.dt, device=DEV)
    wide[:, :512] = b.q.flatten(1)
    out = torch.zeros(b.T, 4 * 128 + 8, dtype=b.dt, device=DEV)
    b.to_device(gap=32)
    plain = b.attend()
    b.attend(q=wide[:, :512], out=out[:, :512])
    assert torch.equal(out[:, :512].reshape_as(plain), plain) and torch.all(out[:, 512:] == 0)
    q = b.q.to(DEV)
    b.attend(q=q, out=q)
    assert torch.equal(q, plain)


@pytest.mark.parametrize("q_lens", [[1, 1, 1], [40, 3, 90]])
def test_attention_on_another_stream_and_in_a_graph(q_lens):
    b = BatchQ4(q_lens, [60, 61, 200], 300, 8, 2, 128, 16, "bf16").to_device()
    plain = b.attend()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = b.attend()
    side.synchronize()
    assert torch.equal(out, plain)
    q, out = b.q.to(DEV), torch.zeros_like(plain)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.attend(q=q, out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, plain)
    b.dev[1] -= 7          # the lengths are read when the graph runs
    b.seq_len -= 7
    graph.replay()
    torch.cuda.synchronize()
    want, mass = b.reference()
    assert np.all(np.abs(f64(out) - want) <= b.bound(want, mass))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q_lens", [[1, 1], [9, 9]])
def test_attention_reports_bad_pages_and_lengths(dtype, q_lens):
    b = BatchQ4(q_lens, [20, 9], 0, 2, 1, 80, 8, dtype, fill=0.0)
    b.page_table[0, 1] = 10 ** 6
    b.to_device()
    out = b.attend()
    assert G.griffin_check_device_status(b.ws) == G.ERR_INVALID_ARG
    G.griffin_workspace_init(b.ws)
    b.k_host = torch.cat((b.k_host, torch.zeros_like(b.k_host[:1])))              # the page reads as zeros
    b.v_host = torch.cat((b.v_host, torch.zeros_like(b.v_host[:1])))
    b.page_table[0, 1] = b.k_host.shape[0] - 1
    want, mass = b.reference()
    assert np.all(np.abs(f64(out) - want) <= b.bound(want, mass))
    b = BatchQ4(q_lens, [16, 9], 0, 2, 1, 64, 8, dtype, fill=0.0, table_extra=0).to_device()
    b.dev[1][0] = 17
    out = b.attend()
    assert G.griffin_check_device_status(b.ws) == G.ERR_INVALID_ARG and torch.isfinite(out).all()


@pytest.mark.parametrize("dtype,q_lens", [("f32", [1, 2]), ("bf16", [1, 2]), ("bf16", [30, 2])])
def test_cache_offsets_beyond_32_bits(dtype, q_lens):
    # caches of 2^32 bytes and more, of which the calls use pages at their end
    hd, page, hkv = 128, 64, 8
    size = Q.block_bytes(page, hd)
    n_pages = (1 << 32) // (size * hkv) + 40
    kb, vb = (torch.empty(n_pages, hkv, size, dtype=torch.uint8, device=DEV) for _ in range(2))
    b = BatchQ4(q_lens, [70, 3], 100, 8, hkv, hd, page, dtype)
    first = n_pages - b.k_host.shape[0]
    kb[first:], vb[first:] = b.k_bytes.to(DEV), b.v_bytes.to(DEV)
    table, pre = (b.page_table + first).to(DEV), (b.prefix_pages + first).to(DEV)
    desc = G.make_attn_desc(8, hkv, hd, page, dtype)
    batch = G.make_attn_batch(b.q_start.to(DEV), b.seq_len.to(DEV), table, b.T, pre, b.prefix)
    ws, cache = G.alloc_attn_workspace(desc, b.T, 2, DEV), G.make_kv_cache_q4(kb, vb)
    out = torch.zeros(b.T, 8, hd, dtype=b.dt, device=DEV)
    G.griffin_attn_prefix_q4(desc, batch, cache, b.q.to(DEV), out, ws)
    want, mass = b.reference()
    assert np.all(np.abs(f64(out) - want) <= b.bound(want, mass))
    G.griffin_kv_append_q4(desc, batch, cache, None, None, b.k.to(DEV), b.v.to(DEV), None, ws)
    k, v = (torch.zeros(b.T, hkv, hd, dtype=b.dt, device=DEV) for _ in range(2))
    G.griffin_kv_read_q4(desc, batch, cache, k, v, ws)
    for x, got in ((b.k, k), (b.v, v)):
        assert np.array_equal(f64(got), Q.values(*Q.quantise(x.float().numpy())))
    assert G.griffin_check_device_status(ws) == G.OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_then_attend_is_one_causal_pass_over_the_tokens(dtype):
    # a prompt in one call and in three pieces: the same cache, and outputs within the roundings of the two
    n, cuts = 200, (0, 70, 71, 200)
    b = BatchQ4([n], [n], 0, 4, 2, 128, 16, dtype, fill=0.0).to_device()
    rope = G.make_rope(G.rope_table(256, 128, device=DEV))
    q, k, v = b.q.to(DEV), b.k.to(DEV), b.v.to(DEV)
    q1 = torch.empty_like(q)
    G.griffin_kv_append_q4(b.desc, b.batch, b.cache, rope, q, k, v, q1, b.ws)
    whole, kb = b.attend(q=q1), b.kb.clone()
    b.kb.fill_(7)
    parts = []
    for lo, hi in zip(cuts, cuts[1:]):
        batch = G.make_attn_batch(torch.tensor([0, hi - lo], dtype=torch.int32, device=DEV),
                                  torch.tensor([hi], dtype=torch.int32, device=DEV), b.dev[2], hi - lo)
        qp, out = torch.empty_like(q[lo:hi]), torch.empty_like(q[lo:hi])
        G.griffin_kv_append_q4(b.desc, batch, b.cache, rope, q[lo:hi], k[lo:hi], v[lo:hi], qp, b.ws)
        G.griffin_attn_prefix_q4(b.desc, batch, b.cache, qp, out, b.ws)
        parts.append(out)
    used = [int(x) for x in b.page_table[0, :-(-n // 16)]]
    row = -(-128 // 64) * 4
    for i, page in enumerate(used):
        m = min(16, n - 16 * i)
        for lo, width in ((0, 64), (16 * 64, row)):
            assert torch.equal(b.kb[page, :, lo:lo + m * width], kb[page, :, lo:lo + m * width])
    # the exact output over what the cache holds: both are within its bound of it
    kk, vv = b.read()
    x, y, z = f64(q1), f64(kk), f64(vv)
    kmax = np.abs(y).max()
    got = [f64(torch.cat(parts)), f64(whole)]
    for t in (0, 69, 70, 71, 128, 199):
        for h in range(4):
            logit = y[:t + 1, h // 2] @ x[t, h] * b.scale
            p = np.exp(logit - logit.max())
            p /= p.sum()
            want, mass = p @ z[:t + 1, h // 2], p @ np.abs(z[:t + 1, h // 2])
            arith = (2 * (128 + 4) * np.abs(x[t, h]).sum() * kmax * b.scale * 2.0 ** -24 + 2 * (t + 9) * 2.0 ** -24 + 2.0 ** -21) * mass
            bound = arith + (0.0 if dtype == "f32" else 2.0 ** -8 * (1.01 * mass + np.abs(want)))
            for g in got:
                assert np.all(np.abs(g[t, h] - want) <= bound + 1e-30)

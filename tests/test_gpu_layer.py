"""The operators around the FF block on the GPU, through the C ABI, against the float64 oracle."""
import numpy as np
import pytest
import torch

from layer_util import DTYPES, Batch, f64
from oracle import layer_oracle as L
from paper_2404_01365_b200 import binding as G

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# ---- norms and the residual stream -------------------------------------------------------------------------------
def norm_case(T, d, dtype, res, pre, post, gate, act="linear", biases=True, w0=0.0, seed=0, pad=0, x_shift=0.0):
    g = torch.Generator().manual_seed(seed)
    dt, rdt = DTYPES[dtype], DTYPES[res]
    rnd = lambda *s, t=dt, m=1.0, b=0.0: (torch.randn(*s, generator=g) * m + b).to(t)
    wide = lambda t, **k: rnd(T, d + pad, t=t, **k)[:, :d]
    y, r = wide(dt, m=0.7), wide(rdt, m=2.0, b=x_shift)
    w = {n: rnd(d, m=0.2, b=1.0 - w0) for n in ("pre_w", "post_w")}
    b = {n: rnd(d, m=0.2) if biases else None for n in ("pre_b", "post_b")}
    gt = {"none": None, "channel": rnd(d), "full": wide(dt)}[gate]
    return y, r, w, b, gt


def check_norm(T, d, dtype, res, pre, post, gate, act="linear", biases=True, w0=0.0, res_scale=1.0, out_scale=1.0, with_y=True,
               pad=0, in_place=False, x_shift=0.0, seed=0):
    y, r, w, b, gt = norm_case(T, d, dtype, res, pre, post, gate, act, biases, w0, seed, pad, x_shift)
    up = lambda t: None if t is None else t.to(DEV) if t.dim() == 1 or pad == 0 else torch.nn.functional.pad(t, (0, pad)).to(DEV)[:, :d]
    desc = G.make_norm_desc(d, dtype, res, pre, post, 1e-5, w0, res_scale, out_scale, act)
    dw = {k: up(v) for k, v in {**w, **b}.items()}
    weights = G.make_norm_weights(dw["pre_w"], dw["pre_b"], dw["post_w"], dw["post_b"])
    yd, rd = up(y) if with_y else None, up(r)
    ro = rd if in_place else torch.full((T, d), 55.0, dtype=rd.dtype, device=DEV)
    h = yd if in_place and with_y else torch.full((T, d), 55.0, dtype=DTYPES[dtype], device=DEV)
    G.griffin_norm_residual(desc, weights, rd, ro, h, yd, up(gt) if with_y else None)
    want_r, want_h = L.norm_residual(f64(r), f64(y) if with_y else None, f64(gt) if with_y else None, pre, post, f64(w["pre_w"]),
                                     f64(b["pre_b"]), f64(w["post_w"]), f64(b["post_b"]), 1e-5, w0, res_scale, out_scale, act)
    # One rounding to the storage type (2^-8 of a bf16 value), and fp32 arithmetic: a handful of roundings per entry
    # and the statistics' sums (d terms, added in trees of depth < 40), relative to the largest entry of the row.
    ulp = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
    rows = lambda a: np.abs(a).max(1, keepdims=True) + 1.0
    slack = 64 * 2.0 ** -24
    assert np.all(np.abs(f64(ro) - want_r) <= ulp[res] * np.abs(want_r) * 1.01 + slack * rows(want_r) * (1 + abs(x_shift)))
    assert np.all(np.abs(f64(h) - want_h) <= ulp[dtype] * np.abs(want_h) * 1.01 + slack * rows(want_h) * (1 + abs(x_shift)))


@pytest.mark.parametrize("d", [8, 248, 256, 264, 512, 1016, 1024, 1032, 2056, 4096, 4104, 8192, 8200, 16384])
@pytest.mark.parametrize("dtype,res", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_norm_residual_widths(d, dtype, res):
    check_norm(3, d, dtype, res, "rms", "rms", "channel", seed=d)


@pytest.mark.parametrize("pre", ["none", "rms", "layer"])
@pytest.mark.parametrize("post", ["none", "rms", "layer"])
@pytest.mark.parametrize("gate,act", [("none", "linear"), ("channel", "sigmoid"), ("full", "tanh"), ("full", "linear")])
@pytest.mark.parametrize("d", [320, 1360])
def test_norm_residual_forms(pre, post, gate, act, d):
    check_norm(5, d, "bf16", "f32", pre, post, gate, act, biases=gate != "none", w0=1.0 if gate == "full" else 0.0, res_scale=0.7,
               out_scale=1.3)


@pytest.mark.parametrize("T", [1, 2, 4, 5, 149, 1000])
@pytest.mark.parametrize("d", [128, 1200])
def test_norm_residual_row_counts_and_strides(T, d):
    check_norm(T, d, "f32", "f32", "layer", "rms", "full", pad=24)
    check_norm(T, d, "bf16", "bf16", "rms", "none", "none", pad=8)


@pytest.mark.parametrize("d", [320, 1360])
def test_norm_residual_in_place_and_without_a_block(d):
    check_norm(6, d, "bf16", "bf16", "rms", "rms", "channel", in_place=True)
    check_norm(6, d, "bf16", "f32", "rms", "none", "none", with_y=False, res_scale=8.0)
    check_norm(6, d, "f32", "f32", "layer", "none", "none", x_shift=100.0)     # a mean far above the spread


def test_norm_residual_outputs_may_be_left_out():
    r = torch.randn(4, 512, device=DEV)
    y = torch.randn(4, 512, device=DEV)
    out = torch.empty_like(r)
    none = G.make_norm_weights()
    G.griffin_norm_residual(G.make_norm_desc(512, "f32", pre="none"), none, r, out, None, y)
    assert torch.equal(out, r + y)
    h, w = torch.empty_like(r), torch.ones(512, device=DEV)
    G.griffin_norm_residual(G.make_norm_desc(512, "f32", pre="rms"), G.make_norm_weights(w), r, None, h)
    assert torch.allclose(h, r * torch.rsqrt((r * r).mean(1, keepdim=True) + 1e-6), rtol=1e-5, atol=1e-6)
    G.griffin_norm_residual(G.make_norm_desc(512, "f32", pre="rms"), G.make_norm_weights(w), r[:0], None, h[:0])   # no rows: nothing


def test_norm_residual_rows_do_not_touch_each_other():
    r = torch.randn(9, 1360, device=DEV)
    r[4, 7], r[6, 11] = float("nan"), float("inf")
    h, w = torch.empty_like(r), torch.ones(1360, device=DEV)
    G.griffin_norm_residual(G.make_norm_desc(1360, "f32", pre="rms"), G.make_norm_weights(w), r, None, h)
    bad = (~torch.isfinite(h)).any(1).cpu().tolist()
    assert [i for i, x in enumerate(bad) if x] == [4, 6]


# ---- the cache ---------------------------------------------------------------------------------------------------
def check_append(b, rot, style, with_q=True, fused=False, in_place=False):
    b.to_device()
    n_pos = b.prefix + int(b.seq_len.max()) + 3
    table = G.rope_table(n_pos, rot, device=DEV) if rot else None
    if fused:      # slices of one projection's output, whose rows are wider than they need be
        qkv = torch.cat((b.q.flatten(1), b.k.flatten(1), b.v.flatten(1), torch.zeros(b.T, 16, dtype=b.dt)), 1).to(DEV)
        nq, nk = b.hq * b.hd, b.hkv * b.hd
        q, k, v = qkv[:, :nq], qkv[:, nq:nq + nk].unflatten(1, (b.hkv, b.hd)), qkv[:, nq + nk:nq + 2 * nk]
    else:
        q, k, v = b.q.to(DEV), b.k.to(DEV), b.v.to(DEV)
    q_out = None if not with_q else q if in_place else torch.full((b.T, b.hq, b.hd), 33.0, dtype=b.dt, device=DEV)
    before_k, before_v = b.kc.clone(), b.vc.clone()
    G.griffin_kv_append(b.desc, b.batch, b.cache, G.make_rope(table, style) if rot else None, q if with_q else None, k, v, q_out, b.ws)
    assert G.griffin_check_device_status(b.ws) == G.OK
    want_k, want_v, want_q = L.kv_append(f64(before_k), f64(before_v), b.q_start.numpy(), b.seq_len.numpy(), b.page_table.numpy(),
                                         b.prefix, f64(b.q), f64(b.k), f64(b.v), None if table is None else f64(table), style)
    # one rounding of the storage type, and two products and a sum in 32 bits: three roundings of values up to |x| + |y|
    ulp = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}[b.dtype]
    near = lambda a, w, size: np.all(np.abs(a - w) <= ulp * np.abs(w) + 4 * 2.0 ** -24 * size)
    size = 2 * float(torch.cat((b.q.flatten(), b.k.flatten())).abs().max())
    touched = np.zeros(want_k.shape[:1] + want_k.shape[2:3], bool)
    for t, s, i in L.places(b.q_start.numpy(), b.seq_len.numpy()):
        if i >= 0:
            touched[b.page_table[s, i // b.page], i % b.page] = True
    got_k, got_v = f64(b.kc), f64(b.vc)
    at = np.broadcast_to(touched[:, None, :, None], got_k.shape)
    assert near(got_k[at], want_k[at], size) and np.array_equal(got_v[at], want_v[at])
    for got, old in ((got_k, before_k), (got_v, before_v)):
        assert np.array_equal(got[~at], f64(old)[~at], equal_nan=True), "an entry that no token stands for was written"
    if with_q:
        n = int(b.q_start[-1])
        got_q = f64(q_out).reshape(b.T, b.hq, b.hd)
        assert near(got_q[:n], want_q[:n], size)
        assert np.all(got_q[n:] == (f64(b.q)[n:] if in_place else 33.0)), "rows behind the last sequence were written"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot,style", [(0, "half"), (16, "pairs"), (64, "half"), (64, "pairs")])
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
def test_append_forms(dtype, rot, style, layout):
    check_append(Batch([3, 1, 7], [19, 1, 40], 21, 4, 2, 72, 16, dtype, layout=layout), rot, style)


@pytest.mark.parametrize("hq,hkv,hd", [(1, 1, 64), (10, 2, 128), (40, 40, 128), (6, 3, 80), (3, 1, 256), (64, 1, 88)])
def test_append_heads(hq, hkv, hd):
    check_append(Batch([1, 4, 1], [1, 9, 130], 0, hq, hkv, hd, 32, "bf16"), hd // 16 * 16, "half", fused=True)


@pytest.mark.parametrize("q_lens,seq_lens", [([1], [1]), ([0, 1, 0, 2, 0], [5, 1, 0, 9, 3]), ([4, 2], [2, 0]), ([700], [700]),
                                             ([1] * 300, list(range(1, 301)))])
def test_append_lengths_empty_sequences_and_padding(q_lens, seq_lens):
    check_append(Batch(q_lens, seq_lens, 5, 2, 1, 64, 8, "bf16", extra_rows=3), 32, "half")


def test_append_in_place_without_queries_and_on_another_stream():
    mk = lambda: Batch([2, 5], [9, 5], 17, 4, 2, 128, 64, "bf16")
    check_append(mk(), 128, "pairs", in_place=True)
    check_append(mk(), 128, "half", with_q=False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        check_append(mk(), 128, "half")


def test_append_reports_what_it_cannot_place():
    def run(b, table):
        b.to_device()
        q_out = torch.full((b.T, b.hq, b.hd), 3.0, dtype=b.dt, device=DEV)
        old = b.kc.clone()
        G.griffin_kv_append(b.desc, b.batch, b.cache, G.make_rope(table), b.q.to(DEV), b.k.to(DEV), b.v.to(DEV), q_out, b.ws)
        return old, q_out, G.griffin_check_device_status(b.ws)

    b = Batch([2, 1], [4, 3], 0, 2, 1, 64, 8, "bf16", fill=0.0)
    b.page_table[1, 0] = 999
    old, q_out, st = run(b, G.rope_table(16, 64, device=DEV))
    assert st == G.ERR_INVALID_ARG and torch.all(q_out[2] == 0) and not torch.all(q_out[0] == 0)
    b = Batch([2], [4], 10, 2, 1, 64, 8, "bf16", fill=0.0)
    old, q_out, st = run(b, G.rope_table(13, 64, device=DEV))            # positions 12 and 13: the second is beyond the table
    assert st == G.ERR_INVALID_ARG and not torch.all(q_out[0] == 0) and torch.all(q_out[1] == 0)
    assert not torch.equal(b.kc, old)
    b = Batch([1], [8], 0, 2, 1, 64, 8, "bf16", fill=0.0, table_extra=0)
    b.seq_len[0] = 9                                                     # beyond the table's only page
    old, q_out, st = run(b, G.rope_table(64, 64, device=DEV))
    assert st == G.ERR_INVALID_ARG and torch.equal(b.kc, old)


# ---- attention ---------------------------------------------------------------------------------------------------
def check_attention(b, rows=None, **kw):
    b.to_device()
    out = b.attend(**kw)
    assert G.griffin_check_device_status(b.ws) == G.OK
    want, mass = b.reference(rows)
    n = int(b.q_start[-1])
    got = f64(out)
    at = slice(0, n) if rows is None else sorted(rows)
    err = np.abs(got[at] - want[at])
    assert np.all(err <= b.bound(want, mass)[at]), (np.nanmax(err / b.bound(want, mass)[at]), np.argwhere(~(err <= b.bound(want, mass)[at]))[:5])
    assert np.all(got[n:] == 77.0), "rows behind the last sequence were written"
    again = b.attend(**kw)
    assert torch.equal(out, again), "the same call gave other bits"
    return out


HEADS = [(1, 1, 64), (8, 8, 128), (8, 2, 128), (6, 2, 80), (5, 1, 128), (4, 4, 256), (8, 1, 200), (64, 1, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", HEADS)
def test_attention_step_behind_a_shared_prefix(dtype, hq, hkv, hd):
    check_attention(Batch([1, 1, 1, 1], [1, 40, 129, 77], 300, hq, hkv, hd, 16, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd", [(2, 2, 64), (4, 1, 128), (3, 1, 80), (2, 1, 256)])
@pytest.mark.parametrize("n", [1, 7, 64, 128, 129, 300])
def test_attention_of_a_prompt(dtype, hq, hkv, hd, n):
    check_attention(Batch([n], [n], 0, hq, hkv, hd, 32, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix", [0, 1, 31, 32, 127, 128, 129, 1000])
def test_attention_prefix_lengths(dtype, prefix):
    check_attention(Batch([1, 2], [1, 33], prefix, 4, 2, 128, 32, dtype))
    check_attention(Batch([1], [5], prefix, 4, 2, 128, 32, dtype))               # one sequence walks the prefix itself


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [8, 16, 64, 128, 256])
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
def test_attention_pages(dtype, page, layout):
    check_attention(Batch([1, 3, 1], [200, 131, 3], 150, 4, 2, 128, page, dtype, layout=layout))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fill", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_attention_does_not_see_what_lies_behind_the_ends(dtype, fill):
    check_attention(Batch([1, 2, 1], [5, 70, 129], 37, 4, 2, 64, 64, dtype, fill=fill))
    check_attention(Batch([1, 2, 1], [5, 70, 129], 37, 2, 1, 256, 32, dtype, fill=fill))
    check_attention(Batch([200], [203], 0, 2, 1, 128, 64, dtype, fill=fill))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("which,value", [("k", float("nan")), ("v", float("nan")), ("k", float("inf")), ("v", -float("inf")), ("q", float("nan"))])
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("hq", [2, 10])
def test_attention_lets_a_seen_value_that_is_not_finite_through(dtype, which, value, hd, hq):
    # one bad entry in a key, a value or a query that is seen (also as the only thing seen): what the formula makes of it
    for prefix, own, at in [(0, 1, 0), (0, 9, 3), (40, 200, 197), (40, 200, 70), (40, 200, 2), (0, 300, 128)] + [(0, 64, i) for i in range(16, 32)]:
        b = Batch([1, 1], [own, 30], prefix, hq, 1, hd, 16, dtype, fill=0.0)
        q = b.q.clone()
        if which == "q":
            q[0, 1, 5] = value
        else:
            q[0, ::2, 5], q[0, 1::2, 5] = 1.5, -1.5         # an infinite key: logits of +inf and of -inf
            t = b.k_host if which == "k" else b.v_host
            t[int(b.page_table[0, at // 16]), 0, at % 16, 5] = value
        with np.errstate(all="ignore"):
            want, mass = L.attention(f64(q), f64(b.k_host), f64(b.v_host), b.q_start.numpy(), b.seq_len.numpy(), b.page_table.numpy(),
                                     b.prefix_pages.numpy(), b.prefix, b.scale)
            bound = b.bound(np.nan_to_num(want, posinf=0.0, neginf=0.0), np.nan_to_num(mass, posinf=0.0))
        if (which, value, prefix + own) == ("k", float("inf"), 1):
            want[0, 1::2] = 0.0                            # no logit above -inf counts as nothing seen
        b.to_device()
        got = f64(b.attend(q=q.to(DEV)))
        assert not np.all(np.isfinite(want))
        assert np.array_equal(np.isnan(want), np.isnan(got)), (prefix, own, at)
        assert np.array_equal(np.isinf(want), np.isinf(got)) and np.all(got[np.isinf(want)] == want[np.isinf(want)])
        fine = np.isfinite(want)
        assert np.all(np.abs(got[fine] - want[fine]) <= bound[fine])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
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
    check_attention(Batch(q_lens, seq_lens, prefix, 4, 2, 64, 16, dtype, extra_rows=2))
    check_attention(Batch(q_lens, seq_lens, prefix, 3, 1, 128, 16, dtype))


@pytest.mark.parametrize("hq,hkv,hd", [(2, 2, 64), (4, 2, 72), (8, 1, 128), (3, 1, 200), (2, 1, 256)])
@pytest.mark.parametrize("page,layout", [(8, "hnd"), (8, "nhd"), (16, "hnd"), (128, "nhd")])
def test_attention_of_a_few_rows(hq, hkv, hd, page, layout):
    # up to 8 rows a block (the kernel for single tokens), the bounds of that, and calls of more behind the same lengths
    group = hq // hkv
    most = 8 // group
    for q_lens, seq_lens, prefix in [([1], [1], 0), ([1], [700], 0), ([most], [333], 90), ([most + 1], [333], 90), ([most, 0], [130, 5], 0),
                                     ([most - most // 2, most // 2], [17, 129], 300), ([most, 1], [17, 129], 300), ([1, 1], [0, 3], 0),
                                     ([3 * most, 1, 1], [3 * most + 5, 40, 16], 0), ([most, 1], [most - 1, 64], 0)]:
        check_attention(Batch(q_lens, seq_lens, prefix, hq, hkv, hd, page, "bf16", layout=layout))


def test_attention_of_few_rows_and_many_blocks():
    # 296 blocks of sequences are the most that the kernel for single tokens takes
    for n in (74, 75):
        check_attention(Batch([1] * n, [(31 * i) % 190 for i in range(n)], 0, 8, 4, 64, 16, "bf16"), rows={0, 1, 7, n - 2, n - 1})
    check_attention(Batch([1] * 8, [(31 * i) % 190 + 1 for i in range(8)], 1100, 37, 37, 64, 16, "bf16"), rows={0, 7})
    check_attention(Batch([1] * 8, [(31 * i) % 190 + 1 for i in range(8)], 1100, 38, 38, 64, 16, "bf16"), rows={0, 7})


def test_attention_of_two_blocks_of_few_rows():
    # 9 to 16 rows of a sequence or of a short prefix, and sequences whose rows are unevenly many
    check_attention(Batch([4], [1500], 0, 8, 2, 128, 16, "bf16"))
    check_attention(Batch([13, 9, 2], [700, 9, 40], 0, 2, 2, 72, 32, "bf16"))
    check_attention(Batch([2, 2], [200, 5], 333, 8, 2, 128, 16, "bf16"))
    check_attention(Batch([1, 3, 0, 1], [20, 90, 4, 1], 1111, 3, 1, 256, 64, "bf16"))
    check_attention(Batch([17, 1], [16, 30], 0, 1, 1, 64, 8, "bf16"))


@pytest.mark.parametrize("fill", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_attention_of_more_rows_does_not_see_what_lies_behind_the_ends(fill):
    check_attention(Batch([4, 2, 3], [5, 70, 129], 37, 4, 2, 64, 64, "bf16", fill=fill))
    check_attention(Batch([4, 2, 3], [5, 70, 129], 37, 2, 1, 256, 32, "bf16", fill=fill))
    check_attention(Batch([9], [40], 37, 2, 2, 128, 16, "bf16", fill=fill))


def test_attention_of_many_sequences():
    b = Batch([1] * 1000, [(13 * i) % 37 for i in range(1000)], 64, 2, 1, 64, 8, "bf16")
    check_attention(b, rows={0, 1, 2, 500, 998, 999})


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_over_a_long_context(dtype):
    check_attention(Batch([1], [9000], 0, 4, 1, 128, 64, dtype))
    check_attention(Batch([1, 1], [37, 900], 7000, 4, 1, 128, 64, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_scale", [0.0, 12.0])
def test_attention_flat_and_sharp(dtype, q_scale):
    # equal logits; and logits that spread over hundreds, so that the running maximum moves by far more than a
    # tile's sum can hold
    check_attention(Batch([1, 4], [300, 700], 200, 4, 2, 128, 64, dtype, q_scale=q_scale))


def test_attention_strided_rows_and_in_place():
    b = Batch([2, 5], [9, 40], 17, 4, 2, 128, 64, "bf16")
    wide = torch.zeros(b.T, 4 * 128 + 24, dtype=b.dt, device=DEV)
    wide[:, :512] = b.q.flatten(1)
    out = torch.zeros(b.T, 4 * 128 + 8, dtype=b.dt, device=DEV)
    b.to_device()
    plain = b.attend()
    b.attend(q=wide[:, :512], out=out[:, :512])
    assert torch.equal(out[:, :512].reshape_as(plain), plain) and torch.all(out[:, 512:] == 0)
    q = b.q.to(DEV)
    b.attend(q=q, out=q)
    assert torch.equal(q, plain)


def test_attention_on_another_stream_and_in_a_graph():
    b = Batch([1, 1, 1], [60, 61, 200], 300, 8, 2, 128, 16, "bf16").to_device()
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
    # the lengths are read when the graph runs
    b.dev[1] -= 7
    b.seq_len -= 7
    graph.replay()
    torch.cuda.synchronize()
    want, mass = b.reference()
    assert np.all(np.abs(f64(out) - want) <= b.bound(want, mass))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_reports_bad_pages_and_lengths(dtype):
    b = Batch([1, 1], [20, 9], 0, 2, 1, 64, 8, dtype, fill=0.0)
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
    b = Batch([1, 1], [16, 9], 0, 2, 1, 64, 8, dtype, fill=0.0, table_extra=0).to_device()
    b.dev[1][0] = 17
    out = b.attend()
    assert G.griffin_check_device_status(b.ws) == G.ERR_INVALID_ARG and torch.isfinite(out).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cache_offsets_beyond_32_bits(dtype):
    # a cache of 2^31 entries and more in k and in v each, of which the call uses pages at its end
    hd, page, hkv = 128, 64, 8
    n_pages = (1 << 31) // (hd * page * hkv) + 40
    dt = DTYPES[dtype]
    kc = torch.empty(n_pages, hkv, page, hd, dtype=dt, device=DEV)
    vc = torch.empty(n_pages, hkv, page, hd, dtype=dt, device=DEV)
    b = Batch([1, 2], [70, 3], 100, 8, hkv, hd, page, dtype)
    first = n_pages - b.k_host.shape[0]
    kc[first:], vc[first:] = b.k_host.to(DEV), b.v_host.to(DEV)
    table, pre = (b.page_table + first).to(DEV), (b.prefix_pages + first).to(DEV)
    desc = G.make_attn_desc(8, hkv, hd, page, dtype)
    batch = G.make_attn_batch(b.q_start.to(DEV), b.seq_len.to(DEV), table, b.T, pre, b.prefix)
    ws, cache = G.alloc_attn_workspace(desc, b.T, 2, DEV), G.make_kv_cache(kc, vc)
    out = torch.zeros(b.T, 8, hd, dtype=dt, device=DEV)
    G.griffin_attn_prefix(desc, batch, cache, b.q.to(DEV), out, ws)
    want, mass = b.reference()
    assert np.all(np.abs(f64(out) - want) <= b.bound(want, mass))
    G.griffin_kv_append(desc, batch, cache, None, None, b.k.to(DEV), b.v.to(DEV), None, ws)
    for t, s, i in L.places(b.q_start.numpy(), b.seq_len.numpy()):
        at = int(b.page_table[s, i // page]) + first
        assert torch.equal(kc[at, :, i % page].cpu(), b.k[t]) and torch.equal(vc[at, :, i % page].cpu(), b.v[t])
    assert G.griffin_check_device_status(ws) == G.OK


def test_append_then_attend_is_one_causal_pass_over_the_tokens():
    # a prompt in one call and in three pieces: the same cache, and outputs within the roundings
    n, cuts = 200, (0, 70, 71, 200)
    b = Batch([n], [n], 0, 4, 2, 128, 16, "bf16", fill=0.0).to_device()
    rope = G.make_rope(G.rope_table(256, 128, device=DEV))
    q, k, v = b.q.to(DEV), b.k.to(DEV), b.v.to(DEV)
    q1 = torch.empty_like(q)
    G.griffin_kv_append(b.desc, b.batch, b.cache, rope, q, k, v, q1, b.ws)
    whole, kc = b.attend(q=q1), b.kc.clone()
    b.kc.zero_()
    parts = []
    for lo, hi in zip(cuts, cuts[1:]):
        batch = G.make_attn_batch(torch.tensor([0, hi - lo], dtype=torch.int32, device=DEV),
                                  torch.tensor([hi], dtype=torch.int32, device=DEV), b.dev[2], hi - lo)
        qp, out = torch.empty_like(q[lo:hi]), torch.empty_like(q[lo:hi])
        G.griffin_kv_append(b.desc, batch, b.cache, rope, q[lo:hi], k[lo:hi], v[lo:hi], qp, b.ws)
        G.griffin_attn_prefix(b.desc, batch, b.cache, qp, out, b.ws)
        parts.append(out)
    assert torch.equal(b.kc, kc)
    assert torch.allclose(torch.cat(parts).float(), whole.float(), atol=2.0 ** -7, rtol=2.0 ** -7)

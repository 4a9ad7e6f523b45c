"""The operators around the FF block at the edges of what their arguments may say: rows of no sequence, workspaces and
lengths at their limits, arrays out of order."""
import numpy as np
import pytest
import torch

from layer_util import Batch, f64
from oracle import layer_oracle as L
from paper_2404_01365_b200 import binding as G

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def behind(lead, q_lens, seq_lens, *args, **kw):
    """A batch whose first sequence's rows begin at `lead`: a slice of a larger batch's arrays."""
    b = Batch([lead] + q_lens, [0] + seq_lens, *args, **kw)
    b.q_start, b.seq_len, b.page_table = b.q_start[1:].clone(), b.seq_len[1:].clone(), b.page_table[1:].clone()
    return b


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lead,q_lens,seq_lens", [(4, [1, 1], [100, 50]), (1, [3], [40]), (3, [0, 2, 5], [30, 9, 5]),
                                                  (7, [2400], [2400]), (2400, [3, 1], [2500, 1])])
def test_append_leaves_rows_in_front_of_the_first_sequence_alone(dtype, lead, q_lens, seq_lens):
    b = behind(lead, q_lens, seq_lens, 21, 2, 1, 64, 16, dtype, extra_rows=2).to_device()
    table = G.rope_table(b.prefix + max(seq_lens) + 1, 64, device=DEV)
    q_out = torch.full((b.T, b.hq, b.hd), 33.0, dtype=b.dt, device=DEV)
    old_k, old_v = b.kc.clone(), b.vc.clone()
    G.griffin_kv_append(b.desc, b.batch, b.cache, G.make_rope(table), b.q.to(DEV), b.k.to(DEV), b.v.to(DEV), q_out, b.ws)
    assert G.griffin_check_device_status(b.ws) == G.OK
    n = int(b.q_start[-1])
    assert torch.all(q_out[:lead] == 33.0) and torch.all(q_out[n:] == 33.0), "rows of no sequence were written"
    want_k, want_v, want_q = L.kv_append(f64(old_k), f64(old_v), b.q_start.numpy(), b.seq_len.numpy(), b.page_table.numpy(), b.prefix,
                                         f64(b.q), f64(b.k), f64(b.v), f64(table))
    touched = np.zeros(want_k.shape[:1] + want_k.shape[2:3], bool)
    for t, s, i in L.places(b.q_start.numpy(), b.seq_len.numpy()):
        touched[b.page_table[s, i // b.page], i % b.page] = True
    at = np.broadcast_to(touched[:, None, :, None], want_k.shape)
    # one rounding of the storage type, and two products and a sum in 32 bits of values up to |x| + |y|
    ulp = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}[dtype]
    size = 2 * float(torch.cat((b.q.flatten(), b.k.flatten())).abs().max())
    near = lambda a, w: np.all(np.abs(a - w) <= ulp * np.abs(w) + 4 * 2.0 ** -24 * size)
    assert near(f64(b.kc)[at], want_k[at]) and np.array_equal(f64(b.vc)[at], want_v[at]) and near(f64(q_out)[lead:n], want_q[lead:n])
    for got, old in ((b.kc, old_k), (b.vc, old_v)):
        assert np.array_equal(f64(got)[~at], f64(old)[~at], equal_nan=True), "an entry that no token stands for was written"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lead,q_lens,seq_lens,prefix", [(4, [1, 1], [100, 50], 70), (1, [3], [40], 0), (200, [130, 2], [130, 9], 50),
                                                         (9, [300], [300], 0)])
def test_attention_leaves_rows_in_front_of_the_first_sequence_alone(dtype, lead, q_lens, seq_lens, prefix):
    b = behind(lead, q_lens, seq_lens, prefix, 4, 2, 64, 16, dtype, extra_rows=2)
    b.q[:lead] = float("nan")
    b.to_device()
    out = b.attend()
    assert G.griffin_check_device_status(b.ws) == G.OK
    n = int(b.q_start[-1])
    assert torch.all(out[:lead] == 77.0) and torch.all(out[n:] == 77.0), "rows of no sequence were written"
    b.q[:lead] = 0.0
    want, mass = b.reference()
    assert np.all(np.abs(f64(out) - want)[lead:n] <= b.bound(want, mass)[lead:n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_lens,seq_lens,prefix,hq,hkv,hd", [
    ([1, 1, 1], [100, 50, 7], 300, 16, 1, 128),      # more rows than the few-row kernel's blocks: partials of the prefix and of own keys
    ([5, 6, 5], [30, 6, 80], 333, 4, 4, 256),        # one accumulator
    ([3], [3000], 0, 8, 1, 64),                      # one sequence, its keys cut over the CTAs
    ([300], [300], 0, 2, 2, 72),
])
def test_attention_with_a_workspace_on_a_16_byte_boundary(dtype, q_lens, seq_lens, prefix, hq, hkv, hd):
    b = Batch(q_lens, seq_lens, prefix, hq, hkv, hd, 16, dtype).to_device()
    plain, n = b.attend(), b.ws.numel()
    room = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    assert room.data_ptr() % 32 == 0
    for at in (0, 16):
        b.ws = room[at:at + n]
        G.griffin_workspace_init(b.ws)
        assert torch.equal(b.attend(), plain) and G.griffin_check_device_status(b.ws) == G.OK
        assert torch.all(room[:at] == 0xA5) and torch.all(room[at + n:] == 0xA5), "written outside the workspace"
        room.fill_(0xA5)


@pytest.mark.parametrize("dtype,tokens,hkv,group,n_seq", [
    ("bf16", 1, 256, 1, 1),       # the few-row kernel, one sequence behind a prefix of 2^30 tokens (one page, again and again)
    ("bf16", 300, 128, 1, 1),     # two row blocks under every head, the second in one row tile
    ("bf16", 256, 256, 1, 1),     # one block of two row tiles
    ("bf16", 2, 256, 4, 2),       # a prefix that is read once for the batch
    ("f32", 1, 128, 1, 1),
    ("f32", 2, 128, 2, 2),
])
def test_attention_of_more_tiles_than_can_be_counted_is_not_run(dtype, tokens, hkv, group, n_seq):
    page, prefix, hd, dt = 1024, 1 << 30, 64, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    desc = G.make_attn_desc(hkv * group, hkv, hd, page, dtype)
    kc, vc = (torch.randn(1, hkv, page, hd, device=DEV, dtype=dt) for _ in range(2))
    pages = torch.zeros(prefix // page, dtype=torch.int32, device=DEV)
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device=DEV)
    starts, lens = ints(0, tokens) if n_seq == 1 else ints(0, 1, tokens), ints(*[0] * n_seq)
    q, out = (torch.full((tokens, hkv * group, hd), x, device=DEV, dtype=dt) for x in (0.1, 77.0))
    ws, cache = G.alloc_attn_workspace(desc, tokens, n_seq, DEV), G.make_kv_cache(kc, vc)
    table = torch.zeros(n_seq, 1, dtype=torch.int32, device=DEV)
    G.griffin_attn_prefix(desc, G.make_attn_batch(starts, lens, table, tokens, pages, prefix), cache, q, out, ws)
    assert G.griffin_check_device_status(ws) == G.ERR_INVALID_ARG
    assert torch.all(out == 77.0)
    # the workspace is fit for the next call
    G.griffin_workspace_init(ws)
    G.griffin_attn_prefix(desc, G.make_attn_batch(starts, lens, table, tokens, pages, page), cache, q, out, ws)
    assert G.griffin_check_device_status(ws) == G.OK
    # a query of equal entries: softmax of 0.1 scale times the keys' sums
    p = torch.softmax(q[0, 0, 0].double() * hd ** -0.5 * kc[0].double().sum(2), 1)
    want = (p[:, None] @ vc[0].double())[:, 0].repeat_interleave(group, 0)
    assert torch.all((out.double() - want[None]).abs() < (2.0 ** -7 if dtype == "bf16" else 2.0 ** -16))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_near_the_end_of_32_bits(dtype):
    # a table of 2^21 entries of one page, so that its row holds 2^31 tokens: place, position and tiles must not run over
    page, hkv, hd, n, dt = 1024, 64, 64, 1300, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    desc = G.make_attn_desc(hkv, hkv, hd, page, dtype)
    kc, vc = (torch.zeros(1, hkv, page, hd, device=DEV, dtype=dt) for _ in range(2))
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device=DEV)
    table, pre = torch.zeros(1, 1 << 21, dtype=torch.int32, device=DEV), torch.zeros(1 << 20, dtype=torch.int32, device=DEV)
    ws, cache = G.alloc_attn_workspace(desc, n, 1, DEV), G.make_kv_cache(kc, vc)
    q, out = (torch.full((n, hkv, hd), x, device=DEV, dtype=dt) for x in (0.1, 77.0))
    rope = G.make_rope(G.rope_table(64, 64, device=DEV))
    for length in (2 ** 31 - 1, 2 ** 30 + n, -2 ** 31):
        for prefix in (0, 1 << 30):
            batch = G.make_attn_batch(ints(0, n), ints(length), table, n, pre if prefix else None, prefix)
            q_out = torch.full_like(q, 33.0)
            G.griffin_kv_append(desc, batch, cache, rope, q, q, q, q_out, ws)
            assert G.griffin_check_device_status(ws) == (G.ERR_INVALID_ARG if length > 0 else G.OK)
            assert torch.all(q_out == 0) and not kc.any() and not vc.any()
            G.griffin_workspace_init(ws)
        if length > 0:      # cut to 2^30 tokens, and those are more tiles than can be counted
            G.griffin_attn_prefix(desc, G.make_attn_batch(ints(0, n), ints(length), table, n), cache, q, out, ws)
            assert G.griffin_check_device_status(ws) == G.ERR_INVALID_ARG and torch.all(out == 77.0)
            G.griffin_workspace_init(ws)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("starts", [(0, 300, 0, 10), (-5000, -3000, 0, 4), (0, 1000000, 5, 10), (290, 200, 100, 300), (5, -2 ** 31, 2 ** 31 - 1, 7)])
@pytest.mark.parametrize("prefix", [0, 100])
def test_rows_that_do_not_ascend_are_reported_and_stay_inside(dtype, starts, prefix):
    b = Batch([100, 100, 100], [120, 150, 100], prefix, 2, 2, 64, 16, dtype, fill=0.0).to_device()
    room = torch.full((b.T + 600, b.hq, b.hd), 77.0, dtype=b.dt, device=DEV)
    out = room[300:300 + b.T]
    good = b.attend()
    b.dev[0].copy_(torch.tensor(starts, dtype=torch.int32))
    b.attend(out=out)
    assert G.griffin_check_device_status(b.ws) == G.ERR_INVALID_ARG
    rope, qd = G.make_rope(G.rope_table(400, 64, device=DEV)), b.q.to(DEV)
    kc = b.kc.clone()
    G.griffin_kv_append(b.desc, b.batch, b.cache, rope, qd, b.k.to(DEV), b.v.to(DEV), out, b.ws)
    torch.cuda.synchronize()
    assert torch.all(room[:300] == 77.0) and torch.all(room[300 + b.T:] == 77.0), "written outside the output"
    b.kc.copy_(kc)
    b.vc.copy_(b.v_host.to(DEV) if b.layout == "hnd" else b.vc)
    b.dev[0].copy_(b.q_start)
    G.griffin_workspace_init(b.ws)
    assert torch.equal(b.attend(), good) and G.griffin_check_device_status(b.ws) == G.OK


@pytest.mark.parametrize("dtype,res", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("pre,post", [("rms", "none"), ("layer", "none"), ("none", "layer"), ("layer", "rms"), ("rms", "layer")])
@pytest.mark.parametrize("d", [320, 1360])
def test_norm_rows_that_are_not_finite(dtype, res, pre, post, d):
    # in the residual stream, the block's output or the gate: what the formula makes of them, and other rows as they were
    dts = {"f32": torch.float32, "bf16": torch.bfloat16}
    g = torch.Generator().manual_seed(d)
    rnd = lambda *s, t=dts[dtype], b=0.0: (torch.randn(*s, generator=g) + b).to(t)
    T, bad = 12, [float("nan"), float("inf"), -float("inf")]
    r, y, gate = rnd(T, d, t=dts[res]), rnd(T, d), rnd(T, d)
    for i, value in enumerate(bad):
        r[i, 5 + 40 * i], y[4 + i, 7 + 50 * i], gate[8 + i, 9 + 60 * i] = value, value, value
    w = [rnd(d, b=1.0) for _ in range(2)]
    b = [rnd(d) for _ in range(2)]
    up = lambda t: t.to(DEV)
    desc = G.make_norm_desc(d, dtype, res, pre, post, 1e-5, 0.0, 0.7, 1.3, "linear")
    weights = G.make_norm_weights(up(w[0]), up(b[0]), up(w[1]), up(b[1]))
    ro, h = torch.empty(T, d, dtype=dts[res], device=DEV), torch.empty(T, d, dtype=dts[dtype], device=DEV)
    G.griffin_norm_residual(desc, weights, up(r), ro, h, up(y), up(gate))
    with np.errstate(all="ignore"):
        want = L.norm_residual(f64(r), f64(y), f64(gate), pre, post, f64(w[0]), f64(b[0]), f64(w[1]), f64(b[1]), 1e-5, 0.0, 0.7, 1.3, "linear")
    ulp = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
    for got, ref, kind in ((f64(ro), want[0], res), (f64(h), want[1], dtype)):
        assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(np.isinf(got), np.isinf(ref))
        assert np.all(got[np.isinf(ref)] == ref[np.isinf(ref)]) and not np.all(np.isfinite(ref[[0, 1, 2, 4, 5, 6, 8, 9, 10]]))
        # one rounding, and fp32 arithmetic relative to the row's largest entry (as the tests of finite rows have it)
        fine = np.isfinite(ref)
        size = np.abs(np.where(fine, ref, 0.0)).max(1, keepdims=True) + 1.0
        err = np.abs(np.where(fine, got, 0.0) - np.where(fine, ref, 0.0))
        assert np.all(err <= ulp[kind] * np.abs(np.where(fine, ref, 0.0)) * 1.01 + 64 * 2.0 ** -24 * size)


@pytest.mark.parametrize("hq,hkv,hd", [(2, 1, 128), (2, 2, 256)])
@pytest.mark.parametrize("n,prefix", [(330, 0), (360, 150), (1024, 40)])
def test_attention_of_many_sequences_beside_a_smaller_ring(hq, hkv, hd, n, prefix):
    # the list of the sequences' first tiles takes the room of one of the ring's five tiles
    lens = [(17 * i) % 140 + 4 for i in range(n)]
    b = Batch([(i % 3) + 1 for i in range(n)], lens, prefix, hq, hkv, hd, 64, "bf16").to_device()
    out = b.attend()
    assert G.griffin_check_device_status(b.ws) == G.OK and torch.isfinite(out).all()
    rows = {0, 1, 2, 3, b.T // 2, b.T - 2, b.T - 1}
    want, mass = b.reference(rows)
    at = sorted(rows)
    assert np.all(np.abs(f64(out)[at] - want[at]) <= b.bound(want, mass)[at])
    assert torch.equal(b.attend(), out)

"""Refusals of the layer operators: every wrong argument is answered on the host, before any CUDA call."""
import ctypes as C

import pytest
import torch

from paper_2404_01365_b200 import binding as G, build

FAKE, ODD = C.c_void_p(0x10000), C.c_void_p(0x10004)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return G.load()


def test_norm_residual_refusals(lib):
    def call(T=2, y=FAKE, ld_y=64, gate=None, ld_gate=0, res=FAKE, ld_res=64, ro=FAKE, ld_ro=64, h=FAKE, ld_h=64,
             w=G.NormWeights(FAKE, None, FAKE, None), d=64, dtype="bf16", res_dtype="bf16", **kw):
        desc = G.make_norm_desc(d, dtype, res_dtype)
        for k, v in kw.items():
            setattr(desc, k, v)
        return lib.griffin_norm_residual(C.byref(desc), C.byref(w), T, y, ld_y, gate, ld_gate, res, ld_res, ro, ld_ro, h, ld_h, None)

    assert lib.griffin_norm_residual(None, None, 1, None, 0, None, 0, None, 0, None, 0, None, 0, None) == G.ERR_INVALID_ARG
    assert call(T=0) == call(T=-1) == call(res=None) == call(d=0) == call(eps=0.0) == call(eps=float("nan")) == G.ERR_INVALID_ARG
    assert call(d=60) == call(res=ODD) == call(y=ODD) == call(ld_y=65) == call(ld_h=68) == G.ERR_ALIGNMENT
    assert call(ld_y=56) == call(ld_res=0) == call(ld_ro=56) == call(ld_h=32) == call(gate=FAKE, ld_gate=56) == G.ERR_INVALID_ARG
    assert call(d=16392) == call(dtype="f32") == call(pre_norm=3) == call(post_norm=-1) == call(gate_act=3) == call(dtype=7) == G.ERR_UNSUPPORTED
    assert call(y=None, gate=FAKE) == call(h=None) == call(h=None, ro=None, pre_norm=0) == G.ERR_INVALID_ARG
    assert call(w=G.NormWeights()) == call(post_norm=1, w=G.NormWeights(FAKE)) == call(post_norm=1, y=None) == G.ERR_INVALID_ARG
    assert call(w=G.NormWeights(ODD)) == call(gate=ODD) == G.ERR_ALIGNMENT


def attn_args(hq=4, hkv=2, hd=64, page=16, dtype="bf16", scale=0.125, n_seq=2, T=3, prefix=0, pages=None, **kw):
    desc = G.make_attn_desc(hq, hkv, hd, page, dtype, scale)
    batch = G.AttnBatch(n_seq, T, FAKE, FAKE, FAKE, 4, prefix, pages)
    cache = G.KVCache(FAKE, FAKE, 8, 2 * 16 * 64, 16 * 64, 64)
    for k, v in kw.items():
        setattr(batch if hasattr(batch, k) else cache, k, v)
    return C.byref(desc), C.byref(batch), C.byref(cache)


BAD = [
    (dict(hq=5), G.ERR_INVALID_ARG), (dict(hq=0), G.ERR_INVALID_ARG), (dict(hkv=0, hq=4), G.ERR_INVALID_ARG),
    (dict(scale=0.0), G.ERR_INVALID_ARG), (dict(scale=-1.0), G.ERR_INVALID_ARG), (dict(scale=float("inf")), G.ERR_INVALID_ARG),
    (dict(scale=float("nan")), G.ERR_INVALID_ARG), (dict(dtype=2), G.ERR_UNSUPPORTED), (dict(hq=130), G.ERR_UNSUPPORTED),
    (dict(hd=56), G.ERR_UNSUPPORTED), (dict(hd=264), G.ERR_UNSUPPORTED), (dict(hd=68), G.ERR_ALIGNMENT),
    (dict(page=4), G.ERR_UNSUPPORTED), (dict(page=24), G.ERR_UNSUPPORTED), (dict(page=2048), G.ERR_UNSUPPORTED),
    (dict(n_seq=0), G.ERR_INVALID_ARG), (dict(T=-1), G.ERR_INVALID_ARG), (dict(prefix=-1), G.ERR_INVALID_ARG),
    (dict(prefix=5), G.ERR_INVALID_ARG), (dict(n_seq=1025), G.ERR_UNSUPPORTED), (dict(q_start=None), G.ERR_INVALID_ARG),
    (dict(seq_len=None), G.ERR_INVALID_ARG), (dict(page_table=None), G.ERR_INVALID_ARG), (dict(table_stride=-1), G.ERR_INVALID_ARG),
    (dict(q_start=C.c_void_p(0x10002)), G.ERR_ALIGNMENT), (dict(k=None), G.ERR_INVALID_ARG), (dict(v=ODD), G.ERR_ALIGNMENT),
    (dict(n_pages=0), G.ERR_INVALID_ARG), (dict(stride_page=2 * 16 * 64 + 4), G.ERR_ALIGNMENT), (dict(stride_head=-64), G.ERR_INVALID_ARG),
    (dict(stride_token=56), G.ERR_INVALID_ARG),
]


@pytest.mark.parametrize("kw,want", BAD, ids=[str(k) for k, _ in BAD])
def test_cache_operators_refuse_the_same_descriptions(lib, kw, want):
    a = attn_args(**kw)
    big = 1 << 40
    assert lib.griffin_kv_append(*a, None, FAKE, 9000, FAKE, 9000, FAKE, 9000, FAKE, 9000, FAKE, None) == want
    assert lib.griffin_attn_prefix(*a, FAKE, 9000, FAKE, 9000, FAKE, big, None) == want


def test_kv_append_refusals(lib):
    a = attn_args()

    def call(rope=None, q=FAKE, ld_q=256, k=FAKE, ld_k=128, v=FAKE, ld_v=128, qo=FAKE, ld_o=256, ws=None, args=a):
        return lib.griffin_kv_append(*args, None if rope is None else C.byref(rope), q, ld_q, k, ld_k, v, ld_v, qo, ld_o, ws, None)

    assert call(k=None) == call(v=None) == call(qo=None) == call(q=None) == call(ld_q=248) == call(ld_k=120) == G.ERR_INVALID_ARG
    assert call(k=ODD) == call(ld_v=132) == call(qo=ODD) == call(ws=ODD) == G.ERR_ALIGNMENT
    assert call(G.Rope(None, 8, 32, 0)) == call(G.Rope(FAKE, 0, 32, 0)) == call(G.Rope(FAKE, 8, 80, 0)) == call(G.Rope(FAKE, 8, 8, 0)) == G.ERR_INVALID_ARG
    assert call(G.Rope(FAKE, 8, 40, 0)) == call(G.Rope(ODD, 8, 32, 0)) == G.ERR_ALIGNMENT
    assert call(G.Rope(FAKE, 8, 32, 2)) == G.ERR_UNSUPPORTED
    assert call(args=attn_args(T=0)) == G.OK                      # no tokens: nothing to do


def test_attn_prefix_refusals_and_workspace(lib):
    desc = G.make_attn_desc(4, 2, 64, 16, "bf16")
    need = G.griffin_attn_workspace_bytes(desc, 3, 2)
    assert need > 256 and G.griffin_attn_workspace_bytes(desc, 3, 3) >= need and G.griffin_attn_workspace_bytes(desc, 4000, 2) >= need
    assert G.griffin_attn_workspace_bytes(G.make_attn_desc(5, 2, 64, 16, "bf16"), 3, 2) == 0
    assert G.griffin_attn_workspace_bytes(desc, -1, 2) == G.griffin_attn_workspace_bytes(desc, 3, 0) == 0

    def call(q=FAKE, ld_q=256, out=FAKE, ld_o=256, ws=FAKE, n=need, args=attn_args()):
        return lib.griffin_attn_prefix(*args, q, ld_q, out, ld_o, ws, n, None)

    assert call(q=None) == call(out=None) == call(ld_q=248) == call(ld_o=0) == G.ERR_INVALID_ARG
    assert call(q=ODD) == call(ld_o=260) == call(ws=ODD) == G.ERR_ALIGNMENT
    assert call(ws=None) == call(n=need - 1) == call(n=0) == G.ERR_WORKSPACE
    assert call(args=attn_args(T=0)) == G.OK


def test_workspace_grows_with_both_counts(lib):
    for shape in ((32, 8, 128, 64, "bf16"), (16, 16, 256, 16, "bf16"), (6, 2, 80, 8, "f32")):
        desc = G.make_attn_desc(*shape)
        sizes = [[G.griffin_attn_workspace_bytes(desc, t, n) for n in (1, 2, 31, 64, 1024)] for t in (0, 1, 64, 1000, 8192)]
        for row in sizes:
            assert row == sorted(row)
        for col in zip(*sizes):
            assert list(col) == sorted(col)


def test_binding_checks_tensors():
    desc = G.make_attn_desc(4, 2, 64, 16, "bf16")
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    assert G._rows(q, 3, 4, 64, desc.dtype, "q") == 256 and G._rows(q.flatten(1), 3, 4, 64, desc.dtype, "q") == 256
    for bad in (q.float(), q[:2], q.transpose(1, 2), q[:, :3], torch.zeros(3, 8, 64, dtype=torch.bfloat16)[:, ::2]):
        with pytest.raises(ValueError):
            G._rows(bad, 3, 4, 64, desc.dtype, "q")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    with pytest.raises(ValueError):
        G.make_attn_batch(i32(3), i32(2).long(), i32(2, 4), 3)
    with pytest.raises(ValueError):
        G.make_attn_batch(i32(2), i32(2), i32(2, 4), 3)
    with pytest.raises(ValueError):
        G.make_attn_batch(i32(3), i32(2), i32(2, 8)[:, :4], 3)
    with pytest.raises(ValueError):
        G.make_kv_cache(torch.zeros(4, 2, 16, 64), torch.zeros(4, 2, 16, 64).half())
    with pytest.raises(ValueError):
        G.make_rope(torch.zeros(4, 32, dtype=torch.float64))
    t = G.rope_table(5, 4, 100.0)
    assert t.shape == (5, 4) and torch.allclose(t[3], torch.tensor([3.0, 0.3, 3.0, 0.3], dtype=torch.float64).float().cos()
                                                * torch.tensor([1., 1, 0, 0]) + torch.tensor([3.0, 0.3, 3.0, 0.3]).sin() * torch.tensor([0., 0, 1, 1]))

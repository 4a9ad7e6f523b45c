"""The format of the cache in 4 bits on the CPU: the oracle's rules against their definitions, the tests' own arrays against
the oracle, and the calls' refusals."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import q4_util as Q
from oracle import layer_oracle as L
from paper_2404_01365_b200 import binding as G, build
from test_layer_abi import BAD, FAKE, ODD, attn_args


def test_scale_is_the_nearest_of_four_bits():
    grid = sorted((8 + m) / 8 * 2.0 ** e for e in range(-21, 11) for m in range(8))[:-1]     # (the last byte is NaN's)
    assert grid[0] == 2.0 ** -21 and grid[-1] == 1792.0
    rng = np.random.default_rng(0)
    for a in np.concatenate((2.0 ** rng.uniform(-20, 13, 500), [0.0, 1e-9, 7.0, 7 * 1.0625, 7 * 1.1875, 12544.0, 1e30])):
        s = L.q4_scale([a] + [0.0] * 15)
        assert s in grid and abs(s - a / 7) == min(abs(g - a / 7) for g in grid)
    assert L.q4_scale([7 * 1.0625] + [0.0] * 15) == 1.0 and L.q4_scale([-7 * 1.1875] + [0.0] * 15) == 1.25    # ties to even
    assert math.isnan(L.q4_scale([math.inf] + [1.0] * 15)) and math.isnan(L.q4_scale([1.0] * 15 + [math.nan]))


def test_no_entry_is_off_by_more_than_half_a_scale():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((400, 16)) * 2.0 ** rng.uniform(-15, 10, (400, 1))
    s = np.array([L.q4_scale(g) for g in x])
    held = L.q4_held(x)
    assert np.all(np.abs(held - x) <= s[:, None] / 2)
    assert np.array_equal(held, held.astype(np.float32)) and torch.equal(torch.from_numpy(held), torch.from_numpy(held).bfloat16().double())
    assert np.array_equal(L.q4_held(held), held) or np.all(np.abs(L.q4_held(held) - held) <= s[:, None])   # near its own grid
    assert np.all(L.q4_held(np.zeros((2, 32))) == 0)
    assert np.array_equal(L.q4_held(np.full((1, 16), 1e6)), np.full((1, 16), 12544.0))
    bad = x[:2].copy()
    bad[0, 3] = np.nan
    assert np.isnan(L.q4_held(bad)[0]).all() and np.isfinite(L.q4_held(bad)[1]).all()


@pytest.mark.parametrize("page,d", [(8, 64), (16, 80), (8, 128), (8, 208), (8, 256)])
def test_pages(page, d):
    rng = np.random.default_rng(d)
    x = (rng.standard_normal((page, d)) * 2.0 ** rng.uniform(-25, 12, (page, 1))).astype(np.float32)
    x[1, 5], x[2] = np.inf, 0
    block = L.q4_pack(x)
    assert block.shape == (Q.block_bytes(page, d),) and Q.block_bytes(page, d) % 16 == 0
    assert np.array_equal(L.q4_unpack(block, page, d), L.q4_held(x), equal_nan=True)
    c, b = Q.quantise(x)
    assert np.array_equal(Q.pack(c, b), block) and np.array_equal(Q.values(c, b), L.q4_held(x), equal_nan=True)
    desc = G.make_attn_desc(2, 2, d, page, "bf16")
    build.build()
    assert G.griffin_kv_q4_block_bytes(desc) == block.size


def q4(args, **kw):
    """The arguments of the calls over a cache in the storage type, for one in 4 bits."""
    old = args[2]._obj
    c = G.KVCacheQ4(old.k, old.v, old.n_pages, old.stride_page, old.stride_head)
    for k, v in kw.items():
        setattr(c, k, v)
    return args[0], args[1], C.byref(c)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return G.load()


def calls(lib, a):
    yield lib.griffin_kv_append_q4(*a, None, FAKE, 9000, FAKE, 9000, FAKE, 9000, FAKE, 9000, FAKE, None)
    yield lib.griffin_kv_read_q4(*a, FAKE, 9000, FAKE, 9000, FAKE, None)
    yield lib.griffin_attn_prefix_q4(*a, FAKE, 9000, FAKE, 9000, FAKE, 1 << 40, None)


@pytest.mark.parametrize("kw,want", [c for c in BAD if not set(c[0]) & {"stride_token", "stride_page", "stride_head"}],
                         ids=[str(k) for k, w in BAD if not set(k) & {"stride_token", "stride_page", "stride_head"}])
def test_the_same_descriptions_are_refused(lib, kw, want):
    assert list(calls(lib, q4(attn_args(**kw)))) == [want] * 3


@pytest.mark.parametrize("kw,want", [(dict(hd=72), G.ERR_UNSUPPORTED), (dict(hd=136), G.ERR_UNSUPPORTED)])
def test_heads_that_groups_do_not_fill_are_refused(lib, kw, want):
    assert list(calls(lib, q4(attn_args(**kw)))) == [want] * 3
    assert G.griffin_kv_q4_block_bytes(G.make_attn_desc(4, 2, kw["hd"], 16, "bf16")) == 0
    with pytest.raises(G.GriffinError):
        G.alloc_kv_cache_q4(G.make_attn_desc(4, 2, kw["hd"], 16, "bf16"), 3, "cpu")


@pytest.mark.parametrize("kw,want", [(dict(stride_page=-16), G.ERR_INVALID_ARG), (dict(stride_head=-16), G.ERR_INVALID_ARG),
                                     (dict(stride_page=8), G.ERR_ALIGNMENT), (dict(stride_head=24), G.ERR_ALIGNMENT),
                                     (dict(k=ODD), G.ERR_ALIGNMENT), (dict(v=None), G.ERR_INVALID_ARG)])
def test_caches_that_are_refused(lib, kw, want):
    assert list(calls(lib, q4(attn_args(), **kw))) == [want] * 3


def test_other_refusals(lib):
    a = q4(attn_args())

    def append(rope=None, q=FAKE, ld_q=256, k=FAKE, ld_k=128, v=FAKE, ld_v=128, qo=FAKE, ld_o=256, ws=None, args=a):
        return lib.griffin_kv_append_q4(*args, None if rope is None else C.byref(rope), q, ld_q, k, ld_k, v, ld_v, qo, ld_o, ws, None)

    def read(k=FAKE, ld_k=128, v=FAKE, ld_v=128, ws=None, args=a):
        return lib.griffin_kv_read_q4(*args, k, ld_k, v, ld_v, ws, None)

    need = G.griffin_attn_workspace_bytes(G.make_attn_desc(4, 2, 64, 16, "bf16"), 3, 2)

    def attn(q=FAKE, ld_q=256, out=FAKE, ld_o=256, ws=FAKE, n=need, args=a):
        return lib.griffin_attn_prefix_q4(*args, q, ld_q, out, ld_o, ws, n, None)

    assert append(k=None) == append(v=None) == append(qo=None) == append(q=None) == append(ld_q=248) == append(ld_k=120) == G.ERR_INVALID_ARG
    assert append(k=ODD) == append(ld_v=132) == append(qo=ODD) == append(ws=ODD) == G.ERR_ALIGNMENT
    assert append(G.Rope(None, 8, 32, 0)) == append(G.Rope(FAKE, 0, 32, 0)) == append(G.Rope(FAKE, 8, 80, 0)) == G.ERR_INVALID_ARG
    assert append(G.Rope(FAKE, 8, 40, 0)) == append(G.Rope(ODD, 8, 32, 0)) == G.ERR_ALIGNMENT
    assert append(G.Rope(FAKE, 8, 32, 2)) == G.ERR_UNSUPPORTED
    assert read(k=None) == read(v=None) == read(ld_k=120) == read(ld_v=0) == G.ERR_INVALID_ARG
    assert read(k=ODD) == read(ld_v=132) == read(ws=ODD) == G.ERR_ALIGNMENT
    assert attn(q=None) == attn(out=None) == attn(ld_q=248) == attn(ld_o=0) == G.ERR_INVALID_ARG
    assert attn(q=ODD) == attn(ld_o=260) == attn(ws=ODD) == G.ERR_ALIGNMENT
    assert attn(ws=None) == attn(n=need - 1) == attn(n=0) == G.ERR_WORKSPACE
    none = q4(attn_args(T=0))
    assert append(args=none) == read(args=none) == attn(args=none) == G.OK
    assert lib.griffin_kv_append_q4(a[0], a[1], None, None, *([FAKE, 256] * 4), None, None) == G.ERR_INVALID_ARG
    assert lib.griffin_kv_q4_block_bytes(None) == 0


def test_the_binding_checks_tensors(monkeypatch):
    def reached():
        raise RuntimeError("not refused")
    monkeypatch.setattr(G, "load", reached)
    BF = torch.bfloat16
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    desc = G.make_attn_desc(4, 2, 64, 16, "bf16")
    n = 16 * 36

    def run(which, cache=None, prefix=0, pages=None, q=torch.zeros(3, 4, 64, dtype=BF), k=torch.zeros(3, 2, 64, dtype=BF)):
        batch = G.make_attn_batch(i32(3), i32(2), i32(2, 4), 3, None if pages is None else i32(pages), prefix)
        cache = G.make_kv_cache_q4(*(u8(8, 2, n) if cache is None else cache() for _ in range(2)))
        if which == "append":
            G.griffin_kv_append_q4(desc, batch, cache, None, q, k, k, torch.zeros_like(q))
        elif which == "read":
            G.griffin_kv_read_q4(desc, batch, cache, k, torch.zeros_like(k))
        else:
            G.griffin_attn_prefix_q4(desc, batch, cache, q, torch.zeros_like(q), u8(64))

    for which in ("append", "read", "attn"):
        for kw in (dict(), dict(prefix=32, pages=2), dict(cache=lambda: u8(8, 3, 2 * n)[:, :2, :n])):
            with pytest.raises(RuntimeError, match="not refused"):
                run(which, **kw)
        for kw in (dict(cache=lambda: u8(8, 2, n - 16)), dict(cache=lambda: u8(8, 4, n)), dict(cache=lambda: u8(8, 2 * n)),
                   dict(cache=lambda: torch.zeros(8, 2, n)), dict(cache=lambda: u8(8, 2, 2 * n)[..., ::2]), dict(prefix=33, pages=2)):
            with pytest.raises(ValueError):
                run(which, **kw)
    for which in ("append", "read"):
        with pytest.raises(ValueError):
            run(which, k=torch.zeros(3, 2, 64))
    for which in ("append", "attn"):
        with pytest.raises(ValueError):
            run(which, q=torch.zeros(2, 4, 64, dtype=BF))
    with pytest.raises(ValueError):
        G.make_kv_cache_q4(u8(8, 2, n), u8(9, 2, n))


def test_calls_without_tokens_do_nothing(lib):
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    desc = G.make_attn_desc(4, 2, 64, 16, "bf16")
    batch, cache = G.make_attn_batch(i32(3), i32(2), i32(2, 4), 0), G.alloc_kv_cache_q4(desc, 8, "cpu")
    q, k, ws = torch.zeros(0, 4, 64, dtype=torch.bfloat16), torch.zeros(0, 2, 64, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.uint8)
    G.griffin_kv_append_q4(desc, batch, cache, None, q, k, k, q, ws)
    G.griffin_kv_read_q4(desc, batch, cache, k, k, ws)
    G.griffin_attn_prefix_q4(desc, batch, cache, q, q, ws)

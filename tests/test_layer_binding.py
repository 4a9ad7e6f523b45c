"""What the Python calls of the layer operators refuse by themselves: tensors that the C ABI gets as bare pointers."""
import pytest
import torch

from paper_2404_01365_b200 import binding as G

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def no_calls(monkeypatch):
    """A call that is not refused would reach the library with the host's pointers: it ends here instead."""
    def reached():
        raise RuntimeError("not refused")
    monkeypatch.setattr(G, "load", reached)


def norm(w, d=64, dtype="bf16", res="f32"):
    dt = {"bf16": BF, "f32": F32}
    r = torch.zeros(3, d, dtype=dt[res])
    G.griffin_norm_residual(G.make_norm_desc(d, dtype, res, post="rms"), w(), r, r, torch.zeros(3, d, dtype=dt[dtype]),
                            torch.zeros(3, d, dtype=dt[dtype]))


def test_norm_weights_are_the_descriptors():
    v = lambda n=64, dt=BF: torch.ones(n, dtype=dt)
    with pytest.raises(RuntimeError, match="not refused"):
        norm(lambda: G.make_norm_weights(v(), None, v(), v()))
    with pytest.raises(RuntimeError, match="not refused"):
        norm(lambda: G.make_norm_weights(v(dt=F32), v(dt=F32), v(dt=F32)), dtype="f32")
    for bad in (lambda: G.make_norm_weights(v(dt=F32), None, v(dt=F32)),             # fp32 weights beside bf16 rows
                lambda: G.make_norm_weights(v(), None, v(dt=F32)),
                lambda: G.make_norm_weights(v(32), None, v(32)),                     # too short
                lambda: G.make_norm_weights(v(), v(32), v()),
                lambda: G.make_norm_weights(v(128), None, v(128)),
                lambda: G.make_norm_weights(v(128)[::2], None, v()),                 # every other entry
                lambda: G.make_norm_weights(v()[None], None, v()[None])):
        with pytest.raises(ValueError):
            norm(bad)
    with pytest.raises(ValueError):
        norm(lambda: G.make_norm_weights(v(), None, v()), dtype="f32")               # bf16 weights beside fp32 rows


def cache_call(which, cache_shape=(8, 2, 16, 64), cache_dtype=BF, prefix=0, pages=None, view=None):
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    desc = G.make_attn_desc(4, 2, 64, 16, "bf16")
    batch = G.make_attn_batch(i32(3), i32(2), i32(2, 4), 3, None if pages is None else i32(pages), prefix)
    mk = lambda: torch.zeros(*cache_shape, dtype=cache_dtype)
    cache = G.make_kv_cache(*(mk() if view is None else view(mk()) for _ in range(2)))
    q, k = torch.zeros(3, 4, 64, dtype=BF), torch.zeros(3, 2, 64, dtype=BF)
    if which == "append":
        G.griffin_kv_append(desc, batch, cache, None, q, k, k, q)
    else:
        G.griffin_attn_prefix(desc, batch, cache, q, torch.zeros_like(q), torch.zeros(1 << 16, dtype=torch.uint8))


@pytest.mark.parametrize("which", ["append", "attention"])
def test_the_cache_is_the_descriptors(which):
    for kw in (dict(), dict(prefix=32, pages=2), dict(prefix=17, pages=2), dict(cache_shape=(8, 16, 2, 64), view=lambda t: t.transpose(1, 2))):
        with pytest.raises(RuntimeError, match="not refused"):
            cache_call(which, **kw)
    for kw in (dict(cache_dtype=F32), dict(cache_shape=(8, 1, 16, 64)), dict(cache_shape=(8, 4, 16, 64)), dict(cache_shape=(8, 2, 8, 64)),
               dict(cache_shape=(8, 2, 32, 64)), dict(cache_shape=(8, 2, 16, 128)), dict(cache_shape=(8, 16, 2, 64)),
               dict(prefix=33, pages=2), dict(prefix=1, pages=0)):
        with pytest.raises(ValueError):
            cache_call(which, **kw)


@pytest.mark.parametrize("which", ["append", "attention"])
def test_structures_made_by_hand_are_left_to_the_abi(which):
    # (their pointers say nothing about what is behind them)
    c = G.KVCache(0x10000, 0x10000, 8, 2 * 16 * 64, 16 * 64, 64)
    b = G.AttnBatch(2, 3, 0x10000, 0x10000, 0x10000, 4, 5, 0x10000)
    q, k = torch.zeros(3, 4, 64, dtype=BF), torch.zeros(3, 2, 64, dtype=BF)
    desc = G.make_attn_desc(4, 2, 64, 16, "bf16")
    with pytest.raises(RuntimeError, match="not refused"):
        if which == "append":
            G.griffin_kv_append(desc, b, c, None, q, k, k, q)
        else:
            G.griffin_attn_prefix(desc, b, c, q, q, torch.zeros(8, dtype=torch.uint8))

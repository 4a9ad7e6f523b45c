"""The small decoder over a cache in 4 bits, end to end against float64.

The float64 model attends over the keys and values that the device's cache holds (which are checked by themselves: each is
within half a scale, and the calls' roundings, of what the model computes), and is given the tokens that the device chose and its
expert sets.  Everything else it computes from the formulas, without pages, prefixes or caches."""
import numpy as np
import pytest
import torch

from oracle import griffin_oracle as O, layer_oracle as L
from paper_2404_01365_b200 import binding as G
from paper_2404_01365_b200.decoder import Decoder, DecoderConfig, random_weights
from layer_util import f64
from test_gpu_decoder import Model64, rel

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Model64Held(Model64):
    def run_held(self, tokens, first, feed_forward, held, slack):
        """Logits from position `first` on; held: per layer (k, v) of every position.  slack: how far, relative to the largest
        entry, a key or value of the device may be off before it is quantised."""
        c, n = self.cfg, len(tokens)
        nq, nk = c.n_q_heads, c.n_kv_heads
        r = self.w["embed"][tokens]
        rms = lambda x, g: np.array([L.norm(row, "rms", g, eps=c.eps) for row in x])
        for i, l in enumerate(self.layers):
            qkv = (rms(r, l["norm_attn"]) @ l["w_qkv"].T).reshape(n, nq + 2 * nk, c.head_dim)
            turned = np.array([[L.rotate(x, self.cos[t], self.sin[t], "half") for x in qkv[t, :nq + nk]] for t in range(n)])
            k, v = held[i]
            for got, want in ((k, turned[:, nq:]), (v, qkv[:, nq + nk:])):
                a = np.abs(want).reshape(n, nk, -1, 16).max(-1)
                off = np.abs(got - want).reshape(n, nk, -1, 16).max(-1)
                # half a scale, which is at most a / 7 and its rounding by 1/16; the largest entry's own error moves the scale, too
                assert np.all(off <= a / 14 * (1 + 1 / 16) + 2 * slack * np.abs(want).max())
            o = np.zeros((n, nq, c.head_dim))
            for t in range(n):
                for h in range(nq):
                    g = h // (nq // nk)
                    x = k[:t + 1, g] @ turned[t, h] * c.head_dim ** -0.5
                    p = np.exp(x - x.max())
                    o[t, h] = p / p.sum() @ v[:t + 1, g]
            r = r + o.reshape(n, -1) @ l["w_o"].T
            r = r + feed_forward(i, rms(r, l["norm_ff"]))
        return (rms(r, self.w["norm_out"]) @ self.w["head"].T)[first:]


# The bounds are those of the decoder over a cache in the storage type: what is given to the model is exact, and the other roundings are
# the same.
@pytest.mark.parametrize("dtype,tol,slack", [("f32", 1e-4, 1e-4), ("bf16", 2.0 ** -5, 2.0 ** -5)])
@pytest.mark.parametrize("act,hq,hkv,hd,page,P", [("swiglu", 4, 2, 64, 16, 37), ("relu", 2, 2, 80, 8, 64), ("geglu_tanh", 4, 1, 128, 32, 5)])
def test_prompt_and_continuations(dtype, tol, slack, act, hq, hkv, hd, page, P):
    cfg = DecoderConfig(vocab=96, d=256, n_layers=2, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, d_ff=512, act=act, dtype=dtype,
                        page_size=page, cache="q4")
    n_seq, steps = 3, 5
    host = random_weights(cfg, seed=3)
    up = lambda t: None if t is None else t.to(DEV)
    weights = {k: [{a: up(b) for a, b in l.items()} for l in v] if k == "layers" else up(v) for k, v in host.items()}
    dec = Decoder(cfg, weights, 64, n_seq, 8, keep=0.5, device=DEV)
    model = Model64Held(cfg, host, 72)
    prompt = torch.randint(0, cfg.vocab, (P,), generator=torch.Generator().manual_seed(5))

    logits = dec.prompt(prompt.to(DEV))
    chosen = [logits.topk(n_seq).indices]
    got = []
    for _ in range(steps):
        got.append(dec.step(chosen[-1]))
        chosen.append(got[-1].argmax(1))
    assert dec.status() == G.OK
    held = [dec.held(i) for i in range(cfg.n_layers)]
    assert held[0][0][0].shape == (P, hkv, hd) and held[0][1][0].shape == (n_seq, steps, hkv, hd)

    want = model.run_held(prompt.numpy(), P - 1, model.full, [tuple(f64(x) for x in h[0]) for h in held], slack)
    assert rel(f64(logits), want[0]) < tol
    sets = [O.compact_experts(dec.experts[i].cpu().numpy(), l["w_gate"], l["w_up"], l["w_down"]) for i, l in enumerate(model.layers)]

    def pruned(i, h):   # the prompt's rows went through the full block
        return np.concatenate((model.full(i, h[:P]), np.array([O.ff_pruned(x, sets[i], act) for x in h[P:]])))
    for s in range(n_seq):
        own = [int(c[s]) for c in chosen[:steps]]
        kv = [tuple(np.concatenate((f64(pre), f64(mine[s]))) for pre, mine in zip(*h)) for h in held]
        want = model.run_held(np.concatenate((prompt.numpy(), own)), P, pruned, kv, slack)
        for t in range(steps):
            assert rel(f64(got[t][s]), want[t]) < tol, (s, t)

    # back to the prompt's end: the same tokens give the same bits
    dec.restart()
    for t in range(steps):
        assert torch.equal(dec.step(chosen[t]), got[t])


def test_refusals():
    cfg = DecoderConfig(vocab=32, d=64, n_layers=1, n_q_heads=1, n_kv_heads=1, head_dim=64, d_ff=64, dtype="f32", page_size=8)
    w = random_weights(cfg, device=DEV)
    with pytest.raises(ValueError):
        Decoder(cfg, w, 8, 2, 2, device=DEV).held(0)
    cfg.cache = "int3"
    with pytest.raises(ValueError):
        Decoder(cfg, w, 8, 2, 2, device=DEV)
    cfg.cache, cfg.head_dim, cfg.n_q_heads = "q4", 72, 1
    with pytest.raises(G.GriffinError):
        Decoder(cfg, random_weights(cfg, device=DEV), 8, 2, 2, device=DEV)
    cfg = DecoderConfig(vocab=32, d=64, n_layers=1, n_q_heads=1, n_kv_heads=1, head_dim=64, d_ff=64, dtype="f32", page_size=8, cache="q4")
    dec = Decoder(cfg, w, 8, 2, 2, device=DEV)
    dec.prompt(torch.zeros(8, dtype=torch.long, device=DEV))
    (pre, _), (own, _) = dec.held(0)
    assert pre.shape == (8, 1, 64) and own.shape == (2, 0, 1, 64)

"""The small decoder end to end against float64: prompt, expert selection, continuations over the shared prompt.

The float64 model is written without pages, prefixes or caches: every position's whole row of keys, straight from the
formulas.  It is given the tokens that the device chose and, behind the prompt, the device's expert sets (the selection is
checked by itself)."""
import numpy as np
import pytest
import torch

from oracle import griffin_oracle as O, layer_oracle as L
from paper_2404_01365_b200 import binding as G
from paper_2404_01365_b200.decoder import Decoder, DecoderConfig, random_weights
from gpu_util import check_expert_set
from layer_util import f64

DEV = "cuda:0"


class Model64:
    def __init__(self, cfg, weights, n_pos):
        self.cfg = cfg
        self.w = {k: f64(v) for k, v in weights.items() if k != "layers"}
        self.layers = [{k: f64(v) for k, v in l.items()} for l in weights["layers"]]
        t = G.rope_table(n_pos, cfg.head_dim, cfg.theta).double().numpy()
        self.cos, self.sin = t[:, :cfg.head_dim // 2], t[:, cfg.head_dim // 2:]

    def run(self, tokens, first, feed_forward):
        """Logits of the positions from `first` on, and what each layer's FF is given there."""
        c, n = self.cfg, len(tokens)
        nq, nk = c.n_q_heads, c.n_kv_heads
        r, seen = self.w["embed"][tokens], []
        rms = lambda x, g: np.array([L.norm(row, "rms", g, eps=c.eps) for row in x])
        for i, l in enumerate(self.layers):
            qkv = (rms(r, l["norm_attn"]) @ l["w_qkv"].T).reshape(n, nq + 2 * nk, c.head_dim)
            turned = np.array([[L.rotate(x, self.cos[t], self.sin[t], "half") for x in qkv[t, :nq + nk]] for t in range(n)])
            o = np.zeros((n, nq, c.head_dim))
            for t in range(n):
                for h in range(nq):
                    g = h // (nq // nk)
                    x = turned[:t + 1, nq + g] @ turned[t, h] * c.head_dim ** -0.5
                    p = np.exp(x - x.max())
                    o[t, h] = p / p.sum() @ qkv[:t + 1, nq + nk + g]
            r = r + o.reshape(n, -1) @ l["w_o"].T
            h = rms(r, l["norm_ff"])
            seen.append(h)
            r = r + feed_forward(i, h)
        return (rms(r, self.w["norm_out"]) @ self.w["head"].T)[first:], seen

    def full(self, i, h):
        l = self.layers[i]
        return O.ff_dense(h, l["w_gate"], l["w_up"], l["w_down"], self.cfg.act)[0]


def rel(a, b):
    return np.linalg.norm(a - b) / np.linalg.norm(b)


# fp32: a product over m entries is off by at most (m + 1) 2^-24 of sum |a b|, typically sqrt(m) of it; with m <= 512 and a
# dozen products in a row, 1e-4 of the norm leaves a factor of ten.  bf16: every tensor between two calls is rounded (2^-9
# of it on average); a dozen such roundings a layer and the residual stream's own, added up as a walk, stay below 2^-5.
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tol", [("f32", 1e-4), ("bf16", 2.0 ** -5)])
@pytest.mark.parametrize("act,hq,hkv,hd,page,P", [("swiglu", 4, 2, 64, 16, 37), ("relu", 2, 2, 80, 8, 64), ("geglu_tanh", 4, 1, 128, 32, 5)])
def test_prompt_and_continuations(dtype, tol, act, hq, hkv, hd, page, P):
    cfg = DecoderConfig(vocab=96, d=256, n_layers=2, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, d_ff=512, act=act, dtype=dtype,
                        page_size=page)
    n_seq, steps = 3, 5
    host = random_weights(cfg, seed=3)
    up = lambda t: None if t is None else t.to(DEV)
    weights = {k: [{a: up(b) for a, b in l.items()} for l in v] if k == "layers" else up(v) for k, v in host.items()}
    dec = Decoder(cfg, weights, 64, n_seq, 8, keep=0.5, device=DEV)
    model = Model64(cfg, host, 72)
    prompt = torch.randint(0, cfg.vocab, (P,), generator=torch.Generator().manual_seed(5))

    logits = dec.prompt(prompt.to(DEV))
    chosen = [logits.topk(n_seq).indices]
    got = []
    for _ in range(steps):
        got.append(dec.step(chosen[-1]))
        chosen.append(got[-1].argmax(1))
    assert dec.status() == G.OK

    want, seen = model.run(prompt.numpy(), P - 1, model.full)
    assert rel(f64(logits), want[0]) < tol
    if dtype == "f32":
        for i, h in enumerate(seen):
            z = O.ff_dense(h, *(model.layers[i][k] for k in ("w_gate", "w_up", "w_down")), act)[1]
            check_expert_set(dec.experts[i].cpu().numpy(), O.flock_score(z), dec.k)
    sets = [O.compact_experts(dec.experts[i].cpu().numpy(), l["w_gate"], l["w_up"], l["w_down"]) for i, l in enumerate(model.layers)]

    def pruned(i, h):   # the prompt's rows went through the full block
        return np.concatenate((model.full(i, h[:P]), np.array([O.ff_pruned(x, sets[i], act) for x in h[P:]])))
    for s in range(n_seq):
        own = [int(c[s]) for c in chosen[:steps]]
        want, _ = model.run(np.concatenate((prompt.numpy(), own)), P, pruned)
        for t in range(steps):
            assert rel(f64(got[t][s]), want[t]) < tol, (s, t)

    # back to the prompt's end: the same tokens give the same bits
    dec.restart()
    for t in range(steps):
        assert torch.equal(dec.step(chosen[t]), got[t])


@pytest.mark.gpu
def test_refusals():
    cfg = DecoderConfig(vocab=32, d=64, n_layers=1, n_q_heads=1, n_kv_heads=1, head_dim=64, d_ff=64, dtype="f32", page_size=8)
    dec = Decoder(cfg, random_weights(cfg, device=DEV), 8, 2, 2, device=DEV)
    two = torch.zeros(2, dtype=torch.long, device=DEV)
    with pytest.raises(ValueError):
        dec.step(two)
    for n in (0, 9):
        with pytest.raises(ValueError):
            dec.prompt(torch.zeros(n, dtype=torch.long, device=DEV))
    dec.prompt(torch.zeros(8, dtype=torch.long, device=DEV))
    for _ in range(2):
        dec.step(two)
    with pytest.raises(ValueError):
        dec.step(two)

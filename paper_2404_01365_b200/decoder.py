"""A small decoder whose layers run through the C ABI: one prompt, several continuations of it.

What each layer does, in the order of its calls (projections are plain torch matrix products):

  h = norm(r)                                 griffin_norm_residual
  q, k, v = h W_qkv; into the cache, rotated  griffin_kv_append
  o = softmax(q K^T) V                        griffin_attn_prefix
  r += o W_o;  h = norm(r)                    griffin_norm_residual
  y = FF(h)                                   griffin_ff_prefill_score (prompt: full block and the statistic), then
                                              griffin_select_topk and griffin_compact_experts;
                                              griffin_ff_decode (generation: the prompt's experts)
  r += y;  h = norm(r) of the next layer      griffin_norm_residual

The prompt's keys and values are kept once.  Its continuations have it as their shared prefix, and the expert set that
the prompt selected as theirs, so a step reads both once for all of them.

  python -m paper_2404_01365_b200.decoder --continuations 8 --steps 32      (random weights)
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass

import torch

from . import binding as G


@dataclass
class DecoderConfig:
    vocab: int
    d: int
    n_layers: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    d_ff: int
    act: str = "swiglu"
    dtype: str = "bf16"
    page_size: int = 64
    eps: float = 1e-6
    theta: float = 10000.0

    @property
    def torch_dtype(self):
        return torch.float32 if self.dtype == "f32" else torch.bfloat16


def random_weights(cfg, seed=0, device="cpu"):
    """Weights of the configuration's shapes: normal, scaled so that every product keeps its input's size."""
    g = torch.Generator(device="cpu").manual_seed(seed)
    rnd = lambda n, m: (torch.randn(n, m, generator=g) * m ** -0.5).to(device=device, dtype=cfg.torch_dtype)
    gain = lambda: (1.0 + 0.1 * torch.randn(cfg.d, generator=g)).to(device=device, dtype=cfg.torch_dtype)
    gated = G.act_is_gated(G.ACT_BY_NAME[cfg.act])
    qkv = (cfg.n_q_heads + 2 * cfg.n_kv_heads) * cfg.head_dim
    layers = [dict(norm_attn=gain(), w_qkv=rnd(qkv, cfg.d), w_o=rnd(cfg.d, cfg.n_q_heads * cfg.head_dim), norm_ff=gain(),
                   w_gate=rnd(cfg.d_ff, cfg.d) if gated else None, w_up=rnd(cfg.d_ff, cfg.d), w_down=rnd(cfg.d, cfg.d_ff))
              for _ in range(cfg.n_layers)]
    return dict(embed=rnd(cfg.vocab, cfg.d) * cfg.d ** 0.5, layers=layers, norm_out=gain(), head=rnd(cfg.vocab, cfg.d))


class Decoder:
    """prompt() once, then step() for every token of the continuations; restart() goes back to the prompt's end."""

    def __init__(self, cfg, weights, max_prompt, n_seq, max_new, keep=0.5, device="cuda"):
        self.cfg, self.w, self.n_seq, self.max_prompt, self.max_new, self.device = cfg, weights, n_seq, max_prompt, max_new, device
        dt, page = cfg.torch_dtype, cfg.page_size
        self.ff = G.make_desc(cfg.d, cfg.d_ff, cfg.act, cfg.dtype)
        self.ff_ws = G.alloc_workspace(self.ff, max_prompt, n_seq, device)
        self.ff_w = [G.make_weights(l["w_gate"], l["w_up"], l["w_down"]) for l in weights["layers"]]
        self.k = G.griffin_k_from_keep_ratio(cfg.d_ff, keep)
        self.score = torch.empty(cfg.n_layers, cfg.d_ff, device=device)
        self.experts = torch.empty(cfg.n_layers, self.k, device=device, dtype=torch.int32)
        self.sets = [G.alloc_compact(self.ff, self.k, device, dt) for _ in range(cfg.n_layers)]
        self.set_arrays = [G.compact_array([s] * n_seq) for s in self.sets]

        self.norm = G.make_norm_desc(cfg.d, cfg.dtype, eps=cfg.eps)
        gains = [g for l in weights["layers"] for g in (l["norm_attn"], l["norm_ff"])] + [weights["norm_out"]]
        self.norm_w = [G.make_norm_weights(g) for g in gains]          # norm_w[2 i]: in front of layer i's attention

        self.attn = G.make_attn_desc(cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, page, cfg.dtype)
        self.attn_ws = G.alloc_attn_workspace(self.attn, max(max_prompt, n_seq), n_seq, device)
        self.rope = G.make_rope(G.rope_table(max_prompt + max_new, cfg.head_dim, cfg.theta, device))
        pre, own = -(-max_prompt // page), -(-max_new // page)
        shape = (pre + n_seq * own, cfg.n_kv_heads, page, cfg.head_dim)
        self.caches = [G.make_kv_cache(torch.empty(shape, device=device, dtype=dt), torch.empty(shape, device=device, dtype=dt))
                       for _ in range(cfg.n_layers)]
        ints = lambda *a: torch.arange(*a, dtype=torch.int32, device=device)
        self.prefix_pages, self.own_pages = ints(pre), ints(pre, pre + n_seq * own).view(n_seq, own)
        self.q_start = ints(n_seq + 1)
        self.seq_len = torch.zeros(n_seq, dtype=torch.int32, device=device)
        self.prompt_len = self.done = 0
        self.batch = None

    def _layers(self, x, batch, feed_forward):
        """The layers over the rows x [T, d], which become the residual stream; the last norm's output."""
        cfg, T = self.cfg, x.shape[0]
        nq, nk = cfg.n_q_heads * cfg.head_dim, cfg.n_kv_heads * cfg.head_dim
        h, o = torch.empty_like(x), torch.empty(T, nq, device=x.device, dtype=x.dtype)
        G.griffin_norm_residual(self.norm, self.norm_w[0], x, None, h)
        for i, l in enumerate(self.w["layers"]):
            qkv = h @ l["w_qkv"].t()
            q, k, v = qkv.split((nq, nk, nk), 1)
            G.griffin_kv_append(self.attn, batch, self.caches[i], self.rope, q, k, v, q, self.attn_ws)
            G.griffin_attn_prefix(self.attn, batch, self.caches[i], q, o, self.attn_ws)
            G.griffin_norm_residual(self.norm, self.norm_w[2 * i + 1], x, x, h, o @ l["w_o"].t())
            y = torch.empty_like(x)
            feed_forward(i, h, y)
            G.griffin_norm_residual(self.norm, self.norm_w[2 * i + 2], x, x, h, y)
        return h

    def prompt(self, tokens):
        """Runs the prompt [P], selects and slices every layer's experts; the logits behind its last token."""
        P = tokens.shape[0]
        if not 0 < P <= self.max_prompt:
            raise ValueError(f"a prompt of {P} tokens; 1 to {self.max_prompt} are expected")
        lens = torch.tensor([0, P, P], dtype=torch.int32, device=self.device)
        batch = G.make_attn_batch(lens[:2], lens[2:], self.prefix_pages[None], P)

        def full(i, h, y):
            G.griffin_ff_prefill_score(self.ff, self.ff_w[i], h, y, self.score[i], self.ff_ws)
        h = self._layers(self.w["embed"][tokens], batch, full)
        G.griffin_select_topk(self.score, self.k, self.experts)
        for i, s in enumerate(self.sets):
            G.griffin_compact_experts(self.ff, self.ff_w[i], self.experts[i], s, self.ff_ws)
        self.prompt_len = P
        self.restart()
        return h[-1] @ self.w["head"].t()

    def restart(self):
        self.seq_len.zero_()
        self.done = 0
        self.batch = G.make_attn_batch(self.q_start, self.seq_len, self.own_pages, self.n_seq, self.prefix_pages, self.prompt_len)

    def step(self, tokens):
        """The next token of every continuation [n_seq]; the logits behind them [n_seq, vocab]."""
        if self.batch is None or self.done == self.max_new:
            raise ValueError("a prompt comes first" if self.batch is None else f"room for {self.max_new} tokens, all used")
        self.done += 1
        self.seq_len += 1       # (the batch reads it when its calls run)

        def pruned(i, h, y):
            G.griffin_ff_decode(self.ff, self.set_arrays[i], None, h, y, self.ff_ws)
        return self._layers(self.w["embed"][tokens], self.batch, pruned) @ self.w["head"].t()

    def status(self):
        """OK, or what a call of the path reported from the device (synchronises)."""
        st = G.griffin_check_device_status(self.ff_ws)
        return st if st != G.OK else G.griffin_check_device_status(self.attn_ws)


def main(argv=None):
    ap = argparse.ArgumentParser(description="One prompt and several continuations of it, random weights.")
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=2048)
    ap.add_argument("--continuations", type=int, default=8)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--keep", type=float, default=0.5)
    a = ap.parse_args(argv)
    cfg = DecoderConfig(vocab=32000, d=4096, n_layers=a.layers, n_q_heads=32, n_kv_heads=8, head_dim=128, d_ff=14336)
    dec = Decoder(cfg, random_weights(cfg, device="cuda"), a.prompt, a.continuations, a.steps, a.keep)
    tokens = torch.randint(0, cfg.vocab, (a.prompt,), generator=torch.Generator().manual_seed(1)).cuda()
    nxt = torch.empty(a.continuations, dtype=torch.long, device="cuda")
    graph = None
    for timed in (False, True):
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
        ev[0].record()
        logits = dec.prompt(tokens)
        ev[1].record()
        nxt.copy_(logits.topk(a.continuations).indices)            # the continuations begin with different tokens
        for _ in range(a.steps):
            if timed:
                graph.replay()
            else:
                nxt.copy_(dec.step(nxt).argmax(1))
        ev[2].record()
        torch.cuda.synchronize()
        if dec.status() != G.OK:
            raise SystemExit("a call reported an error: " + G.status_string(dec.status()))
        if timed:
            print(f"prompt of {a.prompt} tokens: {ev[0].elapsed_time(ev[1]):.2f} ms; {a.steps} steps of {a.continuations} "
                  f"continuations: {ev[1].elapsed_time(ev[2]) / a.steps * 1e3:.0f} us a step of {a.layers} layers")
            continue
        dec.restart()                                              # a step as a graph: the lengths are counted on the device
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            nxt.copy_(dec.step(nxt).argmax(1))


if __name__ == "__main__":
    main()

"""Inputs of the layer operators' tests: a batch over a paged cache, drawn from a seed."""
import numpy as np
import torch

from oracle import layer_oracle as L
from paper_2404_01365_b200 import binding as G

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def f64(t):
    return None if t is None else t.detach().to("cpu", torch.float64).numpy()


class Batch:
    """n_seq sequences behind a shared prefix: q_lens new tokens each, the last of seq_lens own ones.  Everything in the
    cache that no token stands for holds `fill`.  layout "hnd": pages [heads, page, D]; "nhd": [page, heads, D]."""

    def __init__(self, q_lens, seq_lens, prefix, hq, hkv, hd, page, dtype, seed=0, fill=float("nan"), layout="hnd", device="cuda:0",
                 q_scale=1.3, extra_rows=0, table_extra=1):
        g = torch.Generator().manual_seed(seed)
        dt = DTYPES[dtype]
        n_pre, n_own = -(-prefix // page), max(max(-(-n // page) for n in seq_lens), 0) + table_extra
        used = n_pre + sum(-(-n // page) for n in seq_lens)
        order = torch.randperm(used + 2, generator=g).to(torch.int32)
        self.prefix_pages = order[:n_pre].clone()
        table = torch.full((len(seq_lens), n_own), -7, dtype=torch.int32)   # entries that nothing may follow
        at = n_pre
        for s, n in enumerate(seq_lens):
            m = -(-n // page)
            table[s, :m] = order[at:at + m]
            at += m
        self.page_table = table
        starts = np.concatenate(([0], np.cumsum(q_lens)))
        self.q_start, self.seq_len = torch.tensor(starts, dtype=torch.int32), torch.tensor(seq_lens, dtype=torch.int32)
        T = int(starts[-1]) + extra_rows
        self.T, self.prefix = T, prefix
        rnd = lambda *shape, s=1.0: (torch.randn(*shape, generator=g) * s).to(dt)
        self.q, self.k, self.v = rnd(T, hq, hd, s=q_scale), rnd(T, hkv, hd), rnd(T, hkv, hd)
        kp, vp = torch.full((used + 2, hkv, page, hd), fill).to(dt), torch.full((used + 2, hkv, page, hd), fill).to(dt)

        self.kmax = 1.0

        def put(pages, n):
            for i in range(n):
                key = rnd(hkv, hd)
                self.kmax = max(self.kmax, float(key.abs().max()))
                kp[pages[i // page], :, i % page] = key
                vp[pages[i // page], :, i % page] = rnd(hkv, hd)
        put(self.prefix_pages, prefix)
        for s, n in enumerate(seq_lens):
            put(table[s], n)
        self.k_host, self.v_host = kp, vp
        self.hq, self.hkv, self.hd, self.page, self.dtype = hq, hkv, hd, page, dtype
        self.dt = dt
        self.device = device
        self.layout = layout
        self.scale = hd ** -0.5

    def to_device(self):
        d = self.device
        self.desc = G.make_attn_desc(self.hq, self.hkv, self.hd, self.page, self.dtype, self.scale)
        up = lambda t: t.to(d)
        if self.layout == "hnd":
            self.kc, self.vc = up(self.k_host), up(self.v_host)
        else:
            self.kc, self.vc = (up(t.transpose(1, 2).contiguous()).transpose(1, 2) for t in (self.k_host, self.v_host))
        self.cache = G.make_kv_cache(self.kc, self.vc)
        self.dev = [up(t) for t in (self.q_start, self.seq_len, self.page_table, self.prefix_pages)]
        self.batch = G.make_attn_batch(self.dev[0], self.dev[1], self.dev[2], self.T, self.dev[3] if self.prefix else None,
                                       self.prefix)
        self.ws = G.alloc_attn_workspace(self.desc, self.T, len(self.seq_len), d)
        return self

    def attend(self, q=None, out=None, stream=None):
        q = self.q.to(self.device) if q is None else q
        out = torch.full((self.T, self.hq, self.hd), 77.0, dtype=self.dt, device=self.device) if out is None else out
        G.griffin_attn_prefix(self.desc, self.batch, self.cache, q, out, self.ws, stream)
        return out

    def reference(self, rows=None):
        clean = lambda t: np.nan_to_num(f64(t), nan=0.0, posinf=0.0, neginf=0.0)
        return L.attention(f64(self.q), clean(self.k_host), clean(self.v_host), self.q_start.numpy(), self.seq_len.numpy(),
                           self.page_table.numpy(), self.prefix_pages.numpy(), self.prefix, self.scale, rows)

    def bound(self, out, mass):
        """Largest error of an output entry.  bf16: the result is rounded once (2^-8 of it) and each probability once
        (2^-8 of it, so 2^-8 of sum p |v|); fp32 arithmetic adds what the last line says.  fp32: a logit is a sum of D
        products in 32 bits, off by at most (D + 4) 2^-24 sum |q k| scale; that much relative error of p, twice (numerator
        and sum), plus one rounding per key in the sums, the output's included."""
        q, kmax = np.abs(f64(self.q)), self.kmax
        logit = q.sum(2).max() * kmax * self.scale            # sum |q k| scale at most
        n = self.prefix + int(self.seq_len.max())
        arith = (2 * (self.hd + 4) * logit * 2.0 ** -24 + 2 * (n + 8) * 2.0 ** -24 + 2.0 ** -21) * mass
        return arith + 1e-30 if self.dtype == "f32" else arith + 2.0 ** -8 * (1.01 * mass + np.abs(out)) + 1e-30

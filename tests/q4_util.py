"""Inputs of the tests of the cache held in 4 bits: its format in numpy, and batches over such a cache."""
import numpy as np
import torch

from layer_util import Batch, f64
from paper_2404_01365_b200 import binding as G

F32 = np.float32


def block_bytes(page, d):
    return page * (d // 2 + -(-d // 64) * 4)


def quantise(x):
    """x [..., D] fp32 -> integers of -7 .. 7 [..., D] and scale bytes [..., D / 16], every operation rounded to fp32."""
    g = np.asarray(x, F32).reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
    ok = np.isfinite(g).all(-1)
    g = np.where(ok[..., None], g, F32(0))
    m, e = np.frexp(np.abs(g).max(-1) / F32(7))
    b = np.clip(np.rint(m * 16).astype(np.int64) - 8 + 8 * (e.astype(np.int64) - 1 + 21), 0, 254)
    b = np.where(m > 0, b, 0)
    c = np.clip(np.rint(g / scale_of(b)[..., None].astype(F32)), -7, 7).astype(np.int64)
    return c.reshape(x.shape), np.where(ok, b, 255)


def scale_of(b):
    return np.where(b == 255, np.nan, np.ldexp(1 + b % 8 / 8, b // 8 - 21))


def values(c, b):
    return c * np.repeat(scale_of(b), 16, -1)


def pack(c, b):
    """Tokens [..., page, D] and their scales to one head's part of a page each [..., bytes]."""
    page, d = c.shape[-2:]
    n = (c + 8).astype(np.uint32).reshape(*c.shape[:-1], d // 8, 4, 2)                   # [..., word, i, entry 2i or 2i + 1]
    i = np.arange(4, dtype=np.uint32)
    words = ((n[..., 0] << (4 * i)) | (n[..., 1] << (4 * i + 16))).sum(-1, dtype=np.uint32)
    codes = words.astype("<u4").view(np.uint8).reshape(*c.shape[:-2], page * d // 2)
    row = -(-d // 64) * 4
    scales = np.zeros((*b.shape[:-1], row), np.uint8)
    scales[..., :d // 16] = b
    return np.concatenate((codes, scales.reshape(*c.shape[:-2], page * row)), -1)


def rotate32(x, table, pos, style):
    """Heads x [T, H, D] turned by their tokens' positions, every product and sum rounded to fp32."""
    x = np.array(x, F32)
    if table is None:
        return x
    n = table.shape[1] // 2
    cos, sin = table[pos, None, :n].astype(F32), table[pos, None, n:].astype(F32)
    lo, hi = (slice(0, n), slice(n, 2 * n)) if style == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b = x[..., lo].copy(), x[..., hi].copy()
    x[..., lo], x[..., hi] = a * cos - b * sin, a * sin + b * cos
    return x


class BatchQ4(Batch):
    """The batch over a cache in 4 bits: k_host and v_host become what the cache holds of them."""

    def __init__(self, *a, **kw):
        kw.pop("layout", None)
        super().__init__(*a, **kw)
        self.requantise()

    def requantise(self):
        for name in ("k", "v"):
            c, b = quantise(getattr(self, name + "_host").float().numpy())
            setattr(self, name + "_bytes", torch.from_numpy(pack(c, b)))
            setattr(self, name + "_host", torch.from_numpy(values(c, b)).to(self.dt))    # (exact)
        self.kmax = float(torch.nan_to_num(self.k_host.float()).abs().max())

    def to_device(self, gap=0):
        d = self.device
        self.desc = G.make_attn_desc(self.hq, self.hkv, self.hd, self.page, self.dtype, self.scale)
        up = lambda t: t.to(d)
        # (gap: bytes between the heads' parts)
        self.kb, self.vb = (up(torch.nn.functional.pad(t, (0, gap), value=0xAB))[..., :t.shape[-1]] for t in (self.k_bytes, self.v_bytes))
        self.cache = G.make_kv_cache_q4(self.kb, self.vb)
        self.dev = [up(t) for t in (self.q_start, self.seq_len, self.page_table, self.prefix_pages)]
        self.batch = G.make_attn_batch(self.dev[0], self.dev[1], self.dev[2], self.T, self.dev[3] if self.prefix else None,
                                       self.prefix)
        self.ws = G.alloc_attn_workspace(self.desc, self.T, len(self.seq_len), d)
        return self

    def attend(self, q=None, out=None, stream=None):
        q = self.q.to(self.device) if q is None else q
        out = torch.full((self.T, self.hq, self.hd), 77.0, dtype=self.dt, device=self.device) if out is None else out
        G.griffin_attn_prefix_q4(self.desc, self.batch, self.cache, q, out, self.ws, stream)
        return out

    def read(self, k=None, v=None):
        mk = lambda: torch.full((self.T, self.hkv, self.hd), 33.0, dtype=self.dt, device=self.device)
        k, v = mk() if k is None else k, mk() if v is None else v
        G.griffin_kv_read_q4(self.desc, self.batch, self.cache, k, v, self.ws)
        return k, v

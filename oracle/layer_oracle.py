"""What surrounds the FF block in a decoder layer, in plain numpy float64: the norms with the residual stream,
rotated keys and values in a paged cache, attention over a shared prefix and own tokens.  One row, one token,
one head at a time; imports nothing from the package.
"""
import math

import numpy as np


def norm(x, kind, w=None, b=None, eps=1e-6, w0=0.0):
    """One row: rms  x / sqrt(mean x^2 + eps) (w0 + w);  layer  (x - mean) / sqrt(var + eps) (w0 + w) + b."""
    x = np.asarray(x, np.float64)
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean()
    out = x / math.sqrt((x * x).mean() + eps) * (w0 + w)
    return out + b if kind == "layer" and b is not None else out


GATES = {"linear": lambda g: g, "sigmoid": lambda g: 1.0 / (1.0 + np.exp(-g)), "tanh": np.tanh}


def norm_residual(res, y=None, gate=None, pre="rms", post="none", pre_w=None, pre_b=None, post_w=None, post_b=None, eps=1e-6,
                  w0=0.0, res_scale=1.0, out_scale=1.0, gate_act="linear"):
    """(res', h) for rows res [T, d]; gate [d] or [T, d]."""
    r_out, h_out = [], []
    for t, r in enumerate(np.asarray(res, np.float64)):
        r = res_scale * r
        if y is not None:
            u = norm(y[t], post, post_w, post_b, eps, w0)
            if gate is not None:
                u = GATES[gate_act](gate if gate.ndim == 1 else gate[t]) * u
            r = r + out_scale * u
        r_out.append(r)
        h_out.append(norm(r, pre, pre_w, pre_b, eps, w0))
    return np.array(r_out), np.array(h_out)


def rotate(x, cos, sin, style):
    """One head's entries x [D] turned by rot/2 angles."""
    x = np.array(x, np.float64)
    n = len(cos)
    for j in range(n):
        a, b = (j, j + n) if style == "half" else (2 * j, 2 * j + 1)
        x[a], x[b] = x[a] * cos[j] - x[b] * sin[j], x[a] * sin[j] + x[b] * cos[j]
    return x


def places(q_start, seq_len):
    """(token, sequence, index among the sequence's own tokens) of every new token; a negative index is padding."""
    return [(t, s, int(seq_len[s]) - (int(q_start[s + 1]) - t))
            for s in range(len(seq_len)) for t in range(int(q_start[s]), int(q_start[s + 1]))]


def kv_append(k_pages, v_pages, q_start, seq_len, page_table, prefix_len, q, k, v, table=None, style="half"):
    """New caches [n_pages, heads, page, D] and the rotated q."""
    k_pages, v_pages = np.array(k_pages, np.float64), np.array(v_pages, np.float64)
    q_out, page = np.array(q, np.float64), k_pages.shape[2]

    def turn(x, pos):
        if table is None:
            return x
        n = table.shape[1] // 2
        return np.array([rotate(h, table[pos, :n], table[pos, n:], style) for h in x])

    for t, s, i in places(q_start, seq_len):
        if i < 0:
            q_out[t] = 0
            continue
        p = int(page_table[s, i // page])
        q_out[t] = turn(q[t], prefix_len + i)
        k_pages[p, :, i % page], v_pages[p, :, i % page] = turn(k[t], prefix_len + i), v[t]
    return k_pages, v_pages, q_out


def gather(pages, which, n):
    """The first n tokens of a list of pages: [n, heads, D]."""
    page = pages.shape[2]
    return np.stack([pages[int(which[i // page]), :, i % page] for i in range(n)]) if n else np.zeros((0,) + pages.shape[1::2])


def attention(q, k_pages, v_pages, q_start, seq_len, page_table, prefix_pages, prefix_len, scale, rows=None):
    """out [T, Hq, D] and, entry for entry, sum_j p_j |v_j| (what rounding errors of p scale with); `rows`: only these tokens."""
    T, hq, _ = q.shape
    hkv = k_pages.shape[1]
    out, mass = np.zeros(q.shape), np.zeros(q.shape)
    kp, vp = gather(k_pages, prefix_pages, prefix_len), gather(v_pages, prefix_pages, prefix_len)
    for t, s, i in places(q_start, seq_len):
        if rows is not None and t not in rows:
            continue
        n = max(i + 1, 0)
        k, v = (np.concatenate((a, gather(b, page_table[s], n))) for a, b in ((kp, k_pages), (vp, v_pages)))
        if len(k) == 0:
            continue
        for h in range(hq):
            x = k[:, h // (hq // hkv)] @ q[t, h] * scale
            p = np.exp(x - x.max())
            p /= p.sum()
            out[t, h] = p @ v[:, h // (hq // hkv)]
            mass[t, h] = p @ np.abs(v[:, h // (hq // hkv)])
    return out, mass

"""Workloads for timing the operators of the cache held in 4 bits: new tokens quantised into it, read back, and attention
of a batch whose sequences share a prefix over it.

`run` computes one pass, either in plain torch operations (own = False) or through the package's entry points
(own = True), on the same inputs.  Head counts and widths are those of the decoder layers whose FF shapes the
package's synthetic workloads use, or generic ones.

The format: 16 consecutive entries of a head are a group with one scale s, max |x| / 7 rounded to 4 significant bits,
and hold rint(x / s) + 8 in 4 bits each.  Scale bytes: 8 (e + 21) + m for s = 2^e (1 + m / 8); 255 makes the group NaN.
Of 8 entries in a 32-bit word, 2i has bits 4i .. 4i+3 and 2i+1 the same of the upper half.  A page holds, per head, the
codes of its tokens and behind them their scales, 4 ceil(D / 64) bytes each.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}
_DEV = "cuda"


# ------------------------------------------------------------------------------------------------------------
# Cases
# ------------------------------------------------------------------------------------------------------------
def _append(n_seq, q_len, prefix, own_len, hq, hkv, hd, page, dtype, rot, style):
    return {"op": "append", "n_seq": n_seq, "q_len": q_len, "prefix": prefix, "own_len": own_len, "hq": hq, "hkv": hkv,
            "hd": hd, "page": page, "dtype": dtype, "rot": rot, "style": style}


def _read(n_seq, own_len, hkv, hd, page, dtype):
    return {"op": "read", "n_seq": n_seq, "q_len": own_len, "prefix": 0, "own_len": own_len, "hq": hkv, "hkv": hkv, "hd": hd,
            "page": page, "dtype": dtype}


def _attn(n_seq, q_len, prefix, own_len, hq, hkv, hd, page, dtype):
    return {"op": "attn", "n_seq": n_seq, "q_len": q_len, "prefix": prefix, "own_len": own_len, "hq": hq, "hkv": hkv,
            "hd": hd, "page": page, "dtype": dtype}


def listed():
    named = {
        # one decode step of 8 continuations, 40 heads (Llama-2-13B): the smallest appends
        "append_step": _append(8, 1, 2048, 256, 40, 40, 128, 64, "bf16", 128, "half"),
        # a whole 4096-token prompt with grouped heads (Mistral-7B) goes into the cache
        "append_prompt": _append(1, 4096, 0, 4096, 32, 8, 128, 64, "bf16", 128, "half"),
        # fp32, partial rotation of adjacent pairs, short pages, ragged drafts
        "append_f32_ragged": _append(37, 29, 301, 411, 12, 4, 80, 16, "f32", 32, "pairs"),
        # ragged sequences of up to 8192 tokens go back to bf16, to be moved elsewhere
        "read_long": _read(5, 8192, 8, 128, 64, "bf16"),
        # fp32, narrow heads, odd lengths: what a check of a small model reads
        "read_f32_odd": _read(3, 531, 4, 80, 16, "f32"),
        # generation for one sequence after a 512-token prompt (Llama-2-7B heads)
        "attn_step_one": _attn(1, 1, 512, 128, 32, 32, 128, 64, "bf16"),
        # 8 continuations of one 2048-token prompt, every query head with its own keys (Llama-2-13B heads)
        "attn_step_shared": _attn(8, 1, 2048, 256, 40, 40, 128, 64, "bf16"),
        # 48 unrelated sequences of up to 4096 tokens, grouped heads (Mistral-7B heads): nothing to share
        "attn_step_own": _attn(48, 1, 0, 4096, 32, 8, 128, 64, "bf16"),
        # 32 continuations of a 32768-token document, grouped heads (Mistral-7B heads)
        "attn_step_long": _attn(32, 1, 32768, 512, 32, 8, 128, 64, "bf16"),
        # the prompt itself: 4096 tokens, causal (Mistral-7B heads)
        "attn_prompt": _attn(1, 4096, 0, 4096, 32, 8, 128, 64, "bf16"),
        # wide heads (Gemma-7B), a few drafted tokens per sequence, pages of 32
        "attn_draft_wide": _attn(6, 5, 1000, 300, 16, 16, 256, 32, "bf16"),
        # fp32 storage, narrow heads, odd lengths
        "attn_step_f32": _attn(5, 1, 1003, 217, 16, 4, 64, 16, "f32"),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("append", "read", "attn", "attn"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    hkv, group = rng.choice((1, 2, 4, 5, 8, 16, 32, 40)), rng.choice((1, 1, 2, 3, 4, 8))
    if hkv * group > 64:
        group = 1
    hq, hd, page = hkv * group, rng.choice((64, 80, 128, 128, 256)), rng.choice((16, 32, 64, 128))
    n_seq, prefix, own_len = _log(rng, 1, 64), _log(rng, 1, 32768) - 1, _log(rng, 1, 4096)
    if op == "read":
        while n_seq * own_len * hkv * hd > 5 * 8192 * 8 * 128 // 2:
            n_seq, own_len = (n_seq + 1) // 2, (own_len * 3 + 3) // 4
        return _read(n_seq, own_len, hkv, hd, page, dtype)
    if op == "append":
        q_len = min(own_len, _log(rng, 1, 512))
        while n_seq * q_len * (hq + hkv) * hd > 4096 * 48 * 128:
            n_seq, q_len = (n_seq + 1) // 2, (q_len + 1) // 2
        prefix = min(prefix, 4096)
        return _append(n_seq, q_len, prefix, own_len, hq, hkv, hd, page, dtype, rng.choice((0, 32, hd - hd % 16)),
                       rng.choice(("half", "pairs")))
    q_len = min(own_len, rng.choice((1, 1, 1, _log(rng, 1, 8), _log(rng, 1, 1024))))
    most = 4e9 if dtype == "f32" else 60e9      # fp32 storage stands for small models and checks
    while 4.0 * n_seq * q_len * hq * hd * (prefix + own_len) > most:
        if n_seq > 1 and rng.random() < 0.5:
            n_seq = (n_seq + 1) // 2
        elif q_len > 8 and rng.random() < 0.5:
            q_len = (q_len + 1) // 2
        else:
            prefix //= 2
            own_len = max(q_len, own_len * 3 // 4)
    while (prefix + n_seq * own_len) * hkv * hd > 32768 * 8 * 128:     # the cache itself
        prefix, own_len = prefix * 3 // 4, max(q_len, own_len * 3 // 4)
        n_seq = (n_seq + 1) // 2 if q_len == own_len else n_seq
    return _attn(n_seq, q_len, prefix, own_len, hq, hkv, hd, page, dtype)


def _lengths(case):
    """New tokens and own tokens (new ones included) of each sequence: a fixed ragged pattern of the case's sizes."""
    r = random.Random(case["n_seq"] * 1000003 + case["q_len"] * 10007 + case["own_len"])
    if case["op"] == "read":       # whole sequences
        lens = [case["own_len"]] + [r.randint(max(1, case["own_len"] // 4), case["own_len"]) for _ in range(case["n_seq"] - 1)]
        return lens, lens
    q = [case["q_len"]] + [r.randint(max(1, case["q_len"] // 2), case["q_len"]) for _ in range(case["n_seq"] - 1)]
    lens = [case["own_len"]] + [r.randint(min(case["own_len"], max(n, case["own_len"] // 4)), case["own_len"]) for n in q[1:]]
    return q, [max(a, b) for a, b in zip(q, lens)]


def work(case):
    b = _BYTES[case["dtype"]]
    q, lens = _lengths(case)
    T, hq, hkv, hd = sum(q), case["hq"], case["hkv"], case["hd"]
    held = 2 * hkv * (hd // 2 + hd // 16)           # of one token in the cache
    if case["op"] == "append":    # q in and out, k and v in, into the cache, and out as the values they became
        return {"bytes": T * (2 * hq * hd * b + 4 * hkv * hd * b + held) + T * case["rot"] * 4,
                "flops": 3 * T * (hq + hkv) * case["rot"] + 12 * T * hkv * hd}
    if case["op"] == "read":
        return {"bytes": T * (held + 2 * hkv * hd * b), "flops": 4 * T * hkv * hd}
    pairs = sum(n * case["prefix"] + n * (l - n) + n * (n + 1) // 2 for n, l in zip(q, lens))
    return {"bytes": (case["prefix"] + sum(lens)) * held + 2 * T * hq * hd * b, "flops": 4 * pairs * hq * hd}


# ------------------------------------------------------------------------------------------------------------
# The format, in plain operations
# ------------------------------------------------------------------------------------------------------------
def _quantise(x):
    """x [..., D] (fp32) -> codes [..., D / 2] and scales [..., D / 16], uint8."""
    g = x.unflatten(-1, (-1, 16))
    a = g.abs().amax(-1)
    ok = torch.isfinite(g).all(-1)
    m, e = torch.frexp(torch.where(ok, a, 0.0) / torch.full_like(a, 7.0))     # m in [1/2, 1)
    b = ((torch.round(m * 16) - 8).int() + 8 * (e - 1 + 21)).clamp(0, 254)    # (a mantissa rounded up to 16 goes on in the exponent)
    b = torch.where(m > 0, b, 0)
    s = torch.ldexp(1 + (b % 8) / 8, b // 8 - 21)
    c = torch.round(torch.where(ok[..., None], g, 0.0) / s[..., None]).clamp(-7, 7).int() + 8
    w = c.flatten(-2).unflatten(-1, (-1, 4, 2))                               # [..., word, i, entry 2i or 2i + 1]
    lo = (w[..., 0, :] | w[..., 1, :] << 4, w[..., 2, :] | w[..., 3, :] << 4)
    codes = torch.stack((lo[0][..., 0], lo[1][..., 0], lo[0][..., 1], lo[1][..., 1]), -1).flatten(-2)
    return codes.to(torch.uint8), torch.where(ok, b, 255).to(torch.uint8)


def _values(codes, scales):
    """What they stand for, fp32."""
    w = codes.int().unflatten(-1, (-1, 2, 2))                                 # [..., word, half, byte]
    c = torch.stack((w & 15, w >> 4), -1).flatten(-2)                         # [..., word, half, i]
    c = c.transpose(-1, -2).flatten(-3) - 8
    b = scales.int()
    s = torch.ldexp(1 + (b % 8) / 8, b // 8 - 21).masked_fill(b == 255, float("nan"))
    return (c.unflatten(-1, (-1, 16)) * s[..., None]).flatten(-2)


def _parts(pages, case):
    """Views of the pages [n, heads, bytes]: codes [n, heads, page, D / 2], scales [n, heads, page, D / 16]."""
    P, hd = case["page"], case["hd"]
    codes, scales = pages[..., :P * hd // 2], pages[..., P * hd // 2:]
    return codes.unflatten(-1, (P, hd // 2)), scales.unflatten(-1, (P, 4 * -(-hd // 64)))[..., :hd // 16]


# ------------------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------------------
def _inputs(case, seed):
    g = torch.Generator(device=_DEV)
    g.manual_seed(seed)
    dt = _DT[case["dtype"]]

    def rand(*shape, dtype=dt, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=g, device=_DEV) * scale + shift).to(dtype)

    s = {"case": case}
    q_lens, lens = _lengths(case)
    n_seq, P, prefix, T = case["n_seq"], case["page"], case["prefix"], sum(q_lens)
    n_pre, n_own = -(-prefix // P), -(-max(lens) // P)
    n_pages = n_pre + sum(-(-l // P) for l in lens) + 3
    pages = torch.randperm(n_pages, generator=g, device=_DEV).to(torch.int32)
    s["prefix_pages"] = pages[:n_pre].clone()
    # rows of the page table are filled as far as the sequence reaches; the rest names page 0
    need = torch.tensor([-(-l // P) for l in lens], device=_DEV)
    first = torch.cumsum(need, 0) - need + n_pre
    col = torch.arange(n_own, device=_DEV)
    at = first[:, None] + col[None, :]
    s["page_table"] = torch.where(col[None, :] < need[:, None], pages[at.clamp(max=n_pages - 1)], torch.zeros_like(pages[:1])).contiguous()
    starts = [0]
    for n in q_lens:
        starts.append(starts[-1] + n)
    s["q_start"] = torch.tensor(starts, dtype=torch.int32, device=_DEV)
    s["seq_len"] = torch.tensor(lens, dtype=torch.int32, device=_DEV)
    s["T"] = T
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    size = P * (hd // 2 + 4 * -(-hd // 64))
    s["k_pages"], s["v_pages"] = (torch.zeros(n_pages, hkv, size, dtype=torch.uint8, device=_DEV) for _ in range(2))
    if case["op"] == "append":
        qkv = rand(T, (hq + 2 * hkv) * hd)                # the fused projection's output; q, k, v are slices of it
        s["qkv"] = qkv
        s["q"] = qkv[:, :hq * hd].unflatten(1, (hq, hd))
        s["k"] = qkv[:, hq * hd:(hq + hkv) * hd].unflatten(1, (hkv, hd))
        s["v"] = qkv[:, (hq + hkv) * hd:].unflatten(1, (hkv, hd))
        rot, n_pos = case["rot"], prefix + max(lens)
        if rot:
            freq = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device=_DEV) * 2 / rot)
            ang = torch.arange(n_pos, dtype=torch.float64, device=_DEV)[:, None] * freq
            s["rope"] = torch.cat((ang.cos(), ang.sin()), 1).float().contiguous()
        else:
            s["rope"] = None
        return s
    # a cache that earlier calls have filled: keys with some channels far larger than the rest, as trained models have them
    wide = 1.0 + 5.0 * (torch.rand(hkv, 1, hd, generator=g, device=_DEV) < 0.03)
    step = max(1, (1 << 24) // (hkv * P * hd))
    for name, scale in (("k_pages", 0.9 * wide / wide.square().mean().sqrt()), ("v_pages", 1.0)):
        codes, scales = _parts(s[name], case)
        for a in range(0, n_pages, step):
            n = min(step, n_pages - a)
            codes[a:a + n], scales[a:a + n] = _quantise(torch.randn(n, hkv, P, hd, generator=g, device=_DEV) * scale)
    if case["op"] == "attn":
        s["q"] = rand(T, hq, hd, scale=1.3)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:   # what the caller of the package keeps beside its data: descriptors, output buffers, a workspace
        from paper_2404_01365_b200 import binding as G
        s["G"] = G
        dt, hq, hkv, hd = _DT[case["dtype"]], case["hq"], case["hkv"], case["hd"]
        s["desc"] = G.make_attn_desc(hq, hkv, hd, case["page"], case["dtype"])
        s["batch"] = G.make_attn_batch(s["q_start"], s["seq_len"], s["page_table"], s["T"], s["prefix_pages"], case["prefix"])
        s["cache"] = G.make_kv_cache_q4(s["k_pages"], s["v_pages"])
        s["ws"] = G.alloc_attn_workspace(s["desc"], s["T"], case["n_seq"], _DEV)
        if case["op"] != "read":
            s["out"] = torch.empty(s["T"], hq, hd, dtype=dt, device=_DEV)
        if case["op"] != "attn":
            s["k_out"], s["v_out"] = (torch.empty(s["T"], hkv, hd, dtype=dt, device=_DEV) for _ in range(2))
        if case["op"] == "append":
            s["rope_desc"] = G.make_rope(s["rope"], case["style"]) if case["rot"] else None
    return s


# ------------------------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------------------------
def run(s):
    op = s["case"]["op"]
    if own:
        G = s["G"]
        if op == "attn":
            G.griffin_attn_prefix_q4(s["desc"], s["batch"], s["cache"], s["q"], s["out"], s["ws"])
            return {"out": s["out"]}
        if op == "append":   # what the new tokens became in the cache is read back
            G.griffin_kv_append_q4(s["desc"], s["batch"], s["cache"], s["rope_desc"], s["q"], s["k"], s["v"], s["out"], s["ws"])
        G.griffin_kv_read_q4(s["desc"], s["batch"], s["cache"], s["k_out"], s["v_out"], s["ws"])
        out = {"k": s["k_out"], "v": s["v_out"]}
        return dict(out, q=s["out"]) if op == "append" else out
    return {"append": _plain_append, "read": _plain_read, "attn": _plain_attn}[op](s)


def _plain_places(s):
    """Sequence and index among its own tokens of every new token."""
    t = torch.arange(s["T"], device=_DEV)
    seq = (t[:, None] >= s["q_start"][None, 1:]).sum(1)
    i = s["seq_len"][seq] - (s["q_start"][seq + 1] - t)
    return seq, i


def _plain_rotate(x, table, rot, style, pos):
    x = x.float()
    if not rot:
        return x
    cos, sin = table[pos, None, :rot // 2], table[pos, None, rot // 2:]
    if style == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_read(s):
    case = s["case"]
    seq, i = _plain_places(s)
    page, slot = s["page_table"][seq, i // case["page"]].long(), i % case["page"]
    out = {}
    for name in ("k", "v"):
        codes, scales = _parts(s[name + "_pages"], case)
        out[name] = _values(codes[page, :, slot], scales[page, :, slot]).to(_DT[case["dtype"]])
    return out


def _plain_append(s):
    case = s["case"]
    seq, i = _plain_places(s)
    pos, P = i + case["prefix"], case["page"]
    page, slot = s["page_table"][seq, i // P].long(), i % P
    q = _plain_rotate(s["q"], s["rope"], case["rot"], case["style"], pos).to(s["q"].dtype)
    for name, x in (("k_pages", _plain_rotate(s["k"], s["rope"], case["rot"], case["style"], pos)), ("v_pages", s["v"].float())):
        codes, scales = _parts(s[name], case)
        codes[page, :, slot], scales[page, :, slot] = _quantise(x)
    return dict(_plain_read(s), q=q)


def _plain_attn(s):
    case = s["case"]
    n_seq, hq, hkv, hd, P, L = case["n_seq"], case["hq"], case["hkv"], case["hd"], case["page"], case["prefix"]
    group, mq = hq // hkv, case["q_len"]
    n_own = s["page_table"].shape[1]
    # queries in a padded [sequence, token] grid, grouped under their key head
    q_len = s["q_start"][1:] - s["q_start"][:-1]
    at = s["q_start"][:-1, None] + torch.arange(mq, device=_DEV)[None]
    q = s["q"].float()[at.clamp(max=s["T"] - 1)].view(n_seq, mq, hkv, group, hd).permute(0, 2, 3, 1, 4).reshape(n_seq, hkv, group * mq, hd)
    pages = [_values(*_parts(s[name], case)) for name in ("k_pages", "v_pages")]
    kp, vp = (c[s["prefix_pages"]].transpose(0, 1).reshape(hkv, s["prefix_pages"].shape[0] * P, hd)[:, :L] for c in pages)
    ko, vo = (c[s["page_table"]].transpose(1, 2).reshape(n_seq, hkv, n_own * P, hd) for c in pages)
    sp = torch.matmul(q.transpose(0, 1).reshape(hkv, n_seq * group * mq, hd), kp.transpose(1, 2)).view(hkv, n_seq, group * mq, L).transpose(0, 1)
    so = torch.matmul(q, ko.transpose(2, 3)).view(n_seq, hkv, group, mq, n_own * P)
    seen = (s["seq_len"] - q_len)[:, None] + torch.arange(mq, device=_DEV)[None]          # last own token that each query sees
    hidden = torch.arange(n_own * P, device=_DEV)[None, None] > seen[:, :, None]
    so = so.masked_fill(hidden[:, None, None], float("-inf")).view(n_seq, hkv, group * mq, n_own * P)
    x = torch.cat((sp, so), 3) * hd ** -0.5
    p = torch.exp(x - x.amax(3, keepdim=True))
    p = p / p.sum(3, keepdim=True)
    op = torch.matmul(p[..., :L].transpose(0, 1).reshape(hkv, n_seq * group * mq, L), vp).view(hkv, n_seq, group * mq, hd).transpose(0, 1)
    o = op + torch.matmul(p[..., L:], vo)
    o = o.view(n_seq, hkv, group, mq, hd).permute(0, 3, 1, 2, 4).reshape(n_seq, mq, hq, hd)
    seq, i = _plain_places(s)
    t = torch.arange(s["T"], device=_DEV) - s["q_start"][seq]
    return {"out": o[seq, t].to(s["q"].dtype)}


# ------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ------------------------------------------------------------------------------------------------------------
def _exact_held(x):
    """The values that x [..., D] becomes: the nearest multiple of its group's scale."""
    x = x.double()
    a = x.reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
    want = a.abs().max(-1, keepdim=True).values / 7
    unit = torch.exp2(torch.floor(torch.log2(want.clamp(min=2.0 ** -60))))
    scale = (torch.round(want / unit * 8) / 8 * unit).clamp(2.0 ** -21, 1792.0)
    return (torch.round(a / scale).clamp(-7, 7) * scale).reshape(x.shape)


def _exact_pages(pages, which, head, case):
    """Tokens of a list of pages under one head, [tokens, D]."""
    P, hd = case["page"], case["hd"]
    raw = pages[which.long(), head].long()
    words, nib = raw[:, :P * hd // 2].reshape(-1, hd // 8, 4), torch.arange(8, device=_DEV)
    word = (words << (8 * torch.arange(4, device=_DEV))).sum(-1)
    code = (word[..., None] >> (4 * (nib // 2 + 4 * (nib % 2)))) & 15         # entry e of a word: nibble e / 2, of the upper half if odd
    row = 4 * -(-hd // 64)
    b = raw[:, P * hd // 2:].reshape(-1, row)[:, :hd // 16].repeat_interleave(16, 1)
    return (code.reshape(-1, hd) - 8).double() * torch.exp2((b // 8 - 21).double()) * (8 + b % 8) / 8


def exact(case, seed):
    s = _inputs(case, seed)
    q_lens, lens = _lengths(case)
    P, prefix, hq, hkv, hd = case["page"], case["prefix"], case["hq"], case["hkv"], case["hd"]
    starts, table = s["q_start"].tolist(), s["page_table"]
    if case["op"] == "read":
        out = {n: torch.empty(s["T"], hkv, hd, dtype=torch.float64, device=_DEV) for n in ("k", "v")}
        for n in range(case["n_seq"]):
            for h in range(hkv):
                for name in out:
                    out[name][starts[n]:starts[n + 1], h] = _exact_pages(s[name + "_pages"], table[n], h, case)[:lens[n]]
        return out
    if case["op"] == "append":
        rot = case["rot"]
        q_out = torch.empty(s["T"], hq, hd, dtype=torch.float64, device=_DEV)
        k_out = torch.empty(s["T"], hkv, hd, dtype=torch.float64, device=_DEV)

        def turned(x, pos):
            x = x.double().clone()
            if rot:
                # the pair as a complex number times cos + i sin of the table
                z = torch.complex(s["rope"][pos, :rot // 2].double(), s["rope"][pos, rot // 2:].double())[:, None]
                lo, hi = (slice(0, rot // 2), slice(rot // 2, rot)) if case["style"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
                w = torch.complex(x[..., lo], x[..., hi]) * z
                x[..., lo], x[..., hi] = w.real, w.imag
            return x

        for n in range(case["n_seq"]):
            a, b = starts[n], starts[n + 1]
            pos = prefix + torch.arange(lens[n] - (b - a), lens[n], device=_DEV)
            q_out[a:b], k_out[a:b] = turned(s["q"][a:b], pos), turned(s["k"][a:b], pos)
        return {"q": q_out, "k": _exact_held(k_out), "v": _exact_held(s["v"])}
    out = torch.empty(s["T"], hq, hd, dtype=torch.float64, device=_DEV)
    for h in range(hkv):
        heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
        k_pre, v_pre = (_exact_pages(c, s["prefix_pages"], h, case)[:prefix] for c in (s["k_pages"], s["v_pages"]))
        for n in range(case["n_seq"]):
            a, b = starts[n], starts[n + 1]
            k, v = (torch.cat((pre, _exact_pages(c, table[n], h, case)[:lens[n]]))
                    for pre, c in ((k_pre, s["k_pages"]), (v_pre, s["v_pages"])))
            last = prefix + lens[n] - (b - a) + torch.arange(b - a, device=_DEV)
            logits = torch.einsum("tgd,ld->gtl", s["q"][a:b, heads].double(), k) / math.sqrt(hd)
            logits = logits + torch.where(torch.arange(k.shape[0], device=_DEV)[None] <= last[:, None], 0.0, -math.inf)
            weights = torch.exp(logits - torch.logsumexp(logits, 2, keepdim=True))
            out[a:b, heads] = torch.einsum("gtl,ld->tgd", weights, v)
    return {"out": out}

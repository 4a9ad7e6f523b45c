"""Workloads for timing the operators around the feed-forward block: norms with the residual stream, the paged
key/value cache, and attention of a batch whose sequences share a prefix.

`run` computes one pass, either in plain torch operations (own = False) or through the package's entry points
(own = True), on the same inputs.  Head counts and widths are those of the decoder layers whose FF shapes the
package's synthetic workloads use, or generic ones.
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
def _norm(T, d, dtype, res, pre, post, gate):
    return {"op": "norm", "T": T, "d": d, "dtype": dtype, "res": res, "pre": pre, "post": post, "gate": gate}


def _append(n_seq, q_len, prefix, own_len, hq, hkv, hd, page, dtype, rot, style):
    return {"op": "append", "n_seq": n_seq, "q_len": q_len, "prefix": prefix, "own_len": own_len, "hq": hq, "hkv": hkv,
            "hd": hd, "page": page, "dtype": dtype, "rot": rot, "style": style}


def _attn(n_seq, q_len, prefix, own_len, hq, hkv, hd, page, dtype):
    return {"op": "attn", "n_seq": n_seq, "q_len": q_len, "prefix": prefix, "own_len": own_len, "hq": hq, "hkv": hkv,
            "hd": hd, "page": page, "dtype": dtype}


def listed():
    named = {
        # one token of one sequence between two blocks of a 4096-wide layer: nothing but latency
        "norm_token": _norm(1, 4096, "bf16", "bf16", "rms", "none", "none"),
        # a 4096-token prompt, norms on both sides of the block, a learned scale per channel, fp32 residual stream
        "norm_prompt_sandwich": _norm(4096, 4096, "bf16", "f32", "rms", "rms", "channel"),
        # fp32, LayerNorm with biases, a gate per token and channel; a row count and a width that divide nothing
        "norm_layer_f32_odd": _norm(1001, 2056, "f32", "f32", "layer", "layer", "full"),
        # one decode step of 8 continuations, 40 heads (Llama-2-13B): the smallest appends
        "append_step": _append(8, 1, 2048, 256, 40, 40, 128, 64, "bf16", 128, "half"),
        # a whole 4096-token prompt with grouped heads (Mistral-7B) goes into the cache
        "append_prompt": _append(1, 4096, 0, 4096, 32, 8, 128, 64, "bf16", 128, "half"),
        # fp32, partial rotation of adjacent pairs, short pages, ragged drafts
        "append_f32_ragged": _append(37, 29, 301, 411, 12, 4, 80, 16, "f32", 32, "pairs"),
        # generation for one sequence after a 512-token prompt (Llama-2-7B heads)
        "attn_step_one": _attn(1, 1, 512, 128, 32, 32, 128, 64, "bf16"),
        # 8 continuations of one 2048-token prompt, every query head with its own keys (Llama-2-13B heads)
        "attn_step_shared": _attn(8, 1, 2048, 256, 40, 40, 128, 64, "bf16"),
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
    op = rng.choice(("norm", "append", "attn", "attn"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "norm":
        d = 8 * _log(rng, 32, 1024)
        if d == 3072:
            d += 8
        T = min(_log(rng, 1, 8192), 4096 * 4096 // d)
        return _norm(T, d, dtype, "f32" if dtype == "f32" else rng.choice(("bf16", "f32")), rng.choice(("rms", "rms", "layer")),
                     rng.choice(("none", "rms", "layer")), rng.choice(("none", "channel", "full")))
    hkv, group = rng.choice((1, 2, 4, 5, 8, 16, 32, 40)), rng.choice((1, 1, 2, 3, 4, 8))
    if hkv * group > 64:
        group = 1
    hq, hd, page = hkv * group, rng.choice((64, 80, 128, 128, 256)), rng.choice((16, 32, 64, 128))
    n_seq, prefix, own_len = _log(rng, 1, 64), _log(rng, 1, 32768) - 1, _log(rng, 1, 2048)
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
    while (prefix + n_seq * own_len) * hkv * hd > 32768 * 16 * 128:     # the cache itself
        prefix, own_len = prefix * 3 // 4, max(q_len, own_len * 3 // 4)
        n_seq = (n_seq + 1) // 2 if q_len == own_len else n_seq
    return _attn(n_seq, q_len, prefix, own_len, hq, hkv, hd, page, dtype)


def _lengths(case):
    """New tokens and own tokens (new ones included) of each sequence: a fixed ragged pattern of the case's sizes."""
    r = random.Random(case["n_seq"] * 1000003 + case["q_len"] * 10007 + case["own_len"])
    q = [case["q_len"]] + [r.randint(max(1, case["q_len"] // 2), case["q_len"]) for _ in range(case["n_seq"] - 1)]
    lens = [case["own_len"]] + [r.randint(min(case["own_len"], max(n, case["own_len"] // 4)), case["own_len"]) for n in q[1:]]
    return q, [max(a, b) for a, b in zip(q, lens)]


def work(case):
    b = _BYTES[case["dtype"]]
    if case["op"] == "norm":
        n, rb = case["T"] * case["d"], _BYTES[case["res"]]
        full = n if case["gate"] == "full" else case["d"] if case["gate"] == "channel" else 0
        params = case["d"] * ((2 if case["pre"] == "layer" else 1) + {"none": 0, "rms": 1, "layer": 2}[case["post"]])
        per = 8 + {"none": 0, "rms": 4, "layer": 6}[case["post"]] + (0 if case["gate"] == "none" else 1)
        return {"bytes": n * (2 * b + 2 * rb) + (full + params) * b, "flops": n * per}
    q, lens = _lengths(case)
    T, hq, hkv, hd = sum(q), case["hq"], case["hkv"], case["hd"]
    if case["op"] == "append":
        return {"bytes": 2 * T * (hq + 2 * hkv) * hd * b + T * case["rot"] * 4, "flops": 3 * T * (hq + hkv) * case["rot"]}
    pairs = sum(n * case["prefix"] + n * (l - n) + n * (n + 1) // 2 for n, l in zip(q, lens))
    return {"bytes": 2 * (case["prefix"] + sum(lens)) * hkv * hd * b + 2 * T * hq * hd * b, "flops": 4 * pairs * hq * hd}


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
    if case["op"] == "norm":
        T, d = case["T"], case["d"]
        s["y"] = rand(T, d, scale=0.7)                                        # the block's output
        s["res"] = rand(T, d, dtype=_DT[case["res"]], scale=3.0, shift=0.2)   # the residual stream, grown over some layers
        s["pre_w"], s["pre_b"] = rand(d, scale=0.1, shift=1.0), rand(d, scale=0.1) if case["pre"] == "layer" else None
        s["post_w"] = rand(d, scale=0.1, shift=1.0) if case["post"] != "none" else None
        s["post_b"] = rand(d, scale=0.1) if case["post"] == "layer" else None
        s["gate"] = {"none": None, "channel": rand(d, scale=0.3, shift=0.5), "full": rand(T, d) if case["gate"] == "full" else None}[case["gate"]]
        return s
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
    if case["op"] == "append":
        qkv = rand(T, (hq + 2 * hkv) * hd)                # the fused projection's output; q, k, v are slices of it
        s["qkv"] = qkv
        s["q"] = qkv[:, :hq * hd].unflatten(1, (hq, hd))
        s["k"] = qkv[:, hq * hd:(hq + hkv) * hd].unflatten(1, (hkv, hd))
        s["v"] = qkv[:, (hq + hkv) * hd:].unflatten(1, (hkv, hd))
        s["k_pages"] = torch.zeros(n_pages, hkv, P, hd, dtype=dt, device=_DEV)
        s["v_pages"] = torch.zeros(n_pages, hkv, P, hd, dtype=dt, device=_DEV)
        rot, n_pos = case["rot"], prefix + max(lens)
        if rot:
            freq = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device=_DEV) * 2 / rot)
            ang = torch.arange(n_pos, dtype=torch.float64, device=_DEV)[:, None] * freq
            s["rope"] = torch.cat((ang.cos(), ang.sin()), 1).float().contiguous()
        else:
            s["rope"] = None
        return s
    s["q"] = rand(T, hq, hd, scale=1.3)
    s["k_pages"] = rand(n_pages, hkv, P, hd, scale=1.1)
    s["v_pages"] = rand(n_pages, hkv, P, hd)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:   # what the caller of the package keeps beside its data: descriptors, output buffers, a workspace
        from paper_2404_01365_b200 import binding as G
        s["G"] = G
        if case["op"] == "norm":
            s["desc"] = G.make_norm_desc(case["d"], case["dtype"], case["res"], pre=case["pre"], post=case["post"], eps=1e-5,
                                         res_scale=1.0, out_scale=0.5)
            s["weights"] = G.make_norm_weights(s["pre_w"], s["pre_b"], s["post_w"], s["post_b"])
            s["res_out"], s["h"] = torch.empty_like(s["res"]), torch.empty_like(s["y"])
            return s
        s["desc"] = G.make_attn_desc(case["hq"], case["hkv"], case["hd"], case["page"], case["dtype"])
        s["batch"] = G.make_attn_batch(s["q_start"], s["seq_len"], s["page_table"], s["T"], s["prefix_pages"], case["prefix"])
        s["cache"] = G.make_kv_cache(s["k_pages"], s["v_pages"])
        s["ws"] = G.alloc_attn_workspace(s["desc"], s["T"], case["n_seq"], _DEV)
        s["out"] = torch.empty(s["T"], case["hq"], case["hd"], dtype=_DT[case["dtype"]], device=_DEV)
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
        if op == "norm":
            G.griffin_norm_residual(s["desc"], s["weights"], s["res"], s["res_out"], s["h"], s["y"], s["gate"])
            return {"res": s["res_out"], "h": s["h"]}
        if op == "append":
            G.griffin_kv_append(s["desc"], s["batch"], s["cache"], s["rope_desc"], s["q"], s["k"], s["v"], s["out"], s["ws"])
            return {"q": s["out"], "k": s["k_pages"], "v": s["v_pages"]}
        G.griffin_attn_prefix(s["desc"], s["batch"], s["cache"], s["q"], s["out"], s["ws"])
        return {"out": s["out"]}
    return {"norm": _plain_norm, "append": _plain_append, "attn": _plain_attn}[op](s)


def _norm_rows(x, kind, w, b):
    if kind == "rms":
        return x * torch.rsqrt((x * x).mean(1, keepdim=True) + 1e-5) * w.float()
    c = x - x.mean(1, keepdim=True)
    return c * torch.rsqrt((c * c).mean(1, keepdim=True) + 1e-5) * w.float() + b.float()


def _plain_norm(s):
    case = s["case"]
    u = s["y"].float()
    if case["post"] != "none":
        u = _norm_rows(u, case["post"], s["post_w"], s["post_b"])
    if s["gate"] is not None:
        u = u * s["gate"].float()
    r = s["res"].float() + 0.5 * u
    h = _norm_rows(r, case["pre"], s["pre_w"], s["pre_b"])
    return {"res": r.to(s["res"].dtype), "h": h.to(s["y"].dtype)}


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


def _plain_append(s):
    case = s["case"]
    seq, i = _plain_places(s)
    pos, P = i + case["prefix"], case["page"]
    page, slot = s["page_table"][seq, i // P].long(), i % P
    dt = s["q"].dtype
    q = _plain_rotate(s["q"], s["rope"], case["rot"], case["style"], pos).to(dt)
    s["k_pages"][page, :, slot] = _plain_rotate(s["k"], s["rope"], case["rot"], case["style"], pos).to(dt)
    s["v_pages"][page, :, slot] = s["v"]
    return {"q": q, "k": s["k_pages"], "v": s["v_pages"]}


def _plain_attn(s):
    case = s["case"]
    n_seq, hq, hkv, hd, P, L = case["n_seq"], case["hq"], case["hkv"], case["hd"], case["page"], case["prefix"]
    group, mq = hq // hkv, case["q_len"]
    n_own = s["page_table"].shape[1]
    # queries in a padded [sequence, token] grid, grouped under their key head
    q_len = s["q_start"][1:] - s["q_start"][:-1]
    at = s["q_start"][:-1, None] + torch.arange(mq, device=_DEV)[None]
    q = s["q"].float()[at.clamp(max=s["T"] - 1)].view(n_seq, mq, hkv, group, hd).permute(0, 2, 3, 1, 4).reshape(n_seq, hkv, group * mq, hd)
    kp, vp = (c[s["prefix_pages"]].transpose(0, 1).reshape(hkv, s["prefix_pages"].shape[0] * P, hd)[:, :L].float() for c in (s["k_pages"], s["v_pages"]))
    ko, vo = (c[s["page_table"]].transpose(1, 2).reshape(n_seq, hkv, n_own * P, hd).float() for c in (s["k_pages"], s["v_pages"]))
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
def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "norm":
        def normed(x, kind, w, b):
            mean = torch.zeros((), dtype=torch.float64, device=_DEV) if kind == "rms" else x.sum(-1, keepdim=True) / case["d"]
            spread = torch.linalg.vector_norm(x - mean, dim=-1, keepdim=True) ** 2 / case["d"]
            out = (x - mean) / torch.sqrt(spread + 1e-5) * w.double()
            return out if b is None else out + b.double()

        y, r = s["y"].double(), s["res"].double()
        u = y if case["post"] == "none" else normed(y, case["post"], s["post_w"], s["post_b"])
        gate = 1.0 if s["gate"] is None else s["gate"].double()
        r = r + gate * u / 2
        return {"res": r, "h": normed(r, case["pre"], s["pre_w"], s["pre_b"])}
    q_lens, lens = _lengths(case)
    P, prefix, hq, hkv, hd = case["page"], case["prefix"], case["hq"], case["hkv"], case["hd"]
    starts, table = s["q_start"].tolist(), s["page_table"].long()
    if case["op"] == "append":
        rot = case["rot"]
        k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
        q_out = torch.empty(s["T"], hq, hd, dtype=torch.float64, device=_DEV)

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
            i = torch.arange(lens[n] - (b - a), lens[n], device=_DEV)
            where = (table[n][i // P], slice(None), i % P)
            q_out[a:b] = turned(s["q"][a:b], prefix + i)
            k_pages[where], v_pages[where] = turned(s["k"][a:b], prefix + i), s["v"][a:b].double()
        return {"q": q_out, "k": k_pages, "v": v_pages}
    out = torch.empty(s["T"], hq, hd, dtype=torch.float64, device=_DEV)
    for h in range(hkv):
        heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
        k_pre, v_pre = (c[s["prefix_pages"].long(), h].reshape(-1, hd)[:prefix].double() for c in (s["k_pages"], s["v_pages"]))
        for n in range(case["n_seq"]):
            a, b = starts[n], starts[n + 1]
            k, v = (torch.cat((pre, c[table[n], h].reshape(-1, hd)[:lens[n]].double()))
                    for pre, c in ((k_pre, s["k_pages"]), (v_pre, s["v_pages"])))
            last = prefix + lens[n] - (b - a) + torch.arange(b - a, device=_DEV)
            logits = torch.einsum("tgd,ld->gtl", s["q"][a:b, heads].double(), k) / math.sqrt(hd)
            logits = logits + torch.where(torch.arange(k.shape[0], device=_DEV)[None] <= last[:, None], 0.0, -math.inf)
            weights = torch.exp(logits - torch.logsumexp(logits, 2, keepdim=True))
            out[a:b, heads] = torch.einsum("gtl,ld->tgd", weights, v)
    return {"out": out}

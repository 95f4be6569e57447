"""Cases of the serving operators between a decoder layer's quantized linears: what a user runs, from one token to long prompts.

A case is one pass through one operator:

  append   sasq_kv_append: rotates the new tokens' queries and keys by their positions and writes keys and values to a paged
           cache, in 16 bits or as int8 codes with a static factor for each kv head
  attend   sasq_paged_attention: causal attention of the new tokens over that cache

Shapes: the attention blocks of the LLaMA-2-7B (32 heads), 13B (40 heads) and 70B (64 heads on 8 kv heads) layers that the
configurations and the benchmark of this repository use, all with 128 channels a head, and generic ones.  The lengths of a case's
sequences follow from the case alone; the order of their pages, and all values, from the seed.

Where `own` is false, run() computes the operators from elementary torch operations in 32 bits, rounded once at the end.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
TABLE = 1 << 17                 # rows of the rotation table: the longest position of any case


def _attend(name, batch, heads, kv_heads, new, past, mix="all", dtype="bf16", cache="16", page=64, order="hnd", dim=128, lse=False):
    return {"name": name, "kind": "attend", "batch": batch, "heads": heads, "kv_heads": kv_heads, "dim": dim, "new": new, "mix": mix,
            "past_lo": past[0], "past_hi": past[1], "dtype": dtype, "cache": cache, "page": page, "order": order, "lse": lse}


def _append(name, batch, heads, kv_heads, new, past, mix="all", dtype="bf16", cache="16", page=64, order="hnd", dim=128, rot=128,
            style="halves", fused=False):
    return {"name": name, "kind": "append", "batch": batch, "heads": heads, "kv_heads": kv_heads, "dim": dim, "new": new, "mix": mix,
            "past_lo": past[0], "past_hi": past[1], "dtype": dtype, "cache": cache, "page": page, "order": order, "rot": rot,
            "style": style, "fused": fused}


def listed():
    return [
        # one user, a short conversation, one token of a 7B model: what a call costs at the least
        _attend("attend one short 7B", 1, 32, 32, 1, (300, 300), dtype="f16", page=16),
        # a served batch of 70B: one token for each of 48 users whose conversations are of all lengths
        _attend("attend batch 70B", 48, 64, 8, 1, (200, 8190)),
        # the same in 13B without shared heads, the cache in int8
        _attend("attend batch 13B int8", 32, 40, 40, 1, (900, 4095), dtype="f16", cache="int8", page=32, order="nhd"),
        # two very long documents, one token each, 70B with an int8 cache
        _attend("attend long 70B int8", 2, 64, 8, 1, (120000, 131000), cache="int8", page=256),
        # a few tokens at once for each user, as when a draft is checked
        _attend("attend drafts 70B", 16, 64, 8, 5, (500, 4000), dtype="f16", cache="int8", page=16),
        # chunks of two new prompts beside ten users who wait for their next token, 13B
        _attend("attend mixed 13B", 12, 40, 40, 509, (100, 6000), mix="mixed", page=64, order="nhd", lse=True),
        # prompts of 7B from the first token: batch 2 x 2048
        _attend("attend prompts 7B", 2, 32, 32, 2048, (0, 0), dtype="f16", page=128),
        # a chunk of 4096 tokens of a long 70B prompt on what is already in the cache
        _attend("attend chunk 70B", 1, 64, 8, 4096, (12281, 12281), page=256),
        # one token of a 7B model appended
        _append("append one 7B", 1, 32, 32, 1, (300, 300), dtype="f16", page=16),
        # one token for each of 200 users of 70B
        _append("append batch 70B", 200, 64, 8, 1, (10, 1500), fused=True),
        # 70B: batch 4 x 2048 new tokens
        _append("append prompts 70B", 4, 64, 8, 2048, (0, 0), page=128),
        # ragged chunks of 13B into an int8 cache, pairs rotated, the products of one fused projection
        _append("append chunks 13B int8", 9, 40, 40, 600, (0, 0), mix="ragged", cache="int8", page=32, order="nhd", style="pairs", fused=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def lengths(case):
    """[(new tokens, tokens already in the cache)] of the case's sequences."""
    r = random.Random("%(batch)d %(new)d %(mix)s %(past_lo)d %(past_hi)d" % case)
    got = []
    for b in range(case["batch"]):
        past = case["past_lo"] if case["past_hi"] <= case["past_lo"] else _log(r, max(1, case["past_lo"]), case["past_hi"])
        new = case["new"]
        if case["mix"] == "ragged":
            new = r.randint(1, new)
        elif case["mix"] == "mixed" and b % 6 != 3:
            new = 1
        got.append((new, past))
    return got


def _size(case):
    """Elements of the padded table of scores, and of the padded keys."""
    ln = lengths(case)
    longest = max(n + p for n, p in ln)
    return case["batch"] * case["heads"] * max(n for n, _ in ln) * longest, case["batch"] * case["kv_heads"] * longest * case["dim"]


def draw(rng):
    limit = max((work(c) for c in listed() if c["kind"] == "attend"), key=lambda w: w["flops"])
    scores, keys = (max(v) for v in zip(*(_size(c) for c in listed() if c["kind"] == "attend")))
    while True:
        heads, kv_heads = rng.choice([(32, 32), (40, 40), (64, 8), (64, 8), (8, 8), (28, 4), (20, 4), (16, 1)])
        dim, page = rng.choice([64, 128, 128, 128]), rng.choice([16, 32, 64, 128, 256])
        common = {"mix": rng.choice(["all", "ragged", "mixed"]), "dtype": rng.choice(["f16", "bf16"]), "cache": rng.choice(["16", "16", "int8"]),
                  "page": page, "order": rng.choice(["hnd", "nhd"]), "dim": dim}
        if rng.random() < 0.65:
            new = rng.choice([1, _log(rng, 2, 16), _log(rng, 17, 4096)])
            lo = _log(rng, 1, 100000)
            c = _attend("", _log(rng, 1, 64), heads, kv_heads, new, (lo - 1, _log(rng, lo, min(131000, 8 * lo))), lse=rng.random() < 0.3, **common)
            if max(_size(c)[0] / scores, _size(c)[1] / keys, work(c)["flops"] / limit["flops"]) > 1:
                continue
        else:
            new = rng.choice([1, _log(rng, 2, 2048)])
            rot = rng.choice([dim, dim, dim // 2])
            c = _append("", _log(rng, 1, 200), heads, kv_heads, new, (0, _log(rng, 2, 2000)), rot=rot,
                        style=rng.choice(["halves", "pairs"]), fused=rng.random() < 0.5, **common)
            if work(c)["bytes"] > 400e6 or _size(c)[1] > keys / 4:
                continue
        del c["name"]
        return c


def work(case):
    ln = lengths(case)
    tokens, D, H, Hk = sum(n for n, _ in ln), case["dim"], case["heads"], case["kv_heads"]
    e = 1 if case["cache"] == "int8" else 2
    if case["kind"] == "append":
        return {"bytes": tokens * D * (4 * H + 4 * Hk + 2 * Hk * e), "flops": 3 * tokens * (H + Hk) * case["rot"] + (2 * tokens * Hk * D if e == 1 else 0)}
    pairs = sum(n * p + n * (n + 1) // 2 for n, p in ln)
    held = sum(n + p for n, p in ln)
    return {"bytes": tokens * H * (4 * D + (4 if case["lse"] else 0)) + held * Hk * 2 * D * e, "flops": 4 * D * H * pairs}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ln, dt = lengths(case), DTYPES[case["dtype"]]
    H, Hk, D, page, B = case["heads"], case["kv_heads"], case["dim"], case["page"], case["batch"]
    new = torch.tensor([n for n, _ in ln], dtype=torch.int32)
    kv_len = torch.tensor([n + p for n, p in ln], dtype=torch.int32)
    cu_q = torch.zeros(B + 1, dtype=torch.int32)
    cu_q[1:] = new.cumsum(0)
    T, longest = int(cu_q[-1]), int(kv_len.max())
    need = (kv_len + page - 1) // page
    pages, width = int(need.sum()) + 3, -(-longest // page) + 1
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)      # a page's place says nothing about its sequence
    first = (need.cumsum(0) - need).cuda()
    col = torch.arange(width, device="cuda")
    table = torch.where(col < need.cuda()[:, None], order[(first[:, None] + col).clamp(max=pages - 1).long()], -1).to(torch.int32)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(dt)

    def cache():
        shape = (pages, Hk, page, D) if case["order"] == "hnd" else (pages, page, Hk, D)
        if case["cache"] == "int8":                                                # factors that clip little: codes over the whole range
            t = torch.randn(shape, generator=g, device="cuda").mul_(30).round_().clamp_(-128, 127).to(torch.int8)
        else:
            t = torch.randn(shape, generator=g, device="cuda").to(dt)
        return t.transpose(1, 2) if case["order"] == "hnd" else t

    s = {"case": dict(case), "T": T, "max_q": int(new.max()), "max_kv": longest, "cu_q": cu_q.cuda(), "kv_len": kv_len.cuda(), "table": table,
         "k_cache": cache(), "v_cache": cache(), "k_scale": None, "v_scale": None}
    if case["cache"] == "int8":
        s["k_scale"] = (torch.rand(Hk, generator=g, device="cuda") + 0.5) / 30
        s["v_scale"] = (torch.rand(Hk, generator=g, device="cuda") + 0.5) / 30
    if case["kind"] == "append":
        if case["fused"]:                                                          # columns of one projection's output
            qkv = normal(T, (H + 2 * Hk), D)
            s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        else:
            s["q"], s["k"], s["v"] = normal(T, H, D), normal(T, Hk, D), normal(T, Hk, D)
        s["k"][..., ::37] *= 4                                                     # the few large channels that keys have
        half = case["rot"] // 2
        angle = torch.arange(TABLE, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["q_out"] = torch.empty((T, H, D), dtype=dt, device="cuda")
    else:
        s["q"] = normal(T, H, D, scale=1.5)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((T, H), dtype=torch.float32, device="cuda") if case["lse"] else None
        s["scale"] = D ** -0.5
    if own:                                                                        # what a serving program keeps: the cache, the step's batch, a workspace
        from paper_2512_14481_amd import binding as lib
        s["lib"] = lib
        s["cache"] = lib.KVCache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
        s["batch"] = lib.KVBatch(s["cu_q"], s["kv_len"], s["table"], T, max_q=s["max_q"], max_kv=s["max_kv"])
        if case["kind"] == "attend":
            s["workspace"] = lib.new_workspace(lib.sasq_paged_attention_workspace(s["cache"], s["batch"], H))
    return s


def _values(codes, scale, dt):
    """What a cache holds: its 16-bit values, or those that its codes stand for."""
    return codes if scale is None else (codes.float() * scale[:, None]).to(dt)


def _of_token(s):
    """Sequence and position of each row."""
    t = torch.arange(s["T"], device="cuda", dtype=torch.int32)
    seq = torch.bucketize(t, s["cu_q"][1:], right=True)
    return seq, s["kv_len"][seq].long() - (s["cu_q"][seq + 1] - t).long()


def _rotated(x, cos, sin, style):
    half = cos.shape[-1]
    a, b = (x[..., :half], x[..., half:2 * half]) if style == "halves" else (x[..., :2 * half:2], x[..., 1:2 * half:2])
    lo, hi = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat((lo, hi), -1) if style == "halves" else torch.stack((lo, hi), -1).flatten(-2)
    return torch.cat((turned, x[..., 2 * half:]), -1)


def _plain_append(s):
    page, dt = s["case"]["page"], s["q"].dtype
    seq, pos = _of_token(s)
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]
    q = _rotated(s["q"].float(), cos, sin, s["case"]["style"]).to(dt)
    k = _rotated(s["k"].float(), cos, sin, s["case"]["style"]).to(dt)
    v = s["v"]
    if s["k_scale"] is not None:
        k = (k.float() * (1.0 / s["k_scale"])[:, None]).round().clamp(-128, 127).to(torch.int8)
        v = (v.float() * (1.0 / s["v_scale"])[:, None]).round().clamp(-128, 127).to(torch.int8)
    at = s["table"][seq, pos // page].long(), pos % page
    s["k_cache"][at] = k
    s["v_cache"][at] = v
    return q


def _plain_attend(s):
    case = s["case"]
    H, Hk, D, page, B, n, m = case["heads"], case["kv_heads"], case["dim"], case["page"], case["batch"], s["max_q"], s["max_kv"]
    q_len = s["cu_q"][1:] - s["cu_q"][:-1]
    i, j = torch.arange(n, device="cuda"), torch.arange(m, device="cuda")
    there = i < q_len[:, None]                                                      # [B, n]: rows that the sequence has
    row = (s["cu_q"][:-1, None] + i).clamp(max=s["T"] - 1)
    q = s["q"][row].float().view(B, n, Hk, H // Hk, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, H // Hk * n, D)
    at = s["table"][:, j // page]                                                   # [B, m]
    held = (at >= 0) & (j < s["kv_len"][:, None])
    at = at.clamp(min=0).long(), (j % page).expand(B, m)
    k, v = s["k_cache"][at].float(), s["v_cache"][at].float()                        # [B, m, Hk, D]
    if s["k_scale"] is not None:
        k, v = k * s["k_scale"][:, None], v * s["v_scale"][:, None]
    v = torch.where(held[:, :, None, None], v, 0.0)
    score = torch.matmul(q, k.permute(0, 2, 3, 1)).mul_(s["scale"]).view(B, Hk, H // Hk, n, m)
    position = (s["kv_len"] - q_len)[:, None] + i
    seen = held[:, None, :] & (j <= position[:, :, None]) & there[:, :, None]        # [B, n, m]
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.view(B, Hk, H // Hk * n, m), v.permute(0, 2, 1, 3)).view(B, Hk, H // Hk, n, D)
    out = torch.where(total > 0, out / total, 0.0).permute(0, 3, 1, 2, 4).reshape(B, n, H, D)
    lse = (top + total.log()).permute(0, 3, 1, 2, 4).reshape(B, n, H)
    return out[there].to(s["q"].dtype), lse[there] if case["lse"] else None


def run(state):
    s, case = state, state["case"]
    if case["kind"] == "append":
        if own:
            q = s["q_out"]
            s["lib"].sasq_kv_append(s["q"], s["k"], s["v"], q, s["cache"], s["batch"], s["cos"], s["sin"],
                                    style=s["lib"].SASQ_ROPE_HALVES if case["style"] == "halves" else s["lib"].SASQ_ROPE_PAIRS)
        else:
            q = _plain_append(s)
        return {"q": q, "k_cache": _values(s["k_cache"], s["k_scale"], q.dtype), "v_cache": _values(s["v_cache"], s["v_scale"], q.dtype)}
    if own:
        out, lse = s["out"], s["lse"]
        s["lib"].sasq_paged_attention(s["q"], out, s["cache"], s["batch"], s["workspace"], s["scale"], lse=lse)
    else:
        out, lse = _plain_attend(s)
    return {"out": out} if lse is None else {"out": out, "lse": lse}


def _exact_append(s):
    case, page = s["case"], s["case"]["page"]
    half, rot = case["rot"] // 2, case["rot"]
    dt = s["q"].dtype
    place = torch.arange(rot, device="cuda")
    if case["style"] == "halves":
        partner, row, sign = (place + half) % rot, place % half, torch.where(place < half, -1.0, 1.0).double()
    else:
        partner, row, sign = place ^ 1, place // 2, torch.where(place % 2 == 0, -1.0, 1.0).double()
    out = {"q": s["q"].double().clone(), "k_cache": s["k_cache"].clone(), "v_cache": s["v_cache"].clone()}
    keys = s["k"].double().clone()
    for b in range(case["batch"]):
        lo, hi, end = int(s["cu_q"][b]), int(s["cu_q"][b + 1]), int(s["kv_len"][b])
        pos = torch.arange(end - (hi - lo), end, device="cuda")
        cos, sin = s["cos"].double()[pos][:, row][:, None], s["sin"].double()[pos][:, row][:, None]
        for x in (out["q"][lo:hi], keys[lo:hi]):
            x[..., :rot] = x[..., :rot] * cos + sign * x[..., partner] * sin
        where = s["table"][b].long()[pos // page], pos % page
        for name, x, scale in (("k_cache", keys[lo:hi], s["k_scale"]), ("v_cache", s["v"][lo:hi].double(), s["v_scale"])):
            if scale is not None:                                                   # the code of the 16-bit value
                x = (x.to(dt).double() * (1.0 / scale).double()[:, None]).round().clamp(-128, 127)
            elif out[name].dtype != torch.float64:
                out[name] = out[name].double()
            out[name][where] = x.to(out[name].dtype)
    for name, scale in (("k_cache", s["k_scale"]), ("v_cache", s["v_scale"])):
        if scale is not None:
            out[name] = out[name].double() * scale.double()[:, None]
    return out


def _exact_attend(s):
    case, page = s["case"], s["case"]["page"]
    H, Hk = case["heads"], case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        lo, hi, end = int(s["cu_q"][b]), int(s["cu_q"][b + 1]), int(s["kv_len"][b])
        j = torch.arange(end, device="cuda")
        where = s["table"][b].long()[j // page], j % page
        later = j > torch.arange(end - (hi - lo), end, device="cuda")[:, None]
        k, v = s["k_cache"][where].double(), s["v_cache"][where].double()
        for h in range(H):
            kv = h // (H // Hk)
            kh, vh = k[:, kv].contiguous(), v[:, kv].contiguous()
            if s["k_scale"] is not None:
                kh, vh = kh * s["k_scale"][kv].double(), vh * s["v_scale"][kv].double()
            score = (s["q"][lo:hi, h].double() @ kh.t().contiguous()) * s["scale"]
            score[later] = -math.inf
            lse[lo:hi, h] = torch.logsumexp(score, -1)
            out[lo:hi, h] = torch.softmax(score, -1) @ vh
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_append(s) if case["kind"] == "append" else _exact_attend(s)

"""The attention-serving operators as they are measured: rotary positions (`rg_rope`), keys and values appended to a
paged cache with the rotation on the way (`rg_kv_append`), and attention of a chunk of new tokens over that cache
(`rg_paged_attention`), each beside its plain form in elementary torch operations.

A case's shapes (lengths of the sequences among them) follow from the case alone, its values from the seed.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BASE = 10000.0


def listed():
    return [
        # training: queries of an 8192-token batch, 32 heads of 128, rotated once in the forward pass
        {"name": "rope_batch_bf16", "op": "rope", "tokens": 8192, "heads": 32, "d": 128, "rot": 128, "style": "half", "axes": 1, "inverse": False, "type": "bf16", "far": 8192},
        # training on video: gradients of rows with time, height and width positions; an odd number of patches, half of each head rotated
        {"name": "rope_video_grad_fp32", "op": "rope", "tokens": 6145, "heads": 16, "d": 80, "rot": 40, "style": "pairs", "axes": 3, "inverse": True, "type": "fp32", "far": 4000},
        # a few draft tokens far into a long text: latency
        {"name": "rope_seven_far_fp16", "op": "rope", "tokens": 7, "heads": 32, "d": 128, "rot": 128, "style": "half", "axes": 1, "inverse": False, "type": "fp16", "far": 1 << 20},
        # serving: 64 sequences get one token each
        {"name": "append_decode_64", "op": "append", "seqs": 64, "q_lo": 1, "q_hi": 1, "ctx_lo": 1, "ctx_hi": 8192, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "style": "half", "axes": 1, "page": 16, "type": "bf16", "shape": 1},
        # serving: prompts of ragged length, pages of 64
        {"name": "append_prompts", "op": "append", "seqs": 5, "q_lo": 500, "q_hi": 4096, "ctx_lo": 0, "ctx_hi": 2000, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "style": "half", "axes": 1, "page": 64, "type": "bf16", "shape": 2},
        # images among the text: three position axes, heads of 64
        {"name": "append_axes_fp16", "op": "append", "seqs": 3, "q_lo": 37, "q_hi": 1031, "ctx_lo": 0, "ctx_hi": 5000, "hq": 16, "hkv": 2, "d": 64, "rot": 64, "style": "half", "axes": 3, "page": 32, "type": "fp16", "shape": 3},
        # one user's next token: latency
        {"name": "attend_decode_1", "op": "attend", "seqs": 1, "q_lo": 1, "q_hi": 1, "ctx_lo": 8191, "ctx_hi": 8191, "hq": 32, "hkv": 8, "d": 128, "page": 16, "window": 0, "split": 256, "lse": False, "type": "bf16", "shape": 4},
        # a serving batch: one token for each of 64 sequences of ragged length
        {"name": "attend_decode_64", "op": "attend", "seqs": 64, "q_lo": 1, "q_hi": 1, "ctx_lo": 100, "ctx_hi": 8191, "hq": 32, "hkv": 8, "d": 128, "page": 16, "window": 0, "split": 512, "lse": False, "type": "bf16", "shape": 5},
        # long documents: few sequences, far apart in length
        {"name": "attend_decode_long", "op": "attend", "seqs": 4, "q_lo": 1, "q_hi": 1, "ctx_lo": 30001, "ctx_hi": 65536, "hq": 64, "hkv": 8, "d": 128, "page": 64, "window": 0, "split": 512, "lse": False, "type": "bf16", "shape": 6},
        # draft tokens checked within a sliding window, heads of 64
        {"name": "attend_drafts_window_fp16", "op": "attend", "seqs": 33, "q_lo": 2, "q_hi": 5, "ctx_lo": 0, "ctx_hi": 6000, "hq": 16, "hkv": 2, "d": 64, "page": 32, "window": 2048, "split": 512, "lse": False, "type": "fp16", "shape": 7},
        # a step that mixes prompts' chunks with short ones, and wants the normalisers too
        {"name": "attend_mixed_lse", "op": "attend", "seqs": 9, "q_lo": 1, "q_hi": 1000, "ctx_lo": 0, "ctx_hi": 3000, "hq": 32, "hkv": 8, "d": 128, "page": 16, "window": 0, "split": 0, "lse": True, "type": "bf16", "shape": 8},
        # a long prompt's next chunk
        {"name": "attend_chunk_4096", "op": "attend", "seqs": 1, "q_lo": 4096, "q_hi": 4096, "ctx_lo": 12288, "ctx_hi": 12288, "hq": 32, "hkv": 8, "d": 128, "page": 64, "window": 0, "split": 0, "lse": False, "type": "bf16", "shape": 9},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "append", "attend", "attend"])
    if op == "rope":
        kind = rng.choice(["bf16", "fp16", "fp32"])
        d = rng.choice([64, 80, 96, 128, 256])
        axes = rng.choice([1, 1, 2, 3])
        rot = rng.choice([d, d, d // 2])
        while True:
            tokens, heads = _log(rng, 1, 16384), _log(rng, 1, 64)
            if tokens * heads * d * (2 if kind == "fp32" else 1) <= 8192 * 32 * 128:
                break
        return {"op": op, "tokens": tokens, "heads": heads, "d": d, "rot": rot, "style": rng.choice(["half", "pairs"]), "axes": axes,
                "inverse": rng.random() < 0.5, "type": kind, "far": _log(rng, 1000, 1 << 20)}
    hkv = rng.choice([1, 2, 4, 8])
    c = {"op": op, "hq": hkv * rng.choice([1, 2, 4, 5, 7, 8]), "hkv": hkv, "d": rng.choice([64, 80, 128, 128]), "page": rng.choice([16, 16, 32, 64, 128]),
         "type": rng.choice(["bf16", "bf16", "fp16"]), "shape": rng.randrange(1 << 30)}
    if op == "append":
        c |= {"rot": rng.choice([c["d"], c["d"] // 2]), "style": rng.choice(["half", "pairs"]), "axes": rng.choice([1, 1, 3])}
    else:
        c |= {"window": rng.choice([0, 0, 0, _log(rng, 100, 4096)]), "lse": rng.random() < 0.3}
    while True:
        seqs, q_hi, ctx_hi = _log(rng, 1, 128), _log(rng, 1, 4096), _log(rng, 1, 65536)
        big = c | {"seqs": seqs, "q_lo": rng.randint(1, q_hi), "q_hi": q_hi, "ctx_lo": rng.randint(0, ctx_hi), "ctx_hi": ctx_hi}
        if rng.random() < 0.4:
            big["q_lo"] = big["q_hi"] = 1
        if op == "attend":
            big["split"] = 512 if big["q_hi"] <= 16 else 0
        q, kv = _lens(big)
        most = 2 ** 28 // (big["hkv"] * big["d"])               # padded keys of all sequences, within half a gigabyte of cache
        pairs = seqs * max(q) * max(kv) * big["hq"]              # the plain form's score matrix
        if seqs * max(kv) <= most and sum(q) <= 16384 and (op == "append" or pairs * big["d"] <= 32 * 4096 * 16384 * 128):
            return big


def _lens(c):
    """New tokens and whole length (new ones included) of each sequence: they follow from the case alone."""
    r = random.Random(c["shape"])
    q = [r.randint(c["q_lo"], c["q_hi"]) for _ in range(c["seqs"])]
    return q, [n + r.randint(c["ctx_lo"], c["ctx_hi"]) for n in q]


def _sections(c):
    """How many of a row's rot/2 angle pairs each axis has: time a quarter, height and width the rest."""
    pairs = c["rot"] // 2
    if c["axes"] == 1:
        return (pairs,)
    if c["axes"] == 2:
        return (pairs - pairs // 2, pairs // 2)
    w = (pairs - pairs // 4) // 2
    return (pairs - 2 * w, w, w)


def _positions(c, g, tokens, far):
    """[axes, tokens] positions up to `far`: text order on the first axis, patch rows and columns on the others."""
    p = torch.randint(0, far, (c["axes"], tokens), generator=g, device=DEV)
    p[0] = p[0].sort().values
    return p.to(torch.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = TYPES[c["type"]]
    st = {"c": c}
    if "rot" in c:
        # one frequency for each rotated pair, in radians for each position
        st["inv_freq"] = BASE ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device=DEV) / c["rot"])
        st["sections"] = _sections(c)
        # which axis each pair turns by
        st["axis"] = torch.repeat_interleave(torch.arange(c["axes"]), torch.tensor(st["sections"])).to(DEV)
    if c["op"] == "rope":
        st["x"] = torch.randn(c["tokens"], c["heads"], c["d"], generator=g, device=DEV).to(t)
        st["pos"] = _positions(c, g, c["tokens"], c["far"])
        st["out"] = torch.empty_like(st["x"])
        return st
    q, kv = _lens(c)
    page, T = c["page"], sum(q)
    per = [-(-n // page) for n in kv]
    pool = sum(per) + 3
    order = torch.randperm(pool, generator=g, device=DEV).to(torch.int32)
    cols = max(per)
    st["max_q"], st["max_len"] = max(q), max(kv)
    # each sequence's pages from the shuffled pool; entries behind its last page name none
    n = torch.tensor(per, device=DEV)
    at = torch.arange(cols, device=DEV)[None, :] + (torch.cumsum(n, 0) - n)[:, None]
    st["table"] = torch.where(torch.arange(cols, device=DEV)[None, :] < n[:, None], order[at.clamp(max=pool - 1)], -1).to(torch.int32)
    st["seq_lens"] = torch.tensor(kv, dtype=torch.int32, device=DEV)
    st["cu_q"] = torch.tensor([0] + q, device=DEV).cumsum(0).to(torch.int32)
    rows = c["hq"] + 2 * c["hkv"]
    qkv = torch.randn(T, rows, c["d"], generator=g, device=DEV).to(t)         # one product's output, as a model has it
    st["q"], st["k"], st["v"] = qkv[:, :c["hq"]], qkv[:, c["hq"]:c["hq"] + c["hkv"]], qkv[:, c["hq"] + c["hkv"]:]
    shape = (pool, page, c["hkv"], c["d"])
    st["k_cache"] = torch.randn(shape, generator=g, device=DEV, dtype=t)
    st["v_cache"] = torch.randn(shape, generator=g, device=DEV, dtype=t)
    st["out"] = torch.empty(T, c["hq"], c["d"], dtype=t, device=DEV)
    if c["op"] == "append":
        st["pos"] = _positions(c, g, T, max(kv)) if c["axes"] > 1 else None   # text: a token's position is its place in the cache
    else:
        st["lse"] = torch.empty(T, c["hq"], dtype=torch.float32, device=DEV) if c["lse"] else None
        st["scale"] = c["d"] ** -0.5
    return st


# ---------------------------------------------------------------- plain forms
def _rotate(x, pos, st, sign):
    """x [T, H, d] in 32 bits, rotated by its positions [axes, T]; angles in 64 bits."""
    c = st["c"]
    half = c["rot"] // 2
    angle = pos.double()[st["axis"]].T * st["inv_freq"]                       # [T, rot/2]
    cos, sin = angle.cos().float()[:, None, :], sign * angle.sin().float()[:, None, :]
    a, b = (x[..., :half], x[..., half:c["rot"]]) if c["style"] == "half" else (x[..., 0:c["rot"]:2], x[..., 1:c["rot"]:2])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat((ra, rb), -1) if c["style"] == "half" else torch.stack((ra, rb), -1).flatten(-2)
    return torch.cat((turned, x[..., c["rot"]:]), -1)


def _places(st):
    """Each token's sequence and its place in it."""
    cu = st["cu_q"].long()
    token = torch.arange(st["q"].shape[0], device=DEV)
    s = torch.searchsorted(cu, token, right=True) - 1
    return s, st["seq_lens"].long()[s] - (cu[s + 1] - token)


def _plain_rope(st):
    return _rotate(st["x"].float(), st["pos"], st, -1.0 if st["c"]["inverse"] else 1.0).to(st["x"].dtype)


def _plain_append(st):
    s, place = _places(st)
    pos = st["pos"] if st["pos"] is not None else place[None, :]
    page = st["table"][s, place // st["c"]["page"]].long()
    slot = place % st["c"]["page"]
    st["k_cache"][page, slot] = _rotate(st["k"].float(), pos, st, 1.0).to(st["k"].dtype)
    st["v_cache"][page, slot] = st["v"]
    return _rotate(st["q"].float(), pos, st, 1.0).to(st["q"].dtype), st["k_cache"], st["v_cache"]


def _plain_attend(st):
    c = st["c"]
    B, n_q, n_k, hkv, G, d = c["seqs"], st["max_q"], st["max_len"], c["hkv"], c["hq"] // c["hkv"], c["d"]
    s, place = _places(st)
    row = torch.arange(st["q"].shape[0], device=DEV) - st["cu_q"].long()[s]
    table = st["table"].clamp(min=0).long()
    key = torch.arange(n_k, device=DEV)
    there = key[None, :] < st["seq_lens"][:, None]                             # [B, n_k]
    k = st["k_cache"][table].flatten(1, 2)[:, :n_k].float()                    # [B, n_k, hkv, d]
    v = st["v_cache"][table].flatten(1, 2)[:, :n_k].float()
    k, v = (torch.where(there[:, :, None, None], x, 0.0).permute(0, 2, 3, 1) for x in (k, v))
    q = torch.zeros(B, n_q, hkv, G, d, device=DEV)
    q[s, row] = st["q"].float().unflatten(1, (hkv, G))
    at = torch.full((B, n_q), -1, device=DEV)
    at[s, row] = place
    seen = (key <= at[:, :, None]) & there[:, None, :]                         # [B, n_q, n_k]
    if c["window"]:
        seen &= key > at[:, :, None] - c["window"]
    seen = seen[:, None, :, None, :]
    score = (q.permute(0, 2, 1, 3, 4).reshape(B, hkv, n_q * G, d) @ k).view(B, hkv, n_q, G, n_k)
    score = torch.where(seen, score.mul_(st["scale"]), -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(B, hkv, n_q * G, n_k) @ v.transpose(2, 3)).view(B, hkv, n_q, G, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 2, 1, 3, 4)[s, row].flatten(1, 2).to(st["q"].dtype)
    if not c["lse"]:
        return o
    return o, (top + total.log()).squeeze(-1).permute(0, 2, 1, 3)[s, row].flatten(1, 2)


# ---------------------------------------------------------------- the framework's calls
def _own(st):
    import paper_2609_11356_b200 as rg
    c = st["c"]
    if "desc" not in st:                                                        # descriptors and workspace are made once
        if "rot" in c:
            st["desc"] = rg.rg_rope_desc(rot_dim=c["rot"], style=rg.RG_ROPE_HALF if c["style"] == "half" else rg.RG_ROPE_PAIRS, sections=st["sections"],
                                         inverse=int(c.get("inverse", False)))
        else:
            st["desc"] = rg.rg_paged_attn_desc(scale=st["scale"], split=c["split"], window=c["window"])
        if c["op"] != "rope":
            st["seqs"] = rg.rg_paged_seqs(st["table"], st["seq_lens"], st["cu_q"], max_q=st["max_q"], max_len=st["max_len"])
        if c["op"] == "attend":
            need = rg.rg_paged_attention_workspace_bytes(st["desc"], st["seqs"], st["q"].shape[0], c["hq"], c["d"])
            st["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
    if c["op"] == "rope":
        return rg.rg_rope(st["desc"], st["x"], st["pos"], st["inv_freq"], st["out"])
    if c["op"] == "append":
        rg.rg_kv_append(st["desc"], st["k"], st["v"], st["inv_freq"], st["k_cache"], st["v_cache"], st["seqs"], pos=st["pos"], q=st["q"], q_out=st["out"])
        return st["out"], st["k_cache"], st["v_cache"]
    rg.rg_paged_attention(st["desc"], st["q"], st["k_cache"], st["v_cache"], st["seqs"], st["out"], lse=st["lse"], ws=st["ws"])
    return (st["out"], st["lse"]) if c["lse"] else st["out"]


def run(state):
    if own:
        return _own(state)
    return {"rope": _plain_rope, "append": _plain_append, "attend": _plain_attend}[state["c"]["op"]](state)


def work(case):
    c = case
    size = 4 if c["type"] == "fp32" else 2
    if c["op"] == "rope":
        n = c["tokens"] * c["heads"]
        return {"bytes": 2 * n * c["d"] * size + 4 * c["axes"] * c["tokens"] + 4 * c["rot"], "flops": 3 * n * c["rot"]}
    q, kv = _lens(c)
    T = sum(q)
    meta = 4 * (2 * len(q) + 1)
    if c["op"] == "append":
        rotated = T * (c["hq"] + c["hkv"])
        return {"bytes": 2 * (rotated + T * c["hkv"]) * c["d"] * size + meta + 4 * T + 4 * c["rot"], "flops": 3 * rotated * c["rot"]}
    w = c["window"] or 1 << 40
    keys = pairs = 0
    for n, m in zip(q, kv):
        first = m - n                                                           # the first new token's place
        keys += m - max(0, first - w + 1)
        if m <= w:                                                              # places first .. m-1 see place + 1 keys each
            pairs += (m * (m + 1) - first * (first + 1)) // 2
        else:
            pairs += sum(min(p + 1, w) for p in range(first, m))
    return {"bytes": 2 * keys * c["hkv"] * c["d"] * size + 2 * T * c["hq"] * c["d"] * size + meta + 4 * sum(-(-m // c["page"]) for m in kv) + (4 * T * c["hq"] if c["lse"] else 0),
            "flops": 4 * pairs * c["hq"] * c["d"]}


# ---------------------------------------------------------------- from the definitions, in 64 bits
def _turned(x, pos, st, sign):
    """Row by row as complex numbers: pair j of a head is multiplied by e^(i sign angle_j)."""
    c = st["c"]
    half = c["rot"] // 2
    x = x.double()
    first = torch.arange(half, device=DEV) * (1 if c["style"] == "half" else 2)
    second = first + (half if c["style"] == "half" else 1)
    angle = torch.empty(x.shape[0], half, dtype=torch.float64, device=DEV)
    at = 0
    for a, n in enumerate(st["sections"]):
        angle[:, at:at + n] = sign * torch.outer(pos[a].double(), st["inv_freq"][at:at + n])
        at += n
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones_like(angle), angle)[:, None, :]
    out = x.clone()
    out[..., first], out[..., second] = z.real, z.imag
    return out


def exact(case, seed):
    st = prepare(case, seed)
    c = case
    if c["op"] == "rope":
        return _turned(st["x"], st["pos"], st, -1.0 if c["inverse"] else 1.0)
    q, kv = _lens(c)
    if c["op"] == "append":
        pos = st["pos"]
        if pos is None:
            pos = torch.cat([torch.arange(m - n, m, device=DEV) for n, m in zip(q, kv)])[None]
        k, kc, vc = _turned(st["k"], pos, st, 1.0), st["k_cache"].double(), st["v_cache"].double()
        at = 0
        for i, (n, m) in enumerate(zip(q, kv)):
            p = torch.arange(m - n, m, device=DEV)
            page = st["table"][i].long()[p // c["page"]]
            kc[page, p % c["page"]] = k[at:at + n]
            vc[page, p % c["page"]] = st["v"][at:at + n].double()
            at += n
        return _turned(st["q"], pos, st, 1.0), kc, vc
    o = torch.zeros(sum(q), c["hq"], c["d"], dtype=torch.float64, device=DEV)
    lse = torch.full((sum(q), c["hq"]), -math.inf, dtype=torch.float64, device=DEV)
    G, at = c["hq"] // c["hkv"], 0
    for i, (n, m) in enumerate(zip(q, kv)):
        pages = st["table"][i, :-(-m // c["page"])].long()
        k, v = (x[pages].flatten(0, 1)[:m].double() for x in (st["k_cache"], st["v_cache"]))
        gap = torch.arange(m - n, m, device=DEV)[:, None] - torch.arange(m, device=DEV)[None, :]
        hidden = (gap < 0) | (gap >= (c["window"] or 1 << 40))
        for h in range(c["hq"]):
            score = (st["q"][at:at + n, h].double() @ k[:, h // G].T * st["scale"]).masked_fill(hidden, -math.inf)
            z = torch.logsumexp(score, -1)
            lse[at:at + n, h] = z
            o[at:at + n, h] = torch.exp(score - z[:, None]) @ v[:, h // G]
        at += n
    return (o, lse) if c["lse"] else o

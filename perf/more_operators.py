"""The operators of serving in four bits as they are measured: products of a few rows with 4-bit weights (`rg_gemv_four`), keys and
values put into a paged cache of 4-bit codes with the rotation on the way and read back (`rg_kv_append_four`, `rg_kv_read_four`), and attention
of new tokens over that cache (`rg_paged_attention_four`), each beside its plain form in elementary torch operations.

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
        # decode, one user: a square projection of one token, latency
        {"name": "gemv_token_square", "op": "gemv", "M": 1, "N": 4096, "K": 4096, "group": 128, "zeros": False, "scales": "bf16", "type": "bf16", "out": "bf16", "bias": False, "act": False, "residual": False},
        # decode, one user: gate and up projection in one product, zero points
        {"name": "gemv_token_up", "op": "gemv", "M": 1, "N": 28672, "K": 4096, "group": 128, "zeros": True, "scales": "fp16", "type": "fp16", "out": "fp16", "bias": False, "act": False, "residual": False},
        # decode, eight users: the product back down onto the residual stream
        {"name": "gemv_eight_down", "op": "gemv", "M": 8, "N": 4096, "K": 14336, "group": 64, "zeros": True, "scales": "bf16", "type": "bf16", "out": "bf16", "bias": False, "act": False, "residual": True},
        # drafts of a few users: 33 rows, odd width, small groups, bias and activation, results in 32 bits
        {"name": "gemv_drafts_odd", "op": "gemv", "M": 33, "N": 11009, "K": 4128, "group": 32, "zeros": False, "scales": "fp32", "type": "bf16", "out": "fp32", "bias": True, "act": True, "residual": False},
        # serving: 64 sequences get one token each
        {"name": "append_decode_64", "op": "append", "seqs": 64, "q_lo": 1, "q_hi": 1, "ctx_lo": 1, "ctx_hi": 8192, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "style": "half", "axes": 1, "page": 16, "type": "bf16", "shape": 1},
        # serving: prompts of ragged length, pages of 64
        {"name": "append_prompts", "op": "append", "seqs": 5, "q_lo": 500, "q_hi": 4096, "ctx_lo": 0, "ctx_hi": 2000, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "style": "half", "axes": 1, "page": 64, "type": "bf16", "shape": 2},
        # one user's next token on 8191 others: latency
        {"name": "attend_decode_1", "op": "attend", "seqs": 1, "q_lo": 1, "q_hi": 1, "ctx_lo": 8191, "ctx_hi": 8191, "hq": 32, "hkv": 8, "d": 128, "page": 16, "window": 0, "split": 256, "lse": False, "type": "bf16", "shape": 4},
        # a serving batch: one token for each of 64 sequences of ragged length
        {"name": "attend_decode_64", "op": "attend", "seqs": 64, "q_lo": 1, "q_hi": 1, "ctx_lo": 100, "ctx_hi": 8191, "hq": 32, "hkv": 8, "d": 128, "page": 16, "window": 0, "split": 512, "lse": False, "type": "bf16", "shape": 5},
        # long documents: few sequences, far apart in length, normalisers kept
        {"name": "attend_decode_long", "op": "attend", "seqs": 4, "q_lo": 1, "q_hi": 1, "ctx_lo": 30001, "ctx_hi": 65536, "hq": 64, "hkv": 8, "d": 128, "page": 64, "window": 0, "split": 512, "lse": True, "type": "bf16", "shape": 6},
        # draft tokens checked within a sliding window, heads of 64
        {"name": "attend_drafts_window", "op": "attend", "seqs": 33, "q_lo": 2, "q_hi": 5, "ctx_lo": 0, "ctx_hi": 6000, "hq": 16, "hkv": 2, "d": 64, "page": 32, "window": 2048, "split": 512, "lse": False, "type": "fp16", "shape": 7},
        # a step that mixes prompts' chunks with short ones
        {"name": "attend_mixed", "op": "attend", "seqs": 9, "q_lo": 1, "q_hi": 1000, "ctx_lo": 0, "ctx_hi": 3000, "hq": 32, "hkv": 8, "d": 128, "page": 16, "window": 0, "split": 0, "lse": True, "type": "bf16", "shape": 8},
        # a long prompt's next chunk
        {"name": "attend_chunk_4096", "op": "attend", "seqs": 1, "q_lo": 4096, "q_hi": 4096, "ctx_lo": 12288, "ctx_hi": 12288, "hq": 32, "hkv": 8, "d": 128, "page": 64, "window": 0, "split": 0, "lse": False, "type": "bf16", "shape": 9},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["gemv", "gemv", "append", "attend", "attend"])
    if op == "gemv":
        kind = rng.choice(["bf16", "bf16", "fp16"])
        c = {"op": op, "M": _log(rng, 1, 64), "group": rng.choice([32, 64, 128]), "zeros": rng.random() < 0.5, "scales": rng.choice(["bf16", "fp16", "fp32"]),
             "type": kind, "out": rng.choice([kind, kind, "fp32"]), "bias": rng.random() < 0.3, "act": rng.random() < 0.3, "residual": rng.random() < 0.3}
        while True:
            n, k = _log(rng, 64, 32768), 32 * _log(rng, 4, 896)
            if n * k <= 28672 * 4096:
                return c | {"N": n, "K": k}
    hkv = rng.choice([1, 2, 4, 8])
    c = {"op": op, "hq": hkv * rng.choice([1, 2, 4, 5, 7, 8]), "hkv": hkv, "d": rng.choice([32, 64, 96, 128, 128, 128]), "page": rng.choice([8, 16, 16, 24, 32, 64, 128, 256]),
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
        most = 2 ** 28 // (big["hkv"] * big["d"])               # padded keys of all sequences
        pairs = seqs * max(q) * max(kv) * big["hq"]              # the plain form's score matrix
        if seqs * max(kv) <= most and sum(q) <= 10752 and (op == "append" or pairs * big["d"] <= 32 * 4096 * 16384 * 128):
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
    w = (pairs - pairs // 4) // 2
    return (pairs - 2 * w, w, w)


def _scale_table():
    """Scale byte b stands for (8 + b % 8) 2^(b // 8 - 22)."""
    b = torch.arange(256, dtype=torch.float64, device=DEV)
    return (8 + b % 8) * torch.exp2(torch.floor(b / 8) - 22)


SHIFTS = (0, 16, 4, 20, 8, 24, 12, 28)                          # where the 8 elements of a 32-bit word lie in it


def _quantise(x):
    """x [..., d] in 64 bits -> codes [..., d] (0 .. 15) and scale bytes [..., d / 16]."""
    table = _scale_table()
    g = x.unflatten(-1, (-1, 16))
    b = torch.searchsorted(7.5 * table, g.abs().amax(-1)).clamp_(max=255)
    code = torch.round(g / table[b][..., None]).clamp_(-8, 7) + 8
    return code.flatten(-2).to(torch.int32), b.to(torch.uint8)


def _words(code):
    """Codes [..., d] -> bytes [..., d / 32, 16] as they lie in the cache."""
    c = code.unflatten(-1, (-1, 8))
    w = c[..., 0].clone()
    for e in range(1, 8):
        w |= c[..., e] << SHIFTS[e]
    return w.view(torch.uint8).unflatten(-1, (-1, 16))


def _parts(cache, d):
    """The code bytes [pages, heads, tiles of 8 slots, d / 32, 8, 16] and scale bytes [pages, heads, tiles, d / 32, 8, 2] of a cache, as views."""
    t = cache.unflatten(-1, (-1, 9 * d // 2))
    return t[..., :4 * d].unflatten(-1, (d // 32, 8, 16)), t[..., 4 * d:].unflatten(-1, (d // 32, 8, 2))


def _values(cache, d):
    """What a cache [..., heads, block] stands for: [..., heads, slots, d] in 32 bits."""
    codes, scales = _parts(cache, d)
    w = codes.contiguous().view(torch.int32)                                  # [..., tiles, d / 32, 8, 4]
    e = (w[..., None] >> torch.tensor(SHIFTS, dtype=torch.int32, device=DEV)).bitwise_and_(15).sub_(8)
    e = e.to(torch.float32).unflatten(-2, (2, 2)).flatten(-2)                # [..., tiles, d / 32, 8, 2 groups, 16]
    e *= _scale_table().float()[scales.long()][..., None]
    return e.flatten(-2).transpose(-3, -2).flatten(-2).flatten(-3, -2)


def _filled(g, pages, heads, page, d):
    """A cache as earlier steps left it: normal values, quantised; made in pieces."""
    cache = torch.empty(pages, heads, page * 9 * d // 16, dtype=torch.uint8, device=DEV)
    step = max(1, 2 ** 25 // (heads * page * d))
    for a in range(0, pages, step):
        part = cache[a:a + step]
        codes, scales = _parts(part, d)
        code, b = _quantise(torch.randn(part.shape[0], heads, page // 8, 8, d, generator=g, device=DEV).double())
        codes.copy_(_words(code).transpose(-3, -2))
        scales.copy_(b.unflatten(-1, (-1, 2)).transpose(-3, -2))
    return cache


def _weights(c, g, st):
    """Normal weights in groups, rounded to 16 levels: symmetric about 8, or between each group's least and largest value."""
    N, K, n = c["N"], c["K"], -(-c["K"] // c["group"])
    st["codes"] = torch.empty(N, K // 2, dtype=torch.uint8, device=DEV)
    st["scales"] = torch.empty(N, n, dtype=TYPES[c["scales"]], device=DEV)
    st["zeros"] = torch.empty(N, n, dtype=torch.uint8, device=DEV) if c["zeros"] else None
    step = max(1, 2 ** 25 // K)
    for a in range(0, N, step):
        w = torch.nn.functional.pad(torch.randn(min(step, N - a), K, generator=g, device=DEV) * K ** -0.5, (0, n * c["group"] - K)).unflatten(-1, (n, c["group"]))
        if c["zeros"]:
            lo, hi = w.amin(-1).clamp(max=0), w.amax(-1).clamp(min=0)
            s = ((hi - lo) / 15).to(TYPES[c["scales"]])
            z = torch.round(-lo / s.float()).clamp(0, 15)
            st["zeros"][a:a + step] = z.to(torch.uint8)
        else:
            s = (w.abs().amax(-1) / 7.5).to(TYPES[c["scales"]])
            z = torch.full_like(s, 8, dtype=torch.float32)
        st["scales"][a:a + step] = s
        u = (torch.round(w / s.float()[..., None]) + z[..., None]).clamp(0, 15).to(torch.uint8).flatten(-2)[:, :K]
        st["codes"][a:a + step] = u[:, 0::2] | u[:, 1::2] << 4


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
    if c["op"] == "gemv":
        _weights(c, g, st)
        st["x"] = torch.randn(c["M"], c["K"], generator=g, device=DEV).to(t)
        o = TYPES[c["out"]]
        st["bias"] = torch.randn(c["N"], generator=g, device=DEV).to(t) if c["bias"] else None
        st["residual"] = torch.randn(c["M"], c["N"], generator=g, device=DEV).to(t) if c["residual"] else None
        st["out"] = torch.empty(c["M"], c["N"], dtype=o, device=DEV)
        return st
    if c["op"] == "append":
        # one frequency for each rotated pair, in radians for each position
        st["inv_freq"] = BASE ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device=DEV) / c["rot"])
        st["sections"] = _sections(c)
        # which axis each pair turns by
        st["axis"] = torch.repeat_interleave(torch.arange(c["axes"]), torch.tensor(st["sections"])).to(DEV)
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
    st["k_cache"], st["v_cache"] = (_filled(g, pool, c["hkv"], page, c["d"]) for _ in range(2))
    st["out"] = torch.empty(T, c["hq"], c["d"], dtype=t, device=DEV)
    if c["op"] == "append":
        st["pos"] = _positions(c, g, T, max(kv)) if c["axes"] > 1 else None   # text: a token's position is its place in the cache
        st["k_out"], st["v_out"] = torch.empty(2, T, c["hkv"], c["d"], dtype=t, device=DEV)
    else:
        st["lse"] = torch.empty(T, c["hq"], dtype=torch.float32, device=DEV) if c["lse"] else None
        st["scale"] = c["d"] ** -0.5
    return st


# ---------------------------------------------------------------- plain forms
def _plain_gemv(st):
    c = st["c"]
    u = torch.stack((st["codes"] & 15, st["codes"] >> 4), -1).flatten(-2).float()
    zero = st["zeros"].float() if c["zeros"] else torch.full_like(st["scales"], 8, dtype=torch.float32)
    u -= zero.repeat_interleave(c["group"], 1)[:, :c["K"]]
    u *= st["scales"].float().repeat_interleave(c["group"], 1)[:, :c["K"]]
    y = st["x"].float() @ u.T
    if c["bias"]:
        y += st["bias"].float()
    if c["act"]:
        y = y / (1 + torch.exp(-y))
    if c["residual"]:
        y += st["residual"].float()
    return y.to(st["out"].dtype)


def _rotate(x, pos, st):
    """x [T, H, d] rotated by its positions [axes, T], in the type of x; angles in 64 bits."""
    c = st["c"]
    half = c["rot"] // 2
    angle = pos.double()[st["axis"]].T * st["inv_freq"]                       # [T, rot/2]
    cos, sin = angle.cos().to(x.dtype)[:, None, :], angle.sin().to(x.dtype)[:, None, :]
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


def _plain_append(st):
    c, t = st["c"], st["q"].dtype
    s, place = _places(st)
    pos = st["pos"] if st["pos"] is not None else place[None, :]
    page = st["table"][s, place // c["page"]].long()
    tile, slot = place % c["page"] // 8, place % 8
    out = [_rotate(st["q"].float(), pos, st).to(t)]
    # keys next to a border between two codes: in 64 bits
    for x, cache in ((_rotate(st["k"].double(), pos, st), st["k_cache"]), (st["v"].double(), st["v_cache"])):
        code, b = _quantise(x)
        codes, scales = _parts(cache, c["d"])
        codes[page, :, tile, :, slot] = _words(code)
        scales[page, :, tile, :, slot] = b.unflatten(-1, (-1, 2))
        codes, scales = codes[page, :, tile, :, slot], scales[page, :, tile, :, slot]      # and back: [T, H, d / 32, 16 and 2]
        w = codes.contiguous().view(torch.int32)
        e = ((w[..., None] >> torch.tensor(SHIFTS, dtype=torch.int32, device=DEV) & 15) - 8).float().flatten(-2).unflatten(-1, (2, 16))
        out.append((e * _scale_table().float()[scales.long()][..., None]).flatten(-3).to(t))
    return tuple(out)


def _plain_attend(st):
    c = st["c"]
    B, n_q, n_k, hkv, G, d = c["seqs"], st["max_q"], st["max_len"], c["hkv"], c["hq"] // c["hkv"], c["d"]
    s, place = _places(st)
    row = torch.arange(st["q"].shape[0], device=DEV) - st["cu_q"].long()[s]
    table = st["table"].clamp(min=0).long()
    key = torch.arange(n_k, device=DEV)
    there = key[None, :] < st["seq_lens"][:, None]                             # [B, n_k]
    # the caches' values once, then each sequence's pages: [pages, hkv, page, d] -> [B, hkv, n_k, d]
    k, v = (_values(x, d)[table].transpose(1, 2).flatten(2, 3)[:, :, :n_k] for x in (st["k_cache"], st["v_cache"]))
    k, v = (torch.where(there[:, None, :, None], x, 0.0) for x in (k, v))
    q = torch.zeros(B, n_q, hkv, G, d, device=DEV)
    q[s, row] = st["q"].float().unflatten(1, (hkv, G))
    at = torch.full((B, n_q), -1, device=DEV)
    at[s, row] = place
    seen = (key <= at[:, :, None]) & there[:, None, :]                         # [B, n_q, n_k]
    if c["window"]:
        seen &= key > at[:, :, None] - c["window"]
    seen = seen[:, None, :, None, :]
    score = (q.permute(0, 2, 1, 3, 4).reshape(B, hkv, n_q * G, d) @ k.transpose(2, 3)).view(B, hkv, n_q, G, n_k)
    score = torch.where(seen, score.mul_(st["scale"]), -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(B, hkv, n_q * G, n_k) @ v).view(B, hkv, n_q, G, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 2, 1, 3, 4)[s, row].flatten(1, 2).to(st["q"].dtype)
    if not c["lse"]:
        return o
    return o, (top + total.log()).squeeze(-1).permute(0, 2, 1, 3)[s, row].flatten(1, 2)


# ---------------------------------------------------------------- the framework's calls
def _own(st):
    import paper_2609_11356_b200 as rg
    c = st["c"]
    if "ready" not in st:                                                       # descriptors, handles and workspace are made once
        st["ready"] = True
        if c["op"] == "gemv":
            st["w"] = rg.rg_weights_four(st["codes"], st["scales"], zeros=st["zeros"], group=c["group"])
        else:
            st["seqs"] = rg.rg_paged_seqs(st["table"], st["seq_lens"], st["cu_q"], max_q=st["max_q"], max_len=st["max_len"])
            st["kc"], st["vc"] = (rg.rg_cache_four(x, page_size=c["page"], dim=c["d"]) for x in (st["k_cache"], st["v_cache"]))
        if c["op"] == "append":
            st["desc"] = rg.rg_rope_desc(rot_dim=c["rot"], style=rg.RG_ROPE_HALF if c["style"] == "half" else rg.RG_ROPE_PAIRS, sections=st["sections"])
        if c["op"] == "attend":
            st["desc"] = rg.rg_paged_attn_desc(scale=st["scale"], split=c["split"], window=c["window"])
            need = rg.rg_paged_attention_workspace_bytes(st["desc"], st["seqs"], st["q"].shape[0], c["hq"], c["d"])
            st["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
    if c["op"] == "gemv":
        return rg.rg_gemv_four(st["w"], st["x"], st["out"], bias=st["bias"], act=int(c["act"]), residual=st["residual"])
    if c["op"] == "append":
        rg.rg_kv_append_four(st["desc"], st["k"], st["v"], st["inv_freq"], st["kc"], st["vc"], st["seqs"], pos=st["pos"], q=st["q"], q_out=st["out"])
        rg.rg_kv_read_four(st["kc"], st["vc"], st["seqs"], st["k_out"], st["v_out"])
        return st["out"], st["k_out"], st["v_out"]
    rg.rg_paged_attention_four(st["desc"], st["q"], st["kc"], st["vc"], st["seqs"], st["out"], lse=st["lse"], ws=st["ws"])
    return (st["out"], st["lse"]) if c["lse"] else st["out"]


def run(state):
    if own:
        return _own(state)
    return {"gemv": _plain_gemv, "append": _plain_append, "attend": _plain_attend}[state["c"]["op"]](state)


def work(case):
    c = case
    size = {"fp32": 4, "bf16": 2, "fp16": 2}
    if c["op"] == "gemv":
        M, N, K, groups = c["M"], c["N"], c["K"], c["N"] * -(-c["K"] // c["group"])
        more = (size[c["type"]] * N if c["bias"] else 0) + (size[c["type"]] * M * N if c["residual"] else 0)
        return {"bytes": N * K // 2 + groups * (size[c["scales"]] + int(c["zeros"])) + M * K * size[c["type"]] + M * N * size[c["out"]] + more, "flops": 2 * M * N * K}
    q, kv = _lens(c)
    T = sum(q)
    meta = 4 * (2 * len(q) + 1)
    if c["op"] == "append":
        rotated = T * (c["hq"] + c["hkv"])
        # rows in, queries out, codes and scales written and read back, their values out
        return {"bytes": 2 * T * c["d"] * (2 * c["hq"] + 4 * c["hkv"]) + 2 * 2 * T * c["hkv"] * 9 * c["d"] // 16 + 2 * meta + 8 * T + 4 * c["rot"], "flops": 3 * rotated * c["rot"]}
    w = c["window"] or 1 << 40
    keys = pairs = 0
    for n, m in zip(q, kv):
        first = m - n                                                           # the first new token's place
        keys += m - max(0, first - w + 1)
        if m <= w:                                                              # places first .. m-1 see place + 1 keys each
            pairs += (m * (m + 1) - first * (first + 1)) // 2
        else:
            pairs += sum(min(p + 1, w) for p in range(first, m))
    return {"bytes": 2 * keys * c["hkv"] * 9 * c["d"] // 16 + 4 * T * c["hq"] * c["d"] + meta + 4 * sum(-(-m // c["page"]) for m in kv) + (4 * T * c["hq"] if c["lse"] else 0),
            "flops": 4 * pairs * c["hq"] * c["d"]}


# ---------------------------------------------------------------- from the definitions, in 64 bits
def _turned(x, pos, st):
    """Row by row as complex numbers: pair j of a head is multiplied by e^(i angle_j)."""
    c = st["c"]
    half = c["rot"] // 2
    x = x.double()
    first = torch.arange(half, device=DEV) * (1 if c["style"] == "half" else 2)
    second = first + (half if c["style"] == "half" else 1)
    angle = torch.empty(x.shape[0], half, dtype=torch.float64, device=DEV)
    at = 0
    for a, n in enumerate(st["sections"]):
        angle[:, at:at + n] = torch.outer(pos[a].double(), st["inv_freq"][at:at + n])
        at += n
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones_like(angle), angle)[:, None, :]
    out = x.clone()
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _in_four_bits(x):
    """What 16 values become: multiples of a step of four significant bits, the smallest one for which 7.5 steps reach the largest of them."""
    g = x.unflatten(-1, (-1, 16))
    m, e = torch.frexp(g.abs().amax(-1, keepdim=True) / 7.5)
    step = torch.ldexp(torch.ceil(16 * m), e - 4).clamp(2.0 ** -19, 7680.0)
    return (torch.round(g / step).clamp(-8, 7) * step).flatten(-2)


def _held(cache, d):
    """The values of blocks [n, block bytes] of one head: [n, slots, d], byte by byte."""
    t = cache.view(cache.shape[0], -1, 9 * d // 2)
    v = torch.empty(cache.shape[0], t.shape[1], 8, d, dtype=torch.float64, device=DEV)
    for chunk in range(d // 32):
        for byte in range(16):
            b = t[:, :, 128 * chunk:128 * chunk + 128].unflatten(-1, (8, 16))[..., byte].double()
            scale = t[:, :, 4 * d + 16 * chunk:4 * d + 16 * chunk + 16].unflatten(-1, (8, 2))[..., byte // 8].double()
            step = (8 + scale % 8) / 8 * 2.0 ** (torch.floor(scale / 8) - 19)
            # bytes 0 .. 3 of a word: elements 0 and 2, 4 and 6, 1 and 3, 5 and 7
            first = 32 * chunk + byte // 4 * 8 + (0, 4, 1, 5)[byte % 4]
            v[..., first], v[..., first + 2] = (b % 16 - 8) * step, (torch.floor(b / 16) - 8) * step
    return v.flatten(1, 2)


def exact(case, seed):
    st = prepare(case, seed)
    c = case
    if c["op"] == "gemv":
        y = torch.zeros(c["M"], c["N"], dtype=torch.float64, device=DEV)
        x = st["x"].double()
        for i in range(st["scales"].shape[1]):
            a, b = i * c["group"], min((i + 1) * c["group"], c["K"])
            byte = st["codes"][:, a // 2:b // 2].double()
            zero = st["zeros"][:, i, None].double() if c["zeros"] else 8.0
            high = torch.floor(byte / 16)
            y += (x[:, a:b:2] @ (byte - 16 * high - zero).T + x[:, a + 1:b:2] @ (high - zero).T) * st["scales"][:, i].double()
        if c["bias"]:
            y += st["bias"].double()
        if c["act"]:
            y *= torch.sigmoid(y)
        return y + st["residual"].double() if c["residual"] else y
    q, kv = _lens(c)
    if c["op"] == "append":
        pos = st["pos"]
        if pos is None:
            pos = torch.cat([torch.arange(m - n, m, device=DEV) for n, m in zip(q, kv)])[None]
        return _turned(st["q"], pos, st), _in_four_bits(_turned(st["k"], pos, st)), _in_four_bits(st["v"].double())
    o = torch.zeros(sum(q), c["hq"], c["d"], dtype=torch.float64, device=DEV)
    lse = torch.full((sum(q), c["hq"]), -math.inf, dtype=torch.float64, device=DEV)
    G, at = c["hq"] // c["hkv"], 0
    for i, (n, m) in enumerate(zip(q, kv)):
        pages = st["table"][i, :-(-m // c["page"])].long()
        gap = torch.arange(m - n, m, device=DEV)[:, None] - torch.arange(m, device=DEV)[None, :]
        hidden = (gap < 0) | (gap >= (c["window"] or 1 << 40))
        for kh in range(c["hkv"]):
            k, v = (_held(x[pages, kh], c["d"]).flatten(0, 1)[:m] for x in (st["k_cache"], st["v_cache"]))
            for h in range(kh * G, kh * G + G):
                score = (st["q"][at:at + n, h].double() @ k.T * st["scale"]).masked_fill(hidden, -math.inf)
                z = torch.logsumexp(score, -1)
                lse[at:at + n, h] = z
                o[at:at + n, h] = torch.exp(score - z[:, None]) @ v
        at += n
    return (o, lse) if c["lse"] else o

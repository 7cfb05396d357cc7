"""Helpers for the tests of rotary positions, the paged cache and attention over it: batches laid out as a server lays them
out, and the definitions in 64 bits."""
import math

import torch

import paper_2609_11356_b200 as rg

DEV = "cuda"
EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}      # half a step, relative


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def inv_freq(rot, base=10000.0):
    return base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)


def rotate64(x, pos, freq, sections, style, sign=1.0):
    """x [T, H, d] rotated in 64 bits; pos [axes, T]."""
    x = x.double()
    half = freq.numel()
    axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections)).to(x.device)
    angle = sign * pos.double()[axis].T * freq
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    first = torch.arange(half, device=x.device) * (1 if style == rg.RG_ROPE_HALF else 2)
    second = first + (half if style == rg.RG_ROPE_HALF else 1)
    a, b = x[..., first], x[..., second]
    y = x.clone()
    y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
    size = x.abs().clone()                                     # what a rounding inside the rotation is relative to
    size[..., first] = size[..., second] = a.abs() + b.abs()
    return y, size


def rotation_bound(y, size, dtype):
    """Angle: the fraction of a turn (at most 1/2) rounded to fp32 is off by 2^-26 of a turn at most: 2 pi 2^-26 < 2^-23 rad.  Sine and
    cosine: 2^-23 each from the function, and the rounding of 2 * fraction is exact.  Products and sum: 3 roundings of 2^-24.  Together under
    2^-21 (|a| + |b|); then one rounding to the output type (2^-25: half of fp16's smallest step)."""
    return 2.0 ** -21 * size + EPS[dtype] * (y.abs() + 2.0 ** -21 * size) + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -140)


class Batch:
    """Sequences with `q[i]` new tokens at the end of `kv[i]` in all, their pages dealt at random from one pool."""

    def __init__(self, q, kv, *, hq, hkv, d, page, dtype=torch.bfloat16, seed=0, spare=3, heads_first=False, garbage=float("nan"), tail_rows=0, spread=1.0):
        g = generator(seed)
        self.q_lens, self.kv_lens, self.hq, self.hkv, self.d, self.page, self.dtype = q, kv, hq, hkv, d, page, dtype
        per = [-(-n // page) for n in kv]
        pool = sum(per) + spare
        order = torch.randperm(pool, generator=g, device=DEV).tolist()
        cols = max(per + [1])
        table = torch.full((len(q), cols), -7, dtype=torch.int32)            # entries behind the last page are never read
        at = 0
        for i, n in enumerate(per):
            table[i, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        self.table = table.to(DEV)
        self.seq_lens = torch.tensor(kv, dtype=torch.int32, device=DEV)
        self.cu_q = torch.tensor([0] + q).cumsum(0).to(torch.int32).to(DEV)
        self.T = sum(q) + tail_rows
        self.Q = (torch.randn(self.T, hq, d, generator=g, device=DEV) * spread).to(dtype)
        shape = (pool, hkv, page, d) if heads_first else (pool, page, hkv, d)
        self.kc = torch.full(shape, garbage, dtype=dtype, device=DEV)
        self.vc = torch.full(shape, garbage, dtype=dtype, device=DEV)
        if heads_first:
            self.kc, self.vc = self.kc.transpose(1, 2), self.vc.transpose(1, 2)
        self.K = [(torch.randn(n, hkv, d, generator=g, device=DEV) * spread).to(dtype) for n in kv]
        self.V = [torch.randn(n, hkv, d, generator=g, device=DEV).to(dtype) for n in kv]
        self.store()

    def where(self, i, n=None):
        n = self.kv_lens[i] if n is None else n
        p = torch.arange(n, device=DEV)
        return self.table[i].long()[p // self.page], p % self.page

    def store(self):
        for i, n in enumerate(self.kv_lens):
            if n:
                page, slot = self.where(i)
                self.kc[page, slot], self.vc[page, slot] = self.K[i], self.V[i]

    def seqs(self, **kw):
        kw.setdefault("max_q", max(self.q_lens + [0]))
        kw.setdefault("max_len", max(self.kv_lens + [0]))
        return rg.rg_paged_seqs(self.table, self.seq_lens, self.cu_q, **kw)


def attend(b, *, scale=None, split=0, window=0, mask=1, out_dtype=None, lse=True, q=None, seqs=None, ws_fill=0xFF):
    """The call, with a poisoned output, normalisers and workspace."""
    q = b.Q if q is None else q
    seqs = b.seqs() if seqs is None else seqs
    d = rg.rg_paged_attn_desc(scale=b.d ** -0.5 if scale is None else scale, split=split, window=window, mask=mask)
    out = torch.full(q.shape, 77.0, dtype=b.dtype if out_dtype is None else out_dtype, device=DEV)
    z = torch.full(q.shape[:2], 77.0, dtype=torch.float32, device=DEV) if lse else None
    need = rg.rg_paged_attention_workspace_bytes(d, seqs, q.shape[0], b.hq, b.d, page_size=b.page)
    ws = torch.full((need,), ws_fill, dtype=torch.uint8, device=DEV) if need else None
    rg.rg_paged_attention(d, q, b.kc, b.vc, seqs, out, lse=z, ws=ws)
    return out, z


def attention64(q, k, v, scale, window=0, mask=1):
    """Rows q [n, hq, d] at the end of k, v [m, hkv, d]: output, normaliser, sum of weights times |v| and the size of the scores' error."""
    n, hq, d = q.shape
    m, hkv = k.shape[:2]
    G = hq // hkv
    q, k, v = q.double(), k.double(), v.double()
    kk, vv = k.repeat_interleave(G, 1).permute(1, 2, 0), v.repeat_interleave(G, 1).permute(1, 0, 2)
    s = q.permute(1, 0, 2) @ kk * scale
    gap = (torch.arange(m - n, m, device=q.device)[:, None] - torch.arange(m, device=q.device)[None, :])
    hidden = torch.zeros_like(gap, dtype=torch.bool) if not mask else (gap < 0) | (gap >= (window or 1 << 40))
    s = s.masked_fill(hidden, -math.inf)
    size = (q.abs().permute(1, 0, 2) @ kk.abs() * scale).masked_fill(hidden, 0).amax(-1)
    z = torch.logsumexp(s, -1)
    w = torch.exp(s - z[..., None])
    w = torch.where(torch.isnan(w), 0.0, w)
    return (w @ vv).permute(1, 0, 2), z.T, (w @ vv.abs()).permute(1, 0, 2), size.T


def attention_bounds(o, mass, size, d, keys, p_dtype, out_dtype):
    """Scores: each of the ceil(d / 16) tensor-core steps rounds a sum of at most `size` by 2^-23 or less, then one fp32 rounding of the
    scaled score's distance from the maximum (2^-24 of at most 2 `size`): ds = (d / 16 + 4) 2^-23 size.  A weight is off by a factor of 1 +- (2 ds + 2^-20)
    with numerator and sum (2^-20: the exponentials and the fp32 sum's order), the narrowed weight by half a step of its type, and the
    keys / 16 steps of the product by 2^-23 of the running sum each; then one rounding."""
    ds = (d / 16 + 4) * 2.0 ** -23 * size
    rel = EPS[p_dtype] + 2 * ds[..., None] + 2.0 ** -20 + (keys / 16 + 16) * 2.0 ** -23
    err = rel * mass
    return err + EPS[out_dtype] * (o.abs() + err) + (2.0 ** -25 if out_dtype == torch.float16 else 0), ds + 2.0 ** -20 * 2 + 2.0 ** -23 * 16


def check(b, out, z, *, scale=None, window=0, mask=1):
    scale = b.d ** -0.5 if scale is None else scale
    at = 0
    for i, (n, m) in enumerate(zip(b.q_lens, b.kv_lens)):
        if n == 0:
            continue
        o, lse, mass, size = attention64(b.Q[at:at + n], b.K[i], b.V[i], scale, window, mask)
        bound, bound_z = attention_bounds(o, mass, size, b.d, m, b.dtype, out.dtype)
        got = out[at:at + n].double()
        off = (got - o).abs() - bound
        assert bool((off <= 0).all()), f"sequence {i} ({n} of {m}): output off by {off.max().item()} more than its bound at {(off == off.max()).nonzero()[0].tolist()}"
        if z is not None:
            offz = (z[at:at + n].double() - lse).abs() - bound_z - 2.0 ** -23 * lse.abs()
            assert bool((offz <= 0).all()), f"sequence {i}: normaliser off by {offz.max().item()} more than its bound"
        at += n
    assert bool((out[at:] == 77.0).all()) and (z is None or bool((z[at:] == 77.0).all())), "rows behind the last sequence were written"

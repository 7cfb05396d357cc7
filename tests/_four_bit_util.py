"""Helpers for the tests of the four-bit operators: the formats in plain torch, written from their definitions, and batches whose caches hold codes."""
import math

import torch

import paper_2609_11356_b200 as rg
from tests._paged_util import DEV, Batch, attention64, attention_bounds

NIBBLE = (0, 4, 1, 5, 2, 6, 3, 7)                            # the nibble of a word that element e of its eight is in


def scale_values(device=DEV):
    return torch.tensor([math.ldexp(8 + b % 8, b // 8 - 22) for b in range(256)], dtype=torch.float64, device=device)


def to_codes(x):
    """x [..., d] in 64 bits -> codes -8..7 [..., d] and scale bytes [..., d / 16]: the smallest scale of which 7.5 reach the group's largest magnitude."""
    x = torch.where(torch.isnan(x), 0.0, x).unflatten(-1, (-1, 16))
    s = scale_values(x.device)
    b = (7.5 * s[:-1] < x.abs().amax(-1)[..., None]).sum(-1)
    c = torch.round(x.clamp(-1e300, 1e300) / s[b][..., None]).clamp(-8, 7)
    return c.flatten(-2).to(torch.int64), b


def from_codes(c, b):
    return (c.unflatten(-1, (-1, 16)) * scale_values(c.device)[b][..., None]).flatten(-2)


def slot_bytes(c, b):
    """Codes and scale bytes of one slot [..., d] -> its bytes as they lie in a tile: [..., d / 32, 16] and [..., d / 32, 2]."""
    w = sum((c[..., e::8] + 8) << (4 * NIBBLE[e]) for e in range(8))
    return torch.stack([(w >> (8 * i)) & 255 for i in range(4)], -1).flatten(-2).unflatten(-1, (-1, 16)).to(torch.uint8), b.unflatten(-1, (-1, 2)).to(torch.uint8)


def tile_views(cache, d):
    """The code bytes [pages, heads, tiles, d / 32, 8, 16] and scale bytes [pages, heads, tiles, d / 32, 8, 2] of a cache tensor."""
    t = cache.unflatten(-1, (-1, 9 * d // 2))
    return t[..., :4 * d].unflatten(-1, (d // 32, 8, 16)), t[..., 4 * d:].unflatten(-1, (d // 32, 8, 2))


def values(cache, d):
    """What a cache tensor holds, in 64 bits: [pages, heads, slots, d]."""
    codes, scales = tile_views(cache, d)
    b = codes.long()
    w = b[..., 0::4] | b[..., 1::4] << 8 | b[..., 2::4] << 16 | b[..., 3::4] << 24                       # [..., chunk, 8, 4]
    c = torch.stack([(w >> (4 * NIBBLE[e])) & 15 for e in range(8)], -1).flatten(-2) - 8               # [..., chunk, 8, 32]
    v = c.unflatten(-1, (2, 16)) * scale_values(cache.device)[scales.long()][..., None]
    return v.flatten(-2).transpose(-3, -2).flatten(-2).flatten(-3, -2)


class Batch4(Batch):
    """A Batch whose caches are random codes and scales all over (so unused slots hold garbage); its 16-bit caches hold the same values."""

    def __init__(self, *a, lowest=128, highest=160, pages_inner=False, **kw):
        super().__init__(*a, **kw)
        g = torch.Generator(device=DEV)
        g.manual_seed(kw.get("seed", 0) + 1000)
        pool, d = self.kc.shape[0], self.d
        block = rg.rg_cache_four_block_bytes(self.page, d)

        def make():
            t = torch.randint(0, 256, (pool, self.hkv, block), generator=g, device=DEV, dtype=torch.uint8)
            if pages_inner:
                t = t.transpose(0, 1).contiguous().transpose(0, 1)
            tile_views(t, d)[1].copy_(torch.randint(lowest, highest, tile_views(t, d)[1].shape, generator=g, device=DEV, dtype=torch.uint8))
            return t

        self.k4, self.v4 = make(), make()
        self.refresh()

    def refresh(self):
        """The 16-bit caches and the sequences' keys and values from the codes."""
        for t, c, rows in ((self.k4, self.kc, self.K), (self.v4, self.vc, self.V)):
            c.copy_(values(t, self.d).transpose(1, 2).to(self.dtype))
            for i, n in enumerate(self.kv_lens):
                if n:
                    page, slot = self.where(i)
                    rows[i] = c[page, slot]
        self.c4 = [rg.rg_cache_four(t, page_size=self.page, dim=self.d) for t in (self.k4, self.v4)]


def attend4(b, *, scale=None, split=0, window=0, mask=1, out_dtype=None, lse=True, q=None, seqs=None):
    """The call, with a poisoned output, normalisers and workspace."""
    q = b.Q if q is None else q
    seqs = b.seqs() if seqs is None else seqs
    d = rg.rg_paged_attn_desc(scale=b.d ** -0.5 if scale is None else scale, split=split, window=window, mask=mask)
    out = torch.full(q.shape, 77.0, dtype=b.dtype if out_dtype is None else out_dtype, device=DEV)
    z = torch.full(q.shape[:2], 77.0, dtype=torch.float32, device=DEV) if lse else None
    need = rg.rg_paged_attention_workspace_bytes(d, seqs, q.shape[0], b.hq, b.d, page_size=b.page)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV) if need else None
    rg.rg_paged_attention_four(d, q, *b.c4, seqs, out, lse=z, ws=ws)
    return out, z


def check4(b, out, z, *, scale=None, window=0, mask=1):
    """The answer against the definition in 64 bits, within attention_bounds and, in fp16, what weights below its normal numbers lose: 2^7 p is narrowed, so a weight p with
    2^7 p < 2^-14 is off by half a subnormal step, 2^-25, at most: p by 2^-32.  The row's sum l is at least 1 (the running maximum is some key's own
    score), so the result is off by at most 2^-32 of the sum of |v| over the keys that it sees: at most those of the sequence."""
    scale = b.d ** -0.5 if scale is None else scale
    at = 0
    for i, (n, m) in enumerate(zip(b.q_lens, b.kv_lens)):
        if n == 0:
            continue
        o, lse, mass, size = attention64(b.Q[at:at + n], b.K[i], b.V[i], scale, window, mask)
        bound, bound_z = attention_bounds(o, mass, size, b.d, m, b.dtype, out.dtype)
        if b.dtype == torch.float16:
            bound = bound + 2.0 ** -32 * b.V[i].double().abs().sum(0).repeat_interleave(b.hq // b.hkv, 0)
        off = (out[at:at + n].double() - o).abs() - bound
        assert bool((off <= 0).all()), f"sequence {i} ({n} of {m}): output off by {off.max().item()} more than its bound at {(off == off.max()).nonzero()[0].tolist()}"
        offz = (z[at:at + n].double() - lse).abs() - bound_z - 2.0 ** -23 * lse.abs()
        assert bool((offz <= 0).all()), f"sequence {i}: normaliser off by {offz.max().item()} more than its bound"
        at += n
    assert bool((out[at:] == 77.0).all()) and bool((z[at:] == 77.0).all()), "rows behind the last sequence were written"

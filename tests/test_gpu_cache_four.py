"""Rows into a paged cache of four-bit codes and back, on the GPU: every byte against the definition in 64 bits."""
import pytest
import torch

import paper_2609_11356_b200 as rg
from tests._four_bit_util import from_codes, scale_values, slot_bytes, tile_views, to_codes, values
from tests._paged_util import DEV, generator, inv_freq, rotate64

pytestmark = pytest.mark.gpu
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(autouse=True)
def healthy():
    yield
    assert rg.rg_device_status() == 0


class Case:
    """New tokens of sequences whose pages lie anywhere, caches full of garbage."""

    def __init__(self, q, kv, *, hkv=2, hq=4, d=64, page=16, dtype=BF, seed=0, tail_rows=0, pages_inner=False, spread=1.0):
        g = generator(seed)
        self.q_lens, self.kv_lens, self.hkv, self.hq, self.d, self.page = q, kv, hkv, hq, d, page
        per = [-(-n // page) for n in kv]
        pool = sum(per) + 2
        order = torch.randperm(pool, generator=g, device=DEV).to(torch.int32)
        self.table = torch.full((len(q), max(per + [1])), -3, dtype=torch.int32, device=DEV)
        at = 0
        for i, n in enumerate(per):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.seq_lens = torch.tensor(kv, dtype=torch.int32, device=DEV)
        self.cu_q = torch.tensor([0] + q).cumsum(0).to(torch.int32).to(DEV)
        self.T = sum(q) + tail_rows
        rows = torch.randn(self.T, hq + 2 * hkv, d, generator=g, device=DEV) * torch.exp(spread * torch.randn(self.T, hq + 2 * hkv, 1, generator=g, device=DEV))
        rows = rows.to(dtype)
        self.q, self.k, self.v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
        shape = (hkv, pool, rg.rg_cache_four_block_bytes(page, d)) if pages_inner else (pool, hkv, rg.rg_cache_four_block_bytes(page, d))
        self.kc, self.vc = (torch.randint(0, 256, shape, generator=g, device=DEV, dtype=torch.uint8) for _ in range(2))
        if pages_inner:
            self.kc, self.vc = self.kc.transpose(0, 1), self.vc.transpose(0, 1)
        self.kh, self.vh = (rg.rg_cache_four(t, page_size=page, dim=d) for t in (self.kc, self.vc))
        self.seqs = rg.rg_paged_seqs(self.table, self.seq_lens, self.cu_q)

    def places(self):
        """Row, page, slot and place of every new token."""
        row, page, slot, place = [], [], [], []
        at = 0
        for i, (n, m) in enumerate(zip(self.q_lens, self.kv_lens)):
            p = torch.arange(m - n, m, device=DEV)
            row.append(torch.arange(at, at + n, device=DEV)); page.append(self.table[i].long()[p // self.page]); slot.append(p % self.page); place.append(p)
            at += n
        return tuple(torch.cat(x) for x in (row, page, slot, place))

    def expect(self, before, x):
        """A cache with rows x [n, hkv, d] (64 bits) at the new tokens' places."""
        row, page, slot, _ = self.places()
        want = before.clone()
        codes, scales = tile_views(want, self.d)
        a, b = slot_bytes(*to_codes(x))
        codes[page, :, slot // 8, :, slot % 8], scales[page, :, slot // 8, :, slot % 8] = a, b
        return want


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("d,page", [(32, 8), (64, 16), (96, 24), (128, 16), (128, 256)])
def test_rows_without_rotation(d, page, dtype):
    c = Case([1, 37, 0, 5], [page + 1, 40, 0, 600], d=d, page=page, dtype=dtype, seed=d + page, tail_rows=3)
    k0, v0 = c.kc.clone(), c.vc.clone()
    rg.rg_kv_append_four(None, c.k, c.v, None, c.kh, c.vh, c.seqs)
    row = c.places()[0]
    assert torch.equal(c.kc, c.expect(k0, c.k[row].double())) and torch.equal(c.vc, c.expect(v0, c.v[row].double()))


# A code comes out otherwise than in the plain 64-bit rotation only for a rotated key within 2^-35 or so of its size (angles of up to 10^5 radians, formed in
# another order) of a border between codes: not among these, and the inputs are fixed.
@pytest.mark.parametrize("style", [rg.RG_ROPE_HALF, rg.RG_ROPE_PAIRS])
@pytest.mark.parametrize("d,rot,sections", [(128, 128, (64,)), (128, 64, (8, 12, 12)), (64, 48, (24,)), (96, 20, (10,)), (32, 2, (1,)), (64, 64, (10, 20, 1, 1))])
@pytest.mark.parametrize("dtype", [BF, HF, F32])
def test_rotated_keys_and_queries(d, rot, sections, style, dtype):
    c = Case([3, 41, 1], [3, 300, 77], d=d, page=16, dtype=dtype, seed=rot, tail_rows=2)
    freq = inv_freq(rot)
    row, page, slot, place = c.places()
    desc = rg.rg_rope_desc(rot_dim=rot, style=style, sections=sections)
    pos = None
    if len(sections) > 1:
        pos = torch.randint(-50, 100000, (len(sections), c.T), generator=generator(9), device=DEV)
    k0, v0 = c.kc.clone(), c.vc.clone()
    q_out = torch.full((c.T, c.hq, d), 77.0, dtype=dtype, device=DEV)
    rg.rg_kv_append_four(desc, c.k, c.v, freq, c.kh, c.vh, c.seqs, pos=pos, q=c.q, q_out=q_out)
    at = pos if pos is not None else torch.cat((place, torch.zeros(2, dtype=torch.int64, device=DEV)))[None]
    k64, _ = rotate64(c.k[row], at[:, row], freq, sections, style)
    assert torch.equal(c.kc, c.expect(k0, k64)) and torch.equal(c.vc, c.expect(v0, c.v[row].double()))
    want = torch.empty_like(q_out)
    rg.rg_rope(desc, c.q, at.contiguous(), freq, want)
    assert torch.equal(q_out[row], want[row])
    assert bool((q_out[len(row):] == 77.0).all()), "rows behind the last sequence were written"


@pytest.mark.parametrize("style,rot", [(rg.RG_ROPE_HALF, 64), (rg.RG_ROPE_HALF, 40), (rg.RG_ROPE_PAIRS, 40)])
def test_queries_in_place(style, rot):
    c = Case([9, 64], [9, 100], hq=16, d=64, seed=3)
    freq = inv_freq(rot)
    desc = rg.rg_rope_desc(rot_dim=rot, style=style)
    want = torch.empty(c.T, c.hq, c.d, dtype=BF, device=DEV)
    rg.rg_kv_append_four(desc, c.k, c.v, freq, c.kh, c.vh, c.seqs, q=c.q, q_out=want)
    rg.rg_kv_append_four(desc, c.k, c.v, freq, c.kh, c.vh, c.seqs, q=c.q, q_out=c.q)
    assert torch.equal(c.q, want)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
def test_strides_and_alignment(dtype):
    """Rows that no vector access can reach, heads outermost, blocks apart; the same bytes as from dense ones."""
    c = Case([5, 20], [30, 20], d=64, dtype=dtype, seed=8, pages_inner=True)
    freq = inv_freq(64)
    desc = rg.rg_rope_desc(rot_dim=64)
    q_want = torch.empty(c.T, c.hq, c.d, dtype=dtype, device=DEV)
    rg.rg_kv_append_four(desc, c.k, c.v, freq, c.kh, c.vh, c.seqs, q=c.q, q_out=q_want)
    block = c.kc.shape[2]
    wide = torch.full((c.kc.shape[0], c.hkv, block + 48), 0xA5, dtype=torch.uint8, device=DEV)
    k2, v2 = wide[:, :, 16:16 + block], torch.zeros_like(c.vc).contiguous()
    odd = torch.empty(c.T, c.hkv, c.d + 3, dtype=dtype, device=DEV)[:, :, 1:c.d + 1]
    odd.copy_(c.k)
    outer = c.v.transpose(0, 1).contiguous().transpose(0, 1)
    q_odd = torch.empty(c.T, c.hq, c.d + 1, dtype=dtype, device=DEV)[:, :, 1:]
    q_odd.copy_(c.q)
    q_out = torch.full((c.T, c.hq, c.d + 2), 5.0, dtype=dtype, device=DEV)
    kh, vh = rg.rg_cache_four(k2, page_size=c.page, dim=c.d), rg.rg_cache_four(v2, page_size=c.page, dim=c.d)
    rg.rg_kv_append_four(desc, odd, outer, freq, kh, vh, c.seqs, q=q_odd, q_out=q_out[:, :, 1:c.d + 1])
    _, page, slot, _ = c.places()
    for a, b in ((c.kc, k2), (c.vc, v2)):
        for x, y in zip(tile_views(a, c.d), tile_views(b, c.d)):
            assert torch.equal(x[page, :, slot // 8, :, slot % 8], y[page, :, slot // 8, :, slot % 8])
    assert torch.equal(q_out[:, :, 1:c.d + 1], q_want) and bool((q_out[:, :, 0] == 5.0).all()) and bool((q_out[:, :, -1] == 5.0).all())
    assert bool((wide[:, :, :16] == 0xA5).all()) and bool((wide[:, :, 16 + block:] == 0xA5).all())
    # and back, into rows of every alignment
    k_out, v_out = torch.full((2, c.T, c.hkv, c.d + 2), 5.0, dtype=F32, device=DEV)
    rg.rg_kv_read_four(kh, vh, c.seqs, k_out[:, :, 1:c.d + 1], v_out[:, :, 1:c.d + 1])
    assert torch.equal(k_out[:, :, 1:c.d + 1].double(), values(k2, c.d)[page, :, slot]) and bool((k_out[:, :, 0] == 5.0).all()) and bool((v_out[:, :, -1] == 5.0).all())


def test_borders_and_extremes():
    """Groups whose largest magnitude is a multiple of 7.5 steps or next to one, ties between codes, tiny and huge numbers, infinities and NaN."""
    s = scale_values()
    x = torch.zeros(256 * 4, 16, dtype=torch.float64, device=DEV)
    up = (7.5 * s).float()
    for i, a in enumerate((up, torch.nextafter(up, torch.full_like(up, 1e30)), torch.nextafter(up, torch.zeros_like(up)), (7 * s).float())):
        x[256 * i:256 * i + 256, 0] = a.double()
    step = s.repeat(4)
    for e in range(1, 16):
        x[:, e] = (e - 8 + 0.5) * step                           # ties of this step
    x[:, 15] = torch.nextafter((2.5 * step).float(), torch.zeros(1024, device=DEV)).double()
    odd = torch.tensor([float("inf"), -float("inf"), float("nan"), 3e38, -3e38, 1e-45, -1e-40, 57600.0, 57601.0, 61440.0, -61440.0, -70000.0, 2.0 ** -20, 2.0 ** -18, 0.0, -0.0], device=DEV)
    extra = torch.stack([odd.double(), torch.full((16,), float("nan"), device=DEV, dtype=torch.float64), torch.zeros(16, device=DEV, dtype=torch.float64), odd.roll(1).double(),
                         torch.where(odd.isfinite() & (odd.abs() < 1e4), odd, 1.0).double(), torch.where(odd.isfinite() & (odd.abs() < 1e-3), odd, 0.0).double()])
    x = torch.cat((x, extra, torch.zeros(2, 16, dtype=torch.float64, device=DEV))).view(-1, 1, 32)
    T = x.shape[0]
    c = Case([T], [T], hkv=1, hq=1, d=32, page=8, dtype=F32)
    x = x.float()
    k0, v0 = c.kc.clone(), c.vc.clone()
    rg.rg_kv_append_four(None, x, -x, None, c.kh, c.vh, c.seqs)
    assert torch.equal(c.kc, c.expect(k0, x.double())) and torch.equal(c.vc, c.expect(v0, -x.double()))


@pytest.mark.parametrize("dtype", [BF, HF, F32])
def test_every_code_and_scale_reads_back_exactly(dtype):
    c = Case([512], [512], hkv=1, hq=1, d=32, page=32, dtype=dtype)
    codes = torch.arange(16, device=DEV).repeat(512, 2) - 8
    b = torch.arange(1024, device=DEV).view(512, 2) % 256
    row, page, slot, _ = c.places()
    a, s = slot_bytes(codes[:, None], b[:, None])
    for t in (c.kc, c.vc):
        x, y = tile_views(t, 32)
        x[page, :, slot // 8, :, slot % 8], y[page, :, slot // 8, :, slot % 8] = a, s
    k_out, v_out = torch.empty(2, 512, 1, 32, dtype=dtype, device=DEV)
    rg.rg_kv_read_four(c.kh, c.vh, c.seqs, k_out, v_out)
    assert torch.equal(k_out.double()[:, 0], from_codes(codes, b)) and torch.equal(k_out, v_out)


def test_reads_whole_sequences_and_leaves_other_rows():
    c = Case([100, 0, 333], [100, 5, 333], d=128, page=24, seed=6, tail_rows=4)
    k_out, v_out = torch.full((2, c.T, c.hkv, c.d), 9.0, dtype=BF, device=DEV)
    rg.rg_kv_read_four(c.kh, c.vh, c.seqs, k_out, v_out)
    row, page, slot, _ = c.places()
    # garbage bytes are finite values, below 2^16 and exact in bf16
    assert torch.equal(k_out[row].double(), values(c.kc, c.d)[page, :, slot]) and torch.equal(v_out[row].double(), values(c.vc, c.d)[page, :, slot])
    assert bool((k_out[len(row):] == 9.0).all()) and bool((v_out[len(row):] == 9.0).all())


def test_bad_places_are_told_and_touch_nothing():
    c = Case([2, 4, 2], [20, 2, 40], d=64, seed=7)                # the second sequence: two tokens without a place
    c.table[0, 1] = 10 ** 6
    c.table[2, 2] = -1
    k0, v0 = c.kc.clone(), c.vc.clone()
    freq = inv_freq(64)
    q_out = torch.full((c.T, c.hq, c.d), 77.0, dtype=BF, device=DEV)
    rg.rg_kv_append_four(rg.rg_rope_desc(rot_dim=64), c.k, c.v, freq, c.kh, c.vh, c.seqs, q=c.q, q_out=q_out)
    assert rg.rg_device_status() == rg.RG_PAGE_CODE_APPEND
    page, slot = c.table[1, :1].long().expand(2), torch.arange(2, device=DEV)
    for before, after in ((k0, c.kc), (v0, c.vc)):
        changed = (values(before, 64) != values(after, 64)).any(-1).any(1)       # [pages, slots]
        changed[page, slot] = False
        assert not bool(changed.any())
    k_out, v_out = torch.full((2, c.T, c.hkv, c.d), 9.0, dtype=BF, device=DEV)
    rg.rg_kv_read_four(c.kh, c.vh, c.seqs, k_out, v_out)
    assert rg.rg_device_status() == rg.RG_PAGE_CODE_READ
    assert not bool(k_out[:4].any()) and not bool(v_out[6:].any()) and torch.equal(v_out[4:6].double(), values(c.vc, 64)[page, :, slot])


def test_a_prompt_at_once_and_token_by_token():
    """The same bytes, whatever comes along, on whichever pages."""
    n = 45
    a = Case([n], [n], d=128, page=16, seed=2)
    freq = inv_freq(128)
    desc = rg.rg_rope_desc(rot_dim=128)
    rg.rg_kv_append_four(desc, a.k, a.v, freq, a.kh, a.vh, a.seqs)
    b = Case([1], [n], d=128, page=64, seed=12)
    for i in range(n):
        b.seq_lens.fill_(i + 1)
        rg.rg_kv_append_four(desc, a.k[i:i + 1], a.v[i:i + 1], freq, b.kh, b.vh, b.seqs)
    outs = []
    for c in (a, b):
        s = rg.rg_paged_seqs(c.table, torch.tensor([n], dtype=torch.int32, device=DEV), torch.tensor([0, n], dtype=torch.int32, device=DEV))
        outs.append(rg.rg_kv_read_four(c.kh, c.vh, s, *torch.empty(2, n, 2, 128, dtype=F32, device=DEV)))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_many_heads_and_tokens():
    c = Case([3000, 1, 77], [3000, 50, 90], hkv=8, hq=32, d=128, page=64, seed=4)
    freq = inv_freq(128)
    k0, v0 = c.kc.clone(), c.vc.clone()
    row, page, slot, place = c.places()
    rg.rg_kv_append_four(None, c.k, c.v, None, c.kh, c.vh, c.seqs)
    assert torch.equal(c.kc, c.expect(k0, c.k[row].double())) and torch.equal(c.vc, c.expect(v0, c.v[row].double()))
    rg.rg_kv_append_four(rg.rg_rope_desc(rot_dim=128), c.k, c.v, freq, c.kh, c.vh, c.seqs)
    k_out, v_out = torch.empty(2, c.T, 8, 128, dtype=F32, device=DEV)
    rg.rg_kv_read_four(c.kh, c.vh, c.seqs, k_out, v_out)
    k64, _ = rotate64(c.k[row], place[None], freq, (64,), rg.RG_ROPE_HALF)
    want = from_codes(*to_codes(k64))
    assert torch.equal(k_out.double(), want) and torch.equal(v_out.double(), from_codes(*to_codes(c.v.double())))


def test_captured_call_follows_the_lengths():
    c = Case([1, 1], [40, 9], d=64, seed=5)
    k_out, v_out = torch.empty(2, 2, c.hkv, c.d, dtype=BF, device=DEV)

    def step():
        rg.rg_kv_append_four(None, c.k, c.v, None, c.kh, c.vh, c.seqs)
        rg.rg_kv_read_four(c.kh, c.vh, c.seqs, k_out, v_out)

    stream = torch.cuda.Stream()
    torch.cuda.synchronize()                                    # the inputs are another stream's work
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for lens in ((33, 1), (48, 16), (17, 8)):
        c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.k.copy_(torch.randn_like(c.k)); c.v.copy_(torch.randn_like(c.v))
        c.kv_lens = list(lens)
        k0 = c.kc.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.kc, c.expect(k0, c.k.double())) and torch.equal(k_out.double(), from_codes(*to_codes(c.k.double())))


def test_offsets_beyond_32_bits():
    """Pages whose blocks lie more than 2^32 bytes into the cache."""
    d, page = 128, 256
    block = rg.rg_cache_four_block_bytes(page, d)
    pages = 2 ** 32 // (2 * block) + 3
    cache = torch.zeros(pages, 2, block, dtype=torch.uint8, device=DEV)
    h = rg.rg_cache_four(cache, page_size=page, dim=d)
    x = torch.randn(3, 2, d, generator=generator(1), device=DEV).to(BF)
    table = torch.tensor([[pages - 1]], dtype=torch.int32, device=DEV)
    s = rg.rg_paged_seqs(table, torch.tensor([page], dtype=torch.int32, device=DEV), torch.tensor([0, 3], dtype=torch.int32, device=DEV))
    rg.rg_kv_append_four(None, x, x, None, h, h, s)
    want = from_codes(*to_codes(x.double()))
    assert torch.equal(values(cache[-1:], d)[0].transpose(0, 1)[-3:], want) and not bool(cache[:-1].any())
    a, b = torch.empty(2, 3, 2, d, dtype=BF, device=DEV)
    rg.rg_kv_read_four(h, h, s, a, b)
    assert torch.equal(a.double(), want) and torch.equal(a, b)

"""Attention over a paged cache of four-bit codes, on the GPU: the same bits as over a 16-bit cache of the same values, and the definition in 64 bits."""
import pytest
import torch

import paper_2609_11356_b200 as rg
from tests._four_bit_util import Batch4, attend4, check4, tile_views
from tests._paged_util import DEV, attend

pytestmark = pytest.mark.gpu
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(autouse=True)
def healthy():
    yield
    assert rg.rg_device_status() == 0


def both(b, **kw):
    """The four-bit call's answer, which has the 16-bit call's bits."""
    o4, z4 = attend4(b, **kw)
    o, z = attend(b, **kw)
    assert torch.equal(o4, o) and torch.equal(z4, z)
    return o4, z4


@pytest.mark.parametrize("split", [0, 128, 256])
@pytest.mark.parametrize("q,kv", [([1], [1]), ([1], [128]), ([1], [129]), ([1, 1, 1], [1, 700, 127]), ([5], [5]), ([127, 1, 130], [127, 300, 513]),
                                  ([1, 0, 3, 0], [257, 0, 3, 40]), ([256], [256]), ([300], [1000])])
def test_lengths(q, kv, split):
    b = Batch4(q, kv, hq=4, hkv=2, d=128, page=16, seed=len(q) + kv[0])
    check4(b, *both(b, split=split))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
def test_head_sizes_and_types(d, dtype):
    b = Batch4([1, 70], [333, 200], hq=6, hkv=2, d=d, page=32, dtype=dtype, seed=d)
    check4(b, *both(b))
    check4(b, *both(b, split=128))
    check4(b, *both(b, out_dtype=F32))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (5, 1), (12, 4), (16, 1), (32, 1), (33, 1), (48, 1), (128, 1), (120, 2), (40, 8)])
@pytest.mark.parametrize("d", [64, 128])
def test_head_groups(hq, hkv, d):
    b = Batch4([1, 9, 40], [150, 9, 260], hq=hq, hkv=hkv, d=d, page=16, seed=hq)
    check4(b, *both(b))
    s = b.seqs(max_q=0)
    o, z = attend4(b, seqs=s)
    assert all(torch.equal(x, y) for x, y in zip((o, z), attend4(b)))
    b = Batch4([1, 1, 1], [150, 9, 1260], hq=hq, hkv=hkv, d=d, page=16, seed=hq)      # single tokens
    check4(b, *both(b))
    check4(b, *both(b, split=256))


@pytest.mark.parametrize("pages_inner", [False, True])
@pytest.mark.parametrize("page", [8, 24, 48, 64, 128, 256, 1000])
@pytest.mark.parametrize("d", [32, 128])
def test_page_sizes(page, pages_inner, d):
    b = Batch4([1, 33, 150], [page * 2 + 3, 33, 1100], hq=4, hkv=2, d=d, page=page, pages_inner=pages_inner, seed=page)
    check4(b, *both(b))
    b = Batch4([1, 1], [page * 2 + 3, 1100], hq=4, hkv=2, d=d, page=page, pages_inner=pages_inner, seed=page)
    check4(b, *both(b, split=256))


@pytest.mark.parametrize("window", [1, 2, 100, 128, 129, 300, 5000])
@pytest.mark.parametrize("split", [0, 256])
def test_sliding_window(window, split):
    b = Batch4([1, 5, 300, 64], [900, 400, 300, 640], hq=8, hkv=2, d=64, page=16, dtype=HF, seed=window)
    check4(b, *both(b, window=window, split=split), window=window)
    b = Batch4([1, 2, 1], [900, 400, 300], hq=8, hkv=2, d=128, page=16, seed=window)
    check4(b, *both(b, window=window, split=split), window=window)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("hq,hkv,most", [(8, 2, 8), (8, 2, 5), (16, 2, 3), (6, 2, 7), (16, 1, 2), (2, 2, 20), (40, 2, 1), (8, 2, 9)])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_a_few_tokens_each(d, hq, hkv, most, dtype):
    """Up to 32 rows a key head, and just more: one tile of rows, two, or the form for many; sequences of every length below, none, and many blocks of keys."""
    q = [most, 1, 0, max(most - 1, 0), most, 1]
    kv = [5000, 1, 700, 128 + most, most, 2300]
    b = Batch4(q, kv, hq=hq, hkv=hkv, d=d, page=16, dtype=dtype, seed=hq + most)
    check4(b, *both(b))
    check4(b, *both(b, split=256))
    check4(b, *both(b, window=300), window=300)


@pytest.mark.parametrize("split", [0, 128])
def test_no_mask(split):
    b = Batch4([1, 130, 40], [500, 130, 257], hq=4, hkv=4, d=128, page=16, seed=3)
    check4(b, *both(b, mask=0, split=split), mask=0)


def test_many_sequences_and_rows_behind_the_last():
    q = [(i * 7) % 4 for i in range(333)]
    kv = [n + (i * 37) % 290 for i, n in enumerate(q)]
    b = Batch4(q, kv, hq=8, hkv=2, d=64, page=16, seed=5, tail_rows=37)
    check4(b, *both(b, split=128))
    check4(b, *both(b))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lowest,highest", [(0, 8), (60, 90), (150, 200), (200, 256), (0, 256)])
def test_scales_of_every_size(dtype, lowest, highest):
    """Tiny values (fp16's subnormal numbers among them) to the largest there are; scores out to infinity leave the same bits as from 16-bit caches."""
    b = Batch4([1, 40], [300, 260], hq=4, hkv=2, d=128, page=16, dtype=dtype, seed=highest, lowest=lowest, highest=highest)
    o4, z4 = attend4(b)
    o, z = attend(b)
    assert torch.equal(o4.view(torch.int16), o.view(torch.int16)) and torch.equal(z4.view(torch.int32), z.view(torch.int32))
    b = Batch4([1, 1], [300, 260], hq=4, hkv=2, d=128, page=16, dtype=dtype, seed=highest, lowest=lowest, highest=highest)
    assert torch.equal(attend4(b)[0].view(torch.int16), attend(b)[0].view(torch.int16))


def test_masked_places_do_not_arrive():
    """Later tokens, unused slots and pages behind the end may hold any byte."""
    b = Batch4([3, 60], [77, 300], hq=4, hkv=2, d=128, page=64, seed=1)
    want = attend4(b)
    used = torch.zeros(b.k4.shape[0], b.page, dtype=torch.bool, device=DEV)
    for i in range(2):
        page, slot = b.where(i)
        used[page, slot] = True
    for t in (b.k4, b.v4):
        for view in tile_views(t, b.d):
            m = ~used.view(-1, 1, b.page // 8, 1, 8, 1)
            view.copy_(torch.where(m, torch.full_like(view, 255), view))
    got = attend4(b)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # a row of a chunk has the bits it has alone, when the later tokens are not there yet
    q, kv = b.q_lens[1], b.kv_lens[1]
    at = b.q_lens[0] + 10
    one = rg.rg_paged_seqs(b.table[1:], torch.tensor([kv - q + 11], dtype=torch.int32, device=DEV), torch.tensor([0, 1], dtype=torch.int32, device=DEV), max_q=1)
    d = rg.rg_paged_attn_desc(scale=b.d ** -0.5)
    out = torch.empty(1, b.hq, b.d, dtype=BF, device=DEV)
    rg.rg_paged_attention_four(d, b.Q[at:at + 1], *b.c4, one, out)
    assert torch.equal(out[0], want[0][at])


def test_bad_pages_read_as_zeros_and_are_told():
    for q in ([1, 1], [3, 200]):
        b = Batch4(q, [300, 400], hq=4, hkv=2, d=128, page=16, seed=1)
        good = attend4(b)[0]
        b.table[0, 3], b.table[0, 5] = 10 ** 6, -1
        o, z = attend4(b)
        assert rg.rg_device_status() == rg.RG_PAGE_CODE_ATTEND
        o16, z16 = attend(b)
        assert rg.rg_device_status() == rg.RG_PAGE_CODE_ATTEND
        assert torch.equal(o, o16) and torch.equal(z, z16) and torch.equal(o[q[0]:], good[q[0]:])


def test_empty_cache_and_empty_batch():
    b = Batch4([2], [2], hq=2, hkv=1, d=64, page=16)
    d = rg.rg_paged_attn_desc(scale=0.125)
    none = torch.empty(0, 1, rg.rg_cache_four_block_bytes(16, 64), dtype=torch.uint8, device=DEV)
    h = rg.rg_cache_four(none, page_size=16, dim=64)
    out = torch.full((2, 2, 64), 5.0, dtype=BF, device=DEV)
    z = torch.empty(2, 2, device=DEV)
    rg.rg_paged_attention_four(d, b.Q, h, h, rg.rg_paged_seqs(b.table, torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)), out, lse=z)
    assert bool((out == 5.0).all())                              # rows of no sequence
    e = torch.empty(0, dtype=torch.int32, device=DEV)
    rg.rg_paged_attention_four(d, b.Q, *b.c4, rg.rg_paged_seqs(torch.empty(0, 3, dtype=torch.int32, device=DEV), e, torch.zeros(1, dtype=torch.int32, device=DEV)), out)
    assert bool((out == 5.0).all())


def test_strided_rows_two_streams_and_repeated_calls():
    b = Batch4([1] * 40, [50 * i + 1 for i in range(40)], hq=8, hkv=2, d=128, page=16, seed=4)
    want, z = attend4(b, split=256)
    wide = torch.full((b.T, 11, 136), float("nan"), dtype=BF, device=DEV)
    wide[:, 2:10, :128] = b.Q
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    torch.cuda.synchronize()
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(attend4(b, split=256, q=wide[:, 2:10, :128]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) and torch.equal(x, z) for o, x in outs)


def test_captured_call_follows_lengths_and_pages():
    b = Batch4([1, 1], [700, 300], hq=8, hkv=2, d=128, page=16, seed=6)
    d = rg.rg_paged_attn_desc(scale=0.1, split=256)
    s = b.seqs(max_len=704)
    need = rg.rg_paged_attention_workspace_bytes(d, s, b.T, b.hq, b.d)
    ws, out = torch.empty(need, dtype=torch.uint8, device=DEV), torch.empty_like(b.Q)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()                                    # the inputs are another stream's work
    with torch.cuda.stream(stream):
        rg.rg_paged_attention_four(d, b.Q, *b.c4, s, out, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        rg.rg_paged_attention_four(d, b.Q, *b.c4, s, out, ws=ws)
    for lens in ((1, 300), (513, 128), (700, 2)):
        b.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        b.table[0] = b.table[0].roll(1)
        graph.replay()
        want = torch.empty_like(out)
        rg.rg_paged_attention(d, b.Q, b.kc, b.vc, s, want, ws=torch.empty_like(ws))
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_codes_beyond_32_bits():
    d, page = 128, 256
    block = rg.rg_cache_four_block_bytes(page, d)
    pages = 2 ** 32 // (2 * block) + 3
    small = Batch4([1, 1], [page, 200], hq=4, hkv=2, d=d, page=page, seed=3)
    want, _ = attend4(small, lse=False)
    caches = []
    for t in (small.k4, small.v4):
        big = torch.zeros(pages, 2, block, dtype=torch.uint8, device=DEV)
        big[-t.shape[0]:] = t
        caches.append(rg.rg_cache_four(big, page_size=page, dim=d))
    s = rg.rg_paged_seqs(small.table + (pages - small.k4.shape[0]), small.seq_lens, small.cu_q, max_q=1)
    out = torch.empty_like(want)
    rg.rg_paged_attention_four(rg.rg_paged_attn_desc(scale=d ** -0.5), small.Q, *caches, s, out)
    assert torch.equal(out, want)

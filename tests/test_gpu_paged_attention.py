"""Attention of new rows over a paged cache, on the GPU against the definition in 64 bits: lengths from one token on, odd
sizes, head layouts, pages that end inside a block, masks, strides, what must not be read, and the order of the arithmetic."""
import pytest
import torch

import paper_2609_11356_b200 as rg
from tests._paged_util import DEV, Batch, attend, check

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def healthy():
    yield
    assert rg.rg_device_status() == 0


@pytest.mark.parametrize("split", [0, 128, 256])
@pytest.mark.parametrize("q,kv", [([1], [1]), ([1], [128]), ([1], [129]), ([1, 1, 1], [1, 700, 127]), ([5], [5]), ([127, 1, 130], [127, 300, 513]),
                                  ([1, 0, 3, 0], [257, 0, 3, 40]), ([256], [256]), ([300], [1000])])
def test_lengths(q, kv, split):
    b = Batch(q, kv, hq=4, hkv=2, d=128, page=16, seed=len(q) + kv[0])
    check(b, *attend(b, split=split))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [8, 64, 72, 80, 96, 128])
def test_head_sizes_and_types(d, dtype):
    b = Batch([1, 70], [333, 200], hq=6, hkv=2, d=d, page=32, dtype=dtype, seed=d)
    check(b, *attend(b))
    check(b, *attend(b, split=128))
    check(b, *attend(b, out_dtype=torch.float32))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (5, 1), (7, 1), (12, 4), (32, 1), (33, 1), (48, 1), (128, 1), (120, 2), (40, 8)])
def test_head_groups(hq, hkv):
    b = Batch([1, 9, 40], [150, 9, 260], hq=hq, hkv=hkv, d=64, page=16, seed=hq)
    check(b, *attend(b))
    check(b, *attend(b, split=128))


@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("page", [8, 24, 48, 64, 128, 256, 1000])
def test_page_sizes(page, heads_first):
    b = Batch([1, 33, 150], [page * 2 + 3, 33, 1100], hq=4, hkv=2, d=128, page=page, heads_first=heads_first, seed=page)
    check(b, *attend(b))
    check(b, *attend(b, split=256))


@pytest.mark.parametrize("window", [1, 2, 100, 128, 129, 300, 5000])
@pytest.mark.parametrize("split", [0, 256])
def test_sliding_window(window, split):
    b = Batch([1, 5, 300, 64], [900, 400, 300, 640], hq=8, hkv=2, d=64, page=16, dtype=HF, seed=window)
    check(b, *attend(b, window=window, split=split), window=window)


@pytest.mark.parametrize("split", [0, 128])
def test_no_mask(split):
    b = Batch([1, 130, 40], [500, 130, 257], hq=4, hkv=4, d=128, page=16, seed=3)
    check(b, *attend(b, mask=0, split=split), mask=0)


def test_many_sequences_and_rows_behind_the_last():
    q = [(i * 7) % 4 for i in range(333)]
    kv = [n + (i * 37) % 290 for i, n in enumerate(q)]
    b = Batch(q, kv, hq=8, hkv=2, d=64, page=16, seed=5, tail_rows=37)
    check(b, *attend(b, split=128))
    check(b, *attend(b))


@pytest.mark.parametrize("spread,scale", [(4.0, None), (1.0, 3.0), (0.01, None)])
def test_wide_and_narrow_scores(spread, scale):
    b = Batch([200, 1], [700, 1500], hq=2, hkv=1, d=128, page=16, seed=9, spread=spread)
    check(b, *attend(b, scale=scale), scale=scale)
    check(b, *attend(b, scale=scale, split=256), scale=scale)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_maximum_that_keeps_rising(dtype):
    """Every block's scores exceed the last one's, by less and by more than the slack of the running maximum."""
    b = Batch([1, 140], [1400, 1024], hq=2, hkv=1, d=64, page=16, dtype=dtype, seed=2)
    for step in (0.02, 0.2):
        u = torch.ones(64, device=DEV) / 8
        b.Q[:] = u.to(dtype)
        for i, m in enumerate(b.kv_lens):
            b.K[i] = ((torch.arange(m, device=DEV) * step)[:, None, None] * u + 0.1 * torch.randn(m, 1, 64, device=DEV)).to(dtype)
        b.store()
        check(b, *attend(b, scale=1.0), scale=1.0)
        check(b, *attend(b, scale=1.0, split=256), scale=1.0)


def test_strided_operands():
    b = Batch([3, 100], [50, 300], hq=4, hkv=2, d=64, page=16, seed=4)
    wide = torch.full((b.T, 9, 72), float("nan"), dtype=BF, device=DEV)
    q = wide[:, 2:6, :64]
    q.copy_(b.Q)
    out_buf = torch.full((b.T, 7, 66), 5.0, dtype=torch.float32, device=DEV)
    out = out_buf[:, 1:5, 1:65]
    z_buf = torch.full((b.T, 6), 5.0, device=DEV)
    rg.rg_paged_attention(rg.rg_paged_attn_desc(scale=0.125), q, b.kc, b.vc, b.seqs(), out, lse=z_buf[:, 1:5])
    check(b, out, z_buf[:, 1:5])
    rest = out_buf.clone()
    rest[:, 1:5, 1:65] = 5.0
    assert bool((rest == 5.0).all()) and bool((z_buf[:, 0] == 5.0).all()) and bool((z_buf[:, 5] == 5.0).all())
    # heads outermost
    q2 = b.Q.transpose(0, 1).contiguous().transpose(0, 1)
    out2 = torch.empty(4, b.T, 64, dtype=BF, device=DEV).transpose(0, 1)
    rg.rg_paged_attention(rg.rg_paged_attn_desc(scale=0.125), q2, b.kc, b.vc, b.seqs(), out2)
    check(b, out2, None)
    # unaligned 16-bit output rows
    out3 = torch.full((b.T, 4, 65), 5.0, dtype=BF, device=DEV)
    rg.rg_paged_attention(rg.rg_paged_attn_desc(scale=0.125), q, b.kc, b.vc, b.seqs(), out3[:, :, 1:])
    check(b, out3[:, :, 1:], None)
    assert bool((out3[:, :, 0] == 5.0).all())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("q_len", [1, 60, 300])
def test_what_is_masked_does_not_arrive(q_len, bad):
    """Keys and values behind a row (later tokens of the same chunk), before its window, and in unused slots hold infinities and NaN."""
    n = 400
    b = Batch([q_len], [n], hq=4, hkv=2, d=64, page=16, seed=q_len, garbage=bad)
    clean, z = attend(b)
    check(b, clean, z)
    if q_len > 1:
        for at in (n - 1, n - q_len + 1, n - q_len // 2):                     # a token of the chunk goes bad
            page, slot = (x[at] for x in b.where(0))
            keep = b.kc[page, slot].clone(), b.vc[page, slot].clone()
            row = at - (n - q_len)
            for split in (0, 128):
                ok, okz = attend(b, split=split)
                b.vc[page, slot, 1, 3] = bad
                got, gz = attend(b, split=split)
                same = torch.equal(got[:row], ok[:row]) and torch.equal(gz, okz)
                assert same, "a later token's value reached an earlier row"
                assert not bool(torch.isfinite(got[row:, 2:, 3]).any()), "a visible value that is not finite was lost"
                assert torch.equal(got[row:, :2], ok[row:, :2]) and torch.equal(got[row:, 2:, 4:], ok[row:, 2:, 4:])
                b.kc[page, slot] = bad
                b.vc[page, slot] = bad
                got, gz = attend(b, split=split)
                assert torch.equal(got[:row], ok[:row]) and torch.equal(gz[:row], okz[:row])
                b.kc[page, slot], b.vc[page, slot] = keep
    w = 50
    ok, okz = attend(b, window=w)
    check(b, ok, okz, window=w)
    page, slot = b.where(0)
    first = n - q_len - w                                                     # the last key that no row sees
    if first >= 0:
        b.kc[page[:first + 1], slot[:first + 1]] = bad
        b.vc[page[:first + 1], slot[:first + 1]] = bad
        got, gz = attend(b, window=w)
        assert torch.equal(got, ok) and torch.equal(gz, okz)


def test_bits_do_not_depend_on_the_batch_the_pages_or_the_chunk():
    q, kv = [1, 37, 200, 1, 4], [777, 500, 900, 64, 1300]
    a = Batch(q, kv, hq=8, hkv=2, d=128, page=16, seed=11)
    for split in (0, 256):
        full, z = attend(a, split=split)
        again, z2 = attend(a, split=split, ws_fill=0)
        assert torch.equal(full, again) and torch.equal(z, z2), "two runs differ"
        for kw in ({"max_q": 0, "max_len": 0}, {"max_q": 4000, "max_len": 100000}, {"max_q": 1, "max_len": 1300}):
            got, gz = attend(a, split=split, seqs=a.seqs(**kw))
            assert torch.equal(got, full) and torch.equal(gz, z), kw
        # other pages, another page size, another order in memory
        other = Batch(q, kv, hq=8, hkv=2, d=128, page=48, seed=99, heads_first=True)
        other.Q, other.K, other.V = a.Q, a.K, a.V
        other.store()
        got, gz = attend(other, split=split)
        assert torch.equal(got, full) and torch.equal(gz, z), "pages"
        # each row of the longest chunk alone, as a single token
        at = q[0] + q[1]
        for r in (0, 1, 63, 64, 150, 199):
            one = Batch([1], [kv[2] - q[2] + r + 1], hq=8, hkv=2, d=128, page=16, seed=5)
            one.Q = a.Q[at + r:at + r + 1]
            one.K, one.V = [a.K[2][:one.kv_lens[0]]], [a.V[2][:one.kv_lens[0]]]
            one.store()
            got, gz = attend(one, split=split)
            assert torch.equal(got[0], full[at + r]) and torch.equal(gz[0], z[at + r]), f"row {r} alone, split {split}"


def test_shared_pages():
    """Two sequences with a common prefix read the same pages."""
    b = Batch([2, 2], [100, 100], hq=4, hkv=2, d=64, page=16, seed=8)
    b.table[1, :4] = b.table[0, :4]
    b.K[1][:64], b.V[1][:64] = b.K[0][:64], b.V[0][:64]
    b.store()
    check(b, *attend(b))


def test_offsets_past_32_bits():
    """Pages that lie more than 2^32 bytes into the cache, by their number and by their stride."""
    hkv, d, page = 1, 64, 8
    pages = 2 ** 31 // (page * d) + 64                                        # 2^31 elements and some: 4.3 GB each
    kc = torch.empty(pages, page, hkv, d, dtype=BF, device=DEV)
    vc = torch.empty(pages, page, hkv, d, dtype=BF, device=DEV)
    b = Batch([1, 3], [60, 31], hq=2, hkv=hkv, d=d, page=page, seed=6)
    far = torch.arange(pages - 40, pages, device=DEV, dtype=torch.int32)
    b.kc, b.vc = kc, vc
    b.table[0, :8], b.table[1, :4] = far[5:13], far[20:24]
    b.store()
    check(b, *attend(b))
    check(b, *attend(b, split=128))
    stride = 2 ** 31 // 16                                                     # 17 pages, the last one past 2^31 elements
    b.kc = torch.as_strided(kc, (17, page, hkv, d), (stride, d, d, 1))
    b.vc = torch.as_strided(vc, (17, page, hkv, d), (stride, d, d, 1))
    b.table[0, :8] = torch.tensor([16, 15, 14, 13, 12, 11, 10, 9])
    b.table[1, :4] = torch.tensor([8, 7, 6, 5])
    b.store()
    check(b, *attend(b))


def test_other_stream_and_captured_graph():
    b = Batch([1, 1, 1], [300, 555, 41], hq=8, hkv=2, d=128, page=16, seed=13, spare=40)
    b.table = torch.cat([b.table, torch.full((3, 4), -7, dtype=torch.int32, device=DEV)], 1)
    seqs = b.seqs(max_len=600)
    d = rg.rg_paged_attn_desc(scale=b.d ** -0.5, split=128)
    ws = torch.zeros(rg.rg_paged_attention_workspace_bytes(d, seqs, b.T, b.hq, b.d), dtype=torch.uint8, device=DEV)
    out, z = torch.full_like(b.Q, 77.0), torch.full((b.T, 8), 77.0, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rg.rg_paged_attention(d, b.Q, b.kc, b.vc, seqs, out, lse=z, ws=ws)
    side.synchronize()
    check(b, out, z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rg.rg_paged_attention(d, b.Q, b.kc, b.vc, seqs, out, lse=z, ws=ws)
    for lens in ([300, 555, 41], [17, 128, 41], [256, 1, 0], [1, 500, 33]):     # replays follow what the arrays hold by then
        b.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(77.0); z.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        cut = Batch([1, 1, 1], [300, 555, 41], hq=8, hkv=2, d=128, page=16, seed=13, spare=40)
        for i, n in enumerate(lens):
            if n == 0:                                                          # a row without a place: zeros, and a code in the health word
                assert bool((out[i] == 0).all()) and bool((z[i] == float("-inf")).all())
                assert rg.rg_device_status() == rg.RG_PAGE_CODE_ATTEND
                cut.K[i], cut.V[i] = cut.K[i][:1], cut.V[i][:1]
                out[i], z[i] = cut.V[i][0].repeat_interleave(4, 0), (cut.Q[i].double() * cut.K[i][0].repeat_interleave(4, 0).double()).sum(-1).float() * b.d ** -0.5
            else:
                cut.K[i], cut.V[i] = cut.K[i][:n], cut.V[i][:n]
        cut.kv_lens = [max(n, 1) for n in lens]
        check(cut, out, z)


def test_pages_and_lengths_outside_are_told_and_touch_nothing():
    b = Batch([1, 4, 2], [300, 200, 90], hq=4, hkv=2, d=64, page=16, seed=21)
    ok, okz = attend(b)
    for split in (0, 128):
        for value in (-1, b.kc.shape[0], 2 ** 31 - 1, -2 ** 31):
            keep = b.table[1, 2].clone()
            b.table[1, 2] = value
            got, z = attend(b, split=split)
            assert rg.rg_device_status() == rg.RG_PAGE_CODE_ATTEND
            assert bool(torch.isfinite(got).all()) and bool(torch.isfinite(z).all())
            if split == 0:
                assert torch.equal(got[0], ok[0]) and torch.equal(got[5:], ok[5:])
            b.table[1, 2] = keep
        for i, n in ((0, 10 ** 6), (1, 2 ** 31 - 1), (2, -5), (1, 2)):            # beyond the table, beyond max_len, below the new rows
            keep = b.seq_lens.clone()
            b.seq_lens[i] = n
            got, z = attend(b, split=split)
            assert rg.rg_device_status() == rg.RG_PAGE_CODE_ATTEND
            others = [r for r in range(7) if r not in ([0], range(1, 5), range(5, 7))[i]]
            if split == 0:
                assert torch.equal(got[others], ok[others]) and torch.equal(z[others], okz[others])
            if n < 0:
                assert bool((got[5:] == 0).all()) and bool((z[5:] == float("-inf")).all())
            if n == 2:
                assert bool((got[1:3] == 0).all()) and bool(torch.isfinite(z[3:5]).all())
            b.seq_lens.copy_(keep)
    assert rg.rg_device_status() == 0


def test_refusals():
    b = Batch([2, 2], [40, 500], hq=4, hkv=2, d=64, page=16, seed=1)
    out = torch.full_like(b.Q, 77.0)
    d = rg.rg_paged_attn_desc(scale=0.125)

    def refused(status, fn):
        with pytest.raises(rg.RgError) as e:
            fn()
        assert e.value.status == status
        torch.cuda.synchronize()
        assert bool((out == 77.0).all())

    run = lambda d=d, q=b.Q, kc=b.kc, vc=b.vc, out=out, **kw: rg.rg_paged_attention(d, q, kc, vc, b.seqs(), out, **kw)
    split = rg.rg_paged_attn_desc(scale=1.0, split=128)
    need = rg.rg_paged_attention_workspace_bytes(split, b.seqs(), 4, 4, 64)
    assert need == 4 * 4 * 4 * 66 * 4                                            # four parts of each row, whole 256-byte lines already
    refused(6, lambda: run(d=split))
    refused(6, lambda: run(d=split, ws=torch.empty(need - 1, dtype=torch.uint8, device=DEV)))
    refused(5, lambda: run(d=split, ws=torch.empty(need + 16, dtype=torch.uint8, device=DEV)[8:]))
    refused(4, lambda: run(kc=b.kc[:, :, :1], vc=b.vc))
    refused(4, lambda: run(kc=b.kc.half(), vc=b.vc.half()))
    refused(5, lambda: run(q=torch.zeros(4, 4, 68, dtype=BF, device=DEV)[:, :, 4:]))
    refused(3, lambda: run(q=b.Q.float(), kc=b.kc.float(), vc=b.vc.float(), out=out.float()))
    refused(4, lambda: run(out=out[:1].expand(4, 4, 64)))
    with pytest.raises(ValueError):
        run(lse=torch.zeros(4, 4, dtype=torch.float64, device=DEV))
    with pytest.raises(ValueError):
        run(q=b.Q.cpu())
    empty = torch.zeros(0, 4, 64, dtype=BF, device=DEV)
    rg.rg_paged_attention(d, empty, b.kc, b.vc, b.seqs(), empty)                 # nothing to do is fine


def test_what_is_visible_and_not_finite_arrives():
    """A NaN key makes the rows that see it NaN, others keep their bits; a score of +inf likewise."""
    for q_len, split in ((1, 0), (1, 128), (150, 0), (150, 128)):
        b = Batch([q_len], [500], hq=4, hkv=2, d=64, page=16, seed=3)
        ok, okz = attend(b, split=split)
        for at in (100, 499 - q_len // 2):
            page, slot = (x[at] for x in b.where(0))
            keep = b.kc[page, slot].clone()
            for bad in (float("nan"), float("inf")):
                b.kc[page, slot, 1, 5] = bad
                got, gz = attend(b, split=split)
                row = max(0, at - (500 - q_len))
                assert torch.equal(got[:row], ok[:row]) and torch.equal(got[:, :2], ok[:, :2])
                hit = got[row:, 2:]
                if bad != bad:
                    assert bool(torch.isnan(hit).all()) and bool(torch.isnan(gz[row:, 2:]).all())
                else:                                                           # +inf or -inf by the query's sign: NaN, or the key drops out
                    up = b.Q[row:, 2:, 5] > 0
                    assert bool(torch.isnan(hit[up]).all()) and bool(torch.isfinite(hit[~up]).all())
                b.kc[page, slot] = keep


@pytest.mark.parametrize("split", [0, 128])
def test_pages_in_front_of_the_window_may_be_gone(split):
    b = Batch([1, 20], [700, 500], hq=4, hkv=2, d=64, page=16, seed=7)
    w = 130
    ok, okz = attend(b, window=w, split=split)
    check(b, ok, okz, window=w)
    for i, (n, m) in enumerate(zip(b.q_lens, b.kv_lens)):
        b.table[i, :(m - n - w + 1) // 16] = -1
    got, gz = attend(b, window=w, split=split)
    assert torch.equal(got, ok) and torch.equal(gz, okz)


@pytest.mark.parametrize("seed", range(24))
def test_drawn_shapes(seed):
    import random
    r = random.Random(seed)
    hkv = r.choice([1, 2, 3, 8])
    n = r.choice([1, 2, 5, 40])
    q = [r.choice([0, 1, 1, r.randint(1, 6), r.randint(1, 200)]) for _ in range(n)]
    kv = [x + r.choice([0, r.randint(0, 300), r.randint(0, 2500)]) for x in q]
    if sum(q) == 0:
        q[0], kv[0] = 1, kv[0] + 1
    b = Batch(q, kv, hq=hkv * r.choice([1, 2, 3, 4, 7, 16]), hkv=hkv, d=r.choice([16, 64, 88, 128]), page=r.choice([8, 16, 40, 128]), dtype=r.choice([BF, HF]), seed=seed,
              heads_first=r.random() < 0.5, tail_rows=r.choice([0, 3]), spread=r.choice([0.3, 1.0, 2.0]))
    window = r.choice([0, 0, r.randint(1, 600)])
    mask = 1 if window else r.choice([1, 1, 0])
    split = r.choice([0, 0, 128, 384, 512])
    seqs = b.seqs(max_q=r.choice([0, 1, max(q)]), max_len=r.choice([0, max(kv)]))
    check(b, *attend(b, window=window, mask=mask, split=split, seqs=seqs, out_dtype=r.choice([None, torch.float32])), window=window, mask=mask)


def test_cache_without_pages():
    """Nothing to read: every row is zeros, and the lengths that say otherwise are told."""
    b = Batch([2, 1], [5, 1], hq=4, hkv=2, d=64, page=16, seed=1)
    kc = torch.zeros(0, 16, 2, 64, dtype=BF, device=DEV)
    for split in (0, 128):
        out, z = torch.full_like(b.Q, 77.0), torch.full((3, 4), 77.0, device=DEV)
        rg.rg_paged_attention(rg.rg_paged_attn_desc(scale=1.0, split=split), b.Q, kc, kc, b.seqs(), out, lse=z)
        assert rg.rg_device_status() == rg.RG_PAGE_CODE_ATTEND
        assert bool((out == 0).all()) and bool((z == float("-inf")).all())


def test_two_calls_at_once_and_back_to_back():
    """Calls on two streams with workspaces of their own, and calls in a row that share one, give what they give alone."""
    a, b = Batch([1] * 8, [900 + 50 * i for i in range(8)], hq=8, hkv=2, d=128, page=16, seed=1), Batch([70, 130], [400, 1300], hq=8, hkv=2, d=128, page=16, seed=2)
    d = rg.rg_paged_attn_desc(scale=0.09, split=128)
    alone = [attend(x, scale=0.09, split=128)[0] for x in (a, b)]
    torch.cuda.synchronize()
    need = [rg.rg_paged_attention_workspace_bytes(d, x.seqs(), x.T, x.hq, x.d) for x in (a, b)]
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [[], []]
    ws = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in need]
    for _ in range(10):
        for i, x in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                outs[i].append(rg.rg_paged_attention(d, x.Q, x.kc, x.vc, x.seqs(), torch.empty_like(x.Q), ws=ws[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, alone[i]) for o in outs[i])
    shared = torch.empty(max(need), dtype=torch.uint8, device=DEV)
    outs = [rg.rg_paged_attention(d, x.Q, x.kc, x.vc, x.seqs(), torch.empty_like(x.Q), ws=shared) for _ in range(10) for x in (a, b)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, alone[i % 2]) for i, o in enumerate(outs))

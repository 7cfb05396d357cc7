"""Paged append and attention at the edges of what their calls allow: tables and positions that sequences or axes share, values and
scores that are not finite or very large, and results that must not depend on which kernel or tile takes a row."""
import random

import pytest
import torch

import paper_2609_11356_b200 as rg
from tests._paged_util import DEV, Batch, attend, attention_bounds, check, inv_freq

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def healthy():
    yield
    assert rg.rg_device_status() == 0


@pytest.mark.parametrize("split", [0, 128])
def test_one_table_row_for_all_sequences(split):
    """Sequences that read one text: the table's row expanded (stride 0) gives what a table of copies gives."""
    b = Batch([2, 3, 1], [300, 300, 300], hq=4, hkv=2, d=64, page=16, seed=3)
    b.table = b.table[:1].repeat(3, 1)
    b.K, b.V = [b.K[0]] * 3, [b.V[0]] * 3
    b.store()
    want, z = attend(b, split=split)
    check(b, want, z)
    b.table = b.table[:1].clone().expand(3, -1)                               # its storage ends with the one row
    got, gz = attend(b, split=split)
    assert torch.equal(got, want) and torch.equal(gz, z)


def test_append_through_one_table_row():
    """Three stages of one text in one call: each sequence's new tokens have places of their own in the shared pages."""
    b = Batch([2, 3, 4], [20, 23, 27], hq=2, hkv=2, d=64, page=16, seed=4, garbage=3.0)
    row = b.table[2:].clone()
    k = torch.randn(9, 2, 64, device=DEV).to(BF)
    ks, vs = [], []
    for table in (row.repeat(3, 1), row.expand(3, -1)):
        kc, vc = torch.full_like(b.kc, 3.0), torch.full_like(b.vc, 3.0)
        b.table = table
        rg.rg_kv_append(None, k, -k, None, kc, vc, b.seqs())
        ks.append(kc); vs.append(vc)
    place = torch.arange(18, 27, device=DEV)
    assert torch.equal(ks[0][row[0].long()[place // 16], place % 16], k)
    assert torch.equal(ks[0], ks[1]) and torch.equal(vs[0], vs[1])


def test_a_wait_that_gave_up_is_told_before_a_bad_page():
    """Both kinds of news unread: the wait is the answer (here the self-test's, which waits 2 ms for nothing), and both words are cleared."""
    import ctypes as C
    from paper_2609_11356_b200 import _cabi
    from paper_2609_11356_b200.api import rg_selftest_bounded_wait
    b = Batch([1], [40], hq=2, hkv=2, d=64, page=16, seed=1)
    b.table[0, 1] = -1
    attend(b)
    rg_selftest_bounded_wait(2_000_000, torch.zeros(1, dtype=torch.int32, device=DEV))
    code = C.c_uint32(0)
    assert _cabi.load().rg_device_status(C.byref(code)) == 8 and code.value == _cabi.RG_SELFTEST_WAIT_CODE
    assert rg.rg_device_status() == 0
    attend(b)
    assert _cabi.load().rg_device_status(C.byref(code)) == 9 and code.value == rg.RG_PAGE_CODE_ATTEND


def _softmax64(q, k, v, scale):
    """attention64 for scores of any size: the weights from the distances to the maximum.  Output, normaliser, sum of weights times |v|."""
    n, m, G = q.shape[0], k.shape[0], q.shape[1] // k.shape[1]
    q, k, v = q.double().permute(1, 0, 2), k.double().repeat_interleave(G, 1).permute(1, 2, 0), v.double().repeat_interleave(G, 1).permute(1, 0, 2)
    s = (q @ k).masked_fill(torch.arange(m - n, m, device=DEV)[:, None] < torch.arange(m, device=DEV)[None], -float("inf"))
    top = s.amax(-1, keepdim=True)
    w = torch.exp((s - top) * scale)
    total = w.sum(-1, keepdim=True)
    w = w / total
    return (w @ v).permute(1, 0, 2), (top * scale + total.log())[..., 0].T, (w @ v.abs()).permute(1, 0, 2)


# q = (a, 1, 0, ...), k_t = (b, r_t, 0, ...): the scores a b + r_t are whole numbers that 24 bits hold, so they carry no rounding
FAR_SCORES = [(BF, 2.0 ** 11, 2.0 ** 11, 1.0), (HF, 2.0 ** 11, -2.0 ** 11, 1.0), (BF, 2.0 ** 11, -2.0 ** 11, 2.0 ** 10), (HF, 2.0 ** 11, 2.0 ** 11, 2.0 ** 8), (BF, 2.0 ** 11, 2.0 ** 11, 2.0 ** 10),
              (HF, 1.0, 8.0, 1e38), (BF, 1.0, -12.0, 1e38), (HF, -1.0, 12.0, 2e38), (BF, 2.0 ** 63, 2.0 ** 63, 3.0), (BF, 2.0 ** 63, -2.0 ** 63, 3.0)]


@pytest.mark.parametrize("split", [0, 128])
@pytest.mark.parametrize("q_len", [1, 7, 150])
@pytest.mark.parametrize("dtype,a,b,scale", FAR_SCORES)
def test_scores_far_from_zero(dtype, a, b, scale, q_len, split):
    """The weights depend on the distances between scores, however large the scores are: where scale times a score is 2^22 and more, and where that
    product is beyond fp32.  Rows of one call lie close to zero too: their neighbours' size is nothing to them."""
    scale = float(torch.tensor(scale, dtype=torch.float32))
    x = Batch([q_len, 2], [700, 300], hq=4, hkv=2, d=64, page=16, dtype=dtype, seed=q_len)
    x.Q.zero_()
    x.Q[..., 0], x.Q[..., 1] = a, 1.0
    g = torch.Generator(device=DEV).manual_seed(5)
    for i, n in enumerate(x.kv_lens):
        x.K[i].zero_()
        x.K[i][..., 0] = b
        x.K[i][..., 1] = torch.randint(0, 12, (n, 2), generator=g, device=DEV).to(dtype) + torch.arange(n, device=DEV)[:, None].div(100).floor().to(dtype)
    near = torch.arange(0, q_len, 3, device=DEV)                              # every third row: scores 0 .. 18 times the scale
    x.Q[near, :, 0] = 0.0
    if scale != 1.0:
        x.Q[near, :, 1] = 0.0
    x.store()
    out, z = attend(x, scale=scale, split=split)
    at = 0
    for i, (n, m) in enumerate(zip(x.q_lens, x.kv_lens)):
        o, lse, mass = _softmax64(x.Q[at:at + n], x.K[i], x.V[i], scale)
        # scores exact; an exponent that a weight above 2^-30 has is off by 32 * 2^-22 at most (the scale times log2(e), the distance times that), but in rows near
        # zero, where scale times maximum (below 32) is rounded: included
        bound, bound_z = attention_bounds(o, mass, torch.zeros_like(lse), 64, m, dtype, out.dtype)
        bound = bound + 2.0 ** -17 * mass
        assert bool(((out[at:at + n].double() - o).abs() <= bound).all())
        finite = lse.abs() < 3.4e38
        # normaliser: maximum times scale rounded, the logarithm added, and the logarithm's own rounding
        off = (z[at:at + n].double() - lse).abs() - (bound_z + 2.0 ** -17 + 2.0 ** -22 * lse.abs())
        assert bool((off[finite] <= 0).all())
        assert bool((z[at:at + n][~finite] == lse[~finite].sign() * float("inf")).all())
        at += n


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("window", [0, 200])
@pytest.mark.parametrize("split", [0, 128])
@pytest.mark.parametrize("dtype,d,hq", [(HF, 64, 4), (BF, 128, 8), (HF, 80, 6)])
def test_visible_values_that_are_not_finite_do_not_depend_on_the_chunk(dtype, d, hq, split, window):
    """Scores so far apart that most weights are 0 in the cache's type: a row that sees one infinity gets it, one that sees both or a NaN gets NaN,
    whether the row comes in a chunk (where the block may be masked for its tile) or alone (where it may not be)."""
    n, m = 230, 700
    b = Batch([n], [m], hq=hq, hkv=2, d=d, page=16, dtype=dtype, seed=d, spread=4.0)
    odd = [(10, 0, 1, INF), (300, 1, 3, INF), (470, 1, 5, -INF), (480, 1, 6, INF), (690, 1, 6, -INF), (520, 0, 7, NAN), (600, 0, d - 1, -INF), (640, 0, d - 1, -INF), (699, 1, 0, INF)]
    clean, cz = attend(b, split=split, window=window)
    for key, head, col, value in odd:
        b.V[0][key, head, col] = value
    b.store()
    got, z = attend(b, split=split, window=window)
    assert torch.equal(z, cz)
    want = torch.full((n, 2, d), 0.0, device=DEV)
    place = torch.arange(m - n, m, device=DEV)
    for key, head, col, value in odd:
        sees = (place >= key) & (place < key + window if window else True)
        want[sees, head, col] += value
    want = want.repeat_interleave(hq // 2, 1)
    touched = want != 0                                                        # NaN != 0 as well
    assert torch.equal(got[~touched], clean[~touched]), "an element that sees numbers only changed"
    if split == 0:                                                             # between parts a weight of 0 may meet an infinity
        assert torch.equal(torch.nan_to_num(got.float()[touched], 7.0, 8.0, 9.0), torch.nan_to_num(want[touched], 7.0, 8.0, 9.0))
    else:
        assert not bool(torch.isfinite(got[touched]).any())
    for r in (0, 1, 50, 100, 127, 160, 200, n - 1):
        one = Batch([1], [m - n + r + 1], hq=hq, hkv=2, d=d, page=32, dtype=dtype, seed=1)
        one.Q, one.K, one.V = b.Q[r:r + 1], [b.K[0][:one.kv_lens[0]]], [b.V[0][:one.kv_lens[0]]]
        one.store()
        alone, az = attend(one, split=split, window=window)
        assert torch.equal(alone[0].view(torch.int16), got[r].view(torch.int16)) and torch.equal(az[0], z[r]), f"row {r} alone"


@pytest.mark.parametrize("q_len", [1, 200])
@pytest.mark.parametrize("what", [NAN, INF])
def test_values_that_are_all_not_finite(q_len, what):
    b = Batch([q_len, 3], [3000, 100], hq=8, hkv=2, d=128, page=16, seed=1)
    ok, okz = attend(b)
    b.V[0] = torch.full_like(b.V[0], what)
    b.store()
    for split in (0, 128):
        got, z = attend(b, split=split)
        assert bool((torch.isnan(got[:q_len]) if what != what else got[:q_len] == INF).all())
        if split == 0:
            assert torch.equal(got[q_len:], ok[q_len:]) and torch.equal(z, okz)


@pytest.mark.parametrize("q_len", [1, 150])
def test_values_that_sum_beyond_fp32(q_len):
    """O overflows although every value is finite: nothing is found, and the element stays what the sum made of it; others are not touched."""
    b = Batch([q_len], [600], hq=4, hkv=2, d=64, page=16, seed=2)
    ok, okz = attend(b)
    b.V[0][:, 1, 9] = 3.0e38
    b.store()
    got, z = attend(b)
    assert torch.equal(z, okz) and torch.equal(got[..., :9], ok[..., :9]) and torch.equal(got[..., 10:], ok[..., 10:]) and torch.equal(got[:, :2], ok[:, :2])
    assert bool((got[:, 2:, 9] == INF).all())


@pytest.mark.parametrize("split", [0, 128])
@pytest.mark.parametrize("window", [0, 150])
@pytest.mark.parametrize("dtype,d,G", [(HF, 64, 5), (HF, 128, 7), (BF, 80, 7), (HF, 80, 1), (BF, 64, 3), (BF, 24, 8), (HF, 128, 4)])
def test_bits_do_not_depend_on_the_form_that_takes_a_row(dtype, d, G, window, split):
    """A row in a long chunk (the form for many rows), alone, and with one to five rows in front of it (the form for few rows at each of its heights)."""
    n, m = 150, 613
    b = Batch([n], [m], hq=2 * G, hkv=2, d=d, page=16, dtype=dtype, seed=d + G, spread=1.5)
    full, z = attend(b, split=split, window=window)
    check(b, full, z, window=window)
    for r in (0, 5, 27, 64, 77, 149):
        for rows in (1, 2, 3, 4, 6):
            if rows > r + 1:
                continue
            end = m - n + r + 1
            few = Batch([rows], [end], hq=2 * G, hkv=2, d=d, page=24, dtype=dtype, seed=3)
            few.Q, few.K, few.V = b.Q[r + 1 - rows:r + 1], [b.K[0][:end]], [b.V[0][:end]]
            few.store()
            got, gz = attend(few, split=split, window=window)
            assert torch.equal(got, full[r + 1 - rows:r + 1]) and torch.equal(gz, z[r + 1 - rows:r + 1]), f"{rows} rows up to row {r}"


@pytest.mark.parametrize("split", [0, 128])
@pytest.mark.parametrize("window", [0, 100])
@pytest.mark.parametrize("form", ["few", "many"])
def test_news_of_odd_values_keeps_to_its_item(form, window, split):
    """Twenty items and more for each CTA: short and long sequences, some without new rows, tiles alone and in pairs, parts that a tile does not
    see.  The odd values of scattered sequences reach those sequences' rows and elements, all of them, and nothing else changes by a bit."""
    r = random.Random(7)
    n = 700 if form == "few" else 260
    q = [r.choice([0, 1, 1, 1]) if form == "few" else r.choice([0, 1, 40, 64, 65, 130, 200]) for _ in range(n)]
    kv = [x + r.choice([0, r.randint(0, 40), r.randint(0, 400)]) for x in q]
    b = Batch(q, kv, hq=16, hkv=8, d=64, page=16, dtype=BF, seed=1, tail_rows=3)
    clean, cz = attend(b, split=split, window=window)
    want = torch.zeros(b.T, 8, 64, dtype=torch.bool, device=DEV)
    at = 0
    for i, (rows, m) in enumerate(zip(q, kv)):
        if rows and r.random() < 0.3:
            key, head, col = r.randrange(m), r.randrange(8), r.randrange(64)
            b.V[i][key, head, col] = r.choice([INF, -INF, NAN])
            place = torch.arange(m - rows, m, device=DEV)
            want[at:at + rows, head, col] = (place >= key) & (place < key + (window or 1 << 30))
        at += rows
    b.store()
    got, z = attend(b, split=split, window=window)
    want = want.repeat_interleave(2, 1)
    assert int(want.sum()) > 100 and torch.equal(z, cz)
    assert not bool(torch.isfinite(got[want]).any()) and torch.equal(got[~want], clean[~want])


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
def test_axes_that_share_their_positions(dtype):
    """One row of positions expanded over the axes is what the row repeated is, alone and on the way into the cache."""
    T = 37
    x = torch.randn(T, 4, 64, device=DEV)
    p = torch.randint(0, 9000, (T,), device=DEV).to(dtype)
    desc, f = rg.rg_rope_desc(rot_dim=64, sections=(8, 12, 12)), inv_freq(64)
    want = rg.rg_rope(desc, x, p.repeat(3, 1), f, torch.empty_like(x))
    assert torch.equal(rg.rg_rope(desc, x, p.expand(3, T), f, torch.empty_like(x)), want)
    assert torch.equal(rg.rg_rope(rg.rg_rope_desc(rot_dim=64), x, p, f, torch.empty_like(x)), want)
    b = Batch([T], [50], hq=2, hkv=2, d=64, page=16, dtype=BF, garbage=3.0)
    k, stored = torch.randn(T, 2, 64, device=DEV).to(BF), []
    for pos in (p.repeat(3, 1), p.expand(3, T)):
        kc, vc = torch.full_like(b.kc, 3.0), torch.full_like(b.vc, 3.0)
        rg.rg_kv_append(desc, k, k, f, kc, vc, b.seqs(), pos=pos)
        stored.append((kc, vc))
    assert torch.equal(stored[0][0], stored[1][0]) and torch.equal(stored[0][1], stored[1][1])


@pytest.mark.parametrize("q_len", [1, 40])
@pytest.mark.parametrize("dtype", [HF, BF])
def test_many_small_weights_next_to_a_large_one(dtype, q_len):
    """One key of weight 1 whose value is 0 and 60000 of weight e^-18, 2^-26, whose values are 1 or -2: together a thousandth, and all of the result.
    In fp16 the narrowed weight is off by half a step of 2^-24, or of its own; scaled by 2^7 that is 2^-32 of the largest weight, which the sum is at
    least.  (Unscaled, 2^-26 narrows to 0.)  In bf16 the half step is the weight's own."""
    n = 60000
    b = Batch([q_len], [n], hq=4, hkv=2, d=64, page=64, dtype=dtype, seed=1)
    b.Q.zero_()
    b.Q[..., 0] = 1.0
    b.K[0].zero_()
    b.K[0][1:, :, 0] = -18.0
    b.V[0].fill_(1.0)
    b.V[0][:, 1, 32:] = -2.0
    b.V[0][0] = 0.0
    b.store()
    for split in (0, 512):
        out, z = attend(b, scale=1.0, split=split, out_dtype=torch.float32)
        o, lse, mass = _softmax64(b.Q, b.K[0], b.V[0], 1.0)
        bound, bound_z = attention_bounds(o, mass, torch.zeros_like(lse), 64, n, dtype, torch.float32)
        small = 2.0 ** -32 * n * b.V[0].abs().double().amax() if dtype == HF else 0.0
        # the exponent, 26 in size, is rounded by 2^-20 at most
        assert bool(((out.double() - o).abs() <= bound + small + 2.0 ** -20 * mass).all()) and bool((o != 0).all())
        # a quarter's running sum takes n / 128 additions, each rounded by 2^-24 of it
        assert bool(((z.double() - lse).abs() <= bound_z + 2.0 ** -20 + n / 128 * 2.0 ** -24).all())
        one, oz = attend(b, scale=1.0, split=split)                            # and in the cache's own type
        assert torch.equal(one, out.to(dtype)) and torch.equal(oz, z)

"""Paged append and attention at the edges of what their calls allow: tables and positions that sequences or axes share, values and
scores that are not finite or very large, and results that must not depend on which kernel or tile takes a row."""
import pytest
import torch

import paper_2609_11356_b200 as rg
from tests._paged_util import DEV, Batch, attend, attention_bounds, check

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

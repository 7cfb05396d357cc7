"""Paged append and attention at the edges of what their calls allow: tables and positions that sequences or axes share, values and
scores that are not finite or very large, and results that must not depend on which kernel or tile takes a row."""
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

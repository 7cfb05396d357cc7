"""How the binding describes tensors of the paged calls whose rows share memory, and what it refuses: no GPU needed."""
import ctypes as C

import pytest
import torch

import paper_2609_11356_b200 as rg
from paper_2609_11356_b200 import _cabi as K, api
from tests.test_paged_host import DESC, SHAPE, WS, append, attend, cache, pos, rope, rows, seqs

I32 = dict(dtype=torch.int32)


def _seqs(table, n):
    return rg.rg_paged_seqs(table, torch.zeros(n, **I32), torch.zeros(n + 1, **I32), max_q=1, max_len=9)


def test_a_table_row_that_all_sequences_share_keeps_its_stride():
    row = torch.arange(64, **I32)[None]
    assert _seqs(row.expand(4, -1), 4).c.table_ld == 0                        # as a dense table it would be read 192 entries past its end
    assert _seqs(row, 1).c.table_ld == 64 and _seqs(row.repeat(4, 1), 4).c.table_ld == 64
    assert _seqs(torch.zeros(4, 80, **I32)[:, 8:72], 4).c.table_ld == 80
    assert _seqs(torch.zeros(8, 64, **I32)[::2], 4).c.table_ld == 128
    assert _seqs(row[:, :1].expand(4, 1), 4).c.table_ld == 0
    for ld in (1, 63):
        with pytest.raises(ValueError, match="overlap"):
            _seqs(torch.zeros(400, **I32).as_strided((4, 64), (ld, 1)), 4)


def test_the_library_takes_one_table_row_for_all_and_no_overlapping_ones():
    for ld in (1, 7):
        assert append(s=seqs(table_ld=ld)) == SHAPE and attend(s=seqs(table_ld=ld)) == SHAPE
    d = rg.rg_paged_attn_desc(scale=1.0, split=128)
    need = lambda ld: K.load().rg_paged_attention_workspace_bytes(C.byref(d), C.byref(seqs(table_ld=ld, table_cols=9, max_len=129)), 16, 10, 4, 64)
    assert need(8) == 0 and need(0) == need(9) > 0                            # 0: refused


def _attend(lse=None, ws=None, split=0):
    """The public call on host tensors: what it refuses for its layout comes before the refusal of the device."""
    q, cache = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(5, 16, 2, 64, dtype=torch.bfloat16)
    rg.rg_paged_attention(rg.rg_paged_attn_desc(scale=1.0, split=split), q, cache, cache, _seqs(torch.zeros(1, 5, **I32), 1), torch.zeros_like(q), lse=lse, ws=ws)


@pytest.mark.parametrize("lse", [torch.zeros(1, 2).expand(4, 2), torch.zeros(9).as_strided((4, 2), (1, 1)), torch.zeros(1, 1).expand(4, 2)])
def test_normalisers_whose_rows_share_memory_are_refused(lse):
    with pytest.raises(ValueError, match="lse"):                              # written as if dense, they would be written past their end
        _attend(lse=lse)


@pytest.mark.parametrize("lse", [torch.zeros(4, 2), torch.zeros(4, 6)[:, 1:3], torch.zeros(8, 2)[::2]])
def test_normalisers_of_any_other_stride_are_not(lse):
    with pytest.raises(ValueError, match="CUDA device"):
        _attend(lse=lse)


def test_a_workspace_has_the_bytes_that_it_holds():
    byte, words = torch.zeros(1, dtype=torch.uint8), torch.zeros(8, 64)
    for ws, n in ((None, 0), (byte.expand(1 << 20), 1), (words[:1].expand(100, 64), 256), (words[:, :1].expand(8, 64), 4 * (7 * 64 + 1)), (words, 2048), (words.T, 2048),
                  (words.view(-1)[::2], 1024), (words[:0], 0), (words[:0].expand(0, 64), 0), (words[:0].T, 0)):
        assert api._workspace(ws) == (None if ws is None else ws.data_ptr(), n)
    a, c = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(2, 2)
    d = rg.rg_desc(cuts=(32,))
    need = rg.rg_gemm_workspace_bytes(d, 2, 2)
    for ws in (byte.expand(need), torch.zeros(need - 1, dtype=torch.uint8)):
        with pytest.raises(rg.RgError) as e:                                  # the expanded byte passed for all of it
            rg.rg_gemm(d, a, a, c, ws=ws)
        assert e.value.status == WS


def test_matrices_whose_rows_share_memory_are_refused():
    """rg_gemm and the reductions: an expanded matrix is not described as a dense one."""
    a, c, v = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(2, 2), torch.zeros(2)
    row = torch.zeros(1, 64, dtype=torch.bfloat16).expand(2, 64)
    over = torch.zeros(80, dtype=torch.bfloat16).as_strided((2, 64), (16, 1))
    for call in (lambda: rg.rg_gemm(rg.rg_desc(), row, a, c), lambda: rg.rg_gemm(rg.rg_desc(), a, over, c), lambda: rg.rg_gemm(rg.rg_desc(), a, a, c[:1].expand(2, 2)),
                 lambda: rg.rg_reduce_rows(rg.rg_desc(), rg.RG_OP_SUM, row, v), lambda: rg.rg_reduce_rows(rg.rg_desc(), rg.RG_OP_SUM, a, v[:1].expand(2))):
        with pytest.raises(rg.RgError) as e:
            call()
        assert e.value.status == SHAPE
    for t, ld in ((a, 64), (a[:1], 64), (torch.zeros(2, 80)[:, :64], 80), (torch.zeros(1, 80)[:, :64], 80), (torch.zeros(4, 64)[::2], 128), (torch.zeros(0, 64), 64),
                  (torch.zeros(3, 1), 1), (v, 1), (torch.zeros(6)[::3], 3), (v[:1], 1), (v[:1].expand(1), 1)):
        assert api._tensor(t).ld == ld


@pytest.mark.parametrize("kw", [{"slot_stride": 0}, {"head_stride": 0}, {"page_stride": 0}, {"head_stride": 32}, {"slot_stride": 64}, {"page_stride": 1024}, {"page_stride": 2047},
                                {"slot_stride": 127}, {"head_stride": 16 * 64 - 1, "slot_stride": 64}, {"pages": 2 ** 31 - 1024, "page_stride": 64, "slot_stride": 2 ** 38, "head_stride": 2 ** 37 - 2 ** 16 - 1},
                                {"pages": 2 ** 31 - 1024, "page_stride": 2 ** 37, "slot_stride": 64, "head_stride": 2 ** 38}])
def test_a_cache_whose_elements_share_memory_is_not_written(kw):
    assert append(kc=cache(**kw), vc=cache(**{k: v for k, v in kw.items() if k == "pages"})) == SHAPE
    assert append(kc=cache(**{k: v for k, v in kw.items() if k == "pages"}), vc=cache(**kw)) == SHAPE


@pytest.mark.parametrize("kw", [{}, {"head_stride": 1024, "slot_stride": 64}, {"page_stride": 4096}, {"page_stride": 128, "slot_stride": 640}, {"page_stride": 64, "slot_stride": 320, "head_stride": 5120},
                                {"page": 1, "slot_stride": 0, "page_stride": 128}, {"pages": 1, "page_stride": 0}, {"slot_stride": 2 ** 38}, {"page_stride": 2 ** 38, "slot_stride": 2 ** 33}])
def test_a_cache_of_any_nested_strides_is(kw):
    assert append(k=rows(0), v=rows(0), kc=cache(**kw), vc=cache(**kw)) == 0    # no tokens: accepted, nothing launched
    heads = cache(heads=1, head_stride=0)
    assert append(k=rows(0, heads=1), v=rows(0, heads=1), kc=heads, vc=heads) == 0


def test_axes_that_share_their_positions():
    """pos.expand(3, T), text under three axes: one row that all of them read."""
    d = rg.rg_rope_desc(rot_dim=64, sections=(8, 12, 12))
    nobody = seqs(n_seqs=0, block_table=None, seq_lens=None, cu_q=None)         # so nothing is launched
    assert append(d=d, pos=pos(3, ld=0), s=nobody) == 0 and append(d=d, pos=pos(3, ld=4), s=nobody) == 0
    assert rope(d=d, x=rows(0), out=rows(0), pos=pos(3, cols=0, ld=0)) == 0
    for ld in (1, 3):
        assert rope(d=d, pos=pos(3, ld=ld)) == SHAPE and append(d=d, pos=pos(3, ld=ld)) == SHAPE


@pytest.mark.parametrize("kw", [{"style": 256}, {"style": -1}, {"inverse": 256}, {"inverse": -256}, {"rot_dim": 2 ** 32 + 64}, {"rot_dim": -64}, {"sections": (2 ** 32 + 32,)}, {"sections": (33, -1)}])
def test_rope_fields_that_do_not_fit_are_refused(kw):
    with pytest.raises(rg.RgError) as e:                                      # 256 is 0 in a byte: another rotation, without a word
        rg.rg_rope_desc(**({"rot_dim": 64} | kw))
    assert e.value.status == DESC


@pytest.mark.parametrize("kw", [{"mask": 256}, {"mask": -1}, {"split": 2 ** 32}, {"split": 2 ** 32 + 128}, {"window": 2 ** 32}, {"window": -1}])
def test_attention_fields_that_do_not_fit_are_refused(kw):
    with pytest.raises(rg.RgError) as e:
        rg.rg_paged_attn_desc(scale=1.0, **kw)
    assert e.value.status == DESC


@pytest.mark.parametrize("kw", [{"max_q": 2 ** 63}, {"max_len": 2 ** 64 + 5}, {"max_q": -1}, {"max_len": -5}])
def test_bounds_that_do_not_fit_are_refused(kw):
    with pytest.raises(rg.RgError) as e:
        rg.rg_paged_seqs(torch.zeros(1, 5, **I32), torch.zeros(1, **I32), torch.zeros(2, **I32), **kw)
    assert e.value.status == SHAPE

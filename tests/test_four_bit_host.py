"""What the four-bit entry points refuse: every check comes before anything is launched, so it needs no GPU.  And how their handles describe tensors."""
import ctypes as C

import pytest
import torch

import paper_2609_11356_b200 as rg
from paper_2609_11356_b200 import _cabi as K
from paper_2609_11356_b200 import api

FAKE = 1 << 20                                               # an address that no refused call may touch
OK, NULL, DESC, UNSUPPORTED, SHAPE, ALIGN, WS = 0, 1, 2, 3, 4, 5, 6


def rows(tokens=4, heads=2, dim=64, dtype=K.RG_BF16, ptr=FAKE, **kw):
    return K.rg_rows_t(ptr, dtype, tokens, heads, dim, kw.get("token_stride", heads * dim), kw.get("head_stride", dim))


def cache(pages=5, page=16, heads=2, dim=64, ptr=FAKE, **kw):
    block = page * dim * 9 // 16
    return K.rg_cache_four_t(ptr, pages, page, heads, dim, kw.get("page_stride", heads * block), kw.get("head_stride", block))


def seqs(**kw):
    a = dict(block_table=FAKE, table_ld=8, table_cols=8, n_seqs=2, seq_lens=FAKE, cu_q=FAKE, max_q=4, max_len=100) | kw
    return K.rg_paged_seqs_t(*a.values())


def w4(**kw):
    a = dict(codes=FAKE, scales=FAKE, zeros=None, rows=32, cols=256, code_ld=128, scale_ld=2, zero_ld=0, group=128, scale_dtype=K.RG_BF16, w_static=0) | kw
    return K.rg_weights_four_t(*a.values())


def matrix(rows_=3, cols=256, dtype=K.RG_BF16, ld=None, ptr=FAKE):
    return K.rg_tensor_t(ptr, dtype, rows_, cols, cols if ld is None else ld)


def _ref(v):
    return C.byref(v) if isinstance(v, C.Structure) else v


def gemv(**kw):
    a = dict(w=w4(), A=matrix(), C=matrix(3, 32), epi=None) | kw
    return K.load().rg_gemv_four(*map(_ref, a.values()), None)


def append(**kw):
    a = dict(d=rg.rg_rope_desc(rot_dim=64), k=rows(), v=rows(), pos=None, f=FAKE, kc=cache(), vc=cache(), s=seqs(), q=None, q_out=None) | kw
    return K.load().rg_kv_append_four(*map(_ref, a.values()), None)


def read(**kw):
    a = dict(kc=cache(), vc=cache(), s=seqs(), k=rows(), v=rows()) | kw
    return K.load().rg_kv_read_four(*map(_ref, a.values()), None)


def attend(**kw):
    a = dict(d=rg.rg_paged_attn_desc(scale=0.1), q=rows(heads=4), kc=cache(), vc=cache(), s=seqs(), out=rows(heads=4), lse=None, lse_ld=0, ws=None, n=0) | kw
    return K.load().rg_paged_attention_four(*map(_ref, a.values()), None)


def epilogue(**kw):
    e = K.rg_epilogue_t()
    for k, v in kw.items():
        setattr(e, k, v)
    return e


@pytest.mark.parametrize("status,kw", [
    (NULL, {"w": None}), (NULL, {"A": None}), (NULL, {"C": None}), (NULL, {"w": w4(codes=None)}), (NULL, {"w": w4(scales=None)}), (NULL, {"A": matrix(ptr=None)}),
    (UNSUPPORTED, {"w": w4(group=16)}), (UNSUPPORTED, {"w": w4(group=256)}), (UNSUPPORTED, {"w": w4(group=0)}), (UNSUPPORTED, {"w": w4(group=-32)}),
    (SHAPE, {"w": w4(scale_dtype=K.RG_F8E4M3)}), (SHAPE, {"w": w4(scale_dtype=K.RG_I32)}), (SHAPE, {"w": w4(w_static=2)}), (SHAPE, {"w": w4(rows=-1)}), (SHAPE, {"w": w4(cols=0), "A": matrix(cols=0)}),
    (UNSUPPORTED, {"w": w4(cols=250), "A": matrix(cols=250, ld=256)}), (SHAPE, {"w": w4(code_ld=112)}), (SHAPE, {"w": w4(scale_ld=1)}), (SHAPE, {"w": w4(zeros=FAKE, zero_ld=1)}),
    (ALIGN, {"w": w4(code_ld=136)}), (ALIGN, {"w": w4(codes=FAKE + 8)}), (ALIGN, {"w": w4(scales=FAKE + 1)}), (ALIGN, {"w": w4(scales=FAKE + 2, scale_dtype=K.RG_F32)}),
    (UNSUPPORTED, {"A": matrix(dtype=K.RG_F32)}), (SHAPE, {"A": matrix(dtype=K.RG_F8E4M3)}), (SHAPE, {"A": matrix(cols=224)}), (SHAPE, {"C": matrix(4, 32)}), (SHAPE, {"C": matrix(3, 31)}),
    (SHAPE, {"A": matrix((1 << 19) + 1), "C": matrix((1 << 19) + 1, 32)}), (SHAPE, {"C": matrix(3, 32, ld=31)}), (ALIGN, {"A": matrix(ptr=FAKE + 2)}), (ALIGN, {"A": matrix(ld=260)}),
    (UNSUPPORTED, {"epi": epilogue(act=2)}), (SHAPE, {"epi": epilogue(bias=FAKE, bias_dtype=K.RG_F8E4M3)}), (SHAPE, {"epi": epilogue(residual=FAKE, ldr=31)}),
    (OK, {"A": matrix(0), "C": matrix(0, 32)}), (OK, {"w": w4(rows=0), "C": matrix(3, 0)}),
])
def test_gemv_refusals(status, kw):
    assert gemv(**kw) == status


@pytest.mark.parametrize("dtype,off", [(K.RG_BF16, 1), (K.RG_F16, 1), (K.RG_F32, 1), (K.RG_F32, 2)])
def test_gemv_refuses_results_and_epilogues_off_their_type(dtype, off):
    """Elements are accessed one by one, each where its type can lie."""
    assert gemv(C=matrix(3, 32, dtype=dtype, ptr=FAKE + off)) == ALIGN
    assert gemv(epi=epilogue(bias=FAKE + off, bias_dtype=dtype)) == ALIGN
    assert gemv(epi=epilogue(residual=FAKE + off, residual_dtype=dtype, ldr=32)) == ALIGN
    # nothing to compute, nothing to access
    assert gemv(A=matrix(0), C=matrix(0, 32, dtype=dtype, ptr=FAKE + off)) == OK


CACHES = [
    (NULL, None), (NULL, cache(ptr=None)), (SHAPE, cache(pages=-1)), (SHAPE, cache(page=0)), (SHAPE, cache(heads=0)), (SHAPE, cache(heads=65536)), (SHAPE, cache(dim=2048)),
    (UNSUPPORTED, cache(dim=48)), (UNSUPPORTED, cache(dim=160)), (UNSUPPORTED, cache(page=12)), (ALIGN, cache(ptr=FAKE + 8)), (ALIGN, cache(head_stride=16 * 36 + 8)),
    (ALIGN, cache(page_stride=2000 * 8 + 8)), (SHAPE, cache(page_stride=-16)), (SHAPE, cache(head_stride=1 << 40)),
]


@pytest.mark.parametrize("status,c", CACHES)
def test_caches_are_checked_everywhere(status, c):
    assert append(kc=c) == status and append(vc=c) == status
    assert read(kc=c) == status and read(vc=c) == status
    assert attend(kc=c) == status and attend(vc=c) == status


@pytest.mark.parametrize("status,kw", [
    (SHAPE, {"kc": cache(head_stride=0)}), (SHAPE, {"vc": cache(page_stride=0)}), (SHAPE, {"kc": cache(page_stride=16 * 36)}), (SHAPE, {"vc": cache(head_stride=16 * 35)}),
    (SHAPE, {"kc": cache(pages=6)}), (SHAPE, {"kc": cache(heads=3), "vc": cache(heads=3)}), (SHAPE, {"kc": cache(dim=32), "vc": cache(dim=32)}), (SHAPE, {"vc": cache(page=8)}),
    (NULL, {"k": None}), (NULL, {"v": rows(ptr=None)}), (SHAPE, {"v": rows(tokens=5)}), (SHAPE, {"v": rows(dtype=K.RG_F16)}), (SHAPE, {"k": rows(dtype=K.RG_F8E4M3)}),
    (NULL, {"s": None}), (NULL, {"s": seqs(cu_q=None)}), (SHAPE, {"s": seqs(table_ld=7)}), (SHAPE, {"s": seqs(n_seqs=-1)}),
    (NULL, {"q": rows(heads=4)}), (NULL, {"f": None}), (ALIGN, {"f": FAKE + 4}), (DESC, {"d": None}), (UNSUPPORTED, {"d": rg.rg_rope_desc(rot_dim=64, inverse=1)}),
    (SHAPE, {"d": rg.rg_rope_desc(rot_dim=128)}), (DESC, {"d": rg.rg_rope_desc(rot_dim=64, sections=(16, 16))}), (DESC, {"d": rg.rg_rope_desc(rot_dim=63)}),
    (SHAPE, {"q": rows(heads=4), "q_out": rows(heads=5)}), (SHAPE, {"q": rows(heads=4), "q_out": rows(heads=4, head_stride=8)}), (SHAPE, {"q": rows(tokens=3), "q_out": rows(tokens=3)}),
    (OK, {"k": rows(tokens=0), "v": rows(tokens=0)}), (OK, {"s": seqs(n_seqs=0)}),
])
def test_append_refusals(status, kw):
    assert append(**kw) == status


@pytest.mark.parametrize("status,kw", [
    (NULL, {"k": None}), (SHAPE, {"k": rows(heads=3), "v": rows(heads=3)}), (SHAPE, {"v": rows(dtype=K.RG_F16)}), (SHAPE, {"k": rows(head_stride=0)}), (SHAPE, {"v": rows(token_stride=64)}),
    (SHAPE, {"k": rows(dim=32), "v": rows(dim=32)}), (SHAPE, {"vc": cache(pages=4)}), (NULL, {"s": None}), (ALIGN, {"k": rows(ptr=FAKE + 1)}),
    (OK, {"k": rows(tokens=0), "v": rows(tokens=0)}), (OK, {"s": seqs(n_seqs=0)}),
])
def test_read_refusals(status, kw):
    assert read(**kw) == status


@pytest.mark.parametrize("status,kw", [
    (NULL, {"d": None}), (DESC, {"d": rg.rg_paged_attn_desc(scale=0.0)}), (DESC, {"d": rg.rg_paged_attn_desc(scale=1.0, split=100)}), (DESC, {"d": rg.rg_paged_attn_desc(scale=1.0, window=5, mask=0)}),
    (NULL, {"q": None}), (UNSUPPORTED, {"q": rows(heads=4, dtype=K.RG_F32), "out": rows(heads=4, dtype=K.RG_F32)}), (SHAPE, {"out": rows(heads=4, dtype=K.RG_F16)}), (SHAPE, {"out": rows(heads=3)}),
    (SHAPE, {"q": rows(heads=3), "out": rows(heads=3)}), (SHAPE, {"kc": cache(dim=32), "vc": cache(dim=32)}), (SHAPE, {"vc": cache(heads=1)}), (SHAPE, {"vc": cache(page=32)}),
    (UNSUPPORTED, {"q": rows(heads=258), "out": rows(heads=258), "kc": cache(), "vc": cache()}), (ALIGN, {"q": rows(heads=4, ptr=FAKE + 8)}), (ALIGN, {"q": rows(heads=4, token_stride=260)}),
    (UNSUPPORTED, {"q": rows(heads=4, token_stride=0)}), (SHAPE, {"out": rows(heads=4, token_stride=0)}), (SHAPE, {"lse": FAKE, "lse_ld": 3}), (SHAPE, {"lse": FAKE + 2, "lse_ld": 4}),
    (WS, {"d": rg.rg_paged_attn_desc(scale=1.0, split=128), "s": seqs(max_len=0)}), (ALIGN, {"d": rg.rg_paged_attn_desc(scale=1.0, split=128), "s": seqs(max_len=0, table_cols=9, table_ld=9), "ws": FAKE + 8, "n": 1 << 30}),
    (OK, {"q": rows(tokens=0, heads=4), "out": rows(tokens=0, heads=4)}), (OK, {"s": seqs(n_seqs=0)}),
])
def test_attention_refusals(status, kw):
    if status == WS:
        kw["s"] = seqs(max_len=0, table_cols=9, table_ld=9)
    assert attend(**kw) == status


def test_block_bytes():
    assert rg.rg_cache_four_block_bytes(16, 128) == 1152 and rg.rg_cache_four_block_bytes(8, 32) == 144
    for page, dim in ((0, 64), (12, 64), (-8, 64), (16, 48), (16, 160), (16, 0), ((1 << 20) + 8, 64)):
        assert rg.rg_cache_four_block_bytes(page, dim) == 0


def test_one_row_has_no_stride():
    """Nothing lies a stride behind a single row, so a view into a wider buffer of any pitch is described as a dense row; several rows keep theirs."""
    buf = torch.zeros(3, 259, dtype=torch.bfloat16)
    for t, ld in ((buf[:1, :256], 256), (buf[2:, 1:257], 256), (buf[:0, :256], 256), (buf[:2, :256], 259), (buf[:1, :256].expand(2, 256), 0)):
        assert api._TENSOR.unpack(api._matrix(t)) == (t.data_ptr(), K.RG_BF16, t.shape[0], 256, ld)


def test_handles_describe_their_tensors():
    t = torch.zeros(3, 2, 1152, dtype=torch.uint8)
    c = rg.rg_cache_four(t, page_size=16, dim=128).c
    assert (c.pages, c.page_size, c.heads, c.dim, c.page_stride, c.head_stride) == (3, 16, 2, 128, 2304, 1152)
    c = rg.rg_cache_four(t.transpose(0, 1).contiguous().transpose(0, 1), page_size=16, dim=128).c
    assert (c.page_stride, c.head_stride) == (1152, 3456)
    for bad, kw in ((t, {"page_size": 32, "dim": 128}), (t.float(), {"page_size": 16, "dim": 128}), (t[0], {"page_size": 16, "dim": 128}), (t[:, :, ::2], {"page_size": 8, "dim": 128})):
        with pytest.raises(ValueError):
            rg.rg_cache_four(bad, **kw)
    with pytest.raises(rg.RgError):
        rg.rg_cache_four(t, page_size=12, dim=128)
    codes, s = torch.zeros(6, 128, dtype=torch.uint8), torch.zeros(6, 2, dtype=torch.float16)
    c = rg.rg_weights_four(codes, s, zeros=torch.zeros(6, 2, dtype=torch.uint8), group=128).c
    assert (c.rows, c.cols, c.code_ld, c.scale_ld, c.zero_ld, c.group, c.scale_dtype) == (6, 256, 128, 2, 2, 128, K.RG_F16)
    assert rg.rg_weights_four(codes[:1].expand(6, 128), s).c.code_ld == 0                       # rows that share memory are the library's to refuse
    for bad in (dict(scales=s[:5]), dict(scales=s, group=64), dict(scales=s.to(torch.uint8)), dict(scales=s, zeros=s), dict(scales=s, zeros=torch.zeros(6, 3, dtype=torch.uint8)), dict(scales=s.T)):
        with pytest.raises(ValueError):
            rg.rg_weights_four(codes, **bad)
    with pytest.raises(rg.RgError):
        rg.rg_weights_four(codes, s, group=-128)
    w = rg.rg_weights_four(codes, s)
    with pytest.raises(ValueError):                              # not on a GPU
        rg.rg_gemv_four(w, torch.zeros(2, 256, dtype=torch.bfloat16), torch.zeros(2, 6, dtype=torch.bfloat16))

"""What the entry points of the positions and the paged cache refuse: every check comes before anything is launched, so it needs no GPU."""
import ctypes as C

import pytest
import torch

import paper_2609_11356_b200 as rg
from paper_2609_11356_b200 import _cabi as K

FAKE = 1 << 20                                               # an address that no refused call may touch
NULL, DESC, UNSUPPORTED, SHAPE, ALIGN, WS = 1, 2, 3, 4, 5, 6


def rows(tokens=4, heads=2, dim=64, dtype=K.RG_BF16, ptr=FAKE, **kw):
    return K.rg_rows_t(ptr, dtype, tokens, heads, dim, kw.get("token_stride", heads * dim), kw.get("head_stride", dim))


def cache(pages=5, page=16, heads=2, dim=64, dtype=K.RG_BF16, ptr=FAKE, **kw):
    return K.rg_cache_t(ptr, dtype, pages, page, heads, dim, kw.get("page_stride", page * heads * dim), kw.get("slot_stride", heads * dim), kw.get("head_stride", dim))


def seqs(**kw):
    a = dict(block_table=FAKE, table_ld=8, table_cols=8, n_seqs=2, seq_lens=FAKE, cu_q=FAKE, max_q=4, max_len=100) | kw
    return K.rg_paged_seqs_t(*a.values())


def pos(rows_=1, cols=4, dtype=K.RG_I32, ld=4, ptr=FAKE):
    return K.rg_tensor_t(ptr, dtype, rows_, cols, ld)


def _ref(v):
    return C.byref(v) if isinstance(v, C.Structure) else v


def rope(**kw):
    a = dict(d=rg.rg_rope_desc(rot_dim=64), x=rows(), pos=pos(), f=FAKE, out=rows()) | kw
    return K.load().rg_rope(*map(_ref, a.values()), None)


def append(**kw):
    a = dict(d=rg.rg_rope_desc(rot_dim=64), k=rows(), v=rows(), pos=None, f=FAKE, kc=cache(), vc=cache(), s=seqs(), q=None, q_out=None) | kw
    return K.load().rg_kv_append(*map(_ref, a.values()), None)


def attend(**kw):
    a = dict(d=rg.rg_paged_attn_desc(scale=0.1), q=rows(heads=4), kc=cache(), vc=cache(), s=seqs(), out=rows(heads=4), lse=None, lse_ld=0, ws=None, n=0) | kw
    return K.load().rg_paged_attention(*map(_ref, a.values()), None)


def _wrong(make, **fields):
    x = make
    for k, v in fields.items():
        setattr(x, k, v)
    return x


@pytest.mark.parametrize("status,kw", [
    (NULL, {"d": None}), (NULL, {"pos": None}), (NULL, {"f": None}), (NULL, {"x": None}), (NULL, {"x": rows(ptr=None)}), (NULL, {"pos": pos(ptr=None)}),
    (DESC, {"d": rg.rg_rope_desc(rot_dim=63)}), (DESC, {"d": rg.rg_rope_desc(rot_dim=0)}), (DESC, {"d": rg.rg_rope_desc(rot_dim=64, sections=(16, 15))}),
    (DESC, {"d": rg.rg_rope_desc(rot_dim=64, style=7)}), (DESC, {"d": _wrong(rg.rg_rope_desc(rot_dim=64), size=3)}), (DESC, {"d": _wrong(rg.rg_rope_desc(rot_dim=64), n_axes=0)}),
    (DESC, {"d": _wrong(rg.rg_rope_desc(rot_dim=64), n_axes=5)}), (DESC, {"d": _wrong(rg.rg_rope_desc(rot_dim=64), inverse=2)}),
    (UNSUPPORTED, {"d": rg.rg_rope_desc(rot_dim=514), "x": rows(dim=600), "out": rows(dim=600)}),
    (SHAPE, {"d": rg.rg_rope_desc(rot_dim=66)}), (SHAPE, {"x": rows(dim=65), "out": rows(dim=65)}), (SHAPE, {"out": rows(tokens=3)}), (SHAPE, {"out": rows(dtype=K.RG_F16)}),
    (SHAPE, {"x": rows(dtype=K.RG_F8E4M3)}), (SHAPE, {"out": rows(token_stride=0)}), (SHAPE, {"out": rows(head_stride=32)}), (SHAPE, {"x": rows(token_stride=-128)}),
    (SHAPE, {"pos": pos(cols=3)}), (SHAPE, {"pos": pos(rows_=2)}), (SHAPE, {"pos": pos(dtype=K.RG_F32)}), (SHAPE, {"d": rg.rg_rope_desc(rot_dim=64, sections=(30, 2)), "pos": pos(2, ld=3)}),
    (SHAPE, {"x": rows(heads=70000), "out": rows(heads=70000)}), (SHAPE, {"x": rows(dim=2000), "out": rows(dim=2000)}),
    (ALIGN, {"f": FAKE + 4}), (ALIGN, {"x": rows(ptr=FAKE + 1)}), (ALIGN, {"pos": pos(dtype=K.RG_I64, ptr=FAKE + 4)}),
])
def test_rope_refuses(status, kw):
    assert rope(**kw) == status


@pytest.mark.parametrize("status,kw", [
    (NULL, {"k": None}), (NULL, {"kc": None}), (NULL, {"s": None}), (NULL, {"f": None}), (NULL, {"q": rows()}), (NULL, {"q_out": rows()}), (NULL, {"s": seqs(block_table=None)}),
    (NULL, {"s": seqs(cu_q=None)}), (NULL, {"kc": cache(ptr=None)}), (DESC, {"d": None}), (DESC, {"d": None, "f": None, "pos": pos()}), (DESC, {"d": rg.rg_rope_desc(rot_dim=64, sections=(16, 16))}),
    (UNSUPPORTED, {"d": rg.rg_rope_desc(rot_dim=64, inverse=1)}), (SHAPE, {"v": rows(heads=1)}), (SHAPE, {"kc": cache(dtype=K.RG_F16)}), (SHAPE, {"kc": cache(heads=1)}),
    (SHAPE, {"vc": cache(pages=4)}), (SHAPE, {"vc": cache(page=8)}), (SHAPE, {"kc": cache(dim=32)}), (SHAPE, {"q": rows(dim=32), "q_out": rows(dim=32)}), (SHAPE, {"q": rows(3), "q_out": rows(3)}),
    (SHAPE, {"s": seqs(n_seqs=-1)}), (SHAPE, {"s": seqs(table_ld=7)}), (SHAPE, {"s": seqs(max_len=-1)}), (SHAPE, {"pos": pos(cols=5)}), (SHAPE, {"kc": cache(slot_stride=-1)}), (ALIGN, {"kc": cache(ptr=FAKE + 1)}),
])
def test_append_refuses(status, kw):
    assert append(**kw) == status


@pytest.mark.parametrize("status,kw", [
    (NULL, {"d": None}), (NULL, {"q": None}), (NULL, {"out": None}), (NULL, {"vc": None}), (NULL, {"s": None}), (NULL, {"q": rows(heads=4, ptr=None)}),
    (DESC, {"d": rg.rg_paged_attn_desc(scale=0.0)}), (DESC, {"d": rg.rg_paged_attn_desc(scale=-1.0)}), (DESC, {"d": rg.rg_paged_attn_desc(scale=float("nan"))}), (DESC, {"d": rg.rg_paged_attn_desc(scale=float("inf"))}),
    (DESC, {"d": rg.rg_paged_attn_desc(scale=1.0, split=64)}), (DESC, {"d": rg.rg_paged_attn_desc(scale=1.0, window=3, mask=0)}), (DESC, {"d": rg.rg_paged_attn_desc(scale=1.0, mask=2)}),
    (DESC, {"d": _wrong(rg.rg_paged_attn_desc(scale=1.0), size=1)}), (DESC, {"d": rg.rg_paged_attn_desc(scale=1.0, split=(1 << 30) + 128)}),
    (UNSUPPORTED, {"q": rows(heads=4, dtype=K.RG_F32)}), (UNSUPPORTED, {"q": rows(heads=4, dim=60), "out": rows(heads=4, dim=60), "kc": cache(dim=60), "vc": cache(dim=60)}),
    (UNSUPPORTED, {"q": rows(heads=4, dim=136), "out": rows(heads=4, dim=136), "kc": cache(dim=136), "vc": cache(dim=136)}), (UNSUPPORTED, {"kc": cache(page=12), "vc": cache(page=12)}),
    (UNSUPPORTED, {"q": rows(heads=258), "out": rows(heads=258)}),
    (SHAPE, {"q": rows(heads=3), "out": rows(heads=3)}), (SHAPE, {"out": rows(heads=4, dtype=K.RG_F16)}), (SHAPE, {"out": rows(heads=2)}), (SHAPE, {"kc": cache(dtype=K.RG_F16)}), (SHAPE, {"vc": cache(heads=4)}),
    (SHAPE, {"vc": cache(pages=6)}), (SHAPE, {"out": rows(heads=4, token_stride=0)}), (SHAPE, {"lse": FAKE, "lse_ld": 3}),
    (ALIGN, {"q": rows(heads=4, ptr=FAKE + 8)}), (ALIGN, {"q": rows(heads=4, head_stride=68)}), (ALIGN, {"kc": cache(slot_stride=132)}), (ALIGN, {"vc": cache(page_stride=2052)}), (ALIGN, {"kc": cache(ptr=FAKE + 2)}),
    (WS, {"d": rg.rg_paged_attn_desc(scale=1.0, split=128), "s": seqs(max_len=0, table_cols=9, table_ld=9)}), (WS, {"d": rg.rg_paged_attn_desc(scale=1.0, split=128), "s": seqs(max_len=129, table_cols=9, table_ld=9), "ws": FAKE, "n": 8}),
    (ALIGN, {"d": rg.rg_paged_attn_desc(scale=1.0, split=128), "s": seqs(max_len=129, table_cols=9, table_ld=9), "ws": FAKE + 4, "n": 1 << 30}),
])
def test_attention_refuses(status, kw):
    assert attend(**kw) == status


@pytest.mark.parametrize("status,kw", [
    # strides of all operands first, then dimensions that repeat an address, then addresses
    (ALIGN, {"q": rows(heads=4, head_stride=68), "kc": cache(slot_stride=0)}), (ALIGN, {"q": rows(heads=4, token_stride=260), "vc": cache(page_stride=0)}), (ALIGN, {"q": rows(heads=4, token_stride=0), "vc": cache(head_stride=68)}),
    (UNSUPPORTED, {"q": rows(heads=4, token_stride=0), "kc": cache(ptr=FAKE + 8)}), (UNSUPPORTED, {"q": rows(heads=4, ptr=FAKE + 8), "vc": cache(head_stride=0)}),
    (SHAPE, {"lse": FAKE, "lse_ld": 3, "kc": cache(slot_stride=132)}), (SHAPE, {"lse": FAKE, "lse_ld": 3, "q": rows(heads=4, ptr=FAKE + 8)}), (UNSUPPORTED, {"q": rows(heads=258, token_stride=258 * 64 + 4), "out": rows(heads=258)}),
])
def test_attention_with_two_faults_names_the_one_that_comes_first(status, kw):
    assert attend(**kw) == status


def test_nothing_to_do_is_fine():
    assert rope(x=rows(0), out=rows(0), pos=pos(cols=0)) == 0
    assert append(k=rows(0), v=rows(0)) == 0 and append(s=seqs(n_seqs=0, block_table=None, seq_lens=None, cu_q=None)) == 0
    assert attend(q=rows(0, heads=4), out=rows(0, heads=4)) == 0 and attend(s=seqs(n_seqs=0, block_table=None, seq_lens=None, cu_q=None)) == 0


def test_workspace_bytes():
    need = lambda split, max_len, cols=100, page=16: K.load().rg_paged_attention_workspace_bytes(C.byref(rg.rg_paged_attn_desc(scale=1.0, split=split)), C.byref(seqs(max_len=max_len, table_cols=cols, table_ld=cols)), page, 10, 4, 64)
    assert need(0, 1000) == 0 and need(128, 128) == 0
    assert need(128, 129) == 10 * 4 * 2 * 66 * 4 // 256 * 256 + (256 if 10 * 4 * 2 * 66 * 4 % 256 else 0)
    assert need(512, 0) == need(512, 1600) == need(512, 10 ** 6)              # the table's capacity is the bound


def test_binding_checks_types_before_the_library():
    t = torch.zeros(2, 3, dtype=torch.int32)
    ok = rg.rg_paged_seqs(t, torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), max_q=1, max_len=9)
    for args in ((t.long(), ok.seq_lens, ok.cu_q), (t, ok.seq_lens.float(), ok.cu_q), (t, ok.seq_lens, ok.cu_q[:2]), (t[:1], ok.seq_lens, ok.cu_q), (t.T, ok.seq_lens, ok.cu_q)):
        with pytest.raises(ValueError):
            rg.rg_paged_seqs(*args)
    x = torch.zeros(4, 2, 64)
    with pytest.raises(ValueError):                                            # host tensors
        rg.rg_rope(rg.rg_rope_desc(rot_dim=64), x, torch.zeros(4, dtype=torch.int32), torch.zeros(32, dtype=torch.float64), x)
    with pytest.raises(rg.RgError):
        rg.rg_rope_desc(rot_dim=10, sections=(1, 1, 1, 1, 1))
    with pytest.raises(rg.RgError):
        rg.rg_paged_attn_desc(scale=1.0, split=-128)

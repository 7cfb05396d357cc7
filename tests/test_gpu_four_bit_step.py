"""The four-bit operators as a server runs them: one layer's decode step (product, append, attention, product), captured once and replayed while the
sequences grow, against the same step in 64 bits."""
import math

import pytest
import torch

import paper_2609_11356_b200 as rg
from tests._four_bit_util import from_codes, to_codes
from tests._paged_util import DEV, EPS, generator, inv_freq, rotate64
from tests.test_gpu_gemv_four import dense, weights

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_decode_steps_in_a_graph():
    S, hq, hkv, d, page, width, steps = 5, 8, 2, 64, 16, 512, 20
    rows = hq + 2 * hkv
    g = generator(1)
    wq, wo = weights(rows * d, width, 64, seed=1), weights(width, hq * d, 64, seed=2)
    W, O = rg.rg_weights_four(wq[0], wq[1], zeros=wq[2], group=64, w_static=1), rg.rg_weights_four(wo[0], wo[1], zeros=wo[2], group=64, w_static=1)
    x, qkv = torch.zeros(S, width, dtype=BF, device=DEV), torch.empty(S, rows * d, dtype=BF, device=DEV)
    heads = qkv.view(S, rows, d)
    q, k, v = heads[:, :hq], heads[:, hq:hq + hkv], heads[:, hq + hkv:]
    per = -(-steps // page)
    kc, vc = (torch.randint(0, 256, (S * per + 1, hkv, rg.rg_cache_four_block_bytes(page, d)), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2))
    kh, vh = rg.rg_cache_four(kc, page_size=page, dim=d), rg.rg_cache_four(vc, page_size=page, dim=d)
    table = torch.randperm(S * per, generator=g, device=DEV).to(torch.int32).view(S, per)
    lens = torch.zeros(S, dtype=torch.int32, device=DEV)
    seqs = rg.rg_paged_seqs(table, lens, torch.arange(S + 1, dtype=torch.int32, device=DEV), max_q=1, max_len=steps)
    freq, rope, desc = inv_freq(d), rg.rg_rope_desc(rot_dim=d), rg.rg_paged_attn_desc(scale=d ** -0.5)
    att, y = torch.empty(S, hq, d, dtype=BF, device=DEV), torch.empty(S, width, dtype=BF, device=DEV)

    def step():
        rg.rg_gemv_four(W, x, qkv)
        rg.rg_kv_append_four(rope, k, v, freq, kh, vh, seqs, q=q, q_out=q)
        rg.rg_paged_attention_four(desc, q, kh, vh, seqs, att)
        rg.rg_gemv_four(O, att.view(S, hq * d), y, residual=x)

    lens.fill_(1)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()                                    # the inputs are another stream's work
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    W64, O64 = dense(*wq, 64), dense(*wo, 64)
    K, V = [], []
    for t in range(steps):
        x.copy_(torch.randn(S, width, generator=g, device=DEV))
        lens.fill_(t + 1)
        graph.replay()
        torch.cuda.synchronize()
        # each stage from the stage before as the framework rounded it, so that the bounds are those of one operator
        qkv64 = (x.double() @ W64.T).view(S, rows, d)
        assert bool(((heads[:, hq:].double() - qkv64[:, hq:]).abs() <= EPS[BF] * qkv64[:, hq:].abs() + 2.0 ** -12 * (x.double().abs() @ W64.abs().T).view(S, rows, d)[:, hq:]).all())
        pos = torch.full((1, S), t, device=DEV)
        K.append(from_codes(*to_codes(rotate64(k, pos, freq, (d // 2,), rg.RG_ROPE_HALF)[0])))
        V.append(from_codes(*to_codes(v.double())))
        q64 = rotate64(qkv64[:, :hq], pos, freq, (d // 2,), rg.RG_ROPE_HALF)[0]
        size = rotate64(qkv64[:, :hq], pos, freq, (d // 2,), rg.RG_ROPE_HALF)[1]
        mass = (x.double().abs() @ W64.abs().T).view(S, rows, d)[:, :hq].amax(-1, keepdim=True)
        assert bool(((q.double() - q64).abs() <= 3 * EPS[BF] * size + 2.0 ** -11 * mass).all())      # rounded before and after the rotation
        kk, vv = torch.stack(K, 2).repeat_interleave(hq // hkv, 1), torch.stack(V, 2).repeat_interleave(hq // hkv, 1)      # [S, hq, t + 1, d]
        p = torch.softmax((kk @ q.double()[..., None]).squeeze(-1) / math.sqrt(d), -1)[:, :, None]
        o = (p @ vv).squeeze(2)
        assert bool(((att.double() - o).abs() <= 3 * EPS[BF] * (p @ vv.abs()).squeeze(2)).all())        # weights and result narrowed
        y64 = att.double().view(S, -1) @ O64.T + x.double()
        assert bool(((y.double() - y64).abs() <= EPS[BF] * y64.abs() + 2.0 ** -12 * (att.double().abs().view(S, -1) @ O64.abs().T + 1)).all())
    assert rg.rg_device_status() == 0

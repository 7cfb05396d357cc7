"""Rotary positions and the paged append on the GPU, against the definition in 64 bits; then the operators as a server runs them."""
import pytest
import torch

import paper_2609_11356_b200 as rg
from tests._paged_util import DEV, Batch, attend, attention64, attention_bounds, generator, inv_freq, rotate64, rotation_bound

pytestmark = pytest.mark.gpu
BF, HF, F4 = torch.bfloat16, torch.float16, torch.float32
HALF, PAIRS = rg.RG_ROPE_HALF, rg.RG_ROPE_PAIRS


@pytest.fixture(autouse=True)
def healthy():
    yield
    assert rg.rg_device_status() == 0


def _within(got, y, size):
    off = (got.double() - y).abs() - rotation_bound(y, size, got.dtype)
    assert bool((off <= 0).all()), f"off by {off.max().item()} more than the bound at {(off == off.max()).nonzero()[0].tolist()}"


@pytest.mark.parametrize("style", [HALF, PAIRS])
@pytest.mark.parametrize("dtype", [BF, HF, F4])
@pytest.mark.parametrize("T,H,d,rot,sections", [(1, 1, 2, 2, (1,)), (3, 5, 64, 64, (32,)), (700, 8, 128, 128, (64,)), (257, 3, 80, 40, (6, 7, 7)), (33, 2, 96, 32, (16, 0)),
                                                (19, 7, 250, 246, (100, 20, 2, 1)), (1030, 1, 512, 512, (128, 128)), (5, 33, 130, 6, (1, 1, 1)), (4001, 2, 16, 16, (8,))])
def test_rope(T, H, d, rot, sections, dtype, style):
    g = generator(T + d)
    x = torch.randn(T, H, d, generator=g, device=DEV).to(dtype)
    pos = torch.randint(-50, 1 << 21, (len(sections), T), generator=g, device=DEV)
    f = inv_freq(rot)
    for inverse in (0, 1):
        desc = rg.rg_rope_desc(rot_dim=rot, style=style, sections=sections, inverse=inverse)
        y, size = rotate64(x, pos, f, sections, style, -1.0 if inverse else 1.0)
        out = torch.full_like(x, 77.0)
        rg.rg_rope(desc, x, pos, f, out)
        _within(out, y, size)
        out32 = rg.rg_rope(desc, x, pos.to(torch.int32), f, torch.empty_like(x))
        assert torch.equal(out, out32), "32-bit and 64-bit positions"
        assert torch.equal(out[..., rot:], x[..., rot:]), "what is not rotated passes through"
        inplace = x.clone()
        rg.rg_rope(desc, inplace, pos, f, inplace)
        assert torch.equal(inplace, out), "in place"


def test_far_positions():
    """Positions of 2^40: a 32-bit angle would be noise."""
    x = torch.randn(9, 2, 64, generator=generator(1), device=DEV)
    pos = (torch.arange(9, device=DEV) + (1 << 40))[None]
    f = inv_freq(64)
    out = rg.rg_rope(rg.rg_rope_desc(rot_dim=64), x, pos, f, torch.empty_like(x))
    y, size = rotate64(x, pos, f, (32,), HALF)
    # the angle itself, formed in 64 bits, carries 2^40 * 2 roundings of 2^-53 on either side: 2^-11 rad here
    assert bool(((out.double() - y).abs() <= 2.0 ** -10 * size).all())


def test_rope_strides_and_rows():
    T, d = 301, 64
    for dtype, pad in ((BF, 3), (F4, 1), (HF, 8)):
        big = torch.randn(T, 6, d + pad, generator=generator(2), device=DEV).to(dtype)
        x = big[:, 1:4, pad:]                                                    # rows that no vector load can read when pad is odd
        pos = torch.arange(T, device=DEV)
        f = inv_freq(d)
        ob = torch.full((4, T, d + pad), 5.0, dtype=dtype, device=DEV)
        out = ob[1:4, :, :d].transpose(0, 1)
        rg.rg_rope(rg.rg_rope_desc(rot_dim=d), x, pos, f, out)
        _within(out, *rotate64(x, pos[None], f, (32,), HALF))
        rest = ob.clone()
        rest[1:4, :, :d] = 5.0
        assert bool((rest == 5.0).all())
        # a row's bits do not depend on its neighbours
        one = rg.rg_rope(rg.rg_rope_desc(rot_dim=d), x[77:78], pos[77:78], f, torch.empty(1, 3, d, dtype=dtype, device=DEV))
        assert torch.equal(one[0], out[77])


def test_gradient_is_the_inverse_rotation():
    T, H, d, sections = 50, 3, 32, (6, 5, 5)
    g = generator(3)
    x = torch.randn(T, H, d, generator=g, device=DEV)
    pos = torch.randint(0, 9000, (3, T), generator=g, device=DEV)
    f = inv_freq(32)
    w = torch.randn(T, H, d, generator=g, device=DEV)
    for style in (HALF, PAIRS):
        grad = rg.rg_rope(rg.rg_rope_desc(rot_dim=d, style=style, sections=sections, inverse=1), w, pos, f, torch.empty_like(w))
        x64 = x.double().requires_grad_()
        y, _ = rotate64(x64, pos, f, sections, style)
        (y * w.double()).sum().backward()
        _, size = rotate64(w, pos, f, sections, style)
        assert bool(((grad.double() - x64.grad).abs() <= rotation_bound(x64.grad, size, F4)).all())
        # against differences of the forward call: the loss is linear, so one step of any length is exact up to rounding
        e = torch.randn(T, H, d, generator=g, device=DEV)
        fwd = lambda v: (rg.rg_rope(rg.rg_rope_desc(rot_dim=d, style=style, sections=sections), v, pos, f, torch.empty_like(v)).double() * w.double()).sum()
        diff, want = fwd(x + e) - fwd(x), (grad.double() * ((x + e) - x).double()).sum()
        # 2 forward sums and one of the gradient, each term within 2^-20 of its operands' size
        room = 2.0 ** -19 * ((x + e).abs().double() + x.abs().double() + e.abs().double()).sum() * float(w.abs().max()) * 2
        assert abs(float(diff - want)) <= float(room)


@pytest.mark.parametrize("dtype", [BF, HF, F4])
@pytest.mark.parametrize("hq,hkv,d,rot,style,page,sections", [(4, 2, 64, 64, HALF, 16, None), (5, 1, 80, 40, PAIRS, 1, None), (1, 1, 6, 2, HALF, 3, None), (8, 8, 128, 128, HALF, 64, (32, 16, 16)),
                                                              (32, 8, 128, 64, PAIRS, 7, (32,))])
def test_append(hq, hkv, d, rot, style, page, sections, dtype):
    q, kv = [1, 0, 37, 300, 1, 2], [1, 0, 37, 513, 260, 77]
    b = Batch(q, kv, hq=hq, hkv=hkv, d=d, page=page, dtype=dtype, seed=d, heads_first=d == 64, garbage=3.0, tail_rows=5)
    g = generator(9)
    qkv = torch.randn(b.T, hq + 2 * hkv, d, generator=g, device=DEV).to(dtype)
    qr, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    place = torch.cat([torch.arange(m - n, m, device=DEV) for n, m in zip(q, kv)] + [torch.zeros(5, dtype=torch.long, device=DEV)])
    pos = None if sections is None else torch.randint(0, 70000, (len(sections), b.T), generator=g, device=DEV)
    sec = sections or (rot // 2,)
    f = inv_freq(rot)
    kc0, vc0 = b.kc.clone(), b.vc.clone()
    out = torch.full((b.T, hq, d), 77.0, dtype=dtype, device=DEV)
    rg.rg_kv_append(rg.rg_rope_desc(rot_dim=rot, style=style, sections=sec), k, v, f, b.kc, b.vc, b.seqs(), pos=pos, q=qr, q_out=out)
    P = place[None] if pos is None else pos
    n = sum(q)
    y, size = rotate64(qr, P, f, sec, style)
    _within(out[:n], y[:n], size[:n])
    assert bool((out[n:] == 77.0).all())
    ky, ks = rotate64(k, P, f, sec, style)
    at = 0
    for i, (a, m) in enumerate(zip(q, kv)):
        if a:
            page_, slot = (x[m - a:] for x in b.where(i))
            _within(b.kc[page_, slot], ky[at:at + a], ks[at:at + a])
            assert torch.equal(b.vc[page_, slot], v[at:at + a])
            b.kc[page_, slot], b.vc[page_, slot] = kc0[page_, slot], vc0[page_, slot]
            at += a
    assert torch.equal(b.kc, kc0) and torch.equal(b.vc, vc0), "slots of other tokens were written"
    # without rotation: a copy
    rg.rg_kv_append(None, k, v, None, b.kc, b.vc, b.seqs())
    at = 0
    for i, (a, m) in enumerate(zip(q, kv)):
        page_, slot = (x[m - a:] for x in b.where(i))
        assert torch.equal(b.kc[page_, slot], k[at:at + a]) and torch.equal(b.vc[page_, slot], v[at:at + a])
        at += a


def test_append_outside_is_told_and_touches_nothing():
    b = Batch([2, 3, 1], [40, 50, 17], hq=2, hkv=2, d=64, page=16, seed=2, garbage=3.0)
    k = torch.randn(6, 2, 64, device=DEV).to(BF)
    for change in ("page", "huge", "long", "short"):
        c = Batch([2, 3, 1], [40, 50, 17], hq=2, hkv=2, d=64, page=16, seed=2, garbage=3.0)
        want_k = c.kc.clone()
        rg.rg_kv_append(None, k, k, None, c.kc, c.vc, c.seqs())
        want_k = c.kc.clone()
        c = Batch([2, 3, 1], [40, 50, 17], hq=2, hkv=2, d=64, page=16, seed=2, garbage=3.0)
        old = c.kc.clone()
        page, slot = (x[47:] for x in c.where(1))
        if change == "page":
            c.table[1] = -3
        elif change == "huge":
            c.table[1] = 2 ** 31 - 1
        elif change == "long":
            c.seq_lens[1] = 2 ** 31 - 1
        else:
            c.seq_lens[1] = 0
        rg.rg_kv_append(None, k, k, None, c.kc, c.vc, c.seqs())
        assert rg.rg_device_status() == rg.RG_PAGE_CODE_APPEND
        want_k[page, slot] = old[page, slot]
        assert torch.equal(c.kc, want_k), change


def test_append_offsets_past_32_bits():
    d, page = 64, 8
    pages = 2 ** 31 // (page * d) + 8
    kc = torch.empty(pages, page, 1, d, dtype=BF, device=DEV)
    b = Batch([5], [13], hq=1, hkv=1, d=d, page=page, seed=2)
    b.table[0] = torch.tensor([pages - 1, pages - 3])
    k = torch.randn(5, 1, d, device=DEV).to(BF)
    rg.rg_kv_append(None, k, k, None, kc, kc, b.seqs())
    assert torch.equal(kc[pages - 3, :5], k)


def test_refusals():
    x = torch.zeros(4, 2, 64, device=DEV)
    pos, f = torch.zeros(4, dtype=torch.int32, device=DEV), inv_freq(64)

    def refused(status, desc, **kw):
        a = {"x": x, "pos": pos, "inv_freq": f, "out": torch.empty_like(x)} | kw
        with pytest.raises(rg.RgError) as e:
            rg.rg_rope(desc, **a)
        assert e.value.status == status

    ok = rg.rg_rope_desc(rot_dim=64)
    refused(2, rg.rg_rope_desc(rot_dim=64, sections=(16, 15)))
    refused(2, rg.rg_rope_desc(rot_dim=64, style=2))
    refused(4, rg.rg_rope_desc(rot_dim=128), inv_freq=inv_freq(128))
    refused(4, ok, out=torch.empty(4, 2, 64, dtype=BF, device=DEV))
    refused(4, ok, out=torch.empty(1, 2, 64, device=DEV).expand(4, 2, 64))
    refused(4, rg.rg_rope_desc(rot_dim=64, sections=(16, 16)))
    for kw in ({"pos": pos.float()}, {"inv_freq": f.float()}, {"inv_freq": inv_freq(32)}, {"x": x.transpose(1, 2)}):
        with pytest.raises((ValueError, TypeError)):
            rg.rg_rope(ok, **({"x": x, "pos": pos, "inv_freq": f, "out": x} | kw))
    b = Batch([2], [5], hq=2, hkv=2, d=64, page=16)
    k = torch.zeros(2, 2, 64, dtype=BF, device=DEV)
    for kw in ({"d": rg.rg_rope_desc(rot_dim=64, inverse=1), "inv_freq": f}, {"d": rg.rg_rope_desc(rot_dim=64), "inv_freq": None}, {"d": rg.rg_rope_desc(rot_dim=64, sections=(16, 16)), "inv_freq": f},
               {"d": None, "inv_freq": None, "k": k.half()}, {"d": None, "inv_freq": f}):
        a = {"k": k, "v": k, "k_cache": b.kc, "v_cache": b.vc, "seqs": b.seqs()} | kw
        with pytest.raises(rg.RgError):
            rg.rg_kv_append(**a)


def test_a_server_s_steps():
    """Prompts in chunks, then single tokens in a captured graph: positions, cache and attention together, against attention over the
    whole rotated texts in 64 bits, and with the same bits whatever the chunks were."""
    hq, hkv, d, page, total = 8, 2, 64, 16, [150, 97]
    f = inv_freq(d)
    g = generator(31)
    text = [torch.randn(n, hq + 2 * hkv, d, generator=g, device=DEV).to(BF) for n in total]
    rope, desc = rg.rg_rope_desc(rot_dim=d), rg.rg_paged_attn_desc(scale=d ** -0.5, split=128)
    table = torch.tensor([[7, 1, 12, 5, 9, 3, 0, 14, 2, 18], [4, 6, 8, 10, 11, 13, 15, -1, -1, -1]], dtype=torch.int32, device=DEV)

    def serve(chunks, decode):
        kc = torch.full((19, page, hkv, d), float("nan"), dtype=BF, device=DEV)
        vc = kc.clone()
        got = [[], []]
        done = [0, 0]
        for n in chunks:
            take = [min(n, t - decode - x) for t, x in zip(total, done)]
            rows = torch.cat([text[i][done[i]:done[i] + take[i]] for i in (0, 1)])
            done = [x + y for x, y in zip(done, take)]
            seqs = rg.rg_paged_seqs(table, torch.tensor(done, dtype=torch.int32, device=DEV), torch.tensor([0, take[0], sum(take)], dtype=torch.int32, device=DEV), max_q=n, max_len=150)
            q = torch.empty(rows.shape[0], hq, d, dtype=BF, device=DEV)
            rg.rg_kv_append(rope, rows[:, hq:hq + hkv], rows[:, hq + hkv:], f, kc, vc, seqs, q=rows[:, :hq], q_out=q)
            ws = torch.empty(rg.rg_paged_attention_workspace_bytes(desc, seqs, rows.shape[0], hq, d), dtype=torch.uint8, device=DEV)
            out = rg.rg_paged_attention(desc, q, kc, vc, seqs, torch.empty_like(q), ws=ws)
            got[0].append(out[:take[0]]); got[1].append(out[take[0]:])
        lens = torch.tensor(done, dtype=torch.int32, device=DEV)
        seqs = rg.rg_paged_seqs(table, lens, torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV), max_q=1, max_len=150)
        rows = torch.empty(2, hq + 2 * hkv, d, dtype=BF, device=DEV)
        q, out = torch.empty(2, hq, d, dtype=BF, device=DEV), torch.empty(2, hq, d, dtype=BF, device=DEV)
        ws = torch.empty(rg.rg_paged_attention_workspace_bytes(desc, seqs, 2, hq, d), dtype=torch.uint8, device=DEV)

        def step():
            lens.add_(1)
            rg.rg_kv_append(rope, rows[:, hq:hq + hkv], rows[:, hq + hkv:], f, kc, vc, seqs, q=rows[:, :hq], q_out=q)
            rg.rg_paged_attention(desc, q, kc, vc, seqs, out, ws=ws)

        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            step()
        for k in range(decode):
            rows.copy_(torch.stack([text[i][total[i] - decode + k] for i in (0, 1)]))
            graph.replay()
            got[0].append(out[:1].clone()); got[1].append(out[1:].clone())
        torch.cuda.synchronize()
        return [torch.cat(x) for x in got]

    a = serve([64, 80], 6)
    b = serve([1, 17, 3, 129], 6)
    c = serve([150], 20)
    for i in (0, 1):
        assert torch.equal(a[i], b[i]) and torch.equal(a[i], c[i]), "the chunks a text came in changed its bits"
        pos = torch.arange(total[i], device=DEV)[None]
        rq, _ = rotate64(text[i][:, :hq], pos, f, (d // 2,), HALF)
        rk, _ = rotate64(text[i][:, hq:hq + hkv], pos, f, (d // 2,), HALF)
        # the operators narrow rotated rows to bf16 on the way; both roundings are made here too, up to ties that fp32 may break differently
        o, _, mass, size = attention64(rq.to(BF), rk.to(BF), text[i][:, hq + hkv:], d ** -0.5)
        bound, _ = attention_bounds(o, mass, size, d, total[i], BF, BF)
        extra = 2 * 2.0 ** -8 * size[..., None] * mass                          # and a rounding that went the other way is a step of one operand
        assert bool(((a[i].double() - o).abs() <= bound + extra).all())

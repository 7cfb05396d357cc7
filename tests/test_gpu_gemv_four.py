"""Products of a few rows with four-bit weights, on the GPU against the definition in 64 bits."""
import pytest
import torch

import paper_2609_11356_b200 as rg
from tests._paged_util import DEV, EPS, generator

pytestmark = pytest.mark.gpu
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


def weights(N, K, group, *, scales=BF, zeros=True, seed=0, pad=0):
    g = generator(seed)
    n = -(-K // group)
    codes = torch.randint(0, 256, (N, K // 2 + pad), generator=g, device=DEV, dtype=torch.uint8)[:, :K // 2]
    s = (torch.randn(N, n + pad, generator=g, device=DEV) * 0.01).to(scales)[:, :n]
    z = torch.randint(0, 16, (N, n + pad), generator=g, device=DEV, dtype=torch.uint8)[:, :n] if zeros else None
    return codes, s, z


def dense(codes, s, z, group):
    K = 2 * codes.shape[1]
    u = torch.stack((codes % 16, codes // 16), -1).flatten(1).double()
    zero = z.double() if z is not None else torch.full_like(s, 8, dtype=torch.float64)
    return (u - zero.repeat_interleave(group, 1)[:, :K]) * s.double().repeat_interleave(group, 1)[:, :K]


def expected(A, W, K, group, out_dtype, bias=None, act=0, residual=None):
    """The definition, and how far off the kernel may be.  A tensor-core step adds 17 numbers, each cut at 2^-24 of the largest or finer, so at most 17 2^-24 of the sum of
    magnitudes; a group has group / 16 of them, then one fused rounding for each of the at most ceil(K / group) groups and one for each of eight parts, 2^-24
    each.  Epilogue: a rounding for each addition; SiLU is off by 2^-20 of its value and passes errors on with a slope below 1.1."""
    y = A.double() @ W.T
    err = (A.double().abs() @ W.abs().T) * 2.0 ** -24 * (17 * group / 16 + -(-K // group) + 8)
    if bias is not None:
        y = y + bias.double()
        err = err + 2.0 ** -24 * (y.abs() + err)
    if act:
        err = 1.1 * err + 2.0 ** -20 * (y * torch.sigmoid(y)).abs()
        y = y * torch.sigmoid(y)
    if residual is not None:
        y = y + residual.double()
        err = err + 2.0 ** -24 * (y.abs() + err)
    return y, err + EPS[out_dtype] * (y.abs() + err) + (2.0 ** -25 if out_dtype == HF else 2.0 ** -149)


def product(A, codes, s, z, group, out_dtype, **kw):
    C = torch.full((A.shape[0], codes.shape[0]), float("nan"), dtype=out_dtype, device=DEV)
    static = kw.pop("w_static", 0)
    return rg.rg_gemv_four(rg.rg_weights_four(codes, s, zeros=z, group=group, w_static=static), A, C, **kw)


def check(A, codes, s, z, group, out_dtype, **kw):
    got = product(A, codes, s, z, group, out_dtype, **kw)
    kw.pop("w_static", None)
    y, bound = expected(A, dense(codes, s, z, group), A.shape[1], group, out_dtype, **kw)
    off = (got.double() - y).abs() - bound
    assert bool((off <= 0).all()), f"off by {off.max().item()} more than the bound"
    return got


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(1, 32), (17, 96), (16, 128), (33, 256), (100, 288), (1000, 4096), (65, 2080), (48, 14336), (5, 2048 + 32)])
@pytest.mark.parametrize("M", [1, 3, 8, 9, 16, 17, 33])
def test_sizes_and_groups(M, N, K, group, zeros):
    A = torch.randn(M, K, generator=generator(M + N), device=DEV).to(BF)
    check(A, *weights(N, K, group, zeros=zeros, seed=K), group, BF)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("out_dtype", [BF, HF, F32])
@pytest.mark.parametrize("scales", [BF, HF, F32])
def test_types(dtype, out_dtype, scales):
    for M, group in ((1, 128), (12, 64), (40, 32)):
        A = torch.randn(M, 1056, generator=generator(M), device=DEV).to(dtype)
        check(A, *weights(70, 1056, group, scales=scales, seed=M), group, out_dtype)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_32_bit_results_are_as_exact_as_a_32_bit_sum(dtype):
    A = torch.randn(8, 14336, generator=generator(1), device=DEV).to(dtype)
    w = weights(256, 14336, 128, scales=F32, seed=2)
    got, y = product(A, *w, 128, F32).double(), A.double() @ dense(*w, 128).T
    # 2^-24 for each rounding of some hundred of like size, which add up like a random walk: well below 2^-20 of the result's size
    assert float((got - y).norm() / y.norm()) < 2.0 ** -20


@pytest.mark.parametrize("M", [1, 5, 20])
@pytest.mark.parametrize("bias,act,residual", [(True, 0, False), (False, 1, False), (False, 0, True), (True, 1, True)])
def test_epilogue(M, bias, act, residual):
    g = generator(7)
    N, K = 131, 512
    A = torch.randn(M, K, generator=g, device=DEV).to(BF)
    for t in (BF, F32):
        b = torch.randn(N, generator=g, device=DEV).to(t) if bias else None
        r = torch.randn(M, N + 3, generator=g, device=DEV).to(t)[:, 1:N + 1] if residual else None
        check(A, *weights(N, K, 64, seed=3), 64, t, bias=b, act=act, residual=r)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(333, 4096), (40, 8224)])
def test_bits_do_not_depend_on_the_other_rows(N, K, group, dtype):
    A = torch.randn(70, K, generator=generator(5), device=DEV).to(dtype)
    w = weights(N, K, group, seed=6)
    whole = product(A, *w, group, F32)
    for lo, hi in ((0, 1), (3, 4), (69, 70), (0, 8), (5, 14), (10, 26), (30, 70), (1, 65)):
        assert torch.equal(product(A[lo:hi], *w, group, F32), whole[lo:hi])
    # nor on the other rows of the weights
    assert torch.equal(product(A[:2], w[0][16:49], w[1][16:49], w[2][16:49], group, F32), whole[:2, 16:49])
    assert torch.equal(product(A, *w, group, F32, w_static=1), whole)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(30011, 2112), (15000, 4096), (7001, 4128), (250, 1056), (129, 544)])
def test_bits_do_not_depend_on_how_many_ctas_share_k(N, K, group):
    """Numbers of rows with 1, 2, 4 and all 8 parts of K a CTA, in one pass over the rows and in two, the last CTA's weights cut."""
    codes, s, z = weights(N, K, group, seed=N)
    A = torch.randn(81, K, generator=generator(5), device=DEV).to(BF)
    full = check(A, codes, s, z, group, F32)
    for M in (1, 2, 3, 8, 9, 16, 17, 24, 25, 32, 33, 40, 41, 72):
        assert torch.equal(product(A[:M].contiguous(), codes, s, z, group, F32), full[:M]), M


def test_strides():
    K, N, M = 544, 90, 11
    codes, s, z = weights(N, K, 32, pad=16, seed=9)
    assert codes.stride(0) == K // 2 + 16
    A = torch.full((M, K + 24), float("nan"), dtype=BF, device=DEV)[:, 8:K + 8]
    A.copy_(torch.randn(M, K, generator=generator(2), device=DEV))
    want = check(A, codes, s, z, 32, BF)
    assert torch.equal(product(A.contiguous(), codes.contiguous(), s.contiguous(), z.contiguous(), 32, BF), want)
    out = torch.full((M, N + 5), 3.0, dtype=BF, device=DEV)
    rg.rg_gemv_four(rg.rg_weights_four(codes, s, zeros=z, group=32), A, out[:, 2:N + 2])
    assert torch.equal(out[:, 2:N + 2], want) and bool((out[:, :2] == 3.0).all()) and bool((out[:, N + 2:] == 3.0).all())


def test_numbers_that_are_not_finite_stay_in_their_row():
    K, N = 512, 40
    A = torch.randn(4, K, generator=generator(2), device=DEV).to(BF)
    w = weights(N, K, 128, zeros=False, seed=1)
    w[0][:, 50] = 0x99                                           # codes 9 and 9: weights above zero times the scale
    clean = product(A, *w, 128, F32)
    A[1, 100], A[2, 100] = float("inf"), float("nan")
    got = product(A, *w, 128, F32)
    assert torch.equal(got[[0, 3]], clean[[0, 3]]) and bool(got[2].isnan().all())
    sign = torch.sign(w[1][:, 100 // 128].float())
    assert torch.equal(got[1], sign * float("inf"))


def test_empty():
    codes, s, z = weights(10, 64, 32)
    assert product(torch.zeros(0, 64, dtype=BF, device=DEV), codes, s, z, 32, BF).shape == (0, 10)
    assert product(torch.zeros(3, 64, dtype=BF, device=DEV), codes[:0], s[:0], z[:0], 32, BF).shape == (3, 0)


def test_back_to_back_on_two_streams_and_in_a_graph():
    """A chain in which every product's result is the next one's input, with the promise about the weights: no call may read early what the one before writes."""
    N = K = 1024
    w = [rg.rg_weights_four(*weights(N, K, 64, seed=i)[:2], group=64, w_static=1) for i in range(6)]
    x0 = torch.randn(2, K, generator=generator(3), device=DEV).to(BF)

    def chain(x):
        for m in w:
            x = rg.rg_gemv_four(m, x, torch.empty(2, N, dtype=BF, device=DEV))
        return x

    want = x0
    for m in w:
        want = rg.rg_gemv_four(m, want, torch.empty(2, N, dtype=BF, device=DEV))
        torch.cuda.synchronize()
    assert bool(want.isfinite().all()) and float(want.abs().max()) > 0
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for i in range(8):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(chain(x0))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = chain(x0)
    for _ in range(5):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("M,K", [(5, 1024), (40, 1024), (12, 2560), (70, 544)])
def test_chains_of_several_rows(M, K):
    """The same with the form for more rows, whose CTAs share K in clusters of several sizes: on two streams at a time, and captured twice."""
    w = [rg.rg_weights_four(*weights(K, K, 128, seed=i)[:2], group=128, w_static=1) for i in range(6)]
    x0 = torch.randn(M, K, generator=generator(3), device=DEV).to(BF)

    def chain(x):
        for m in w:
            x = rg.rg_gemv_four(m, x, torch.empty(M, K, dtype=BF, device=DEV))
        return x

    want = x0
    for m in w:
        want = rg.rg_gemv_four(m, want, torch.empty(M, K, dtype=BF, device=DEV))
        torch.cuda.synchronize()
    assert bool(want.isfinite().all()) and float(want.abs().max()) > 0
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs, graphs = [], []
    for i in range(8):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(chain(x0))
    torch.cuda.synchronize()
    for stream in streams:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            outs.append(chain(x0))
    for _ in range(3):
        for stream, graph in zip(streams, graphs):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_codes_beyond_32_bits():
    """Rows of weights more than 2^32 bytes apart from the first."""
    K, N = 64, 40
    ld = 2 ** 32 // 32
    store = torch.zeros((N - 1) * ld + K // 2, dtype=torch.uint8, device=DEV)
    codes = store.as_strided((N, K // 2), (ld, 1))
    c, s, z = weights(N, K, 32, seed=4)
    codes.copy_(c)
    A = torch.randn(3, K, generator=generator(2), device=DEV).to(BF)
    assert torch.equal(product(A, codes, s, z, 32, F32), product(A, c, s, z, 32, F32))


@pytest.mark.parametrize("pitch", [513, 515, 524])
def test_one_row_of_a_buffer_of_any_pitch(pitch):
    """A single token's row, contiguous and aligned, out of a buffer whose rows lie an odd number of elements apart; results and residual likewise."""
    K, N = 512, 40
    w = weights(N, K, 64, seed=3)
    A, out = torch.full((2, pitch), float("nan"), dtype=BF, device=DEV), torch.full((2, pitch), 3.0, dtype=BF, device=DEV)
    A[0, :K] = torch.randn(K, generator=generator(4), device=DEV).to(BF)
    r = torch.randn(2, N + 1, generator=generator(5), device=DEV)[:1, :N]
    want = check(A[:1, :K].clone(), *w, 64, BF, residual=r.clone())
    rg.rg_gemv_four(rg.rg_weights_four(w[0], w[1], zeros=w[2], group=64), A[:1, :K], out[:1, 1:N + 1], residual=r)
    assert torch.equal(out[:1, 1:N + 1], want) and bool((out[0, :1] == 3.0).all()) and bool((out[0, N + 1:] == 3.0).all()) and bool((out[1] == 3.0).all())


@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("N,K", [(250, 32), (250, 288), (129, 1056), (70, 1312), (333, 2080), (5000, 544), (15000, 1312)])
def test_sums_that_vanish_have_the_same_zero_in_every_number_of_rows(N, K, out_dtype):
    """Products below the smallest number of either sign: a group's scaled sum is rounded to a zero with its sign.  One to eight parts of K, whose missing ones some
    forms add as zeros and others do not; a row's zeros have the same bits in all of them."""
    codes, _, z = weights(N, K, 32, seed=K)
    s = torch.full((N, -(-K // 32)), 2.0 ** -100, dtype=F32, device=DEV) * torch.where(torch.arange(N, device=DEV) % 2 == 0, 1.0, -1.0)[:, None]
    A = torch.full((41, K), 2.0 ** -70, dtype=BF, device=DEV) * torch.where(torch.arange(41, device=DEV) % 3 == 0, 1.0, -1.0)[:, None].to(BF)
    for M in (1, 2, 4, 5, 8, 17, 33, 41):
        assert not bool(product(A[:M], codes, s, z, 32, out_dtype).view(torch.int16).any()), M


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(40, 1056), (4736, 288), (4737, 544), (8864, 2080), (8865, 544), (9472, 544), (9473, 2080), (14208, 544), (14209, 1056), (18944, 2080), (18945, 544), (30011, 544)])
def test_one_to_five_rows_on_weights_of_every_size(N, K, group, dtype):
    """Either side of every number of weights' rows at which up to five rows of A go to another tile, another number of warps or the other kernel: against the definition,
    and the same bits whatever comes along."""
    codes, s, z = weights(N, K, group, seed=N + K)
    A = torch.randn(6, K, generator=generator(N), device=DEV).to(dtype)
    full = check(A, codes, s, z, group, F32)
    for M in (1, 2, 3, 4, 5):
        assert torch.equal(product(A[:M].contiguous(), codes, s, z, group, F32), full[:M]), M
        assert torch.equal(product(A[6 - M:].contiguous(), codes, s, z, group, F32, w_static=1), full[6 - M:]), M


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(1, 32), (17, 96), (16, 128), (33, 256), (100, 288), (1000, 4096), (65, 2080), (48, 14336), (5, 2048 + 32)])
@pytest.mark.parametrize("M", [2, 4, 5])
def test_sizes_and_groups_at_the_border_of_the_kernels(M, N, K, group, zeros):
    A = torch.randn(M, K, generator=generator(M + N), device=DEV).to(BF)
    check(A, *weights(N, K, group, zeros=zeros, seed=K), group, BF)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(333, 4096), (40, 8224)])
def test_bits_of_four_and_five_rows(N, K, group, dtype):
    A = torch.randn(10, K, generator=generator(5), device=DEV).to(dtype)
    w = weights(N, K, group, seed=6)
    whole = product(A, *w, group, F32)
    for lo, hi in ((0, 4), (0, 5), (3, 7), (5, 10), (6, 10)):
        assert torch.equal(product(A[lo:hi], *w, group, F32), whole[lo:hi])

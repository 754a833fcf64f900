"""Products of microscaled matrices on the GPU against the same products of their values in binary64.

Tolerance: the products of codes and scales are exact; a sum of n blocks of 128 is at most n + 32 additions to a binary32
accumulator (the parts of a split contraction joined), each of which may cut a result rather than round it: 2^-23 of
what has been summed, which is never more than S = sum |a b|.  So |error| <= (n + 32) 2^-23 S; inside an instruction 128
terms are added to within 2^-23 of their magnitudes, another 2^-23 S.  A bf16 result is off by 2^-8 of itself more."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_08040_amd as fq
from tests import gpu_util as gu

F64 = torch.float64


def matrix(rows, cols, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((rows, cols), device="cuda", generator=g) * torch.exp(torch.randn((rows, 1), device="cuda", generator=g))
    return (scale * x).to(torch.bfloat16)


def values(q, side):
    return fq.fq_mx_dequantize(q, side, out_dtype=torch.float32).to(F64)


def operands(op, A, B):
    """Both with the contraction last, [M, K] and [N, K], in binary64."""
    r, c = fq.FQ_MX_ROWS, fq.FQ_MX_COLS
    if op == fq.FQ_OP_NT:
        return values(A, r), values(B, r)
    if op == fq.FQ_OP_NN:
        return values(A, r), values(B, c).T
    return values(A, c).T, values(B, c).T


def check(got, a, b):
    """got against a b^T."""
    want, size = a @ b.T, a.abs() @ b.abs().T
    bound = (-(-a.shape[1] // 128) + 33) * 2.0 ** -23 * size
    if got.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (want.abs() + bound)
    bad = (got.to(F64) - want).abs() > bound
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())


def shapes(op, M, N, K):
    """Shapes of A and B for an M x N output over a contraction of K."""
    return {fq.FQ_OP_NT: ((M, K), (N, K)), fq.FQ_OP_NN: ((M, K), (K, N)), fq.FQ_OP_TN: ((K, M), (K, N))}[op]


def pair(op, M, N, K, seed=0):
    sa, sb = shapes(op, M, N, K)
    return (fq.fq_mx_quantize(matrix(*sa, seed + 1), sides=fq.FQ_MX_BOTH),
            fq.fq_mx_quantize(matrix(*sb, seed + 2, 0.02), sides=fq.FQ_MX_BOTH, rule=fq.FQ_MX_COVER))


OPS = {"NT": fq.FQ_OP_NT, "NN": fq.FQ_OP_NN, "TN": fq.FQ_OP_TN}
SIZES = [(1, 1, 1), (1, 4096, 1024), (5, 33, 31), (16, 16, 128), (17, 65, 129), (33, 200, 700), (64, 64, 2048),
         (130, 70, 1), (257, 300, 515), (300, 513, 96), (1000, 40, 260), (520, 776, 1544),
         (1025, 1100, 130), (1111, 1300, 385), (1300, 2050, 1000)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("op", OPS)
def test_products(op, M, N, K):
    A, B = pair(OPS[op], M, N, K)
    a, b = operands(OPS[op], A, B)
    for dt in (torch.float32, torch.bfloat16):
        gu.announce(f"mx gemm {op} {M}x{N}x{K} {dt}")
        check(fq.fq_mx_gemm(OPS[op], A, B, out_dtype=dt), a, b)


# (compute units the planner is told of, M, N, K, the tiles that follow): workgroups that walk over several tiles, edges
# in both directions, contractions of one block and of odd and even numbers of them, shorter than the ring of stages
TILED = [(1, 512, 512, 2048, fq.FQ_MX_FORM_256x256), (2, 700, 900, 2100, fq.FQ_MX_FORM_256x256),
         (1, 500, 1020, 1921, fq.FQ_MX_FORM_256x256), (3, 1000, 700, 1700, fq.FQ_MX_FORM_256x256),
         (3, 1000, 530, 1700, fq.FQ_MX_FORM_128x128), (1, 1024, 1024, 100, fq.FQ_MX_FORM_128x128),
         (1, 2048, 2048, 200, fq.FQ_MX_FORM_256x256), (1, 1000, 1010, 300, fq.FQ_MX_FORM_256x256),
         (256, 4090, 4096, 1000, fq.FQ_MX_FORM_256x256),
         (1, 300, 300, 100, fq.FQ_MX_FORM_128x128), (1, 129, 400, 1, fq.FQ_MX_FORM_128x128),
         (2, 400, 333, 256, fq.FQ_MX_FORM_128x128), (1, 257, 131, 300, fq.FQ_MX_FORM_128x128),
         (3, 500, 420, 513, fq.FQ_MX_FORM_128x256), (4, 500, 420, 513, fq.FQ_MX_FORM_128x128),
         (3, 100, 500, 300, fq.FQ_MX_FORM_128x256), (5, 383, 250, 300, fq.FQ_MX_FORM_128x256),
         (1, 639, 999, 1500, fq.FQ_MX_FORM_128x256), (8, 250, 700, 2100, fq.FQ_MX_FORM_128x256),
         (256, 2040, 4090, 1921, fq.FQ_MX_FORM_128x256), (1, 140, 1000, 700, fq.FQ_MX_FORM_256x256),
         (1, 70, 1000, 700, fq.FQ_MX_FORM_128x128), (8, 130, 150, 900, fq.FQ_MX_FORM_64x64),
         (4, 60, 500, 600, fq.FQ_MX_FORM_64x64), (4, 30, 500, 600, fq.FQ_MX_FORM_32x64),
         (4, 100, 60, 1200, fq.FQ_MX_FORM_32x64)]


@pytest.mark.parametrize("cus,M,N,K,tiles", TILED)
def test_tiles(cus, M, N, K, tiles, monkeypatch):
    monkeypatch.setenv("FQ_GEMM_CUS", str(cus))
    assert fq.fq_mx_gemm_form(M, N, K)[0] == tiles
    op = [fq.FQ_OP_NT, fq.FQ_OP_NN, fq.FQ_OP_TN][(M + N + K) % 3]
    A, B = pair(op, M, N, K, K)
    a, b = operands(op, A, B)
    for dt in (torch.float32, torch.bfloat16):
        gu.announce(f"mx tiles {tiles} cus {cus} {M}x{N}x{K} {dt}")
        for ldc in (N, N + 1, N + 8):
            out = torch.full((M, ldc), 9.0, dtype=dt, device="cuda")
            fq.fq_mx_gemm(op, A, B, out=out[:, :N])
            check(out[:, :N], a, b)
            assert (out[:, N:] == 9.0).all()


@pytest.mark.parametrize("n,k", [(40, 300), (400, 400), (700, 700)])
def test_a_matrix_with_itself(n, k):
    """One tensor as both operands, either side."""
    q = fq.fq_mx_quantize(matrix(n, k, 4), sides=fq.FQ_MX_BOTH)
    for op in OPS if n == k else ("NT", "TN"):
        gu.announce(f"mx product of a {n} x {k} matrix with itself, op {op}")
        check(fq.fq_mx_gemm(OPS[op], q, q), *operands(OPS[op], q, q))


def test_products_of_small_integers_are_exact():
    """Whole numbers up to 6 at scale 1 and sums below 2^24: nothing may round."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    grid = torch.tensor([0.0, 1.0, 2.0, 3.0, 4.0, 6.0], device="cuda")
    for M, N, K in [(3, 5, 64), (70, 130, 384), (260, 514, 1030)]:
        x, w = (grid[torch.randint(0, 6, (n, K), device="cuda", generator=g)] * torch.sign(
            torch.randn((n, K), device="cuda", generator=g)) for n in (M, N))
        x[:, ::32] = w[:, ::32] = 4.0                                # every group's scale is 1
        A, B = fq.fq_mx_quantize(x.to(torch.bfloat16)), fq.fq_mx_quantize(w.to(torch.bfloat16))
        assert torch.equal(fq.fq_mx_gemm(fq.FQ_OP_NT, A, B).to(F64), x.to(F64) @ w.to(F64).T)


@pytest.mark.parametrize("M,N,K", [(7, 50, 300), (300, 280, 200)])
def test_strided_outputs_keep_their_neighbours(M, N, K):
    A, B = pair(fq.FQ_OP_NT, M, N, K)
    want = {dt: fq.fq_mx_gemm(fq.FQ_OP_NT, A, B, out_dtype=dt) for dt in (torch.float32, torch.bfloat16)}
    for dt, w in want.items():
        for off, pad in [(0, 3), (1, 0), (4, 4), (8, 8)]:
            out = torch.full((M, off + N + pad), 9.0, dtype=dt, device="cuda")
            fq.fq_mx_gemm(fq.FQ_OP_NT, A, B, out=out[:, off:off + N])
            assert torch.equal(out[:, off:off + N], w)
            assert (out[:, :off] == 9.0).all() and (out[:, off + N:] == 9.0).all()


@pytest.mark.parametrize("M,N,K", [(4, 40, 200), (200, 300, 400)])
def test_non_finite_groups_reach_their_outputs_only(M, N, K):
    x, w = matrix(M, K, 1), matrix(N, K, 2)
    x[2, 70], w[33, 100] = float("nan"), float("-inf")
    A, B = fq.fq_mx_quantize(x), fq.fq_mx_quantize(w)
    got = fq.fq_mx_gemm(fq.FQ_OP_NT, A, B)
    hit = torch.zeros((M, N), dtype=torch.bool, device="cuda")
    hit[2, :] = hit[:, 33] = True
    assert torch.equal(got.isnan(), hit)
    x[2, 70], w[33, 100] = 0.0, 0.0
    clean = fq.fq_mx_gemm(fq.FQ_OP_NT, fq.fq_mx_quantize(x), fq.fq_mx_quantize(w))
    assert torch.equal(got[~hit], clean[~hit])


def test_scales_at_the_ends():
    """Scale bytes from 0 up: products of large and small scales, without infinities in between."""
    x = matrix(40, 256, 1)
    for e in (-126, -100, 60, 120):
        a = (x.float() * 2.0 ** min(e, 100) * (2.0 ** (e - 100) if e > 100 else 1.0)).to(torch.bfloat16)
        b = (matrix(50, 256, 2).float() * 2.0 ** -e if e > -126 else matrix(50, 256, 2).float() * 2.0 ** 100).to(torch.bfloat16)
        A, B = fq.fq_mx_quantize(a), fq.fq_mx_quantize(b)
        check(fq.fq_mx_gemm(fq.FQ_OP_NT, A, B), *operands(fq.FQ_OP_NT, A, B))


def test_empty_products():
    for M, N, K in [(0, 5, 64), (5, 0, 64), (5, 7, 0), (300, 300, 0)]:
        A, B = (fq.fq_mx_quantize(torch.empty((n, K), dtype=torch.bfloat16, device="cuda")) for n in (M, N))
        out = torch.full((M, N), 5.0, device="cuda")
        fq.fq_mx_gemm(fq.FQ_OP_NT, A, B, out=out)
        assert not out.any()
        y = torch.full((M, N), 5.0, dtype=torch.bfloat16, device="cuda")
        fq.fq_mx_linear(torch.empty((M, K), dtype=torch.bfloat16, device="cuda"), B, out=y)
        assert not y.any()
    torch.cuda.synchronize()


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 500, 4096), (2, 77, 333), (16, 48, 1000), (17, 256, 96), (33, 300, 513),
                                   (200, 130, 260), (600, 520, 300)])
def test_linear_is_quantize_and_multiply(M, N, K):
    """Bit for bit, for either rule, strided x and both outputs; xq given or not."""
    wide = matrix(M, K + 3, 5)
    for x in (matrix(M, K, 4), wide[:, 3:], wide[:, :K]):
        for rule in (fq.FQ_MX_FLOOR, fq.FQ_MX_COVER):
            W = fq.fq_mx_quantize(matrix(N, K, 6, 0.02))
            q = fq.fq_mx_quantize(x, rule=rule)
            for dt in (torch.float32, torch.bfloat16):
                gu.announce(f"mx linear {M}x{N}x{K} rule {rule} {dt} pitch {x.stride(0)}")
                want = fq.fq_mx_gemm(fq.FQ_OP_NT, q, W, out_dtype=dt)
                assert torch.equal(fq.fq_mx_linear(x, W, rule=rule, out_dtype=dt), want)
                y = torch.empty((M, N), dtype=dt, device="cuda")
                fq.fq_mx_linear(x, W, xq=fq.MxTensor(M, K, fq.FQ_MX_BOTH), rule=rule, out=y)
                assert torch.equal(y, want)


def test_linear_of_every_tail():
    """A last group of 1 to 32 values, in each quarter of a block of 128: neighbours of the row do not get in."""
    big = matrix(3, 1100, 8)
    gu.announce("mx linear, contractions of 1 to 1056")
    for K in [*range(1, 34), *range(64, 97), *range(127, 162), 250, 1001, 1023, *range(1025, 1057)]:
        x, W = big[:, 7:7 + K], fq.fq_mx_quantize(matrix(20, K, K))
        assert torch.equal(fq.fq_mx_linear(x, W), fq.fq_mx_gemm(fq.FQ_OP_NT, fq.fq_mx_quantize(x), W)), K


def test_linear_with_non_finite_tokens():
    x, W = matrix(5, 300, 1), fq.fq_mx_quantize(matrix(64, 300, 2))
    clean = fq.fq_mx_linear(x, W)
    x[1, 7], x[3, 299] = float("inf"), float("nan")
    y = fq.fq_mx_linear(x, W)
    assert y[[1, 3]].isnan().all() and torch.equal(y[[0, 2, 4]], clean[[0, 2, 4]])


@pytest.mark.parametrize("M,K,N", [(96, 160, 224), (131, 77, 300)])
def test_a_layers_step(M, K, N):
    """Forward and the two gradients of Y = X W^T, each against the product of the quantized values; and the gradients
    against differences of the loss sum(dY * Y) with Y the plain product: the formulas dX = dY W, dW = dY^T X."""
    x, w, dy = matrix(M, K, 1), matrix(N, K, 2, 0.05), matrix(M, N, 3, 1e-3)
    qx, qw = (fq.fq_mx_quantize(t, sides=fq.FQ_MX_BOTH) for t in (x, w))
    qdy = fq.fq_mx_quantize_sr(dy, 11, sides=fq.FQ_MX_BOTH)
    y = fq.fq_mx_gemm(fq.FQ_OP_NT, qx, qw)
    dx, dw = fq.fq_mx_gemm(fq.FQ_OP_NN, qdy, qw), fq.fq_mx_gemm(fq.FQ_OP_TN, qdy, qx)
    check(y, *operands(fq.FQ_OP_NT, qx, qw))
    check(dx, *operands(fq.FQ_OP_NN, qdy, qw))
    check(dw, *operands(fq.FQ_OP_TN, qdy, qx))
    assert dx.shape == x.shape and dw.shape == w.shape
    # differences of a loss that is linear in x, at the values the gradient's operands stand for: exact up to rounding
    g, wv = values(qdy, fq.FQ_MX_ROWS), values(qw, fq.FQ_MX_COLS)
    for i, k in [(0, 0), (M - 1, K - 1), (M // 2, K // 3)]:
        e = torch.zeros((M, K), dtype=F64, device="cuda")
        e[i, k] = 1.0
        loss = lambda t: (g * (t @ wv.T)).sum()
        diff = (loss(e) - loss(-e)) / 2
        size = (g[i].abs() * wv[:, k].abs()).sum()
        assert abs(diff - dx[i, k].to(F64)) <= (-(-N // 128) + 33) * 2.0 ** -23 * size


def test_results_do_not_depend_on_the_stream_or_on_repetition():
    A, B = pair(fq.FQ_OP_NT, 300, 513, 1000)
    x, W = matrix(3, 1000, 5), B
    want, lin = fq.fq_mx_gemm(fq.FQ_OP_NT, A, B), fq.fq_mx_linear(x, W)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(side):
            a = fq.fq_mx_gemm(fq.FQ_OP_NT, A, B)
            b = fq.fq_mx_linear(x, W)
        c = fq.fq_mx_gemm(fq.FQ_OP_NT, A, B, stream=side)
        side.synchronize()
        assert torch.equal(a, want) and torch.equal(b, lin) and torch.equal(c, want)


def test_a_step_replays_from_a_graph():
    M, K, N = 64, 256, 384
    W = fq.fq_mx_quantize(matrix(N, K, 1, 0.02), sides=fq.FQ_MX_BOTH)
    x, dy = matrix(M, K, 2), matrix(M, N, 3)
    qx, qdy, xq = fq.MxTensor(M, K, fq.FQ_MX_BOTH), fq.MxTensor(M, N, fq.FQ_MX_BOTH), fq.MxTensor(1, K)
    y, dx, dw, t = (torch.empty(s, device="cuda") for s in ((M, N), (M, K), (N, K), (1, N)))

    def step():
        fq.fq_mx_quantize(x, out=qx)
        fq.fq_mx_gemm(fq.FQ_OP_NT, qx, W, out=y)
        fq.fq_mx_quantize_sr(dy, 5, out=qdy)
        fq.fq_mx_gemm(fq.FQ_OP_NN, qdy, W, out=dx)
        fq.fq_mx_gemm(fq.FQ_OP_TN, qdy, qx, out=dw)
        fq.fq_mx_linear(x[:1], W, xq=xq, out=t)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    gu.announce("capturing an mx step")
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        x.copy_(matrix(M, K, 10 + rep))
        dy.copy_(matrix(M, N, 20 + rep))
        step()
        want = [v.clone() for v in (y, dx, dw, t)]
        for v in (y, dx, dw, t):
            v.zero_()
        torch.cuda.synchronize()
        gu.announce(f"replay {rep}")
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, dx, dw, t), want))


@pytest.mark.parametrize("cus,M,N,K", [(256, 1100, 2000, 700), (3, 500, 420, 513), (2, 700, 900, 500)])
def test_large_tiles_replay_from_a_graph(cus, M, N, K, monkeypatch):
    """Tiles through LDS, one output of either type."""
    monkeypatch.setenv("FQ_GEMM_CUS", str(cus))
    tiles = fq.fq_mx_gemm_form(M, N, K)[0]
    assert tiles == {256: fq.FQ_MX_FORM_128x128, 3: fq.FQ_MX_FORM_128x256, 2: fq.FQ_MX_FORM_256x256}[cus]
    x, w = matrix(M, K, 1), matrix(N, K, 2)
    qx, qw = fq.MxTensor(M, K), fq.MxTensor(N, K)
    y, z = torch.empty((M, N), device="cuda"), torch.empty((M, N), dtype=torch.bfloat16, device="cuda")

    def step():
        fq.fq_mx_quantize(w, out=qw)
        fq.fq_mx_linear(x, qw, xq=qx, out=y)
        fq.fq_mx_gemm(fq.FQ_OP_NT, qx, qw, out=z)

    graph = torch.cuda.CUDAGraph()
    gu.announce(f"capturing products in tiles {tiles}")
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        x.copy_(matrix(M, K, 10 + rep))
        w.copy_(matrix(N, K, 20 + rep))
        step()
        want = y.clone(), z.clone()
        y.zero_(), z.zero_()
        torch.cuda.synchronize()
        gu.announce(f"replay {rep}")
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(z, want[1])


def test_two_products_at_once():
    """Products and a quantizer on three streams share nothing."""
    A, B = pair(fq.FQ_OP_NT, 1500, 1700, 900)
    P, Q = pair(fq.FQ_OP_TN, 2300, 4100, 400, 7)
    x = matrix(900, 1000, 3)
    want = fq.fq_mx_gemm(fq.FQ_OP_NT, A, B), fq.fq_mx_gemm(fq.FQ_OP_TN, P, Q), fq.fq_mx_quantize_sr(x, 9, sides=fq.FQ_MX_BOTH)
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [torch.empty_like(want[0]), torch.empty_like(want[1]), fq.MxTensor(900, 1000, fq.FQ_MX_BOTH)]
    torch.cuda.synchronize()
    gu.announce("three mx calls at once")
    for _ in range(20):
        fq.fq_mx_gemm(fq.FQ_OP_NT, A, B, out=got[0], stream=streams[0])
        fq.fq_mx_gemm(fq.FQ_OP_TN, P, Q, out=got[1], stream=streams[1])
        fq.fq_mx_quantize_sr(x, 9, out=got[2], stream=streams[2])
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert all(torch.equal(got[2].view(f), want[2].view(f)) for f in ("codes", "scales", "codes_t", "scales_t"))


def test_native_calls_are_the_ctypes_calls(monkeypatch):
    """Results, errors, the current stream: the same with and without the native module."""
    pytest.importorskip("paper_2503_08040_amd._fqnative")
    x, big = matrix(40, 96, 1), matrix(300, 96, 2)
    W = fq.fq_mx_quantize(matrix(50, 96, 3), sides=fq.FQ_MX_BOTH)
    assert fq._native is not None
    side = torch.cuda.Stream()

    def calls():
        out = []
        q, s = fq.MxTensor(40, 96, fq.FQ_MX_BOTH), fq.MxTensor(40, 96, fq.FQ_MX_BOTH)
        with torch.cuda.stream(side):
            fq.fq_mx_quantize(x, out=q, rule=fq.FQ_MX_COVER)
            fq.fq_mx_quantize_sr(x, -1, out=s)
            for t in (q, s):
                out += [t.view(f).clone() for f in ("codes", "scales", "codes_t", "scales_t")]
                out += [fq.fq_mx_dequantize(t), fq.fq_mx_dequantize(t, fq.FQ_MX_COLS, out_dtype=torch.float32)]
            y = torch.zeros((40, 60), device="cuda")
            out += [fq.fq_mx_gemm(fq.FQ_OP_NT, q, W), fq.fq_mx_gemm(fq.FQ_OP_NT, s, W, out=y[:, 5:55]), y.clone(),
                    fq.fq_mx_linear(x, W, xq=q, out_dtype=torch.bfloat16), fq.fq_mx_linear(big, W), fq.fq_mx_linear(x[:1], W)]
        side.synchronize()
        return out

    def errors():
        got = []
        q = fq.MxTensor(40, 96)
        for call in (lambda: fq.fq_mx_quantize(x, out=q, rule=5), lambda: fq.fq_mx_quantize(big, out=q),
                     lambda: fq.fq_mx_quantize_sr(big, 1, out=q), lambda: fq.fq_mx_dequantize(q, fq.FQ_MX_COLS),
                     lambda: fq.fq_mx_gemm(fq.FQ_OP_TN, q, W), lambda: fq.fq_mx_gemm(9, q, W),
                     lambda: fq.fq_mx_gemm(fq.FQ_OP_NT, q, W, out_dtype=torch.float16),
                     lambda: fq.fq_mx_linear(x, W, xq=fq.MxTensor(41, 96)), lambda: fq.fq_mx_linear(x[:, :95], W),
                     lambda: fq.fq_mx_quantize(x.float(), out=q), lambda: fq.fq_mx_quantize(x.cpu(), out=q),
                     lambda: fq.fq_mx_quantize_sr(x, 1.5, out=q), lambda: fq.fq_mx_gemm(fq.FQ_OP_NT, q, W, out=x)):
            with pytest.raises(Exception) as e:
                call()
            got.append((type(e.value), str(e.value)))
        return got

    native, native_errors = calls(), errors()
    monkeypatch.setattr(fq, "_native", None)
    assert native_errors == errors()
    assert all(torch.equal(a, b) for a, b in zip(native, calls()))


def test_far_offsets():
    """More than 2^31 elements: the last block row of the quantizer, of what is read back and of a product against the
    same calls on that block row alone, bit for bit."""
    rows, cols, first = 70000, 40960, 546 * 128
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    for r in range(0, rows, 7000):
        x[r:r + 7000] = matrix(min(7000, rows - r), cols, r)
    gu.announce("mx quantize of more than 2^31 elements")
    q, part = fq.fq_mx_quantize(x, sides=fq.FQ_MX_BOTH), fq.fq_mx_quantize(x[first:], sides=fq.FQ_MX_BOTH)
    assert torch.equal(q.view("codes")[first // 16:], part.view("codes"))
    assert torch.equal(q.view("scales")[first // 64:], part.view("scales"))
    assert torch.equal(q.view("codes_t")[:, first // 128:], part.view("codes_t"))
    assert torch.equal(q.view("scales_t")[:, first // 128:], part.view("scales_t"))
    for side in (fq.FQ_MX_ROWS, fq.FQ_MX_COLS):
        assert torch.equal(fq.fq_mx_dequantize(q, side)[first:], fq.fq_mx_dequantize(part, side))
    del q, part
    A, tail, B = (fq.fq_mx_quantize(t) for t in (x[:, :100], x[first:, :100], x[:cols, 100:200]))
    gu.announce("mx product of more than 2^31 elements")
    y = fq.fq_mx_gemm(fq.FQ_OP_NT, A, B, out_dtype=torch.bfloat16)
    # one block of 128: a single matrix instruction per output, whatever the tiles
    assert torch.equal(y[first:], fq.fq_mx_gemm(fq.FQ_OP_NT, tail, B, out_dtype=torch.bfloat16))
    assert torch.equal(y[:50], fq.fq_mx_gemm(fq.FQ_OP_NT, fq.fq_mx_quantize(x[:50, :100]), B, out_dtype=torch.bfloat16))

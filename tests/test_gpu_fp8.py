"""fls_quantize and fls_fp8_gemm against plain definitions in 64 bits.

Quantising is exact: every byte is compared.  A product is compared twice: on small whole numbers, where every sum is exact and C has to
agree bit for bit whatever the order of additions, and on ordinary values.  There C may be off by its one rounding (half a step:
2^-11 of the value, 2^-25 below fp16's normal range) and by what one matrix instruction cuts off its 128 products; the
hardware keeps at least 13 bits of their sum of magnitudes, so 2^-13 of that sum over k, and 2-norms by 2^-11 / sqrt(3) for roundings
spread evenly over half a step and 2^-14 for cuts that fall either way.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fls():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2309_10285_amd as f

    f.lib()
    return f


def e4m3_table():
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7.0), m / 8.0 * 2.0 ** -6)
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c >= 128, -v, v)


TABLE = e4m3_table()


def ref_quantize(W):
    """(values in e4m3 as float64, scale bytes) of fp16 W, from the definition."""
    M, K = W.shape
    blocks, stride = -(-K // 128), -(-K // 512) * 4
    w = np.zeros((M, blocks * 128))
    w[:, :K] = W.astype(np.float64)
    w = w.reshape(M, blocks, 128)
    finite = np.where(np.isfinite(w), np.abs(w), 0.0).max(-1)
    e = np.zeros((M, blocks), dtype=int)
    for x in range(-40, 17):  # the smallest power that is enough, found by trying
        e = np.where((finite > 448 * 2.0 ** (x - 1)) | ((finite > 0) & (x == -40)), x, e)
    v = w * 2.0 ** -e[..., None]
    with np.errstate(divide="ignore", invalid="ignore"):
        step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6))) - 3)
        q = np.where(np.isfinite(v), np.rint(v / step) * step, np.nan)
    s = np.full((M, stride), 127, dtype=np.uint8)
    s[:, :blocks] = e + 127
    return q.reshape(M, -1)[:, :K], s


def quantize(fls, W):
    import torch

    q, s = fls.fls_quantize(torch.from_numpy(W).cuda())
    return q.view(torch.uint8).cpu().numpy(), s.view(torch.uint8).cpu().numpy()


def same(values, codes):
    got = TABLE[codes]
    return np.array_equal(got, values, equal_nan=True) and np.array_equal(np.signbit(got), np.signbit(values) | (np.isnan(values) & np.signbit(got)))


@pytest.mark.parametrize("M,K", [(1, 16), (3, 112), (7, 128), (5, 144), (64, 512), (65, 528), (129, 1040), (200, 2048), (63, 7168)])
def test_quantize_is_exact(fls, M, K):
    g = np.random.default_rng(M * 10007 + K)
    W = (g.standard_normal((M, K)) * np.exp2(g.integers(-26, 15, (M, -(-K // 128))).repeat(128, 1)[:, :K])).clip(-65504, 65504).astype(np.float16)
    W[g.random((M, K)) < 0.1] = 0
    codes, scales = quantize(fls, W)
    q, s = ref_quantize(W)
    assert np.array_equal(scales, s)
    assert same(q, codes)


def test_quantize_borders_zeros_infinities_and_nan(fls):
    W = np.zeros((16, 256), dtype=np.float16)
    W[0, :128] = np.linspace(-448, 448, 128)                       # scale 1
    W[1, 5], W[1, 6], W[1, 7] = 448, 2.0 ** -9, 2.0 ** -10          # smallest subnormal of e4m3, half of it: to even
    W[2, 5], W[2, 6] = np.float16(448.25), 1.0                     # just past the border: one power more
    W[3, 130] = 65504                                              # the largest fp16
    W[4, 9] = 2.0 ** -24                                           # the smallest
    W[5, :128] = 17 + 2 * (np.arange(128) % 8)                     # half way between two values: to even
    W[5, 0] = 448
    W[6, 3], W[6, 4], W[6, 5] = np.inf, -np.inf, 2.0               # scale of the finite values
    W[7, 200], W[7, 201] = np.nan, -3.0
    W[8, :128] = np.inf                                            # no finite value: scale 1
    W[9, 0] = -0.0
    W[10, :] = -448
    W[11, 0], W[11, 1] = 1.75, 2.0 ** -14
    W[12, 0], W[12, 1] = np.nextafter(np.float16(1.75), np.float16(2)), 2.0 ** -14
    codes, scales = quantize(fls, W)
    q, s = ref_quantize(W)
    assert np.array_equal(scales, s)
    assert same(q, codes)
    assert scales[11, 0] == 127 - 8 and scales[12, 0] == 127 - 7 and scales[0, 0] == 127 and scales[15, 1] == 127


def run(fls, W, X, fill=7.0):
    import torch

    (M, K), N = W.shape, X.shape[0]
    Wq, Ws = fls.fls_quantize(torch.from_numpy(W).cuda())
    fls.ensure_fp8_workspace(M, K, N)
    C = torch.full((N + 2, M), fill, dtype=torch.float16, device="cuda")
    fls.fls_fp8_gemm(Wq, Ws, torch.from_numpy(X).cuda(), C[1:N + 1], M, K, N) if (M * 2) % 16 == 0 else fls.fls_fp8_gemm(Wq, Ws, torch.from_numpy(X).cuda(), C[:N], M, K, N)
    out = C.cpu().numpy()
    lo = 1 if (M * 2) % 16 == 0 else 0
    assert (out[:lo] == fill).all() and (out[lo + N:] == fill).all(), "rows beside C were written"
    return out[lo:lo + N]


SHAPES = [(1, 16, 1), (16, 128, 1), (17, 144, 16), (5, 400, 3), (64, 1040, 15), (1000, 528, 7), (257, 2048, 13), (1024, 1024, 1),
          (130, 640, 17), (63, 1024, 32), (300, 400, 33), (129, 4096, 64), (64, 9216, 50),
          (1, 16, 65), (256, 128, 256), (255, 272, 100), (257, 384, 257), (1000, 1152, 300), (513, 4096, 129), (40, 16384, 70), (3000, 640, 700),
          (777, 1040, 1111), (4097, 512, 2049), (2048, 8192, 16), (128, 32768, 8), (128, 32768, 40), (100, 32768, 90),
          (128, 33040, 5), (70, 65552, 60), (300, 2304, 200), (260, 7184, 130), (5000, 2560, 20), (9000, 2064, 300), (33000, 272, 14), (2000, 9216, 1), (1100, 5136, 1000)]


@pytest.mark.parametrize("M,K,N", SHAPES)
def test_whole_numbers_are_exact(fls, M, K, N):
    """W and X of -2 ... 2 with a 16 in some blocks (e4m3 holds them whatever the scale), few enough for |C| <= 2048 and sums exact in fp32."""
    g = np.random.default_rng(M + 31 * K + 7 * N)
    W = (g.integers(-2, 3, (M, K)) * (g.random((M, K)) < min(1.0, 200 / K))).astype(np.float16)
    X = (g.integers(-2, 3, (N, K)) * (g.random((N, K)) < 0.5)).astype(np.float16)
    W[:, :: 640] = 16
    X[:, 3:: 1280] = -16
    ref = X.astype(np.float64) @ W.astype(np.float64).T
    assert np.abs(ref).max() <= 2048
    assert np.array_equal(run(fls, W, X).astype(np.float64), ref)


@pytest.mark.parametrize("M,K,N", SHAPES)
def test_ordinary_values(fls, M, K, N):
    g = np.random.default_rng(5 + M + 31 * K + 7 * N)
    W = (g.standard_normal((M, K)) * 0.02).astype(np.float16)
    X = (g.standard_normal((N, K)) * np.where(g.random(K) < 0.01, 20, 1)).astype(np.float16)
    (q, s), (x, t) = ref_quantize(W), ref_quantize(X)
    w = q * np.exp2(s.astype(float) - 127).repeat(128, 1)[:, :K]
    x = x * np.exp2(t.astype(float) - 127).repeat(128, 1)[:, :K]
    ref, size = x @ w.T, np.abs(x) @ np.abs(w).T
    got = run(fls, W, X).astype(np.float64)
    assert (np.abs(got - ref) <= 2.0 ** -11 * np.abs(ref) + 2.0 ** -13 * size + 2.0 ** -25).all()
    if ref.size >= 4096:
        assert np.linalg.norm(got - ref) <= (2.0 ** -11 / 3 ** 0.5 + 2.0 ** -14) * np.linalg.norm(ref)


@pytest.mark.parametrize("N", [5, 40, 300])
def test_not_a_number_stays_where_it_is(fls, N):
    """Inf or NaN in a token makes that token's row of C NaN; in a row of W, that column.  Nothing else."""
    M, K = 300, 656
    g = np.random.default_rng(N)
    W, X = g.integers(1, 3, (M, K)).astype(np.float16), g.integers(1, 3, (N, K)).astype(np.float16)
    W[17, 640], X[2, 100], X[N - 1, 655] = np.nan, np.inf, -np.inf
    out = run(fls, W, X)
    bad = np.zeros((N, M), dtype=bool)
    bad[:, 17] = bad[2] = bad[N - 1] = True
    assert np.array_equal(np.isnan(out), bad)
    assert np.isfinite(out[~bad]).all()


def test_scales_of_another_maker(fls):
    """Any e4m3 codes and any scales: those behind the last block are not used."""
    import torch

    g = np.random.default_rng(77)
    M, K, N = 96, 272, 3
    for N in (3, 48, 130):
        codes = g.integers(0, 0x58, (M, K)).astype(np.uint8) | (g.integers(0, 2, (M, K)) << 7).astype(np.uint8)
        scales = np.full((M, 4), 255, dtype=np.uint8)  # NaN
        scales[:, :3] = g.integers(110, 135, (M, 3))
        X = g.standard_normal((N, K)).astype(np.float16)
        x, t = ref_quantize(X)
        x = x * np.exp2(t.astype(float) - 127).repeat(128, 1)[:, :K]
        w = TABLE[codes] * np.exp2(scales.astype(float) - 127).repeat(128, 1)[:, :K]
        ref, size = x @ w.T, np.abs(x) @ np.abs(w).T
        keep = np.abs(ref) < 60000
        fls.ensure_fp8_workspace(M, K, N)
        C = torch.empty((N, M), dtype=torch.float16, device="cuda")
        fls.fls_fp8_gemm(torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn), torch.from_numpy(scales).cuda().view(torch.float8_e8m0fnu),
                         torch.from_numpy(X).cuda(), C, M, K, N)
        got = C.cpu().numpy().astype(np.float64)
        assert (np.abs(got - ref) <= 2.0 ** -11 * np.abs(ref) + 2.0 ** -13 * size + 2.0 ** -25)[keep].all()


@pytest.mark.parametrize("M,K,N", [(1024, 1024, 1), (512, 16384, 24), (600, 4096, 500)])
def test_same_bits_each_time_and_in_a_graph(fls, M, K, N):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(3)
    Wq, Ws = fls.fls_quantize((torch.randn(M, K, generator=gen, device="cuda") * 0.02).half())
    X = torch.randn(N, K, generator=gen, device="cuda").half()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        fls.ensure_fp8_workspace(M, K, N)
        C, D = torch.zeros(N, M, dtype=torch.float16, device="cuda"), torch.zeros(N, M, dtype=torch.float16, device="cuda")
        side.wait_stream(torch.cuda.default_stream())
        fls.fls_fp8_gemm(Wq, Ws, X, C, M, K, N)
        call = fls.prepare_fp8_gemm(Wq, Ws, X, D, M, K, N)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        for i in range(4):
            X.copy_(torch.randn(N, K, generator=gen, device="cuda").half())
            D.zero_()
            graph.replay()
            fls.fls_fp8_gemm(Wq, Ws, X, C, M, K, N)
            side.synchronize()
            assert torch.equal(C, D) and C.abs().max() > 0


def test_a_matrix_past_32_bits(fls):
    """Elements and bytes of W past 2^32: its last rows against the same rows alone."""
    import torch

    M, K = (1 << 20) + 77, 4112
    gen = torch.Generator(device="cuda").manual_seed(6)
    W = torch.empty(M, K, dtype=torch.float16, device="cuda")
    rows = [0, 1, 522247, 522248, 1044495, 1044496] + list(range(M - 130, M))  # the rows in which 2^32 bytes of fp16 and of e4m3 are full
    W.fill_(0.5)
    W[rows] = torch.randn(len(rows), K, generator=gen, device="cuda").half()
    Wq, Ws = fls.fls_quantize(W)
    part = W[rows]
    del W
    q, s = fls.fls_quantize(part)
    assert torch.equal(Wq.view(torch.uint8)[rows], q.view(torch.uint8)) and torch.equal(Ws.view(torch.uint8)[rows], s.view(torch.uint8))
    plain = q.double() * torch.exp2(s.view(torch.uint8).double() - 127).repeat_interleave(128, 1)[:, :K]
    for N in (3, 40, 100):
        X = torch.randint(-2, 3, (N, K), generator=gen, device="cuda").half()  # exact in e4m3
        fls.ensure_fp8_workspace(M, K, N)
        C = torch.empty(N, M, dtype=torch.float16, device="cuda")
        fls.fls_fp8_gemm(Wq, Ws, X, C, M, K, N)
        ref, size = X.double() @ plain.T, X.double().abs() @ plain.abs().T
        got = C[:, rows].double()
        assert ((got - ref).abs() <= 2.0 ** -11 * ref.abs() + 2.0 ** -13 * size + 2.0 ** -25).all()
        half = X.double().sum(1) * 0.5
        assert ((C[:, 2000:3000].double() - half[:, None]).abs() <= (2.0 ** -11 * half.abs() + 2.0 ** -13 * X.double().abs().sum(1) * 0.5)[:, None]).all()


def test_refusals_in_the_binding(fls):
    import torch

    W = torch.zeros(8, 32, dtype=torch.float16, device="cuda")
    X, C = torch.zeros(3, 32, dtype=torch.float16, device="cuda"), torch.zeros(3, 8, dtype=torch.float16, device="cuda")
    for bad in (W.float(), W.cpu(), W.T, W[0]):
        with pytest.raises(AssertionError):
            fls.fls_quantize(bad)
    with pytest.raises(fls.FlsError) as e:
        fls.fls_quantize(W[:, :24].contiguous())
    assert e.value.code == fls.EINVAL
    Wq, Ws = fls.fls_quantize(W)
    fls.ensure_fp8_workspace(8, 32, 3)
    for bad in ((W, Ws, X, C), (Wq, Ws.view(torch.uint8), X, C), (Wq, Ws[:, :3], X, C), (Wq, Ws, X.float(), C), (Wq, Ws, X[:2], C), (Wq, Ws, X, C.T), (Wq, Ws, X.cpu(), C)):
        with pytest.raises(AssertionError):
            fls.fls_fp8_gemm(*bad, 8, 32, 3)


def test_next_to_the_dense_and_the_sparse_product(fls):
    """One workspace serves all products of a layer in turn."""
    import torch

    M, K, N = 1024, 2048, 24
    gen = torch.Generator(device="cuda").manual_seed(9)
    W, X = (torch.randn(M, K, generator=gen, device="cuda") * 0.02).half(), torch.randn(N, K, generator=gen, device="cuda").half()
    Wq, Ws = fls.fls_quantize(W)
    blob, _ = fls.fls_compress(W)
    fls.ensure_workspace(M, K, N)
    fls.ensure_fp8_workspace(M, K, N)
    out = [torch.empty(N, M, dtype=torch.float16, device="cuda") for _ in range(5)]
    fls.fls_dense_gemm(W, X, out[0], M, K, N)
    fls.fls_fp8_gemm(Wq, Ws, X, out[1], M, K, N)
    fls.fls_spmm(blob, X, out[2], M, K, N)
    fls.fls_fp8_gemm(Wq, Ws, X, out[3], M, K, N)
    fls.fls_dense_gemm(W, X, out[4], M, K, N)
    fls.fls_check_workspace()
    fls.fls_forget(blob)
    d = out[0].double()
    assert torch.equal(out[1], out[3]) and (out[4].double() - d).norm() <= 1e-3 * d.norm() and (out[2].double() - d).norm() <= 1e-3 * d.norm()
    # e4m3 rounds each operand by at most 2^-4 of a value, evenly spread: two of 2^-4 / sqrt(3) rms at most, and the sum of K products keeps that share
    assert (out[1].double() - d).norm() <= 2 ** 0.5 * 2.0 ** -4 / 3 ** 0.5 * d.norm()

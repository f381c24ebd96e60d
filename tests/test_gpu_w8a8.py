"""The 8-bit linears against exact integer sums: codes, scales and outputs have one right
value each, so every comparison is of bits."""
import numpy as np
import pytest

from tests.test_gpu_attn import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pk():
    import paper_2606_08761_amd as pk
    return pk


def quantized(x):
    """Scales (binary32 of the exact quotient: both operands have 24 bits, one rounding) and
    codes: x / s in 64 bits is 2^-53 off at most, and a quotient of 11 and 24 bits that is no tie
    is 2^-32 or more from one."""
    v = x.astype(np.float64)
    s = np.abs(x).max(axis=1).astype(np.float32) / np.float32(127)
    d = s.astype(np.float64)[:, None]
    q = np.divide(v, d, out=np.zeros_like(v), where=d > 0)
    return np.clip(np.rint(q), -127, 127).astype(np.int8), s


def product(A, sa, W, sw):
    """Exact sums (below 2^53 in 64 bits), then binary32 products, then binary16."""
    P = A.astype(np.float64) @ W.astype(np.float64).T
    with np.errstate(over="ignore", invalid="ignore"):
        return (P.astype(np.float32) * sa[:, None] * sw[None]).astype(np.float16)


def codes(g, rows, K):
    return g.integers(-127, 128, (rows, K)).astype(np.int8)


def scales(g, n):
    return (g.random(n) * 1e-3 + 1e-4).astype(np.float32)


def same(a, b):
    a, b = a.cpu().numpy().view(np.uint16), b.view(np.uint16)
    zero = (a & 0x7FFF == 0) & (b & 0x7FFF == 0)
    return bool(((a == b) | zero).all())


@pytest.mark.parametrize("M,K", [(1, 32), (3, 96), (5, 512), (4, 544), (2, 2048), (300, 2080), (3, 4096), (300, 8192), (2, 8224), (300, 28672),
                                 (2, 32768), (2, 32800), (1, 131040)])
def test_quantizer(pk, M, K):
    g = np.random.default_rng(M + K)
    x = (g.standard_normal((M, K)) * 10.0 ** g.uniform(-4, 3, (M, 1))).astype(np.float16)
    if M > 2:
        x[0] = 0
        x[1] = g.integers(-254, 255, K) * 0.5   # scale 1, ties
        x[1, 7] = 127.0
        x[2] = g.integers(-3, 4, K) * 2.0 ** -24  # subnormal values
    q, s = pk.apex4_quantize_act8(dev(x))
    want_q, want_s = quantized(x)
    assert np.array_equal(s.cpu().numpy(), want_s)
    assert np.array_equal(q.cpu().numpy(), want_q)


def test_every_tie_and_neighbour(pk):
    """Values at and next to every border of the codes, for scales whose quotients land there."""
    rows = []
    for top in (127.0, 254.0, 63.5, 1.0, 0.1, 1000.0, 65504.0, 2.0 ** -14 * 127, 3.1415927):
        t = np.float16(top)
        k = np.arange(-127, 127) + 0.5
        v = np.float16(k * (np.float32(t) / np.float32(127)))
        rows.append(np.concatenate((v, np.nextafter(v, np.float16(np.inf)), np.nextafter(v, np.float16(-np.inf)), np.full(6, t, np.float16)))[:768])
    x = np.stack(rows)
    x = np.where(np.abs(x) > x[:, -1:], x[:, -1:], x)
    q, s = pk.apex4_quantize_act8(dev(x))
    want_q, want_s = quantized(x)
    assert np.array_equal(s.cpu().numpy(), want_s) and np.array_equal(q.cpu().numpy(), want_q)


def test_infinities_and_nan_stay_in_their_row(pk):
    g = np.random.default_rng(1)
    x = g.standard_normal((20, 64)).astype(np.float16)
    w = codes(g, 40, 64)
    sw = scales(g, 40)
    for m in (1, 20):
        clean = pk.apex4_w8a8_linear(dev(x[:m]), dev(w), dev(sw)).cpu().numpy()
        for bad in (np.inf, -np.inf, np.nan):
            y = x[:m].copy()
            y[m // 2, 5] = bad
            got = pk.apex4_w8a8_linear(dev(y), dev(w), dev(sw)).cpu().numpy()
            assert np.isnan(got[m // 2]).all()
            rest = np.arange(m) != m // 2
            assert np.array_equal(got[rest], clean[rest])


SIZES = [(1, 1, 32), (1, 100, 96), (2, 33, 160), (8, 16, 128), (7, 1001, 1056), (9, 17, 4128), (16, 520, 8192), (17, 40, 32), (32, 4096, 256),
         (20, 5003, 544), (32, 9000, 160), (33, 70, 96), (64, 8192, 512), (50, 8225, 192), (64, 8200, 128), (65, 64, 32), (65, 8193, 416),
         (130, 260, 2048), (128, 16384, 128), (300, 520, 1056), (257, 4100, 96), (513, 1001, 160), (700, 10240, 288), (1030, 8191, 64),
         (2048, 8192, 128), (3000, 2100, 32), (4100, 4097, 160),
         # each tile, and K that ends inside a stage
         (1544, 7211, 672), (2241, 7191, 672), (1795, 8253, 672), (3203, 2319, 672), (1290, 8101, 672), (578, 8238, 672), (389, 8230, 672),
         (291, 8251, 672), (65, 8209, 672), (131, 8459, 672), (83, 102, 672), (194, 8243, 672), (2057, 7187, 160), (1296, 8086, 288),
         (2577, 579, 160), (2725, 133, 160)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(pk, M, N, K):
    g = np.random.default_rng(M + N + K)
    A, W, sa, sw = codes(g, M, K), codes(g, N, K), scales(g, M), scales(g, N)
    assert same(pk.apex4_w8a8_gemm(dev(A), dev(sa), dev(W), dev(sw)), product(A, sa, W, sw))


@pytest.mark.parametrize("K", [32, 128, 160, 256, 640, 736, 768, 800, 896, 928, 1024, 1056, 1152, 1280, 2080, 4128])
def test_stages_of_few_rows(pk, K):
    """Fewer stages than buffers, as many, some more; even and odd counts, the last one whole or
    not: of narrow tiles, and of weights streamed once."""
    g = np.random.default_rng(K)
    for M, N in ((33, 100), (64, 65), (25, 70), (9, 4130), (32, 4129), (24, 333), (17, 4096), (8, 40)):
        A, W, sa, sw = codes(g, M, K), codes(g, N, K), scales(g, M), scales(g, N)
        assert same(pk.apex4_w8a8_gemm(dev(A), dev(sa), dev(W), dev(sw)), product(A, sa, W, sw))


@pytest.mark.parametrize("M,N,K", [(1, 64, 32), (1, 333, 8192), (1, 40, 28672), (1, 33, 32768), (1, 20, 32800), (2, 100, 1056), (20, 520, 544), (100, 333, 224)])
def test_linear_is_the_two_calls(pk, M, N, K):
    g = np.random.default_rng(M + N + K)
    x, w = g.standard_normal((M, K)).astype(np.float16), g.standard_normal((N, K)).astype(np.float16)
    W, sw = pk.apex4_quantize_act8(dev(w))
    y = pk.apex4_w8a8_linear(dev(x), W, sw)
    q, s = quantized(x)
    assert same(y, product(q, s, W.cpu().numpy(), sw.cpu().numpy()))
    assert same(pk.apex4_w8a8_gemm(dev(q), dev(s), W, sw), y.cpu().numpy())
    layer = pk.W8A8Linear(dev(w))
    assert layer(dev(x)).equal(y) and layer(dev(x)[:, None]).equal(y[:, None])
    # what the layer is for: near the product of the numbers themselves.  A code is half a step
    # off at most, so an output by 2^-8 (2^-7 of a code of 64 on average) of sums of K products
    ref = x.astype(np.float64) @ w.astype(np.float64).T
    off = (np.abs(x).max(1)[:, None] * np.abs(w).astype(np.float64).sum(1)[None] + np.abs(w).max(1)[None] * np.abs(x).astype(np.float64).sum(1)[:, None]) / 254
    assert (np.abs(y.cpu().numpy() - ref) <= 1.02 * off + 2.0 ** -11 * np.abs(ref) + 1e-6).all()


def test_the_largest_sums(pk):
    """K at its limit with codes of one sign, -128 among them: below 2^31."""
    K = 131040
    for M, N in ((1, 20), (70, 70)):
        A, W = np.full((M, K), -128, np.int8), np.full((N, K), -128, np.int8)
        W[1::2] = 127
        sa, sw = np.full(M, 2.0 ** -20, np.float32), np.full(N, 2.0 ** -8, np.float32)
        assert same(pk.apex4_w8a8_gemm(dev(A), dev(sa), dev(W), dev(sw)), product(A, sa, W, sw))


@pytest.mark.parametrize("N,K", [(96, 256), (4100, 96)])
def test_a_row_does_not_depend_on_the_batch(pk, N, K):
    g = np.random.default_rng(5)
    x, W, sw = g.standard_normal((600, K)).astype(np.float16), dev(codes(g, N, K)), dev(scales(g, N))
    whole = pk.apex4_w8a8_linear(dev(x), W, sw)
    for m in (1, 2, 8, 9, 16, 32, 64, 65, 130, 300, 599):
        assert pk.apex4_w8a8_linear(dev(x[:m]), W, sw).equal(whole[:m])


def test_results_past_binary16(pk):
    """Overflow to infinity, underflow to zero, and scales of zero, as the roundings say."""
    A, W = np.full((4, 64), 127, np.int8), np.full((5, 64), 127, np.int8)
    W[1] = -127
    sa, sw = np.array([1.0, 1e-12, 0.0, 1e30], np.float32), np.array([1.0, 1.0, 1e-20, 0.06346, 1e30], np.float32)
    for rows in (4, 100):
        a, s = np.resize(A, (rows, 64)), np.resize(sa, rows)
        assert same(pk.apex4_w8a8_gemm(dev(a), dev(s), dev(W), dev(sw)), product(a, s, W, sw))


def test_nothing_behind_the_outputs_is_written(pk):
    import torch
    g = np.random.default_rng(7)
    for M, N, K in ((1, 33, 96), (9, 35, 160), (70, 131, 32), (300, 515, 128)):
        A, W, sa, sw = codes(g, M, K), codes(g, N, K), scales(g, M), scales(g, N)
        room = torch.full((M * N + 4096,), 7.0, dtype=torch.float16, device="cuda")
        pk.apex4_w8a8_gemm(dev(A), dev(sa), dev(W), dev(sw), Y=room[:M * N].view(M, N))
        assert same(room[:M * N].view(M, N), product(A, sa, W, sw)) and (room[M * N:] == 7.0).all()


def test_no_rows(pk):
    import torch
    W, sw = torch.zeros((8, 64), dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda")
    assert pk.apex4_w8a8_linear(torch.zeros((0, 64), dtype=torch.float16, device="cuda"), W, sw).shape == (0, 8)
    layer = pk.W8A8Linear(torch.ones((8, 64), dtype=torch.float16, device="cuda"))
    assert layer(torch.zeros((3, 0, 64), dtype=torch.float16, device="cuda")).shape == (3, 0, 8)


def test_operands_past_2_gib(pk):
    """Row offsets of more than 31 bits, in weights and in outputs."""
    import torch
    g = np.random.default_rng(11)
    K, N = 8192, 300000  # 2.3 GiB of codes
    W = torch.randint(-127, 128, (N, K), dtype=torch.int8, device="cuda")
    sw = torch.full((N,), 1e-4, device="cuda")
    rows = np.array([0, 1, 262143, 262144, 299999])
    for M in (1, 20, 200):
        A, sa = codes(g, M, K), scales(g, M)
        y = pk.apex4_w8a8_gemm(dev(A), dev(sa), W, sw)
        assert same(y[:, rows], product(A, sa, W[rows].cpu().numpy(), sw.cpu().numpy()[rows]))


def test_more_rows_and_channels_than_a_grid_has(pk):
    """2^22 and more rows to quantize, 2^26 and more channels."""
    import torch
    M, K = (1 << 22) + 5, 32
    x = torch.randn((M, K), device="cuda", dtype=torch.float16)
    q, s = pk.apex4_quantize_act8(x)
    rows = torch.tensor([0, 1, (1 << 21) - 1, 1 << 21, (1 << 22) - 1, 1 << 22, M - 1], device="cuda")
    want_q, want_s = quantized(x[rows].cpu().numpy())
    assert np.array_equal(q[rows].cpu().numpy(), want_q) and np.array_equal(s[rows].cpu().numpy(), want_s)
    N = (1 << 26) + 100
    W, sw = torch.randint(-127, 128, (N, K), dtype=torch.int8, device="cuda"), torch.rand(N, device="cuda")
    cols = torch.tensor([0, 31, 1 << 20, (1 << 26) - 1, 1 << 26, N - 1], device="cuda")
    for m in (1, 3):
        y = pk.apex4_w8a8_linear(x[:m], W, sw)
        qa, sa = quantized(x[:m].cpu().numpy())
        assert same(y[:, cols], product(qa, sa, W[cols].cpu().numpy(), sw[cols].cpu().numpy()))


@pytest.mark.parametrize("M,N,K", [(1, 24, 64), (1, 20, 32800), (3, 40, 96), (70, 36, 160)])
def test_scratch_made_here_or_given(pk, M, N, K):
    """Both buffers, one of them or neither: the same bits.  Both given, they hold the codes
    and scales afterwards (but for a token that is quantized on the way)."""
    import torch
    g = np.random.default_rng(M + K)
    x, W, sw = dev(g.standard_normal((M, K)).astype(np.float16)), dev(codes(g, N, K)), dev(scales(g, N))
    want = pk.apex4_w8a8_linear(x, W, sw)
    A, s = torch.full((M, K), 5, dtype=torch.int8, device="cuda"), torch.full((M,), 5.0, device="cuda")
    assert pk.apex4_w8a8_linear(x, W, sw, A_8_work=A, s_a_work=s).equal(want)
    q, t = quantized(x.cpu().numpy())
    if M > 1:
        assert same(pk.apex4_w8a8_gemm(A, s, W, sw), want.cpu().numpy()) and np.array_equal(A.cpu().numpy(), q) and np.array_equal(s.cpu().numpy(), t)
    assert pk.apex4_w8a8_linear(x, W, sw, A_8_work=A).equal(want) and pk.apex4_w8a8_linear(x, W, sw, s_a_work=s).equal(want)
    layer = pk.W8A8Linear(dev(g.standard_normal((N, K)).astype(np.float16)))
    y = layer(x)
    assert layer(x[0]).equal(y[0]) and layer(x.expand(2, M, K)).equal(y.expand(2, M, N))
    with pytest.raises(ValueError):
        pk.apex4_w8a8_linear(x, W, sw, A_8_work=A[:, :32])
    with pytest.raises(TypeError):
        pk.apex4_w8a8_linear(x, W, sw, A_8_work=A, s_a_work=s.half())
    with pytest.raises(ValueError):
        pk.apex4_w8a8_linear(x, W, sw, A_8_work=A.cpu(), s_a_work=s)
    for odd in (K - 8, K - 1):
        with pytest.raises(pk.Apex4Error):
            pk.apex4_w8a8_linear(x[:, :odd].contiguous(), W[:, :odd].contiguous(), sw)


def test_rows_with_gaps_on_another_stream(pk):
    """The layer's own copy of such rows is made on the stream of the call."""
    import torch
    g = np.random.default_rng(12)
    layer = pk.W8A8Linear(dev(g.standard_normal((64, 128)).astype(np.float16)))
    wide = dev(g.standard_normal((4096, 256)).astype(np.float16))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(50):
            wide.mul_(-1.0)
        wide.add_(1.0)
    y = layer(wide[:, 64:192], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert y.equal(layer(wide[:, 64:192].contiguous()))


def test_captured_and_on_another_stream(pk):
    import torch
    g = np.random.default_rng(8)
    W, sw = dev(codes(g, 500, 1024)), dev(scales(g, 500))
    xs = [dev(g.standard_normal((m, 1024)).astype(np.float16)) for m in (1, 12, 40, 300)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    eager = [pk.apex4_w8a8_linear(x, W, sw, stream=side) for x in xs]
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = [pk.apex4_w8a8_linear(x, W, sw) for x in xs]
    for i in range(3):
        if i:
            for x in xs:
                x.mul_(-1.0)
        for y in out:
            y.fill_(float("nan"))
        graph.replay()
        for x, y, e in zip(xs, out, eager):
            assert y.equal(pk.apex4_w8a8_linear(x, W, sw)) and y.equal(e if i % 2 == 0 else -e)

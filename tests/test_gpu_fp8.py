"""8-bit products with block scales, and their quantisation, against plain 64-bit implementations."""
import numpy as np
import pytest

from tests.block_reference import SMALLEST, U

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DT = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def ccdc():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_1805_01993_b200 import build, ccdc as mod

    build.build_library()
    mod.lib()
    return mod


def f64(t):
    return t.float().double().cpu().numpy()


# ---------------------------------------------------------------- quantisation
GRID = np.array([s * m for s in (1, -1) for m in [n * 2.0 ** -9 for n in range(8)] +
                 [(8 + n) * 2.0 ** (e - 3) for e in range(-6, 9) for n in range(8) if (e, n) != (8, 7)]])


def nearest(v):
    """nearest e4m3 values, ties to the even mantissa, from the list of all of them"""
    pos = np.unique(np.abs(GRID))
    a = np.abs(v)
    hi = np.clip(np.searchsorted(pos, a), 1, len(pos) - 1)
    lo = hi - 1
    down, up = a - pos[lo], pos[hi] - a
    take = np.where(down < up, lo, np.where(up < down, hi, np.where(lo % 2 == 0, lo, hi)))      # mantissas alternate
    return np.copysign(pos[take], v)


def quantised(x, rows):
    """(values, scales) of a matrix by the definition"""
    M, K = x.shape
    scales = np.zeros((-(-M // rows), -(-K // 128)))
    q = np.zeros_like(x)
    for i in range(scales.shape[0]):
        for b in range(scales.shape[1]):
            at = np.s_[i * rows:(i + 1) * rows, b * 128:(b + 1) * 128]
            most = np.abs(x[at]).max()
            e = -126
            while 448 * 2.0 ** e < most:
                e += 1
            scales[i, b] = 2.0 ** e
            q[at] = nearest(x[at] / scales[i, b])
    return q, scales


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("M,K,pad,shift", [(1, 1, 0, 0), (1, 128, 0, 0), (3, 129, 0, 0), (5, 300, 4, 3), (40, 512, 8, 8), (130, 263, 1, 0),
                                           (257, 136, 0, 0), (7, 1, 2, 1)])
def test_quantise(ccdc, M, K, pad, shift, rows, dtype):
    rng = np.random.default_rng(M + K)
    v = rng.normal(size=M * (K + pad) + shift) * 2.0 ** rng.integers(-12, 12, M * (K + pad) + shift)
    x = torch.from_numpy(v).to(DT[dtype]).cuda()[shift:].view(M, K + pad)[:, :K]
    q, scales = ccdc.quantize_fp8(x, rows)
    want_q, want_s = quantised(f64(x), rows)
    assert q.dtype is E4M3 and q.shape == x.shape and np.array_equal(f64(scales), want_s) and np.array_equal(f64(q), want_q)
    # into given tensors, nothing beside them
    big = torch.full((M, -(-K // 16) * 16 + 16), 3, dtype=torch.uint8, device="cuda")
    into = torch.full_like(scales, 5)
    ccdc.quantize_fp8(x, rows, out=big.view(E4M3)[:, :K], scales=into)
    assert torch.equal(into, scales) and torch.equal(big[:, :K], q.view(torch.uint8)) and bool((big[:, K:] == 3).all())


def test_quantise_edges(ccdc):
    """borders of the scales, ties, zeros, the smallest and the largest magnitudes, infinities and NaN"""
    x = torch.zeros((8, 256), device="cuda")
    x[0, 0], x[0, 1] = 448.0, 0.5                       # exactly the largest value: scale 1
    x[1, 0] = float(np.nextafter(np.float32(448), np.float32(500)))     # just above: 2
    x[2, :7] = torch.tensor([448, 17, 19, 1.0625, -1.1875, 2.0 ** -10, 3 * 2.0 ** -10])    # ties
    x[3, 128:] = 1e-42
    x[4, 3], x[4, 200] = 3.4e38, -3.4e38
    x[5, 5], x[5, 200] = float("inf"), 1.0
    x[6, 128] = float("nan")
    q, s = ccdc.quantize_fp8(x)
    assert s[0].tolist() == [1.0, 2.0 ** -126] and s[1, 0] == 2 and s[7].tolist() == [2.0 ** -126] * 2
    assert q[2, :7].float().tolist() == [448, 16, 20, 1.0, -1.25, 0, 2.0 ** -8]
    assert s[3, 1] == 2.0 ** -126 and s[4].tolist() == [2.0 ** 120] * 2
    assert bool(s[5, 0].isnan()) and bool(q[5, :128].float().isnan().all()) and s[5, 1] == 2.0 ** -8
    assert bool(s[6, 1].isnan()) and s[6, 0] == 2.0 ** -126 and not q[6, :128].float().any()
    t, st = ccdc.quantize_fp8(x, 128)
    assert st.shape == (1, 2) and bool(st.isnan().all()) and bool(t.float().isnan().all())
    stack = torch.randn((3, 200, 144), device="cuda").bfloat16()
    q, s = ccdc.quantize_fp8(stack, 128)
    assert s.shape == (3, 2, 2)
    for e in range(3):
        a, b = ccdc.quantize_fp8(stack[e], 128)
        assert torch.equal(q[e].view(torch.uint8), a.view(torch.uint8)) and torch.equal(s[e], b)
    back, sb = ccdc.quantize_fp8(stack.transpose(1, 2).contiguous(), 128)       # blocks transpose with the matrix
    assert torch.equal(back.float(), q.float().transpose(1, 2)) and torch.equal(sb, s.transpose(1, 2))
    none, sn = ccdc.quantize_fp8(stack[0, :0])
    assert none.shape == (0, 144) and sn.shape == (0, 2)


# ---------------------------------------------------------------- products
def eight_bits(rng, rows, K, pad=0, whole=False):
    """e4m3 rows of stride a multiple of 16 bytes; what lies behind K in a row is NaN"""
    ld = -(-K // 16) * 16 + pad
    v = rng.integers(-8, 9, (rows, K)) if whole else rng.normal(size=(rows, K)) * 2.0 ** rng.integers(-3, 6, (rows, K))
    t = torch.full((rows, ld), float("nan"), device="cuda")
    t[:, :K] = torch.from_numpy(v).float().cuda()
    return t.clamp_(-448, 448).to(E4M3)[:, :K]


def ends_of(rng, M, E):
    """offsets with empty experts, one of one row, and rows behind the last"""
    cuts = np.sort(rng.integers(0, M + 1, E))
    if E > 2:
        cuts[E // 2] = cuts[E // 2 - 1]
    return np.concatenate([[0], np.sort(cuts)])


def reference(x, xs, w, ws, offsets):
    """(y, the terms' size) in 64 bits; w [E][N][K], offsets host"""
    M, K = x.shape
    N = w.shape[1]
    y, size = np.zeros((M, N)), np.zeros((M, N))
    dx = x * np.repeat(xs, 128, 1)[:, :K]
    for e in range(w.shape[0]):
        a, b = offsets[e], offsets[e + 1]
        dw = w[e] * np.repeat(np.repeat(ws[e], 128, 0)[:N], 128, 1)[:, :K]
        y[a:b] = dx[a:b] @ dw.T
        size[a:b] = np.abs(dx[a:b]) @ np.abs(dw).T
    return y, size


def bound(want, size, K, dtype):
    """The tensor cores align 32 products and the sum so far to the largest and drop what lies 24 bits below: four steps of 33
    terms a block, each off by at most 2^-23 of the block's size.  Then a product of scales, a product and a sum a block."""
    blocks = -(-K // 128)
    return (4 * 33 * 2.0 ** -23 + (blocks + 2) * 2.0 ** -24) * size * (1 + U[dtype]) + U[dtype] * np.abs(want) + SMALLEST[dtype]


SIZES = [(1, 1, 1), (1, 128, 128), (2, 129, 127), (7, 5, 300), (8, 1000, 256), (9, 64, 15), (15, 257, 640), (16, 33, 129), (17, 384, 1024),
         (31, 130, 2048), (33, 200, 128), (64, 96, 4000), (65, 513, 384), (100, 128, 777), (128, 256, 256), (129, 127, 512), (200, 640, 144),
         (257, 300, 1100), (500, 129, 64), (1000, 600, 900)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(ccdc, M, N, K):
    rng = np.random.default_rng(M * N + K)
    x, w = eight_bits(rng, M, K, 16), eight_bits(rng, N, K)
    kb, nb = -(-K // 128), -(-N // 128)
    xs = torch.from_numpy(rng.random((M, kb)) + 0.1).float().cuda()
    ws = torch.from_numpy(rng.random((nb, kb)) * 2.0 ** rng.integers(-20, 20, (nb, kb))).float().cuda()
    want, size = reference(f64(x), f64(xs), f64(w)[None], f64(ws)[None], [0, M])
    for dtype in DT:
        y = ccdc.matmul_fp8(x, xs, w, ws, out_dtype=DT[dtype])
        tol = bound(want, size, K, dtype)
        got = f64(y) if dtype != "float16" else np.where(np.abs(want) + tol > 65504, want, f64(y))     # beyond fp16
        assert got.shape == want.shape and (np.abs(got - want) <= tol).all(), dtype
    by_column = xs.t().contiguous().t()                 # scales laid out the other way: the same bits
    assert torch.equal(ccdc.matmul_fp8(x, by_column, w, ws, out_dtype=torch.float32), ccdc.matmul_fp8(x, xs, w, ws, out_dtype=torch.float32))
    ccdc.block_status()


@pytest.mark.parametrize("M,N,K,E", [(1, 64, 128, 4), (5, 130, 200, 3), (16, 128, 384, 1), (40, 300, 256, 16), (64, 257, 1000, 9), (130, 96, 512, 130),
                                     (300, 640, 300, 5), (700, 129, 256, 2), (900, 256, 640, 40), (1500, 385, 512, 3), (2000, 64, 128, 1024)])
def test_product_by_expert(ccdc, M, N, K, E):
    rng = np.random.default_rng(M + N + K)
    kb, nb = -(-K // 128), -(-N // 128)
    x = eight_bits(rng, M, K)
    w = eight_bits(rng, E * N, K, 16 if E < 100 else 0)
    w = w.as_strided((E, N, K), (N * w.stride(0), w.stride(0), 1))
    xs = torch.from_numpy(rng.random((M, kb)) + 0.1).float().cuda()
    ws = torch.from_numpy(rng.random((E, nb, kb)) + 0.1).float().cuda()
    for offsets in (ends_of(rng, M, E), np.array([0] * E + [M]), np.array([0] + [M] * E), np.zeros(E + 1, int)):
        want, size = reference(f64(x), f64(xs), f64(w), f64(ws), offsets)
        on = torch.from_numpy(offsets).int().cuda()
        big = torch.full((M, N + 3), 7.0, dtype=torch.bfloat16, device="cuda")
        y = ccdc.matmul_fp8(x, xs, w, ws, offsets=on, out=big[:, :N])
        assert (np.abs(f64(y) - want) <= bound(want, size, K, "bfloat16")).all()
        assert not y[int(offsets[-1]):].any() and bool((big[:, N:] == 7).all())
    ccdc.block_status()


@pytest.mark.parametrize("M,N,K", [(1, 300, 5000), (20, 129, 2000), (300, 256, 1536), (1111, 520, 700)])
def test_whole_numbers_are_exact(ccdc, M, N, K):
    """sums of whole numbers below 2^24 have one value in any order"""
    rng = np.random.default_rng(K)
    x, w = eight_bits(rng, M, K, whole=True), eight_bits(rng, N, K, whole=True)
    ones = torch.ones((M, -(-K // 128)), device="cuda"), torch.ones((-(-N // 128), -(-K // 128)), device="cuda")
    y = ccdc.matmul_fp8(x, ones[0], w, ones[1], out_dtype=torch.float32)
    assert np.array_equal(f64(y), f64(x) @ f64(w).T)


def test_nan_and_infinity_stay_in_their_rows(ccdc):
    for M in (3, 40, 300):
        rng = np.random.default_rng(M)
        N, K = 200, 300
        source = torch.from_numpy(rng.normal(size=(M, K))).float().cuda()
        source[1, 5] = float("inf")
        x, xs = ccdc.quantize_fp8(source)
        w, ws = eight_bits(rng, 2 * N, K), torch.ones((2, 2, 3), device="cuda")
        w = w.as_strided((2, N, K), (N * w.stride(0), w.stride(0), 1))
        w[0, 150, 7] = float("nan")
        offsets = torch.tensor([0, 2, M - 1], dtype=torch.int32, device="cuda")
        y = ccdc.matmul_fp8(x, xs, w, ws, offsets=offsets, out_dtype=torch.float32)
        want = torch.zeros((M, N), dtype=torch.bool, device="cuda")
        want[1], want[:2, 150] = True, True
        assert torch.equal(y.isnan(), want) and not y[M - 1].any()


def test_offsets_outside_the_rows(ccdc):
    """entries beyond M count as M and a decrease as an empty expert: nothing outside is read or written"""
    rng = np.random.default_rng(1)
    M, N, K, E = 50, 70, 140, 4
    x, w = eight_bits(rng, M, K), eight_bits(rng, E * N, K)
    w = w.as_strided((E, N, K), (N * w.stride(0), w.stride(0), 1))
    xs, ws = torch.ones((M, 2), device="cuda"), torch.ones((E, 1, 2), device="cuda")

    def call(o):
        return ccdc.matmul_fp8(x, xs, w, ws, offsets=torch.tensor(o, dtype=torch.int32, device="cuda"), out_dtype=torch.float32)

    assert torch.equal(call([0, 20, 1 << 30, 60, 90]), call([0, 20, 50, 50, 50]))
    assert torch.equal(call([7, 20, 10, 40, 50]), call([0, 20, 20, 40, 50]))
    assert torch.equal(call([0, -5, 20, 20, 45]), call([0, 0, 20, 20, 45]))


def test_gradient_with_the_transposed_weight(ccdc):
    """dx = dy w by the same call; the product is linear in x, so differences give the same"""
    rng = np.random.default_rng(12)
    M, N, K = 70, 384, 256
    weight = torch.from_numpy(rng.normal(size=(N, K))).float().cuda()
    w, ws = ccdc.quantize_fp8(weight, 128)
    wt, wts = ccdc.quantize_fp8(weight.t().contiguous(), 128)
    dy, dys = ccdc.quantize_fp8(torch.from_numpy(rng.normal(size=(M, N))).float().cuda())
    x, xs = ccdc.quantize_fp8(torch.from_numpy(rng.normal(size=(M, K))).float().cuda())
    y = f64(ccdc.matmul_fp8(x, xs, w, ws, out_dtype=torch.float32))
    dx = f64(ccdc.matmul_fp8(dy, dys, wt, wts, out_dtype=torch.float32))
    left = f64(dy) * np.repeat(f64(dys), 128, 1)        # <dy, y(x)> = <dx, x>
    right = f64(x) * np.repeat(f64(xs), 128, 1)
    a, b = (left * y).sum(), (dx * right).sum()
    assert abs(a - b) <= 2.0 ** -14 * (np.abs(left * y).sum() + np.abs(dx * right).sum()) and abs(a) > 0


def test_streams_and_graphs(ccdc):
    rng = np.random.default_rng(2)
    for M, N, K, E in ((1, 512, 2048, 0), (48, 300, 700, 6), (600, 512, 640, 4)):
        source = torch.from_numpy(rng.normal(size=(M, K))).bfloat16().cuda()
        w, ws = ccdc.quantize_fp8(torch.from_numpy(rng.normal(size=(max(E, 1), N, K))).bfloat16().cuda(), 128)
        offsets = torch.from_numpy(ends_of(rng, M, E)).int().cuda() if E else None
        if not E:
            w, ws = w[0], ws[0]

        def both(stream=None):
            x, xs = ccdc.quantize_fp8(source, stream=stream)
            return xs, ccdc.matmul_fp8(x, xs, w, ws, offsets=offsets, out_dtype=torch.float16, stream=stream)

        want = both()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        got = both(side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            one = both()
        with torch.cuda.graph(other):
            two = both()
        source.neg_()
        graph.replay()
        other.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(one[1], -want[1]) and torch.equal(two[1], -want[1]) and torch.equal(both()[1], one[1])
    ccdc.block_status()


def test_no_rows(ccdc):
    x, xs = ccdc.quantize_fp8(torch.empty((0, 256), device="cuda"))
    w, ws = ccdc.quantize_fp8(torch.randn((128, 256), device="cuda"), 128)
    assert ccdc.matmul_fp8(x, xs, w, ws).shape == (0, 128)


def test_more_than_two_to_the_31_elements(ccdc):
    """the last of many experts, and the last of many rows, against the same rows alone"""
    E, N, K = 36, 8192, 8192
    w = torch.zeros((E, N, K), dtype=torch.uint8, device="cuda").view(E4M3)
    last = torch.randn((N, K), device="cuda").to(E4M3)
    w[E - 1] = last
    ws = torch.rand((E, N // 128, K // 128), device="cuda")
    x, xs = ccdc.quantize_fp8(torch.randn((40, K), device="cuda"))
    offsets = torch.tensor([0] * E + [40], dtype=torch.int32, device="cuda")
    # another launch may cut k elsewhere: the 64 blocks are joined in another order, with scales below 1
    y = ccdc.matmul_fp8(x, xs, w, ws, offsets=offsets, out_dtype=torch.float32)
    z = ccdc.matmul_fp8(x, xs, last, ws[E - 1].contiguous(), out_dtype=torch.float32)
    size = (x.float() * xs.repeat_interleave(128, 1)).abs() @ last.float().abs().t()
    assert bool(((y - z).abs() <= 2 * 64 * 2.0 ** -24 * size).all())
    del w, y, z, size
    M, K, N = (1 << 31) // 8192 + 100, 8192, 128
    x = torch.zeros((M, K), dtype=torch.uint8, device="cuda").view(E4M3)
    x[-64:] = torch.randn((64, K), device="cuda").to(E4M3)
    xs = torch.rand((64, M), device="cuda").t()
    y = ccdc.matmul_fp8(x, xs, last[:N], ws[0, :1].contiguous(), out_dtype=torch.float32)
    z = ccdc.matmul_fp8(x[-64:].clone(), xs[-64:].clone(), last[:N], ws[0, :1].contiguous(), out_dtype=torch.float32)
    # other tiles may cut k elsewhere: 64 blocks joined in another order
    assert float((y[-64:] - z).abs().max()) <= 64 * 2.0 ** -24 * float(z.abs().max()) * 8 and not y[:-64].any()
    ccdc.block_status()

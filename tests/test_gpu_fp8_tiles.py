"""8-bit products of several tiles a block: stages, accumulators and scales that go on from tile to tile, and stores of a tile
under the next one's products.  Whole numbers and scales of 1/2, 1 and 2 give sums below 2^24 quarters, which are exact in any
order, so every element has one value."""
import pytest

from tests.test_gpu_fp8 import DT, E4M3, ccdc        # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def tile(M, N, K, E, sms):
    """(SMs to a tile, its tokens, its weight rows, parts of k): the rule by which the library chooses"""
    nb, kb, each, most_split = -(-N // 128), -(-K // 128), -(-M // max(E, 1)), 8

    def most(nt, wide):
        return (M // nt + min(E + 1, M) if E else -(-M // nt)) * wide

    def cuts(tiles, blocks):
        splits = 1
        while splits < most_split and tiles * splits * 2 <= blocks and 2 * splits <= kb:
            splits *= 2
        return splits

    if each <= 64:
        nt = 16 if each <= 8 else 32 if each <= 16 else 64
        return 1, nt, 128, cuts(most(nt, nb), 2 * sms)
    wide = (nb + 1) // 2
    splits = cuts(most(128, wide), sms)

    def rounds(nt, at_once):
        tiles = (M // nt + (E + 1) // 2 if E else -(-M // nt)) * wide
        return -(-max(tiles, 1) // at_once)

    if each > 128 and rounds(256, sms // 2) * (kb + 5) <= rounds(128, sms // splits) * (kb // splits + 5) + (5 if splits > 1 else 0):
        return 2, 256, 256, 1
    return 1, 128, 256, splits


# rows, weight rows, k (an odd number of blocks in most), experts; the tile
CASES = [(600, 900, 870, 128, 16), (5, 115200, 390, 0, 16), (1400, 1200, 870, 100, 32), (15, 115100, 260, 0, 32), (2500, 1900, 640, 64, 64),
         (50, 115199, 390, 0, 64), (2000, 6000, 870, 20, 128), (100, 115001, 390, 0, 128), (5000, 2999, 850, 0, 256), (5000, 3001, 600, 8, 256),
         (9000, 2048, 1000, 5, 128)]


@pytest.mark.parametrize("M,N,K,E,tokens", CASES)
def test_several_tiles_a_block(ccdc, M, N, K, E, tokens):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    cg, nt, nw, splits = tile(M, N, K, E, sms)
    assert nt == tokens and splits == 1
    g = torch.Generator(device="cuda").manual_seed(M + N)

    def whole(rows):                            # rows at multiples of 16 bytes, NaN behind their ends
        t = torch.full((rows, -(-K // 16) * 16), float("nan"), device="cuda")
        t[:, :K] = torch.randint(-8, 9, (rows, K), generator=g, device="cuda")
        return t.to(E4M3)[:, :K]

    def scales(*shape):
        return torch.tensor([0.5, 1.0, 2.0], device="cuda")[torch.randint(0, 3, shape, generator=g, device="cuda")]

    kb, nb = -(-K // 128), -(-N // 128)
    x, xs = whole(M), scales(M, kb)
    w, ws = whole(max(E, 1) * N), scales(max(E, 1), nb, kb)
    w = w.as_strided((max(E, 1), N, K), (N * w.stride(0), w.stride(0), 1))
    left = M - 3 if E else M                    # rows behind the last expert's
    if E:
        share = torch.rand(E, generator=g, device="cuda") + 0.7
        ends = (share.cumsum(0) / share.sum() * left).round().int()
        offsets = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), ends])
        at = offsets.tolist()
    else:
        offsets, at = None, [0, M]
    tiles = sum(-(-(b - a) // nt) for a, b in zip(at, at[1:])) * -(-N // nw)
    assert tiles >= 3 * (sms // 2 if cg == 2 else sms if nt == 128 else 2 * sms)
    want = torch.zeros((M, N), dtype=torch.float64, device="cuda")
    full = x.float() * xs.repeat_interleave(128, 1)[:, :K]
    for e, (a, b) in enumerate(zip(at, at[1:])):
        weight = w[e].float() * ws[e].repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
        want[a:b] = full[a:b].double() @ weight.double().t()
    assert float(want.abs().max()) < 2.0 ** 22
    if not E:
        w, ws = w[0], ws[0]
    for dtype in DT.values():
        for pad in (0, 3, 32):                  # whole sectors where N allows, rows that start anywhere
            big = torch.full((M, N + pad), 7.0, dtype=dtype, device="cuda")
            y = ccdc.matmul_fp8(x, xs, w, ws, offsets=offsets, out=big[:, :N])
            wrong = (y != want.float().to(dtype)).nonzero()
            assert wrong.numel() == 0, (dtype, pad, wrong.shape[0], wrong[0].tolist())
            assert bool((big[:, N:] == 7).all())
    ccdc.block_status()

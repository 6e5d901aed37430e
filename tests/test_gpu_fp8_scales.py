"""8-bit products at the ends of the scales' range: products of two scales from 2^-126 to 2^100, exact with whole numbers."""
import pytest

from tests.test_gpu_fp8 import E4M3, ccdc        # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("M", [3, 12, 40, 100, 1500])
def test_ends_of_the_scales(ccdc, M):
    N, K = 300, 384
    g = torch.Generator(device="cuda").manual_seed(M)
    x, w = (torch.randint(-8, 9, (rows, K), generator=g, device="cuda").float().to(E4M3) for rows in (M, N))
    sums = x.double() @ w.double().t()
    for a, b in ((-126, 0), (-63, -63), (0, -126), (-126, 100), (100, 0), (50, 50), (-100, 126)):
        xs, ws = torch.full((M, 3), 2.0 ** a, device="cuda"), torch.full((3, 3), 2.0 ** b, device="cuda")
        y = ccdc.matmul_fp8(x, xs, w, ws, out_dtype=torch.float32)
        assert torch.equal(y.double(), sums * 2.0 ** (a + b)), (a, b)

"""Distillation of more rows than run at once: blocks take row after row, fetch the next under the current one, and keep two
rows' slots.  Every row has targets and is compared with 64 bits."""
import pytest

from tests.block_reference import SMALLEST, U
from tests.test_gpu_distill import DT, ccdc         # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def bounds(z, ids, values, dloss, T, lse, u, tiny):
    """(loss, its bound, dz, its bound) in 64 bits on the device.  The sum of exponentials: each has 2^-22 (approximate
    exponential) and three roundings of (z - top) / T, whose mean over s is at most log V; a thread adds V / 32 of them at most (one
    warp to a row) and 60 more sums and rescalings join them."""
    M, V = z.shape
    e32 = 2.0 ** -24
    sums = 2.0 ** -22 + e32 * (3 * float(torch.log(torch.tensor(V + 1.0))) + V / 32 + 60)
    zt, ids = z.double() / T, ids.long()
    there = (ids >= 0) & (ids < V)
    at = ids.masked_fill(~there, 0)
    v = (values.double() / T).masked_fill(~there, -float("inf"))
    whole = torch.logsumexp(v, 1) if lse is None else lse.double()
    log_t = (v - whole[:, None]).masked_fill(~there, 0.0)
    t = log_t.exp() * there
    top = zt.amax(1, keepdim=True)
    log_s = zt - torch.logsumexp(zt, 1, keepdim=True)
    loss = (t * (log_t - log_s.gather(1, at))).sum(1)
    away = top - zt
    loss_tol = t.sum(1) * sums + (t * away.gather(1, at)).sum(1) * 2 * e32 + e32 * loss.abs()
    target = torch.zeros_like(zt).scatter_add_(1, at, t)
    g, Ps = (dloss.double() / T)[:, None], t.sum(1, keepdim=True) * log_s.exp()
    dz = g * (Ps - target)
    dz_tol = g.abs() * (Ps * (sums + 2.0 ** -22 + e32 * (3 * away + 6)) + target * 4 * e32) * (1 + u) + u * dz.abs() + tiny
    return loss, loss_tol, dz, dz_tol


# rows, logits, slots, threads that walk a row (a warp for the teacher beside them), blocks to a row in 16 bits and in binary32
CASES = [(15000, 257, 9, 32, 1, 1), (15000, 1001, 5, 32, 1, 1), (9400, 3001, 40, 64, 1, 1), (5400, 10007, 33, 128, 1, 1),
         (650, 70001, 70, 256, 3, 5)]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,V,k,threads,blocks,blocks32", CASES)
def test_more_rows_than_run_at_once(ccdc, M, V, k, threads, blocks, blocks32, dtype):
    if dtype == "float32":
        V, blocks = V // 2 if blocks == 1 else V, blocks32
    # the most blocks that an SM holds: by its 2048 threads and 32 blocks; parts of a cluster's rows take over 45 KiB
    most = min(32, 2048 // (threads + 32)) if blocks == 1 else 4
    assert M * blocks >= 3 * most * torch.cuda.get_device_properties(0).multi_processor_count
    g = torch.Generator(device="cuda").manual_seed(V)
    for T, kind, whole, pad in ((1.0, torch.int32, False, 0), (2.5, torch.int64, True, 5)):
        z = torch.randn((M, V + pad), generator=g, device="cuda").mul_(2).to(DT[dtype])[:, :V]
        ids = torch.randint(0, V, (M, k), generator=g, device="cuda")
        ids[:, 1:] = torch.where(torch.rand((M, k - 1), generator=g, device="cuda") < 0.2, -1, ids[:, 1:])
        ids = ids.to(kind)
        values = torch.randn((M, k), generator=g, device="cuda").mul_(2).to(DT[dtype])
        dloss = torch.rand(M, generator=g, device="cuda") + 0.5
        lse = torch.logsumexp(values.float() / T, 1) + 0.25 if whole else None
        how = dict(temperature=T, teacher_lse=lse)
        is_loss, loss_tol, is_dz, dz_tol = bounds(z, ids, values, dloss, T, lse, U[dtype], SMALLEST[dtype])

        def check(loss, dz=None):
            over = (loss.double() - is_loss).abs() - loss_tol
            assert float(over.max()) <= 0, ("loss", float(over.max()), int(over.argmax()))
            if dz is not None:
                over = (dz.double() - is_dz).abs_().sub_(dz_tol)
                assert float(over.max()) <= 0, ("dz", float(over.max()), divmod(int(over.argmax()), V))

        check(ccdc.distill_forward(z, ids, values, **how))
        loss, stats = ccdc.distill_forward(z, ids, values, save=True, **how)
        check(loss, ccdc.distill_backward(dloss, z, ids, values, stats, **how))
        check(*ccdc.distill(dloss, z, ids, values, **how))
        other = torch.full((M, V + 3), 7.0, dtype=DT[dtype], device="cuda")             # rows that start elsewhere
        check(*ccdc.distill(dloss, z, ids, values, dlogits=other[:, :V], **how))
        assert bool((other[:, V:] == 7).all())
        other.fill_(7)
        ccdc.distill_backward(dloss, z, ids, values, stats, dlogits=other[:, :V], **how)
        check(loss, other[:, :V])
        assert bool((other[:, V:] == 7).all())
        loss, dz = ccdc.distill(dloss, z, ids, values, dlogits=z, **how)                # in place, last
        assert dz.data_ptr() == z.data_ptr()
        check(loss, dz)

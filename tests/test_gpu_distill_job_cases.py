"""The distillation job's Map of few rows, where experts are left without any, and at another temperature; its operators on two
streams at once."""
import pytest

from tests.test_gpu_distill_job import ccdc, student_gradients, unit        # noqa: F401  (ccdc: the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def student_at(x, told, params, choose, T):
    """loss and gradients at temperature T, which is loss at 1 of logits and words divided by it"""
    at, values, lse = told
    scaled = {**params, "w_words": params["w_words"].double() / T}
    loss, grads = student_gradients(x, (at, values.double() / T, lse), scaled, choose)
    return loss, [g / T if name == "w_words" else g for name, g in zip(params, grads)]


@pytest.mark.parametrize("rows,T", [(1, 1.0), (3, 1.0), (3, 2.5), (40, 0.7)])
def test_few_rows(ccdc, rows, T):
    """gradients of experts without rows are zero whatever the partition held"""
    from paper_1805_01993_b200 import distill_job as job

    D, F, E, V, choose = 48, 80, 16, 150, 2
    params = job.make_parameters(D, F, E, V, torch.float32)
    x = torch.randn((rows, D), generator=torch.Generator(device="cuda").manual_seed(rows), device="cuda")
    at, values, _ = job.teacher_top(x, job.make_teacher(D, F, E, V, torch.float32), choose, V)
    told = at, values, torch.logsumexp(values / T, 1)               # all logits are there
    row = torch.full((job.gradient_words(D, F, E, V),), float("nan"), device="cuda")
    loss = job.map_file(x, told, params, choose, row, temperature=T)
    want, grads = student_at(x, told, params, choose, T)
    assert abs(float(loss) - float(want)) <= 1e-5 * abs(float(want))
    start = 0
    z = unit(x.double()) * params["w_pre"].double()
    there = torch.zeros(E, dtype=torch.bool, device="cuda")
    there[torch.softmax(z @ params["w_router"].double().t(), 1).topk(choose, 1).indices.reshape(-1)] = True
    for name, g in zip(params, grads):
        got = row[start:start + g.numel()].double().view(g.shape)
        start += g.numel()
        # chains of about ten binary32 operators, each off by some 2^-21 of its result's norm
        assert float((got - g).norm() / g.norm()) <= 1e-5, name
        if name in ("w_gate", "w_up", "w_down"):
            assert not got[~there].any() and bool((~there).any() or rows == 40)


def test_two_streams_at_once(ccdc):
    """calls and replays on two streams leave the bits of one after the other"""
    g = torch.Generator(device="cuda").manual_seed(2)

    def inputs(M, E, D, V):
        w = ccdc.quantize_fp8(torch.randn((E, 512, D), generator=g, device="cuda").bfloat16(), 128)
        words = ccdc.quantize_fp8(torch.randn((V, 512), generator=g, device="cuda").bfloat16(), 128)
        return (torch.randint(-1, E, (M, 2), generator=g, device="cuda"), torch.randn((M, D), generator=g, device="cuda").bfloat16(), w, words,
                torch.randint(0, V, (M, 9), generator=g, device="cuda"), torch.randn((M, 9), generator=g, device="cuda"),
                torch.rand(M, generator=g, device="cuda"))

    def pass_of(ids, x, w, words, at, values, dloss):
        order = ccdc.expert_sort(ids, w[0].shape[0])
        xs = ccdc.expert_dispatch(x, order)
        ys = ccdc.matmul_fp8(*ccdc.quantize_fp8(xs), *w, offsets=order.offsets)
        y = ccdc.expert_combine(ys, order)
        logits = ccdc.matmul_fp8(*ccdc.quantize_fp8(y), *words)
        loss, dz = ccdc.distill(dloss, logits, at, values, temperature=2.0)
        return *order, y, logits, loss, dz

    sets = [inputs(900, 6, 640, 3000), inputs(30, 9, 384, 20000)]       # pairs of SMs and cut k; few rows
    want = [pass_of(*s) for s in sets]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(pass_of(*sets[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        for r in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(r, want[i]))
    graphs, outs = [], []
    for s in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(pass_of(*s))
        graphs.append(graph)
    for _ in range(5):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i]))
    ccdc.block_status()

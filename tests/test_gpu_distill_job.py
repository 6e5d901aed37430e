"""The operators together: a teacher in 8 bits, a student of experts, the distillation loss, and the coded shuffle of its gradients."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ccdc():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_1805_01993_b200 import build, ccdc as mod

    build.build_library()
    mod.lib()
    return mod


def unit(v):
    return v / (v.square().mean(1, keepdim=True) + 1e-5).sqrt()


def student_gradients(x, told, params, choose):
    """loss and gradients in 64 bits by automatic differentiation"""
    leaves = {k: v.double().requires_grad_() for k, v in params.items()}
    x = x.double()
    z = unit(x) * leaves["w_pre"]
    w, ids = torch.softmax(z @ leaves["w_router"].t(), 1).topk(choose, 1)
    y = torch.zeros_like(x)
    for e in range(params["w_router"].shape[0]):
        h = z @ leaves["w_gate"][e].t()
        part = (h * torch.sigmoid(h) * (z @ leaves["w_up"][e].t())) @ leaves["w_down"][e].t()
        y = y + part * (w * (ids == e)).sum(1, keepdim=True)
    out = unit(x + unit(y) * leaves["w_post"]) * leaves["w_out"]
    at, values, lse = told
    log_t = values.double() - lse.double()[:, None]
    log_s = torch.log_softmax(out @ leaves["w_words"].t(), 1).gather(1, at)
    loss = (log_t.exp() * (log_t - log_s)).sum(1).mean()
    return loss.detach(), torch.autograd.grad(loss, [leaves[k] for k in params])


def test_distill_job(ccdc):
    """Map, shuffle and Reduce: the Reduce output is the sum over the files, a file's gradients are those of automatic
    differentiation, and a second run leaves the same bits"""
    from paper_1805_01993_b200 import distill_job as job

    sizes = dict(nodes=4, load=2, files=6, rows=45, width=64, inner=96, experts=5, choose=2, words=333, top=20, seed=7, dtype=torch.float32)
    total, per_file, plan, losses = job.run(**sizes)
    direct, size = per_file.double().sum(0), per_file.double().abs().sum(0)
    assert bool(((total.double() - direct).abs() <= 1e-5 * size + 1e-30).all())
    params = job.make_parameters(64, 96, 5, 333, torch.float32)
    teacher = job.make_teacher(64, 96, 5, 333, torch.float32)
    g = torch.Generator(device="cuda").manual_seed(7)
    data = [torch.randn((45, 64), generator=g, device="cuda") for _ in range(6)]
    for n in (0, 5):
        told = job.teacher_top(data[n], teacher, 2, 20)
        loss, grads = student_gradients(data[n], told, params, 2)
        assert abs(float(losses[n]) - float(loss)) <= 1e-5 * abs(float(loss))
        at = 0
        for name, want in zip(params, grads):
            got = per_file[n][at:at + want.numel()].double().view(want.shape)
            at += want.numel()
            # chains of about ten binary32 operators, each off by some 2^-21 of its result's norm
            assert float((got - want).norm() / want.norm()) <= 1e-5, (n, name)
    again = job.run(**sizes)
    assert torch.equal(again[1], per_file) and torch.equal(again[0], total)


def test_replicas(ccdc):
    """a file mapped twice, from other addresses, leaves the same bits; so does the teacher's answer"""
    from paper_1805_01993_b200 import distill_job as job

    D, F, E, V = 128, 200, 6, 1000
    params = job.make_parameters(D, F, E, V, torch.bfloat16)
    teacher = job.make_teacher(D, F, E, V, torch.bfloat16)
    x = torch.randn((33, D), device="cuda").bfloat16()
    told = job.teacher_top(x, teacher, 3, 16)
    assert all(torch.equal(a, b) for a, b in zip(told, job.teacher_top(x.clone(), teacher, 3, 16)))
    words = job.gradient_words(D, F, E, V)
    a, b = torch.zeros(words, device="cuda"), torch.ones(words + 64, device="cuda")[64:]
    job.map_file(x, told, params, 3, a)
    job.map_file(x.clone(), tuple(t.clone() for t in told), {k: v.clone() for k, v in params.items()}, 3, b)
    assert torch.equal(a, b) and bool(a.isfinite().all())


def test_teacher_in_8_bits(ccdc):
    """the teacher's logits against 64 bits with the same 8-bit weights: three quantisations of rows, each element off by 2^-4 of
    itself at most and 2^-4 / sqrt(3) / sqrt(2) in the mean, independent; 3 times their joint size is allowed"""
    from paper_1805_01993_b200 import distill_job as job

    D, F, E, V, choose = 256, 384, 4, 700, 2
    teacher = job.make_teacher(D, F, E, V, torch.float32)
    x = torch.randn((60, D), device="cuda")
    at, values, lse = job.teacher_top(x, teacher, choose, V)

    def stored(name):
        q, s = teacher[name]
        n, k = q.shape[-2:]
        return q.double() * s.double().repeat_interleave(128, -2)[..., :n, :].repeat_interleave(128, -1)[..., :k]

    z = unit(x.double())
    w, ids = torch.softmax(z @ teacher["router"].double().t(), 1).topk(choose, 1)
    y = torch.zeros_like(z)
    for e in range(E):
        a = torch.nn.functional.silu(z @ stored("up")[e].t()) @ stored("down")[e].t()
        y += a * (w * (ids == e)).sum(1, keepdim=True)
    want = unit(x.double() + y) @ stored("words").t()
    got = torch.zeros_like(want).scatter_(1, at, values.double())
    assert float((got - want).norm() / want.norm()) <= 3 * 3 ** 0.5 * 2.0 ** -4 / 6 ** 0.5
    assert float((lse.double() - torch.logsumexp(got, 1)).abs().max()) <= 1e-5


def test_command(ccdc, capsys):
    from paper_1805_01993_b200 import distill_job as job

    job.main(["--rows", "20", "--files", "6", "--words", "300", "--experts", "3", "--width", "64", "--inner", "64"])
    assert "difference from the direct sum" in capsys.readouterr().out

"""A coded gradient job of a student of experts that learns from a teacher's top logits, end to end on one GPU.

    python -m paper_1805_01993_b200.distill_job [--nodes 4 --load 2 --files 6 --rows 256 --width 256 --inner 512 --experts 8 --choose 2
                                                 --words 4096 --top 32]

Every file is a batch of token rows.  A frozen teacher, whose products run in 8 bits, gives each row its top logits:

    z = norm(x);  rows sorted by expert, a = silu(z W1[e]^T), W2[e] a back with weights;  logits = norm(x + .) Wv^T

The Map of a file runs the student, a block of feed-forward experts, forward and backward:

    z = norm(x) w_pre;  experts and weights from softmax(z w_router^T);  y = sum of weight * feed-forward_e(z) over a row's experts
    out = norm(x + norm(y) w_post) w_out;  logits = out w_words^T;  loss = distillation from the teacher's top logits

and writes the parameters' gradients, in binary32, into the partition of each node that stores the file; the compressed coded
shuffle then sums them over all files.

Replicas of a file have to agree bit by bit: rows are sorted stably, sums have one order, and the teacher answers once per file
(its logits are part of the file).
"""
from __future__ import annotations

import argparse

from .block_job import _count

PARAMETERS = ("w_gate", "w_up", "w_down", "w_router", "w_pre", "w_post", "w_out", "w_words")


def shapes(D, F, E, V):
    return {"w_gate": (E, F, D), "w_up": (E, F, D), "w_down": (E, D, F), "w_router": (E, D), "w_pre": (D,), "w_post": (D,), "w_out": (D,),
            "w_words": (V, D)}


def gradient_words(D, F, E, V):
    return sum(_count(s) for s in shapes(D, F, E, V).values())


def make_parameters(D, F, E, V, dtype, seed=0):
    import torch

    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=g, device="cuda") * std + mean).to(dtype)

    std = {"w_gate": D ** -0.5, "w_up": D ** -0.5, "w_down": F ** -0.5, "w_router": D ** -0.5, "w_words": 2 * D ** -0.5}
    return {name: randn(*shape, std=std[name]) if name in std else randn(*shape, std=0.1, mean=1.0)
            for name, shape in shapes(D, F, E, V).items()}


def make_teacher(D, F, E, V, dtype, seed=1):
    """The teacher's weights: 8-bit values and scales of 128 x 128 blocks, and its router."""
    import torch

    from . import ccdc

    g = torch.Generator(device="cuda").manual_seed(seed)

    def eight_bits(*shape, std):
        return ccdc.quantize_fp8((torch.randn(shape, generator=g, device="cuda") * std).to(dtype), 128)

    return {"up": eight_bits(E, F, D, std=D ** -0.5), "down": eight_bits(E, D, F, std=F ** -0.5), "words": eight_bits(V, D, std=2 * D ** -0.5),
            "router": (torch.randn((E, D), generator=g, device="cuda") * D ** -0.5).to(dtype), "unit": torch.ones(D, dtype=dtype, device="cuda")}


def route(z, w_router, choose):
    """(ids [M][choose], their weights, all probabilities): the largest of softmax(z w_router^T)"""
    import torch

    p = torch.softmax(z.float() @ w_router.float().t(), 1)
    w, ids = p.topk(choose, 1)
    return ids, w, p


def teacher_top(x, teacher, choose, top):
    """(ids, values [rows][top], logsumexp of all logits): what a file keeps of the teacher's answer"""
    import torch

    from . import ccdc

    z = ccdc.residual_norm_forward(x, w_pre=teacher["unit"])[1]
    ids, w, _ = route(z, teacher["router"], choose)
    order = ccdc.expert_sort(ids, teacher["router"].shape[0])
    a = ccdc.matmul_fp8(*ccdc.quantize_fp8(ccdc.expert_dispatch(z, order)), *teacher["up"], offsets=order.offsets, out_dtype=x.dtype)
    a = torch.nn.functional.silu(a)
    y = ccdc.matmul_fp8(*ccdc.quantize_fp8(a), *teacher["down"], offsets=order.offsets, out_dtype=x.dtype)
    out = ccdc.residual_norm_forward(x, ccdc.expert_combine(y, order, w), w_pre=teacher["unit"])[1]
    logits = ccdc.matmul_fp8(*ccdc.quantize_fp8(out), *teacher["words"], out_dtype=torch.float32)
    values, at = logits.topk(top, 1)
    return at, values, torch.logsumexp(logits, 1)


def map_file(x, told, params, choose, row, temperature=1.0, act="silu"):
    """Forward and backward of one file's rows; the gradients go into ``row`` (binary32, the file's partition row).
    ``told``: (ids, values, logsumexp) of the teacher at this temperature.  Returns the mean loss, a tensor on the device."""
    import torch

    from . import ccdc

    f32 = torch.float32
    E, F, D = params["w_gate"].shape
    into, at = {}, 0
    for name, shape in shapes(D, F, E, params["w_words"].shape[0]).items():
        into[name] = row[at:at + _count(shape)].view(shape)
        at += _count(shape)
    weights = [(params["w_gate"][e], params["w_up"][e], params["w_down"][e]) for e in range(E)]
    _, z, stats_in = ccdc.residual_norm_forward(x, w_pre=params["w_pre"], save=True)
    ids, w, p = route(z, params["w_router"], choose)
    order = ccdc.expert_sort(ids, E)
    zs = ccdc.expert_dispatch(z, order)
    ends = order.offsets.tolist()               # the feed-forward calls take their rows from the host
    ys, saved = torch.empty_like(zs), []
    for e in range(E):
        rows = slice(ends[e], ends[e + 1])
        saved.append(ccdc.ffn_forward(zs[rows], *weights[e], act=act, save=True, out=ys[rows])[1])
    y = ccdc.expert_combine(ys, order, w)
    join = dict(w_post=params["w_post"], w_pre=params["w_out"])
    _, out, stats_out = ccdc.residual_norm_forward(x, y, save=True, **join)
    logits = out @ params["w_words"].t()
    teacher_ids, values, lse = told
    share = torch.full((x.shape[0],), 1.0 / max(1, x.shape[0]), device=x.device)
    loss, dlogits = ccdc.distill(share, logits, teacher_ids, values, temperature=temperature, teacher_lse=lse, dlogits=logits)
    torch.mm(dlogits.float().t(), out.float(), out=into["w_words"])
    dout = dlogits @ params["w_words"]
    dx, dy, _, _, _ = ccdc.residual_norm_backward(None, dout, x, y, stats_out, grad_dtype=f32, dw_post=into["w_post"], dw_pre=into["w_out"], **join)
    dys, dw = ccdc.expert_combine_backward(dy, ys, order, w)
    dzs = torch.zeros_like(zs)
    for e in range(E):
        rows = slice(ends[e], ends[e + 1])
        ccdc.ffn_backward(dys[rows], zs[rows], *weights[e], saved[e], act=act, grad_dtype=f32, dx=dzs[rows], dw_gate=into["w_gate"][e],
                          dw_up=into["w_up"][e], dw_down=into["w_down"][e])
    # the weights are probabilities of the chosen experts: back through the softmax over all of them
    dp = torch.zeros_like(p).scatter_(1, ids, dw)
    dscores = p * (dp - (p * dp).sum(1, keepdim=True))
    torch.mm(dscores.t(), z.float(), out=into["w_router"])
    dz = (ccdc.expert_dispatch_backward(dzs, order).float() + dscores @ params["w_router"].float()).to(x.dtype)
    ccdc.residual_norm_backward(dx, dz, x, None, stats_in, w_pre=params["w_pre"], grad_dtype=f32, dw_pre=into["w_pre"])
    return loss.mean()


def run(nodes=4, load=2, files=6, rows=256, width=256, inner=512, experts=8, choose=2, words=4096, top=32, seed=20180501, dtype=None):
    """Teacher, Map, shuffle and Reduce; returns (full gradient [words], the files' gradients [files][words], the plan, losses)."""
    import torch

    from . import ccdc

    dtype = torch.bfloat16 if dtype is None else dtype
    params = make_parameters(width, inner, experts, words, dtype)
    teacher = make_teacher(width, inner, experts, words, dtype)
    count = gradient_words(width, inner, experts, words)
    Q = nodes
    B = -(-count // (Q * 4)) * 4                    # a slice of the gradient per Reduce function, the last one padded
    plan = ccdc.Plan(nodes, load, files, Q, B, "float32")
    part = plan.alloc_partitions()
    g = torch.Generator(device="cuda").manual_seed(seed)
    data = [torch.randn((rows, width), generator=g, device="cuda").to(dtype) for _ in range(files)]
    told = [teacher_top(x, teacher, choose, top) for x in data]
    losses = [None] * files
    for k in range(nodes):                          # every node maps its own copies of its files
        for i, n in enumerate(plan.node_files(k)):
            row = part[k][i * Q * B:(i + 1) * Q * B]
            row[count:] = 0
            losses[n] = map_file(data[n], told[n], params, choose, row)
    coded, out, ws = plan.alloc(plan.coded_bytes), plan.alloc(plan.out_bytes), plan.alloc(plan.workspace_bytes)
    plan.shuffle(part, coded, out, ws)
    torch.cuda.synchronize()
    ccdc.block_status()
    per_file = torch.empty((files, count), device="cuda")
    for k in range(nodes):
        for i, n in enumerate(plan.node_files(k)):
            per_file[n] = part[k][i * Q * B:i * Q * B + count]
    return out[:count], per_file, plan, losses


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("nodes", 4), ("load", 2), ("files", 6), ("rows", 256), ("width", 256), ("inner", 512), ("experts", 8), ("choose", 2),
                          ("words", 4096), ("top", 32)):
        ap.add_argument(f"--{name}", type=int, default=default)
    a = ap.parse_args(argv)
    total, per_file, plan, losses = run(**vars(a))
    direct = per_file.double().sum(0)
    err = float((total.double() - direct).norm() / direct.norm())
    print(f"{a.files} files of {a.rows} x {a.width} rows on {a.nodes} nodes, load {a.load}, {a.choose} of {a.experts} experts: gradient of "
          f"{total.numel()} words, mean loss {sum(float(v) for v in losses) / len(losses):.4f}, {plan.coded_bits / 8e6:.2f} MB multicast, "
          f"difference from the direct sum {err:.2e}")


if __name__ == "__main__":
    main()

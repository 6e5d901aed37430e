"""A coded gradient job of one transformer feed-forward sub-block, end to end on one GPU.

    python -m paper_1805_01993_b200.block_job [--nodes 4 --load 2 --files 6 --rows 256 --width 512 --inner 1024]

Every file is a batch of token rows.  Its Map runs the sub-block

    z = norm(x) w_pre;  y = feed-forward(z);  out = x + drop(gate * norm(y) w_post)

forward and backward (the loss is the mean square of ``out``) and writes the parameters' gradients, in binary32,
straight into the partition of each node that stores the file.  The compressed coded shuffle then sums the gradients
over all files, and every node ends with its slices of the full gradient.

Coded computing needs the replicas of a file to agree bit by bit (a node cancels from a packet what it computed itself).
The block operators add in fixed orders without atomics, and the dropout mask depends on (seed, element) alone: each file
draws from its own range of elements, so every node that maps it draws the same mask.
"""
from __future__ import annotations

import argparse

PARAMETERS = ("w_gate", "w_up", "w_down", "w_pre", "w_post", "gate")


def shapes(D, F):
    return {"w_gate": (F, D), "w_up": (F, D), "w_down": (D, F), "w_pre": (D,), "w_post": (D,), "gate": (D,)}


def make_parameters(D, F, dtype, seed=0):
    import torch

    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=g, device="cuda") * std + mean).to(dtype)

    return {"w_gate": randn(F, D, std=D ** -0.5), "w_up": randn(F, D, std=D ** -0.5), "w_down": randn(D, F, std=F ** -0.5),
            "w_pre": randn(D, std=0.1, mean=1.0), "w_post": randn(D, std=0.1, mean=1.0), "gate": randn(D, std=0.3, mean=0.5)}


def gradient_words(D, F):
    return sum(_count(s) for s in shapes(D, F).values())


def _count(shape):
    n = 1
    for s in shape:
        n *= s
    return n


def map_file(x, params, p, seed, offset, row, act="silu"):
    """Forward and backward of one file's rows; the gradients go into ``row`` (binary32, the file's partition row).
    Returns the loss, a tensor on the device."""
    import torch

    from . import ccdc

    M, D = x.shape
    F = params["w_gate"].shape[0]
    into, at = {}, 0
    for name, shape in shapes(D, F).items():
        into[name] = row[at:at + _count(shape)]
        at += _count(shape)
    weights = params["w_gate"], params["w_up"], params["w_down"]
    join = dict(w_post=params["w_post"], gate=params["gate"], rows_per_gate=max(M, 1), p=p, seed=seed, offset=offset)
    _, z, stats_in = ccdc.residual_norm_forward(x, w_pre=params["w_pre"], save=True)
    y, saved = ccdc.ffn_forward(z, *weights, act=act, save=True)
    out, _, stats_out = ccdc.residual_norm_forward(x, y, save=True, **join)
    loss = out.float().square().mean()
    dout = (out.float() * (2.0 / out.numel())).to(out.dtype)
    f32 = torch.float32
    dx, dy, _, _, _ = ccdc.residual_norm_backward(dout, None, x, y, stats_out, grad_dtype=f32, dw_post=into["w_post"],
                                                  dgate=into["gate"], **join)
    dz, *_ = ccdc.ffn_backward(dy, z, *weights, saved, act=act, grad_dtype=f32, dw_gate=into["w_gate"],
                               dw_up=into["w_up"], dw_down=into["w_down"])
    ccdc.residual_norm_backward(dx, dz, x, None, stats_in, w_pre=params["w_pre"], grad_dtype=f32, dw_pre=into["w_pre"])
    return loss


def run(nodes=4, load=2, files=6, rows=256, width=512, inner=1024, p=0.1, seed=20180501, dtype=None):
    """Map, shuffle and Reduce; returns (full gradient [words], the files' gradients [files][words], the plan)."""
    import torch

    from . import ccdc

    dtype = torch.bfloat16 if dtype is None else dtype
    params = make_parameters(width, inner, dtype)
    words = gradient_words(width, inner)
    Q = nodes
    B = -(-words // (Q * 4)) * 4                    # a slice of the gradient per Reduce function, the last one padded
    plan = ccdc.Plan(nodes, load, files, Q, B, "float32")
    part = plan.alloc_partitions()
    g = torch.Generator(device="cuda").manual_seed(seed)
    data = [torch.randn((rows, width), generator=g, device="cuda").to(dtype) for _ in range(files)]
    losses = [None] * files
    for k in range(nodes):                          # every node maps its own copies of its files
        for i, n in enumerate(plan.node_files(k)):
            row = part[k][i * Q * B:(i + 1) * Q * B]
            row[words:] = 0
            losses[n] = map_file(data[n], params, p, seed, n * rows * width, row)
    coded, out, ws = plan.alloc(plan.coded_bytes), plan.alloc(plan.out_bytes), plan.alloc(plan.workspace_bytes)
    plan.shuffle(part, coded, out, ws)
    torch.cuda.synchronize()
    ccdc.block_status()
    per_file = torch.empty((files, words), device="cuda")
    for k in range(nodes):
        for i, n in enumerate(plan.node_files(k)):
            per_file[n] = part[k][i * Q * B:i * Q * B + words]
    return out[:words], per_file, plan, losses


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("nodes", 4), ("load", 2), ("files", 6), ("rows", 256), ("width", 512), ("inner", 1024)):
        ap.add_argument(f"--{name}", type=int, default=default)
    ap.add_argument("--drop", type=float, default=0.1)
    a = ap.parse_args(argv)
    total, per_file, plan, losses = run(a.nodes, a.load, a.files, a.rows, a.width, a.inner, a.drop)
    direct = per_file.double().sum(0)
    err = float((total.double() - direct).norm() / direct.norm())
    print(f"{a.files} files of {a.rows} x {a.width} rows on {a.nodes} nodes, load {a.load}: gradient of {total.numel()} words, "
          f"mean loss {sum(float(v) for v in losses) / len(losses):.4f}, {plan.coded_bits / 8e6:.2f} MB multicast, "
          f"difference from the direct sum {err:.2e}")


if __name__ == "__main__":
    main()

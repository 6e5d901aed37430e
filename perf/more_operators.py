"""Cases, plain forms and exact values of the operators of a distillation job of an expert block: tokens
sorted by expert and back, the distillation loss from a teacher's top logits, and the 8-bit product with a
scale for each block of 128.

A file of such a job is a batch of token rows ("M") with the teacher's top logits.  The teacher's products
run in 8 bits; the student's tokens are sorted by expert, go through the experts' feed-forward blocks and
come back weighted; the distillation loss starts the backward pass.

``own`` chooses between the plain form (elementary torch operations in 32 bits, rounded once) and the
framework's calls.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
MOST_ROUTED = 16384 * 8 * 4096          # sorted elements of the largest listed case
MOST_LOGITS = 4096 * 131072
MOST_PRODUCT = 8192 * 8192 * 8192       # multiplications
MOST_WEIGHTS = 1 << 29                  # bytes of 8-bit weights


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one token of a running answer to eight of its experts and back: latency of three small calls
        experts("experts_token", "forward", 1, 4096, 8, 128, "bf16"),
        # a small serving batch, some slots served by another process
        experts("experts_serve", "forward", 64, 2048, 8, 256, "fp16", weights="own", ids="int64", drop=0.1),
        # odd width and rows, an odd number of experts, gradients in the 32 bits of the shuffle's words
        experts("experts_train_ragged", "train", 1999, 1001, 3, 60, "fp32", drop=0.1, pad=5),
        # a large file through a block of many experts, forward and backward
        experts("experts_train_large", "train", 16384, 4096, 8, 64, "bf16"),
        # the loss of one row, as in a check of the student
        distill("distill_row", "forward", 1, 32000, 16, "bf16", 1.0),
        # a file that ends anywhere over an odd vocabulary; loss and gradient in one call
        distill("distill_ragged", "step", 300, 50257, 64, "fp16", 2.0, ids="int64"),
        # 32-bit logits, whose loss is scaled only after all files are known: two calls
        distill("distill_fp32", "train", 1024, 32000, 50, "fp32", 1.0, lse=True),
        # a large file over a large vocabulary
        distill("distill_large", "step", 4096, 131072, 128, "bf16", 2.0),
        # one token through a wide teacher's layer: bound by reading the weight once
        fp8("fp8_token", 1, 16384, 4096, 0, "bf16"),
        # a serving batch sorted by expert: a few rows for each of many weights
        fp8("fp8_experts_serve", 200, 2048, 4096, 64, "bf16"),
        # a file's rows sorted over experts of ragged widths
        fp8("fp8_experts_ragged", 2999, 1419, 1000, 12, "fp16", pad=8),
        # a large file through a dense layer
        fp8("fp8_prompt", 8192, 8192, 8192, 0, "bf16"),
    ]


def experts(name, way, M, D, k, E, dtype, weights="fp32", ids="int32", drop=0.0, pad=0):
    return {"name": name, "op": "experts", "way": way, "M": M, "D": D, "k": k, "E": E, "dtype": dtype,
            "weights": weights, "ids": ids, "drop": drop, "pad": pad}


def distill(name, way, M, V, k, dtype, T, ids="int32", lse=False, pad=0):
    return {"name": name, "op": "distill", "way": way, "M": M, "V": V, "k": k, "dtype": dtype, "T": T, "ids": ids,
            "lse": lse, "pad": pad}


def fp8(name, M, N, K, E, dtype, pad=0):
    return {"name": name, "op": "fp8", "M": M, "N": N, "K": K, "E": E, "dtype": dtype, "pad": pad}


def draw(rng):
    def size(low, high, step=1):
        v = math.exp(rng.uniform(math.log(low), math.log(high)))
        return min(high, max(low, int(round(v / step)) * step))

    def width(low, high):       # widths are mostly multiples of 64, sometimes of 8, sometimes odd
        kind = rng.random()
        return size(low, high, 64) if kind < 0.6 else size(low, high, 8) if kind < 0.8 else min(high - 1, size(low, high) | 1)

    op = rng.choice(["experts", "distill", "fp8"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    pad = rng.choice([0, 0, 8, 5])
    half = 2 if dtype == "fp32" else 1
    if op == "experts":
        while True:
            M, D, E = size(1, 16384), width(64, 8192), size(2, 512)
            k = min(size(1, 16), E)
            if M * k * D <= MOST_ROUTED // half:
                break
        c = experts("", rng.choice(["forward", "train"]), M, D, k, E, dtype, rng.choice(["fp32", "own"]),
                    rng.choice(["int32", "int64"]), rng.choice([0.0, 0.1, 0.5]), pad)
    elif op == "distill":
        while True:
            M, V = size(1, 16384), width(1000, 200000)
            if M * V <= MOST_LOGITS // half:
                break
        c = distill("", rng.choice(["forward", "train", "step"]), M, V, size(1, 256), dtype, rng.choice([1.0, 2.0, 0.7]),
                    rng.choice(["int32", "int64"]), rng.random() < 0.4, pad)
    else:
        while True:
            M, N, K = size(1, 16384), width(64, 16384), width(64, 16384)
            E = 0 if rng.random() < 0.5 else size(2, 128)
            if M * N * K <= MOST_PRODUCT and max(E, 1) * N * K <= MOST_WEIGHTS:
                break
        c = fp8("", M, N, K, E, dtype, pad)
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 29)
    t = TYPES[case["dtype"]]
    M = case["M"]
    s = dict(case)

    def randn(rows, cols, std=1.0, pad=0):
        return torch.randn((rows, cols + pad), generator=g, device="cuda").mul_(std).to(t)[:, :cols]

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    if case["op"] == "experts":
        D, k, E, pad = case["D"], case["k"], case["E"], case["pad"]
        # router scores with some experts more popular than others
        scores = torch.randn((M, E), generator=g, device="cuda") + 0.7 * torch.randn((1, E), generator=g, device="cuda")
        top, ids = scores.topk(k, 1)
        ids = torch.where(rand(M, k) < case["drop"], -1, ids)
        s["ids"] = ids.to(torch.int32 if case["ids"] == "int32" else torch.int64)
        s["w"] = torch.softmax(top, 1).to(torch.float32 if case["weights"] == "fp32" else t)
        s["x"] = randn(M, D, pad=pad)
        s["ys"] = randn(M * k, D)                       # what the experts return
        if case["way"] == "train":
            s["dy"] = randn(M, D, 0.02, pad=pad)
            s["dxs"] = randn(M * k, D, 0.02)            # what the experts' backward pass returns
    elif case["op"] == "distill":
        V, k, T = case["V"], case["k"], case["T"]
        z = torch.empty((M, V + case["pad"]), dtype=t, device="cuda")
        ids = torch.empty((M, k), dtype=torch.int64, device="cuda")
        s["values"] = torch.empty((M, k), dtype=t, device="cuda")
        s["teacher_lse"] = torch.empty(M, device="cuda") if case["lse"] else None
        for a in range(0, M, 512):                      # the student has learned most of what the teacher says
            b = min(a + 512, M)
            teacher = torch.randn((b - a, V), generator=g, device="cuda").mul_(2.5)
            s["values"][a:b], ids[a:b] = teacher.topk(k, 1)
            if case["lse"]:
                s["teacher_lse"][a:b] = torch.logsumexp(teacher / T, 1)
            z[a:b, :V] = teacher.mul_(0.8).add_(torch.randn((b - a, V), generator=g, device="cuda"))
        s["z"] = z[:, :V]
        short = (rand(M) * 8 * k).clamp_(1, k).floor()  # one row in eight brings fewer logits, padding rows bring none
        short = torch.where(rand(M) < 0.02, 0.0, short)
        ids = torch.where(torch.arange(k, device="cuda") < short[:, None], ids, -1)
        s["ids"] = ids.to(torch.int32 if case["ids"] == "int32" else torch.int64)
        # a mean over rows with the temperature's square; 16-bit gradients of narrow range are scaled up
        scale = T * T * (2048.0 if case["dtype"] == "fp16" else 1.0 / M)
        s["dloss"] = (0.5 + rand(M)) * scale
    else:
        N, K, E = case["N"], case["K"], case["E"]
        s["x"] = randn(M, K, pad=case["pad"])
        blocks = [stored_weight(torch.randn((N, K), generator=g, device="cuda").mul_(K ** -0.5)) for _ in range(max(E, 1))]
        ld = -(-K // 16) * 16                           # rows of 8-bit tensors start at multiples of 16 bytes
        s["w"] = torch.zeros((len(blocks), N, ld), dtype=torch.float8_e4m3fn, device="cuda")
        for e, (q, _) in enumerate(blocks):
            s["w"][e, :, :K] = q
        s["w"] = s["w"][:, :, :K]
        s["w_scales"] = torch.stack([v for _, v in blocks])
        s["offsets"], s["ends"] = None, [M]
        if E:
            share = torch.exp(torch.randn(E, generator=g, device="cuda"))
            chosen = torch.multinomial(share, M, replacement=True, generator=g)
            counts = torch.bincount(chosen, minlength=E)
            s["offsets"] = torch.cat([torch.zeros(1, device="cuda"), counts.cumsum(0)]).to(torch.int32)
            s["ends"] = s["offsets"][1:].tolist()       # the plain form's host copy
        else:
            s["w"], s["w_scales"] = s["w"][0], s["w_scales"][0]
    return s


def stored_weight(w):
    """(8-bit values, scales [N/128][K/128]) of a weight as it is stored"""
    N, K = w.shape
    padded = torch.zeros((-(-N // 128) * 128, -(-K // 128) * 128), device=w.device)
    padded[:N, :K] = w
    tiles = padded.view(padded.shape[0] // 128, 128, -1, 128)
    scale = (tiles.abs().amax((1, 3)) / 448).clamp_min(2.0 ** -126)
    q = (tiles / scale[:, None, :, None]).view_as(padded)[:N, :K]
    return q.to(torch.float8_e4m3fn), scale


# ---------------------------------------------------------------- one pass
def run(s):
    return run_own(s) if own else PLAIN[s["op"]](s)


def run_own(s):
    from paper_1805_01993_b200 import ccdc

    if s["op"] == "experts":
        order = ccdc.expert_sort(s["ids"], s["E"])
        r = {"offsets": order.offsets, "slots": order.slots, "places": order.places,
             "xs": ccdc.expert_dispatch(s["x"], order), "y": ccdc.expert_combine(s["ys"], order, s["w"])}
        if s["way"] == "train":
            r["dys"], r["dw"] = ccdc.expert_combine_backward(s["dy"], s["ys"], order, s["w"])
            r["dx"] = ccdc.expert_dispatch_backward(s["dxs"], order)
        return r
    if s["op"] == "distill":
        how = dict(temperature=s["T"], teacher_lse=s["teacher_lse"])
        if s["way"] == "forward":
            return {"loss": ccdc.distill_forward(s["z"], s["ids"], s["values"], **how)}
        if s["way"] == "step":
            loss, dz = ccdc.distill(s["dloss"], s["z"], s["ids"], s["values"], **how)
        else:
            loss, stats = ccdc.distill_forward(s["z"], s["ids"], s["values"], save=True, **how)
            dz = ccdc.distill_backward(s["dloss"], s["z"], s["ids"], s["values"], stats, **how)
        return {"loss": loss, "dz": dz}
    q, scales = ccdc.quantize_fp8(s["x"])
    return {"scales": scales, "y": ccdc.matmul_fp8(q, scales, s["w"], s["w_scales"], offsets=s["offsets"],
                                                   out_dtype=s["x"].dtype)}


def experts_plain(s):
    t = TYPES[s["dtype"]]
    M, D, k, E = s["M"], s["D"], s["k"], s["E"]
    ids = s["ids"].long().view(-1)
    valid = (ids >= 0) & (ids < E)
    key = torch.where(valid, ids, E)
    order = torch.sort(key, stable=True).indices
    counts = torch.zeros(E + 1, dtype=torch.int64, device="cuda").index_add_(0, key, torch.ones_like(key))
    offsets = torch.cat([torch.zeros_like(counts[:1]), counts[:E].cumsum(0)])
    filled = torch.arange(M * k, device="cuda") < offsets[E]
    slots = torch.where(filled, order, -1)
    places = torch.zeros_like(order)
    places[order] = torch.arange(M * k, device="cuda")
    places = torch.where(valid, places, -1).view(M, k)
    row = torch.where(filled, order // k, 0)
    at = places.clamp_min(0)
    present = (places >= 0)[:, :, None]
    w = s["w"].float()
    xs = torch.where(filled[:, None], s["x"].float()[row], 0.0).to(t)

    def back(rows, weights):
        total = torch.zeros((M, D), device="cuda")
        for j in range(k):
            total += torch.where(present[:, j], rows[at[:, j]].float() * weights[:, j, None], 0.0)
        return total.to(t)

    r = {"offsets": offsets.int(), "slots": slots.int(), "places": places.int(), "xs": xs, "y": back(s["ys"], w)}
    if s["way"] == "train":
        dy = s["dy"].float()
        dys = dy[row] * w.view(-1)[torch.where(filled, order, 0)][:, None]
        r["dys"] = torch.where(filled[:, None], dys, 0.0).to(t)
        dw = [torch.where(present[:, j, 0], (s["ys"][at[:, j]].float() * dy).sum(1), 0.0) for j in range(k)]
        r["dw"] = torch.stack(dw, 1).to(s["w"].dtype)
        r["dx"] = back(s["dxs"], torch.ones_like(w))
    return r


def distill_plain(s):
    T, V = s["T"], s["V"]
    z = s["z"].float() / T
    ids = s["ids"].long()
    valid = (ids >= 0) & (ids < V)
    at = torch.where(valid, ids, 0)
    v = torch.where(valid, s["values"].float() / T, -math.inf)
    if s["teacher_lse"] is None:
        top = v.amax(1, keepdim=True)
        top = torch.where(top > -math.inf, top, 0.0)
        log_t = v - top - torch.log(torch.exp(v - top).sum(1, keepdim=True))
    else:
        log_t = v - s["teacher_lse"][:, None]
    t = torch.where(valid, torch.exp(log_t), 0.0)
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    log_s = z.gather(1, at) - top - torch.log(total)
    r = {"loss": torch.where(t > 0, t * (log_t - log_s), 0.0).sum(1)}
    if s["way"] != "forward":
        c = (s["dloss"] / T)[:, None]
        e *= c * t.sum(1, keepdim=True) / total
        r["dz"] = e.scatter_add_(1, at, -c * t).to(TYPES[s["dtype"]])
    return r


def fp8_plain(s):
    t = TYPES[s["dtype"]]
    M, N, K = s["M"], s["N"], s["K"]
    padded = torch.zeros((M, -(-K // 128) * 128), device="cuda")
    padded[:, :K] = s["x"].float()
    blocks = padded.view(M, -1, 128)
    # the smallest power of two that brings the block to 448 = 1.75 * 2^8 at most
    fraction, exponent = torch.frexp(blocks.abs().amax(2))
    exponent = (exponent - 1 + (fraction > 0.875).int() - 8).clamp_min(-126)
    scales = torch.ldexp(torch.ones_like(fraction), exponent)
    x = ((blocks / scales[:, :, None]).to(torch.float8_e4m3fn).float() * scales[:, :, None]).view(M, -1)[:, :K]
    y = torch.zeros((M, N), dtype=t, device="cuda")
    weights, wide = s["w"].view(-1, N, K) if s["E"] else s["w"][None], s["w_scales"].view(-1, -(-N // 128), -(-K // 128))
    start = 0
    for e, end in enumerate(s["ends"]):
        if end > start:
            scale = wide[e].repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
            y[start:end] = (x[start:end] @ (weights[e].float() * scale).t()).to(t)
        start = end
    return {"scales": scales, "y": y}


PLAIN = {"experts": experts_plain, "distill": distill_plain, "fp8": fp8_plain}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    M = case["M"]
    if case["op"] == "experts":
        D, k = case["D"], case["k"]
        train = case["way"] == "train"
        kept = M * k * (1 - case["drop"])               # rows that are there; the others are written as zeros
        one = M + M * k if case["drop"] == 0 else M + kept
        rows = 2 * M + M * k + kept                     # x in, sorted rows out; sorted rows in, y out
        if train:
            rows += M + kept + M * k + one              # dy and the experts' rows in, dys out; dxs in, dx out
        small = M * k * ((8 if case["ids"] == "int64" else 4) + 8) + M * k * 4 * (2 if train else 1)
        return {"bytes": int(size * D * rows + small), "flops": int(D * kept * (6 if train else 2))}
    if case["op"] == "distill":
        V, k = case["V"], case["k"]
        small = M * (k * ((8 if case["ids"] == "int64" else 4) + size) + 8)
        way = case["way"]
        # logits in; with the gradient also out (a second call has to read them again)
        passes = {"forward": 1, "step": 2, "train": 3}[way]
        return {"bytes": size * M * V * passes + small, "flops": M * V * (4 if way == "forward" else 6)}
    N, K, E = case["N"], case["K"], max(case["E"], 1)
    return {"bytes": size * M * (K + N) + min(E, M) * N * K + 4 * M * -(-K // 128), "flops": 2 * M * N * K}


# ---------------------------------------------------------------- exact values
def exact(case, seed):
    """The same outputs from the definitions in 64 bits, one slot, row block or weight at a time; gradients by automatic
    differentiation where the case is small enough for it, else from the derivative."""
    s = prepare(case, seed)
    return {"experts": exact_experts, "distill": exact_distill, "fp8": exact_fp8}[case["op"]](s)


def exact_experts(s):
    M, D, k, E = s["M"], s["D"], s["k"], s["E"]
    ids = s["ids"].cpu().numpy().astype(np.int64).reshape(-1)
    slots = np.full(M * k, -1, np.int64)
    places = np.full(M * k, -1, np.int64)
    inside = np.flatnonzero((ids >= 0) & (ids < E))
    by_expert = inside[np.argsort(ids[inside], kind="stable")]
    slots[: len(by_expert)] = by_expert
    places[by_expert] = np.arange(len(by_expert))
    offsets = np.searchsorted(ids[by_expert], np.arange(E + 1))
    n = len(by_expert)
    slot = torch.from_numpy(by_expert).cuda()
    token = slot // k
    r = {key: torch.from_numpy(v.astype(np.int32)).cuda() for key, v in
         (("offsets", offsets), ("slots", slots), ("places", places.reshape(M, k)))}
    w = s["w"].double().view(-1)[slot]
    xs = torch.zeros((M * k, D), dtype=torch.float64, device="cuda")
    xs[:n] = s["x"].double()[token]
    r["xs"] = xs
    r["y"] = torch.zeros((M, D), dtype=torch.float64, device="cuda").index_add_(0, token, s["ys"][:n].double() * w[:, None])
    if s["way"] == "train":
        dy = s["dy"].double()[token]
        dys = torch.zeros_like(xs)
        dys[:n] = dy * w[:, None]
        r["dys"] = dys
        dw = torch.zeros(M * k, dtype=torch.float64, device="cuda")
        dw[slot] = (dy * s["ys"][:n].double()).sum(1)
        r["dw"] = dw.view(M, k)
        r["dx"] = torch.zeros((M, D), dtype=torch.float64, device="cuda").index_add_(0, token, s["dxs"][:n].double())
    return r


def exact_distill(s):
    M, V, T = s["M"], s["V"], s["T"]
    losses, grads = [], []
    for a in range(0, M, 256):
        b = min(a + 256, M)
        z = s["z"][a:b].double().requires_grad_(s["way"] != "forward")
        ids = s["ids"][a:b].long()
        valid = (ids >= 0) & (ids < V)
        v = (s["values"][a:b].double() / T).masked_fill(~valid, -math.inf)
        if s["teacher_lse"] is None:
            whole = torch.logsumexp(v, 1, keepdim=True)
            whole = whole.masked_fill(~valid.any(1, keepdim=True), 0.0)
        else:
            whole = s["teacher_lse"][a:b, None].double()
        log_t = (v - whole).masked_fill(~valid, 0.0)
        t = torch.exp(log_t) * valid
        log_s = torch.log_softmax(z / T, 1).gather(1, ids.masked_fill(~valid, 0))
        loss = (t * (log_t - log_s)).sum(1)
        losses.append(loss.detach())
        if s["way"] != "forward":
            grads.append(torch.autograd.grad(loss, z, s["dloss"][a:b].double())[0].to(torch.float64))
    r = {"loss": torch.cat(losses)}
    if grads:
        r["dz"] = torch.cat(grads)
    return r


def exact_fp8(s):
    M, N, K = s["M"], s["N"], s["K"]
    y = torch.zeros((M, N), dtype=torch.float64, device="cuda")
    x = torch.empty((M, K), dtype=torch.float64, device="cuda")
    scales = torch.empty((M, -(-K // 128)), dtype=torch.float64, device="cuda")
    for b in range(scales.shape[1]):
        part = s["x"][:, 128 * b:128 * b + 128].double()
        least = part.abs().amax(1) / 448
        scale = torch.full_like(least, 2.0 ** -126)
        for e in range(-125, 121):                      # powers of two, the first that is large enough
            scale = torch.where(scale < least, torch.full_like(least, 2.0 ** e), scale)
        scales[:, b] = scale
        x[:, 128 * b:128 * b + 128] = nearest_e4m3(part / scale[:, None]) * scale[:, None]
    weights = s["w"] if s["E"] else s["w"][None]
    wide = s["w_scales"] if s["E"] else s["w_scales"][None]
    n, c = torch.arange(N, device="cuda") // 128, torch.arange(K, device="cuda") // 128
    start = 0
    for e, end in enumerate(s["ends"]):
        if end > start:
            y[start:end] = torch.nn.functional.linear(x[start:end], weights[e].double() * wide[e].double()[n][:, c])
        start = end
    return {"scales": scales, "y": y}


def nearest_e4m3(v):
    """The nearest values of four exponent and three mantissa bits (bias 7, largest 448), ties to even."""
    _, exponent = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), (exponent - 1).clamp_min(-6) - 3)
    return (torch.round(v / step) * step).clamp(-448, 448)

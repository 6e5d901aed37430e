"""Cases, plain forms and exact values of the block operators: the gated feed-forward block, the norms
around it with gate, dropout and residual scale, and the dropout itself.

A file of a gradient job is a batch of token rows; its Map runs these operators forward and backward and
leaves parameter gradients, which the shuffle sums.  Rows ("M") are tokens, D the model width, F the
inner width of the feed-forward block.

``own`` chooses between the plain form (elementary torch operations in 32 bits, rounded once) and the
framework's calls.
"""
import math
from functools import reduce

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
LARGEST = 18 * 8192 * 4096 * 16384      # operations of the largest listed case


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one token of a running answer: bound by reading the three weight matrices once
        ffn("ffn_token", "forward", 1, 4096, 16384, "bf16", "silu"),
        # a small serving batch
        ffn("ffn_tokens24", "forward", 24, 2048, 8192, "fp16", "gelu"),
        # a prompt, or an evaluation batch
        ffn("ffn_prompt", "forward", 2048, 4096, 8192, "bf16", "silu"),
        # a file of 512 rows (the row count of the linear-regression Map) through a small block
        ffn("ffn_train_512", "train", 512, 1024, 4096, "bf16", "silu"),
        # the 8/3 * D inner width, odd, and a file of packed sequences that ends anywhere
        ffn("ffn_train_ragged", "train", 777, 1024, 2731, "fp16", "gelu_tanh"),
        # a large file through a large block
        ffn("ffn_train_large", "train", 8192, 4096, 16384, "bf16", "silu"),
        # gradients that have to carry the 32 bits of the shuffle's words
        ffn("ffn_train_fp32", "train", 1024, 1024, 4096, "fp32", "silu"),
        # between two blocks of a running answer: the smallest call
        norm("norm_token", "forward", 1, 4096, "bf16", "rms", "channel", 0.0),
        # odd width and rows, words of 32 bits, a layer norm, one gate for every 250 rows
        norm("norm_train_ragged", "train", 1999, 1001, "fp32", "layer", "group", 0.1, per=250),
        # the training form at the rows of two large files
        norm("norm_train_large", "train", 16384, 4096, "bf16", "rms", "group", 0.1, per=1024),
        # one row
        drop("dropout_row", "forward", 1, 8192, "bf16", 0.1),
        # the gradient-sized buffer: 20 slices of 1.28 M words, forward and backward
        drop("dropout_gradient", "train", 20, 1280000, "fp32", 0.1),
    ]


def ffn(name, way, M, D, F, dtype, act, pad=0):
    return {"name": name, "op": "ffn", "way": way, "M": M, "D": D, "F": F, "dtype": dtype, "act": act, "pad": pad}


def norm(name, way, M, D, dtype, kind, gate, p, per=1, pad=0):
    return {"name": name, "op": "norm", "way": way, "M": M, "D": D, "dtype": dtype, "kind": kind, "gate": gate,
            "per": per, "p": p, "alpha": 0.75, "pad": pad}


def drop(name, way, M, D, dtype, p, pad=0):
    return {"name": name, "op": "dropout", "way": way, "M": M, "D": D, "dtype": dtype, "p": p, "pad": pad}


def draw(rng):
    def size(low, high, step=1):
        v = math.exp(rng.uniform(math.log(low), math.log(high)))
        return min(high, max(low, int(round(v / step)) * step))

    def width(low, high):       # widths are mostly multiples of 64, sometimes of 8, sometimes odd
        kind = rng.random()
        return size(low, high, 64) if kind < 0.6 else size(low, high, 8) if kind < 0.8 else size(low, high) | 1

    op = rng.choice(["ffn", "ffn", "norm", "dropout"])
    way = rng.choice(["forward", "train"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    pad = rng.choice([0, 0, 8, 5])
    if op == "ffn":
        while True:
            M, D, F = size(1, 8192), width(128, 4096), width(128, 16384)
            if 18 * M * D * F <= LARGEST // (4 if dtype == "fp32" else 1):
                break
        # the step in relu's derivative makes 32-bit gradients hang on the last bit of a product: 16-bit types only
        acts = ["silu", "gelu", "gelu_tanh"] + ([] if dtype == "fp32" else ["relu"])
        c = ffn("", way, M, D, F, dtype, rng.choice(acts), pad)
    elif op == "norm":
        M, D = size(1, 16384), width(64, 8192)
        while M * D > 16384 * 4096:
            M = size(1, 16384)
        c = norm("", way, M, D, dtype, rng.choice(["rms", "layer"]), rng.choice(["none", "channel", "group", "row"]),
                 rng.choice([0.0, 0.1, 0.5]), per=size(1, max(1, M)), pad=pad)
        c["per"] = 1 if c["gate"] == "row" else c["per"]
    else:
        M, D = size(1, 16384), width(64, 16384)
        while M * D > 1 << 26:
            M = size(1, 16384)
        c = drop("", way, M, D, dtype, rng.choice([0.05, 0.1, 0.5]), pad)
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 17)
    t = TYPES[case["dtype"]]
    M, D = case["M"], case["D"]

    def randn(rows, cols, std=1.0, mean=0.0, pad=0):
        v = torch.randn((rows, cols + pad), generator=g, device="cuda")
        return v.mul_(std).add_(mean).to(t)[:, :cols]

    s = dict(case)
    s["seed"] = (int(seed) * 7919 + 12345) % (1 << 62)
    if case["op"] == "ffn":
        F = case["F"]
        s["x"] = randn(M, D, pad=case["pad"])               # what a norm hands to the block
        s["w_gate"] = randn(F, D, D ** -0.5)
        s["w_up"] = randn(F, D, D ** -0.5)
        s["w_down"] = randn(D, F, F ** -0.5)
        if case["way"] == "train":
            s["dy"] = randn(M, D, 0.02, pad=case["pad"])
    elif case["op"] == "norm":
        s["x"] = randn(M, D, 2.0, 0.1, pad=case["pad"])     # the residual stream
        s["y"] = randn(M, D, 0.7, pad=case["pad"])          # what the block returned
        s["w_post"] = randn(1, D, 0.1, 1.0).view(D)
        s["w_pre"] = randn(1, D, 0.1, 1.0).view(D)
        s["per"] = M if case["gate"] == "channel" else case["per"]
        s["gate_values"] = None if case["gate"] == "none" else randn(-(-M // s["per"]), D, 0.3, 0.5)
        if case["way"] == "train":
            s["dout"] = randn(M, D, 0.02, pad=case["pad"])
            s["dz"] = randn(M, D, 0.02, pad=case["pad"])
    else:
        s["x"] = randn(M, D, pad=case["pad"])
        if case["way"] == "train":
            s["dy"] = randn(M, D, 0.02, pad=case["pad"])
    return s


# ---------------------------------------------------------------- one pass
EPS = 1e-5


def run(s):
    return run_own(s) if own else PLAIN[s["op"]](s)


def run_own(s):
    from paper_1805_01993_b200 import ccdc

    train = s["way"] == "train"
    if s["op"] == "ffn":
        w = (s["w_gate"], s["w_up"], s["w_down"])
        if not train:
            return {"y": ccdc.ffn_forward(s["x"], *w, act=s["act"])}
        y, saved = ccdc.ffn_forward(s["x"], *w, act=s["act"], save=True)
        dx, dwg, dwu, dwd = ccdc.ffn_backward(s["dy"], s["x"], *w, saved, act=s["act"])
        return {"y": y, "dx": dx, "dw_gate": dwg, "dw_up": dwu, "dw_down": dwd}
    if s["op"] == "norm":
        how = dict(w_post=s["w_post"], w_pre=s["w_pre"], gate=s["gate_values"], rows_per_gate=s["per"],
                   alpha=s["alpha"], p=s["p"], seed=s["seed"], kind=s["kind"], eps=EPS)
        if not train:
            out, z = ccdc.residual_norm_forward(s["x"], s["y"], **how)
            return {"out": out, "z": z}
        out, z, stats = ccdc.residual_norm_forward(s["x"], s["y"], save=True, **how)
        dx, dy, dw_post, dw_pre, dgate = ccdc.residual_norm_backward(s["dout"], s["dz"], s["x"], s["y"], stats, **how)
        return {"out": out, "z": z, "dx": dx, "dy": dy, "dw_post": dw_post, "dw_pre": dw_pre, "dgate": dgate}
    y = ccdc.dropout(s["x"], s["p"], s["seed"])
    return {"y": y, "dx": ccdc.dropout(s["dy"], s["p"], s["seed"])} if train else {"y": y}


def act_plain(h, act):
    """(act(h), act'(h))"""
    if act == "silu":
        s = 1 / (1 + torch.exp(-h))
        return h * s, s * (1 + h * (1 - s))
    if act == "gelu":
        c = 0.5 * (1 + torch.erf(h * math.sqrt(0.5)))
        return h * c, c + h * torch.exp(-0.5 * h * h) * (1 / math.sqrt(2 * math.pi))
    if act == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (h + 0.044715 * h * h * h))
        return 0.5 * h * (1 + t), 0.5 * (1 + t) + 0.5 * h * (1 - t * t) * k * (1 + 3 * 0.044715 * h * h)
    return torch.where(h > 0, h, 0.0), torch.where(h > 0, 1.0, 0.0)


def ffn_plain(s):
    t = TYPES[s["dtype"]]
    x, wg, wu, wd = (s[k].float() for k in ("x", "w_gate", "w_up", "w_down"))
    h, u = x @ wg.t(), x @ wu.t()
    f, df = act_plain(h, s["act"])
    a = f * u
    r = {"y": (a @ wd.t()).to(t)}
    if s["way"] == "train":
        dy = s["dy"].float()
        da = dy @ wd
        dh, du = da * u * df, da * f
        r["dx"] = (dh @ wg + du @ wu).to(t)
        r["dw_gate"], r["dw_up"], r["dw_down"] = (dh.t() @ x).to(t), (du.t() @ x).to(t), (dy.t() @ a).to(t)
    return r


def keep_plain(s, M, D):
    """Dropout factors [M][D]: Philox 4x32 in 10 rounds, key = the seed's two words, counter = element / 8; element e
    takes 16 bits of the 128 and is kept where they are at least round(65536 p)."""
    cut = int(s["p"] * 65536 + 0.5)
    if cut == 0:
        return None
    n = M * D
    c = torch.arange(-(-n // 8), dtype=torch.int64, device="cuda")

    def mul(a, m):      # (high, low) words of a 32-bit product, without leaving 63 bits
        low = (a & 0xFFFF) * m
        mid = (a >> 16) * m + (low >> 16)
        return mid >> 16, ((mid & 0xFFFF) << 16) | (low & 0xFFFF)

    def step(v, i):
        k0 = ((s["seed"] & 0xFFFFFFFF) + i * 0x9E3779B9) & 0xFFFFFFFF
        k1 = ((s["seed"] >> 32) + i * 0xBB67AE85) & 0xFFFFFFFF
        (h0, l0), (h1, l1) = mul(v[0], 0xD2511F53), mul(v[2], 0xCD9E8D57)
        return h1 ^ v[1] ^ k0, l1, h0 ^ v[3] ^ k1, l0

    zero = torch.zeros_like(c)
    v = torch.stack(reduce(step, range(10), (c & 0xFFFFFFFF, c >> 32, zero, zero)), 1)
    bits = torch.stack((v & 0xFFFF, v >> 16), 2).view(-1)[:n].view(M, D)
    return torch.where(bits >= cut, 65536 / (65536 - cut), 0.0)


def unit_plain(v, kind):
    """(the normalised rows, 1 / their deviation)"""
    v = v - v.mean(1, keepdim=True) if kind == "layer" else v
    r = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * r, r


def unit_back_plain(dn, n, r, kind):
    dn = dn - dn.mean(1, keepdim=True) if kind == "layer" else dn
    return r * (dn - n * (dn * n).mean(1, keepdim=True))


def norm_plain(s):
    t = TYPES[s["dtype"]]
    M, D = s["M"], s["D"]
    x, y, w_post, w_pre = (s[k].float() for k in ("x", "y", "w_post", "w_pre"))
    group = torch.arange(M, device="cuda") // s["per"]
    n, r = unit_plain(y, s["kind"])
    q = n * w_post
    gate = s["gate_values"]
    g = None if gate is None else gate.float()[group]
    keep = keep_plain(s, M, D)
    c = 1.0 if keep is None else keep
    cg = c if g is None else c * g
    out = s["alpha"] * x + q * cg
    m, ro = unit_plain(out, s["kind"])
    res = {"out": out.to(t), "z": (m * w_pre).to(t)}
    if s["way"] == "train":
        dout, dz = s["dout"].float(), s["dz"].float()
        res["dw_pre"] = (dz * m).sum(0).to(t)
        d = dout + unit_back_plain(dz * w_pre, m, ro, s["kind"])
        res["dx"] = (s["alpha"] * d).to(t)
        if g is not None:
            res["dgate"] = torch.zeros(gate.shape, device="cuda").index_add_(0, group, d * c * q).to(t)
        else:
            res["dgate"] = None
        dq = d * cg
        res["dw_post"] = (dq * n).sum(0).to(t)
        res["dy"] = unit_back_plain(dq * w_post, n, r, s["kind"]).to(t)
    return res


def dropout_plain(s):
    t = TYPES[s["dtype"]]
    keep = keep_plain(s, s["M"], s["D"])
    r = {"y": (s["x"].float() * keep).to(t)}
    if s["way"] == "train":
        r["dx"] = (s["dy"].float() * keep).to(t)
    return r


PLAIN = {"ffn": ffn_plain, "norm": norm_plain, "dropout": dropout_plain}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    M, D = case["M"], case["D"]
    size = 4 if case["dtype"] == "fp32" else 2
    train = case["way"] == "train"
    if case["op"] == "ffn":
        F = case["F"]
        # forward: x and the weights in, y out; backward: dy and the same in, dx and three gradients out
        return {"bytes": size * (2 * M * D + 3 * D * F + (2 * M * D + 3 * D * F if train else 0)),
                "flops": (18 if train else 6) * M * D * F}
    if case["op"] == "norm":
        gates = {"none": 0, "channel": 1, "group": -(-M // case["per"]), "row": M}[case["gate"]]
        return {"bytes": size * ((8 if train else 4) * M * D + (2 + gates) * D * (2 if train else 1)),
                "flops": (40 if train else 14) * M * D}
    return {"bytes": size * M * D * (4 if train else 2), "flops": M * D * (2 if train else 1)}


# ---------------------------------------------------------------- exact values
def exact(case, seed):
    """The same outputs from the definitions in 64 bits; the gradients by automatic differentiation."""
    s = prepare(case, seed)
    train = case["way"] == "train"
    M, D = case["M"], case["D"]

    def leaf(name):
        return None if s.get(name) is None else s[name].double().requires_grad_(train)

    if case["op"] == "ffn":
        x, wg, wu, wd = (leaf(k) for k in ("x", "w_gate", "w_up", "w_down"))
        h = torch.nn.functional.linear(x, wg)
        f = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu,
             "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[case["act"]](h)
        y = torch.nn.functional.linear(f * torch.nn.functional.linear(x, wu), wd)
        if not train:
            return {"y": y}
        dx, dwg, dwu, dwd = torch.autograd.grad(y, (x, wg, wu, wd), s["dy"].double())
        return {"y": y.detach(), "dx": dx, "dw_gate": dwg, "dw_up": dwu, "dw_down": dwd}
    keep = exact_keep(M, D, case["p"], s["seed"])
    if case["op"] == "dropout":
        r = {"y": s["x"].double() * keep}
        if train:
            r["dx"] = s["dy"].double() * keep
        return r
    x, y, w_post, w_pre, gate = (leaf(k) for k in ("x", "y", "w_post", "w_pre", "gate_values"))

    def unit(v, w):
        if case["kind"] == "layer":
            return torch.nn.functional.layer_norm(v, (D,), w, None, EPS)
        return v / (v.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w

    q = unit(y, w_post) * keep
    if gate is not None:
        q = q * gate.repeat_interleave(s["per"], 0)[:M]
    out = case["alpha"] * x + q
    z = unit(out, w_pre)
    if not train:
        return {"out": out, "z": z}
    wanted = [("dx", x), ("dy", y), ("dw_post", w_post), ("dw_pre", w_pre)] + ([("dgate", gate)] if gate is not None else [])
    grads = torch.autograd.grad((out, z), [v for _, v in wanted], (s["dout"].double(), s["dz"].double()))
    return {"out": out.detach(), "z": z.detach(), "dgate": None, **dict(zip((k for k, _ in wanted), grads))}


def exact_keep(M, D, p, seed):
    """Dropout factors from the generator's definition, in unsigned 64-bit words on the host."""
    cut = int(p * 65536 + 0.5)
    blocks = -(-M * D // 8)
    c0 = np.arange(blocks, dtype=np.uint64)
    c1, c2, c3 = c0 >> np.uint64(32), np.zeros_like(c0), np.zeros_like(c0)
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    c0 = c0 & low
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        a, b = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
        c0, c1, c2, c3 = (b >> half) ^ c1 ^ np.uint64(k0), b & low, (a >> half) ^ c3 ^ np.uint64(k1), a & low
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = np.stack([c0, c1, c2, c3], 1).astype("<u4")
    bits = words.view("<u2").reshape(-1)[: M * D].reshape(M, D)
    kept = torch.from_numpy(bits >= cut).cuda()
    return kept.double() * (65536.0 / (65536 - cut))

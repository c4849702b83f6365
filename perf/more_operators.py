"""The layers in front of a language model's loss, as cases that can be timed and compared.

Three operators: the product of a linear layer with bias, activation and residual in one call, and its gradient; the softmax cross
entropy of a linear head over a large vocabulary, loss alone or with both gradients, whose logits are never kept; dropout from a
counter-based generator with the residual's addition.  Sizes are those of ``kimad_synth``'s GPT-2-shaped and Llama-shaped sets and its
ResNets, or lie around them.

Products take 16-bit operands and sum in 32 bits.  A linear layer's activation is of the sum in 32 bits; the sum that is kept for the
backward pass is rounded to the layer's type, and the gradient reads that.  Dropout: element i of a tensor goes by 16 bits of
Philox 4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011), half i % 2 of word
(i / 2) % 4 of block i / 8, with the seed as key and (block, offset) as counter; it is dropped where they are below round(65536 p).
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
GELU_C = math.sqrt(2.0 / math.pi)        # gelu in its tanh form, z / (1 + exp(-2 c (z + 0.044715 z^3)))


def listed():
    return [
        # serving: one token through the gate projection of the Llama-shaped set; bound by the weights' bytes
        dict(name="linear_token", op="linear", M=1, N=5632, K=2048, type="bf16", out="bf16", act="silu", bias=False, residual=False, keep=False, pad=0),
        # ResNet's thousand classes over an odd width, a ragged batch, everything in the epilogue, logits in 32 bits
        dict(name="linear_odd", op="linear", M=77, N=1000, K=513, type="f16", out="f32", act="relu", bias=True, residual=True, keep=True, pad=3),
        # training: 8192 tokens through the gate projection of the Llama-shaped set, the sum kept for the backward pass
        dict(name="linear_up", op="linear", M=8192, N=5632, K=2048, type="bf16", out="bf16", act="silu", bias=False, residual=False, keep=True, pad=0),
        # training: and back to the residual stream, which it adds to
        dict(name="linear_down", op="linear", M=8192, N=2048, K=5632, type="bf16", out="bf16", act="none", bias=True, residual=True, keep=False, pad=0),
        # a small batch's gradient of a layer without activation, the weights' in the 32 bits that a round compresses
        dict(name="linear_grad_small", op="linear_grad", M=100, N=1000, K=513, type="bf16", dw="f32", act="none", pad=0),
        # training: the gradient of linear_up
        dict(name="linear_grad_up", op="linear_grad", M=8192, N=5632, K=2048, type="bf16", dw="bf16", act="silu", pad=0),
        # scoring one next token under the Llama-shaped head; latency counts
        dict(name="xent_row", op="xent", rows=1, vocab=32000, dim=2048, type="bf16", grad=False, pad=0),
        # evaluation: the loss alone of 8192 tokens over the GPT-2-shaped head
        dict(name="xent_eval", op="xent", rows=8192, vocab=50257, dim=768, type="bf16", grad=False, pad=0),
        # training: loss and both gradients
        dict(name="xent_train", op="xent", rows=8192, vocab=50257, dim=768, type="bf16", grad=True, pad=0),
        # a ragged small batch over odd sizes in fp16 (with a loss scale)
        dict(name="xent_odd", op="xent", rows=333, vocab=32001, dim=513, type="f16", grad=True, pad=1),
        # one token's hidden vector; latency counts
        dict(name="dropout_token", op="dropout", rows=1, cols=768, type="bf16", p=0.1, residual=False, pad=0),
        # training: the residual stream of 8192 tokens of the Llama-shaped set, the branch dropped and added
        dict(name="dropout_batch", op="dropout", rows=8192, cols=5632, type="bf16", p=0.1, residual=True, pad=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["linear", "linear", "linear", "linear_grad", "linear_grad", "xent", "xent", "xent", "dropout", "dropout"])
    kind = rng.choice(["f16", "bf16", "bf16"])
    pad = rng.choice([0, 0, 0, 1, 24])
    while True:
        if op in ("linear", "linear_grad"):
            c = dict(op=op, M=_log(rng, 1, 16384), N=_log(rng, 1, 32000), K=_log(rng, 1, 16384), type=kind, pad=pad)
            if rng.random() < 0.5:       # half of them of sizes that a model would have
                c["N"], c["K"] = max(64, c["N"] // 64 * 64), max(64, c["K"] // 64 * 64)
            if op == "linear":
                c.update(out=rng.choice([kind, kind, "f32"]), act=rng.choice(list(ACTS)), bias=rng.random() < 0.5, residual=rng.random() < 0.5, keep=rng.random() < 0.3)
            else:
                c["act"] = rng.choice(list(ACTS))
                c["dw"] = rng.choice([kind, "f32"]) if c["act"] == "none" else kind
            fits = c["M"] * c["N"] * c["K"] <= 9.4e10 and max(c["M"] * c["N"], c["N"] * c["K"], c["M"] * c["K"]) <= 6e7
        elif op == "xent":
            c = dict(op=op, rows=_log(rng, 1, 8192), vocab=_log(rng, 2, 262144), dim=_log(rng, 8, 4096), type=kind, grad=rng.random() < 0.6, pad=pad)
            if rng.random() < 0.5:
                c["dim"] = max(64, c["dim"] // 64 * 64)
            fits = c["rows"] * c["vocab"] * c["dim"] <= 3.1e11 and c["rows"] * c["vocab"] <= 4.1e8 and c["vocab"] * c["dim"] <= 1.4e8
        else:
            c = dict(op=op, rows=_log(rng, 1, 16384), cols=_log(rng, 1, 32000), type=rng.choice(["f32", "f16", "bf16"]), p=rng.choice([0.05, 0.1, 0.25, 0.5]),
                     residual=rng.random() < 0.5, pad=pad)
            fits = c["rows"] * c["cols"] * BYTES[c["type"]] <= 9.2e7
        if fits:
            return c


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _padded(x, pad):
    """x in a buffer whose rows are `pad` longer; what stands there belongs to somebody else."""
    if not pad:
        return x
    out = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=x.dtype, device=x.device)
    out[:, :x.shape[1]] = x
    return out[:, :x.shape[1]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    s = dict(case)
    kind, pad = TYPES[case["type"]], case["pad"]
    if case["op"] in ("linear", "linear_grad"):
        # activations of a normalised stream, weights that keep their size
        M, N, K = case["M"], case["N"], case["K"]
        s["x"] = _padded(randn(M, K).to(kind), pad)
        s["w"] = _padded((randn(N, K) / math.sqrt(K)).to(kind), pad)
        if case["op"] == "linear":
            s["b"] = (0.1 * randn(N)).to(kind) if case["bias"] else None
            s["r"] = _padded(randn(M, N).to(kind), pad) if case["residual"] else None
        else:
            s["z"] = _padded((s["x"] @ s["w"].t()).to(kind), pad) if case["act"] != "none" else None
            s["dy"] = _padded((0.1 * randn(M, N)).to(kind), pad)
    elif case["op"] == "xent":
        rows, vocab, dim = case["rows"], case["vocab"], case["dim"]
        s["x"] = _padded(randn(rows, dim).to(kind), pad)
        s["w"] = _padded((randn(vocab, dim) * (2.0 / math.sqrt(dim))).to(kind), pad)
        target = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
        # one row in sixteen has no label (padding of the batch); fp16 training scales its loss
        s["target"] = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.0625, -1, target).to(torch.int32) if rows > 1 else target
        s["weight"] = torch.full((rows,), (1024.0 if case["type"] == "f16" else 1.0) / rows, device="cuda")
    else:
        s["x"] = _padded(randn(case["rows"], case["cols"]).to(kind), pad)
        s["r"] = _padded(randn(case["rows"], case["cols"]).to(kind), pad) if case["residual"] else None
        s["seed"], s["offset"] = (seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 63), seed + 7      # (a training step's number, say)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------

def run(state):
    return (_own if own else _plain)[state["op"]](state)


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return z / (1 + torch.exp(-2 * GELU_C * (z + 0.044715 * z * z * z)))
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        g = 1 / (1 + torch.exp(-2 * GELU_C * (z + 0.044715 * z * z * z)))
        return g + z * g * (1 - g) * 2 * GELU_C * (1 + 3 * 0.044715 * z * z)
    g = 1 / (1 + torch.exp(-z))
    return g + z * g * (1 - g)


def _plain_linear(s):
    kind = TYPES[s["type"]]
    z = s["x"].float() @ s["w"].float().t()
    if s["bias"]:
        z = z + s["b"].float()
    y = _act(z, s["act"])
    if s["residual"]:
        y = y + s["r"].float()
    out = {"y": y.to(TYPES[s["out"]])}
    if s["keep"]:
        out["z"] = z.to(kind)
    return out


def _plain_linear_grad(s):
    dz = s["dy"].float()
    if s["act"] != "none":
        dz = dz * _act_slope(s["z"].float(), s["act"])
    return {"dx": (dz @ s["w"].float()).to(TYPES[s["type"]]), "dw": (dz.t() @ s["x"].float()).to(TYPES[s["dw"]]), "db": dz.sum(0)}


def _plain_xent(s):
    x, w = s["x"].float(), s["w"].float()
    t = s["target"].long()
    live = (t >= 0).float()
    weight = s["weight"] * live
    z = x @ w.t()
    top = z.amax(1)
    lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
    out = {"loss": weight * (lse - z.gather(1, t.clamp(min=0)[:, None])[:, 0]), "lse": lse * live}
    if s["grad"]:
        g = torch.exp(z - lse[:, None])
        g.scatter_add_(1, t.clamp(min=0)[:, None], -torch.ones_like(live)[:, None])
        g *= weight[:, None]
        out["dx"], out["dw"] = (g @ w).to(s["x"].dtype), (g.t() @ x).to(s["w"].dtype)
    return out


def _philox(counter, key):
    """Ten rounds on int64 tensors that hold 32-bit numbers; counter: four of them, key: two numbers."""
    low = 0xFFFFFFFF
    c0, c1, c2, c3 = counter
    k0, k1 = key
    for _ in range(10):
        # (products of 32-bit numbers wrap in a signed 64-bit number, with the right bits)
        p, q = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((q >> 32) & low) ^ c1 ^ k0, q & low, ((p >> 32) & low) ^ c3 ^ k1, p & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _plain_dropout(s):
    rows, cols = s["x"].shape
    n, low = rows * cols, 0xFFFFFFFF
    block = torch.arange(-(-n // 8), device="cuda")
    offset = torch.full_like(block, s["offset"])
    words = _philox((block & low, block >> 32, offset & low, offset >> 32), (s["seed"] & low, s["seed"] >> 32))
    halves = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], 1).view(-1)[:n].view(rows, cols)
    border = round(65536 * s["p"])
    y = torch.where(halves >= border, s["x"].float() * (65536.0 / (65536 - border)), 0.0)
    if s["residual"]:
        y = y + s["r"].float()
    return y.to(s["x"].dtype)


_plain = {"linear": _plain_linear, "linear_grad": _plain_linear_grad, "xent": _plain_xent, "dropout": _plain_dropout}


def _own_linear(s):
    import paper_2312_08053_amd as kimad
    y = torch.empty(s["M"], s["N"], dtype=TYPES[s["out"]], device="cuda")
    z = torch.empty(s["M"], s["N"], dtype=s["x"].dtype, device="cuda") if s["keep"] else None
    kimad.kimad_linear(s["x"], s["w"], y, bias=s["b"], residual=s["r"], act=ACTS[s["act"]], z=z)
    return {"y": y, "z": z} if s["keep"] else {"y": y}


def _own_linear_grad(s):
    import paper_2312_08053_amd as kimad
    dx = torch.empty(s["M"], s["K"], dtype=s["x"].dtype, device="cuda")
    dw = torch.empty(s["N"], s["K"], dtype=TYPES[s["dw"]], device="cuda")
    db = torch.empty(s["N"], device="cuda")
    kimad.kimad_linear_grad(s["dy"], s["x"], s["w"], z=s["z"], act=ACTS[s["act"]], dx=dx, dw=dw, db=db)
    return {"dx": dx, "dw": dw, "db": db}


def _own_xent(s):
    import paper_2312_08053_amd as kimad
    out = {"loss": torch.empty(s["rows"], device="cuda"), "lse": torch.empty(s["rows"], device="cuda")}
    if s["grad"]:
        out["dx"] = torch.empty(s["rows"], s["dim"], dtype=s["x"].dtype, device="cuda")
        out["dw"] = torch.empty(s["vocab"], s["dim"], dtype=s["w"].dtype, device="cuda")
    kimad.kimad_linear_xent(s["x"], s["w"], s["target"], row_weight=s["weight"], **out)
    return out


def _own_dropout(s):
    import paper_2312_08053_amd as kimad
    y = torch.empty(s["rows"], s["cols"], dtype=s["x"].dtype, device="cuda")
    kimad.kimad_dropout(s["x"], y, s["p"], s["seed"], offset=s["offset"], residual=s["r"])
    return y


_own = {"linear": _own_linear, "linear_grad": _own_linear_grad, "xent": _own_xent, "dropout": _own_dropout}


# ---- what a pass cannot do without -------------------------------------------------------------------------------------

def work(case):
    if case["op"] == "linear":
        # operands read once, the result (and the kept sum) written once
        M, N, K = case["M"], case["N"], case["K"]
        b = 2 * (M * K + N * K) + M * N * BYTES[case["out"]] + 2 * N * case["bias"] + 2 * M * N * (case["residual"] + case["keep"])
        return {"bytes": b, "flops": 2 * M * N * K}
    if case["op"] == "linear_grad":
        M, N, K = case["M"], case["N"], case["K"]
        b = 2 * M * N * (1 if case["act"] == "none" else 2) + 2 * (M * K + N * K) + 2 * M * K + N * K * BYTES[case["dw"]] + 4 * N
        return {"bytes": b, "flops": 4 * M * N * K}
    if case["op"] == "xent":
        # the logits once; with gradients two more products of the same size
        R, V, D = case["rows"], case["vocab"], case["dim"]
        return {"bytes": 2 * (R + V) * D * (2 if case["grad"] else 1) + 16 * R, "flops": 2 * R * V * D * (3 if case["grad"] else 1)}
    n = case["rows"] * case["cols"]
    return {"bytes": n * BYTES[case["type"]] * (3 if case["residual"] else 2), "flops": 3 * n}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def _sigmoid_of(z, act):
    return torch.sigmoid(z if act == "silu" else math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3))


def _keeps(n, seed, offset, p):
    """Which of n elements stay, on the host: Philox on numpy's unsigned numbers."""
    import numpy as np
    u64 = np.uint64
    mask, half = u64(0xFFFFFFFF), u64(32)
    block = np.arange((n + 7) // 8, dtype=np.uint64)
    ctr = [block & mask, block >> half, np.full_like(block, offset & 0xFFFFFFFF), np.full_like(block, offset >> 32)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for r in range(10):
        a, b = u64(0xD2511F53) * ctr[0], u64(0xCD9E8D57) * ctr[2]
        k = [u64((key[0] + r * 0x9E3779B9) % (1 << 32)), u64((key[1] + r * 0xBB67AE85) % (1 << 32))]
        ctr = [(b >> half) ^ ctr[1] ^ k[0], b & mask, (a >> half) ^ ctr[3] ^ k[1], a & mask]
    random16 = np.stack(ctr, 1).astype("<u4").view("<u2").reshape(-1)[:n]
    return torch.from_numpy(random16 >= int(math.floor(65536 * p + 0.5)))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        z = torch.mm(s["x"].double(), s["w"].double().t().contiguous())
        if case["bias"]:
            z += s["b"].double()
        y = torch.relu(z) if case["act"] == "relu" else z if case["act"] == "none" else z * _sigmoid_of(z, case["act"])
        out = {"y": y + s["r"].double() if case["residual"] else y}
        return {**out, "z": z} if case["keep"] else out
    if case["op"] == "linear_grad":
        dz = s["dy"].double()
        if case["act"] == "relu":
            dz = torch.where(s["z"] > 0, dz, 0.0)
        elif case["act"] != "none":
            z = s["z"].double()
            g = _sigmoid_of(z, case["act"])
            inner = 1.0 if case["act"] == "silu" else math.sqrt(8 / math.pi) * (1 + 0.134145 * z ** 2)
            dz = dz * g * (1 + z * (1 - g) * inner)
        return {"dx": torch.mm(dz, s["w"].double()), "dw": torch.mm(dz.t().contiguous(), s["x"].double()), "db": dz.sum(0)}
    if case["op"] == "xent":
        x, w, t = s["x"].double(), s["w"].double(), s["target"].long()
        log_p = torch.log_softmax(torch.mm(x, w.t().contiguous()), 1)
        there = t >= 0
        weight = torch.where(there, s["weight"].double(), 0.0)
        picked = log_p.gather(1, t.clamp(min=0)[:, None])[:, 0]
        # lse = z - log p at any column
        lse = (x * w[0]).sum(1) - log_p[:, 0]
        out = {"loss": -weight * picked, "lse": torch.where(there, lse, 0.0)}
        if case["grad"]:
            g = torch.exp(log_p)
            g[torch.arange(len(t), device="cuda")[there], t[there]] = torch.expm1(picked[there])
            g *= weight[:, None]
            out["dx"], out["dw"] = torch.mm(g, w), torch.mm(g.t().contiguous(), x)
        return out
    keep = _keeps(case["rows"] * case["cols"], s["seed"], s["offset"], case["p"]).cuda().view(case["rows"], case["cols"])
    kept = 65536 - int(math.floor(65536 * case["p"] + 0.5))
    y = torch.where(keep, s["x"].double() * 65536 / kept, 0.0)
    return y + s["r"].double() if case["residual"] else y

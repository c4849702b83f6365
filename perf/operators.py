"""The operators of a low-bandwidth training round of a language model's head, as cases that can be timed and compared.

Five operators: quantisation to microscaled 4-bit floats (rows, and rows and columns in one call) with its reading back,
the product of two such matrices, the worker's update in 4 bits with error feedback, the server's side of it, and the
distillation loss from a teacher's top logits with its gradient.  Sizes are those of ``kimad_synth``'s GPT-2-shaped and
Llama-shaped sets, its perceptron and ResNets, or lie around them.

The 4-bit format: blocks of 32 along a row share a scale 2^(byte - 127), an element is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6
with a sign.  Four blocks are a word: 64 bytes of codes (two to a byte, the first one low) and one 32-bit word of scale
bytes.  A matrix of R rows has its codes as [R, 64 W] bytes and its scales as [W, R] words, W = ceil(columns / 128), filled up
with zeros.  An update is laid out layer by layer: layer i begins at word floor(layer_start[i] / 128) + i.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
GAMMA = 0.0625                           # the server's step size


def listed():
    return [
        # serving: one token's hidden vector (the Llama-shaped set's width) before a product; latency counts
        dict(name="quantise_token", op="quantise", rows=1, cols=2048, type="bf16", both=False, pad=0),
        # training: the embedding of the GPT-2-shaped set, as the forward product and the gradient's product read it
        dict(name="quantise_embedding", op="quantise", rows=50257, cols=768, type="f32", both=True, pad=0),
        # serving: one token through the Llama-shaped set's head
        dict(name="matmul_token", op="matmul", M=1, N=32000, K=2048, type="bf16"),
        # ResNet's thousand classes over an odd width, a ragged batch
        dict(name="matmul_odd", op="matmul", M=77, N=1000, K=513, type="f32"),
        # training: 8192 tokens through the gate projection of the Llama-shaped set
        dict(name="matmul_tokens", op="matmul", M=8192, N=5632, K=2048, type="bf16"),
        # training: the gradient of the GPT-2-shaped embedding, summed over 8192 tokens
        dict(name="matmul_weight_grad", op="matmul", M=50257, N=768, K=8192, type="f32"),
        # the smallest set of layers: a worker's update and its place in the server's copy and model
        dict(name="update_mlp", op="update", arch="mlp", L=0, d=0, seed=0, shift=0),
        # the headline set
        dict(name="update_gpt2", op="update", arch="gpt2", L=0, d=0, seed=0, shift=0),
        # the server's side of a round of four workers, headline set
        dict(name="server_gpt2_4", op="server", arch="gpt2", L=0, d=0, seed=0, shift=0, workers=4),
        # one row of the Llama-shaped vocabulary in fp32, loss and gradient at once
        dict(name="distill_row", op="distill", mode="both", rows=1, vocab=32000, k=16, type="f32", T=2.0, pad=0),
        # a training batch over the GPT-2-shaped vocabulary (an odd row length: rows are not aligned), loss and gradient at once
        dict(name="distill_batch", op="distill", mode="both", rows=8192, vocab=50257, k=64, type="bf16", T=1.0, pad=0),
        # the gradient behind a forward pass of its own, rows of a padded buffer
        dict(name="distill_backward", op="distill", mode="backward", rows=1000, vocab=32001, k=100, type="f32", T=4.0, pad=31),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantise", "quantise", "matmul", "matmul", "matmul", "update", "server", "distill", "distill", "distill"])
    kind = rng.choice(["f32", "f16", "bf16"])
    while True:
        if op == "quantise":
            c = dict(op=op, rows=_log(rng, 1, 65536), cols=_log(rng, 1, 50257), type=kind, both=rng.random() < 0.5, pad=rng.choice([0, 0, 1, 24]))
            fits = c["rows"] * c["cols"] <= 3.8e7
        elif op == "matmul":
            c = dict(op=op, M=_log(rng, 1, 16384), N=_log(rng, 16, 50257), K=_log(rng, 32, 16384), type=kind)
            fits = c["M"] * c["N"] * c["K"] <= 3.1e11 and c["M"] * c["N"] <= 1.2e8
        elif op in ("update", "server"):
            c = dict(op=op, arch="ragged", L=_log(rng, 1, 400), d=_log(rng, 2000, 120_000_000), seed=rng.randrange(1 << 20),
                     shift=rng.choice([0, 0, 1, 2]))
            fits = c["L"] <= c["d"] // 4
            if op == "server":
                c["workers"] = rng.choice([1, 2, 3, 4, 8, 16])
                fits = fits and c["d"] * (c["workers"] + 1) <= 6e8
        else:
            c = dict(op=op, mode=rng.choice(["both", "both", "forward", "backward"]), rows=_log(rng, 1, 8192), vocab=_log(rng, 100, 262144),
                     k=_log(rng, 1, 256), type=kind, T=rng.choice([0.7, 1.0, 2.0, 4.0]), pad=rng.choice([0, 0, 1, 48]))
            fits = c["rows"] * c["vocab"] <= (2.0e8 if kind == "f32" else 4.0e8) and c["k"] <= c["vocab"]
        if fits:
            return c


def _sizes(case):
    if case["arch"] == "ragged":
        # sizes spread over their logarithm, scaled to the total; odd ones and ones of a few entries among them
        r = random.Random(case["seed"])
        w = [math.exp(r.uniform(0.0, 9.0)) for _ in range(case["L"])]
        return [max(1, int(x * case["d"] / sum(w))) for x in w]
    if case["arch"] == "mlp":
        return [784 * 256, 256, 256 * 128, 128, 128 * 10, 10]
    out = [50257 * 768, 1024 * 768]      # GPT-2-shaped: embeddings, twelve blocks of twelve tensors, the last norm
    for _ in range(12):
        out += [768, 768, 768 * 3 * 768, 3 * 768, 768 * 768, 768, 768, 768, 768 * 4 * 768, 4 * 768, 4 * 768 * 768, 768]
    return out + [768, 768]


# ---- the 4-bit format in elementary operations (32 bits) ---------------------------------------------------------------

def _scale_bytes(amax):
    """The scale byte of blocks with these largest magnitudes: two below the exponent of the largest, 255 for Inf and NaN."""
    e = amax.view(torch.int32) >> 23
    return torch.where(e == 255, e, (e - 2).clamp(min=0))


def _round4(x):
    """x [..., 32] float32 -> (codes int32 [..., 32], scale bytes int32 [...])."""
    byte = _scale_bytes(x.abs().amax(-1))
    inv = ((254 - byte).clamp(min=1) << 23).view(torch.float32)
    y = x.abs() * inv[..., None]
    code = (y > 0.25).int() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)
    return code + 8 * (x < 0).int(), byte


def _values4(codes, byte):
    """The values that codes [..., 32] and scale bytes [...] stand for, float32."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    table = torch.cat([table, -table])
    scale = torch.where(byte == 0, torch.full_like(byte, 0x00400000), byte << 23).view(torch.float32)
    return table[codes] * torch.where(byte == 255, float("nan"), scale)[..., None]


def _blocks(x):
    """Rows of x [R, C] as float32 blocks [R, 4 W, 32], filled up with zeros."""
    rows, cols = x.shape
    words = -(-cols // 128)
    full = torch.zeros(rows, words * 128, dtype=torch.float32, device=x.device)
    full[:, :cols] = x
    return full.view(rows, 4 * words, 32)


def _pack(codes, byte):
    """codes [R, 4 W, 32], bytes [R, 4 W] -> the stored form: uint8 [R, 64 W], int32 [W, R]."""
    rows, blocks = byte.shape
    c = codes.view(rows, blocks * 16, 2)
    b = byte.to(torch.uint8).view(rows, blocks // 4, 4).transpose(0, 1).contiguous()
    return (c[..., 0] | c[..., 1] << 4).to(torch.uint8), b.view(torch.int32).view(blocks // 4, rows)


def _unpack(codes, scales):
    """The stored form -> codes int32 [R, 4 W, 32], bytes int32 [R, 4 W]."""
    words, rows = scales.shape
    c = torch.stack([codes & 15, codes >> 4], -1).int().view(rows, 4 * words, 32)
    return c, scales.view(torch.uint8).view(words, rows, 4).transpose(0, 1).reshape(rows, 4 * words).int()


def _layout(sizes, starts):
    """Where every entry of the layers stands among the words of an update: float positions int64 [d]."""
    at = 128 * (starts[:-1] // 128 + torch.arange(len(sizes), device=starts.device)) - starts[:-1]
    n = starts[1:] - starts[:-1]
    return torch.arange(sum(sizes), device=starts.device) + torch.repeat_interleave(at, n)


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _padded(x, pad):
    """x in a buffer whose rows are `pad` longer."""
    if not pad:
        return x
    out = torch.zeros(x.shape[0], x.shape[1] + pad, dtype=x.dtype, device=x.device)
    out[:, :x.shape[1]] = x
    return out[:, :x.shape[1]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    state = dict(case)
    if case["op"] == "quantise":
        # activations and weights: normal values, columns of different scale (outlier channels)
        x = randn(case["rows"], case["cols"]) * torch.exp(randn(case["cols"]))
        state.update(x=_padded(x.to(TYPES[case["type"]]), case["pad"]))
    elif case["op"] == "matmul":
        # what the quantiser wrote before: activations (columns of different scale) by weights (rows of different scale)
        M, N, K = case["M"], case["N"], case["K"]
        state["a"], state["a_scales"] = _pack(*_round4(_blocks(randn(M, K) * torch.exp(randn(K)))))
        state["b"], state["b_scales"] = _pack(*_round4(_blocks(randn(N, K) * torch.exp(0.5 * randn(N, 1)))))
    elif case["op"] in ("update", "server"):
        sizes = _sizes(case)
        d, L = sum(sizes), len(sizes)
        n = torch.tensor(sizes, device="cuda")
        starts = torch.zeros(L + 1, dtype=torch.int64, device="cuda")
        starts[1:] = torch.cumsum(n, 0)
        words, shift = d // 128 + L, case["shift"]
        scale = torch.repeat_interleave(10.0 ** (-5.0 + 3.0 * torch.rand(L, generator=gen, device="cuda")), n)
        state.update(sizes=sizes, starts=starts, words=words, d=d)

        def flat(factor):                # the layers back to back, `shift` elements into their allocation
            out = torch.empty(d + shift, device="cuda")[shift:]
            return out.copy_(randn(d) * scale * factor)

        state["x"] = torch.empty(d + shift, device="cuda")[shift:].copy_(0.02 * randn(d))
        if case["op"] == "update":
            # a round in the middle of training: the estimator is halfway, the server's copy equals the worker's
            state.update(g=flat(1.0), h=flat(0.5))
            state["hat"] = torch.empty(d + shift, device="cuda")[shift:].copy_(state["h"])
            state.update(codes=torch.empty(words, 64, dtype=torch.uint8, device="cuda"), scales=torch.empty(words, dtype=torch.int32, device="cuda"))
        else:
            # what the workers sent, and the server's copies of their estimators
            M = case["workers"]
            at = _layout(sizes, starts)
            state["codes"] = torch.empty(M, words, 64, dtype=torch.uint8, device="cuda")
            state["scales"] = torch.empty(M, words, dtype=torch.int32, device="cuda")
            pitch = d + (-d) % 4         # the copies lie in one allocation, each on a 16-byte border of its own (and shifted)
            state["hats"] = torch.empty(M, pitch + 4, device="cuda")[:, shift:shift + d]
            for m in range(M):
                full = torch.zeros(words * 128, device="cuda")
                full[at] = randn(d) * scale
                codes, packed = _pack(*_round4(full.view(words, 4, 32)))
                state["codes"][m], state["scales"][m] = codes, packed[0]
                state["hats"][m] = randn(d) * scale
            state["weights"] = [(1.0 + m) / (M * (M + 1) / 2) for m in range(M)]
    else:
        rows, vocab, k = case["rows"], case["vocab"], case["k"]
        z = 3.0 * randn(rows, vocab)
        teacher = z + 2.0 * randn(rows, vocab)
        val, idx = teacher.topk(k, dim=1)
        idx = idx.to(torch.int32)
        # one row in eight has fewer entries than k, one in sixteen does not count (padding of the batch)
        count = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.125, torch.randint(0, k + 1, (rows,), generator=gen, device="cuda"), k)
        idx = torch.where(torch.arange(k, device="cuda") < count[:, None], idx, -1)
        weight = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.0625, 0.0, 1.0 / rows)
        state.update(z=_padded(z.to(TYPES[case["type"]]), case["pad"]), idx=idx.contiguous(), val=val.contiguous(), weight=weight)
        if case["mode"] == "backward":
            zf = state["z"].float()
            top = zf.amax(1)
            state["stats"] = torch.stack([top, torch.exp((zf - top[:, None]) / case["T"]).sum(1)], 1).contiguous()
    return state


# ---- one pass ----------------------------------------------------------------------------------------------------------

def run(state):
    return (_own if own else _plain)[state["op"]](state)


def _plain_quantise(s):
    def back(x):
        codes, byte = _round4(_blocks(x))
        return _values4(codes, byte).view(x.shape[0], -1)[:, :x.shape[1]].to(torch.bfloat16)
    x = s["x"]
    return {"rows": back(x), "columns": back(x.t())} if s["both"] else {"rows": back(x)}


def _plain_matmul(s):
    a, b = (_values4(*_unpack(s[n], s[n + "_scales"])).view(s[n].shape[0], -1) for n in ("a", "b"))
    return (a @ b.t()).to(TYPES[s["type"]])


def _plain_update(s):
    at = _layout(s["sizes"], s["starts"])
    full = torch.zeros(s["words"] * 128, device="cuda")
    full[at] = s["g"] - s["h"]
    codes, byte = _round4(full.view(s["words"], 4, 32))
    sent = _values4(codes, byte).view(-1)[at]
    s["h"] += sent
    s["hat"] += sent
    s["x"] -= GAMMA * s["hat"]
    return {"h": s["h"], "hat": s["hat"], "x": s["x"]}


def _plain_server(s):
    at = _layout(s["sizes"], s["starts"])
    M, words = s["scales"].shape
    codes, byte = _unpack(s["codes"].view(M * words, 64), s["scales"].view(1, M * words))
    s["hats"] += _values4(codes, byte).view(M, words * 128)[:, at]
    s["x"] -= GAMMA * (torch.tensor(s["weights"], device="cuda")[:, None] * s["hats"]).sum(0)
    return {"hats": s["hats"], "x": s["x"]}


def _plain_distill(s):
    T, z, idx = s["T"], s["z"].float(), s["idx"].long()
    there = idx >= 0
    t = torch.where(there, s["val"], -math.inf) / T
    p = torch.exp(t - t.amax(1, keepdim=True).clamp(min=-3e38))
    p = p / p.sum(1, keepdim=True).clamp(min=1e-30)              # (a row without entries: zeros)
    live = (there.any(1) & (s["weight"] != 0)).float()[:, None]
    weight = s["weight"][:, None] * live
    out = {}
    if s["mode"] == "backward":
        top, total = s["stats"][:, :1], s["stats"][:, 1:]
    else:
        top = z.amax(1, keepdim=True)
        total = torch.exp((z - top) / T).sum(1, keepdim=True)
        log_q = (z.gather(1, idx.clamp(min=0)) - top) / T - torch.log(total)
        log_p = torch.log(torch.where(p > 0, p, 1.0))
        out["loss"] = (weight * T * T * (p * (log_p - log_q)).sum(1, keepdim=True)).view(-1)
        out["stats"] = torch.where(live > 0, torch.cat([top, total], 1), 0.0)   # (rows that do not count are not read)
    if s["mode"] != "forward":
        q = torch.exp((z - top) / T) / total
        out["grad"] = (weight * T * q.scatter_add(1, idx.clamp(min=0), -p)).to(s["z"].dtype)
    return out


_plain = {"quantise": _plain_quantise, "matmul": _plain_matmul, "update": _plain_update, "server": _plain_server, "distill": _plain_distill}


def _own_quantise(s):
    import paper_2312_08053_amd as kimad
    x = s["x"]
    rows, cols = x.shape
    codes, scales = kimad.mx4_empty(rows, cols, x.device)
    codes_t, scales_t = kimad.mx4_empty(cols, rows, x.device) if s["both"] else (None, None)
    kimad.kimad_mx4_quantise(x, codes, scales, codes_t, scales_t)
    out = {"rows": torch.empty(rows, cols, dtype=torch.bfloat16, device=x.device)}
    kimad.kimad_mx4_dequantise(codes, scales, out["rows"])
    if s["both"]:
        out["columns"] = torch.empty(cols, rows, dtype=torch.bfloat16, device=x.device)
        kimad.kimad_mx4_dequantise(codes_t, scales_t, out["columns"])
    return out


def _own_matmul(s):
    import paper_2312_08053_amd as kimad
    out = torch.empty(s["M"], s["N"], dtype=TYPES[s["type"]], device="cuda")
    kimad.kimad_mx4_matmul(s["a"], s["a_scales"], s["b"], s["b_scales"], s["K"], out)
    return out


def _own_update(s):
    import paper_2312_08053_amd as kimad
    kimad.kimad_mx4_compress_ef(s["g"], s["h"], s["starts"], s["codes"], s["scales"])
    kimad.kimad_mx4_server_apply([(s["codes"], s["scales"])], [s["hat"]], [1.0], s["starts"], s["d"], s["x"], GAMMA)
    return {"h": s["h"], "hat": s["hat"], "x": s["x"]}


def _own_server(s):
    import paper_2312_08053_amd as kimad
    kimad.kimad_mx4_server_apply(list(zip(s["codes"], s["scales"])), list(s["hats"]), s["weights"], s["starts"], s["d"], s["x"], GAMMA)
    return {"hats": s["hats"], "x": s["x"]}


def _own_distill(s):
    import paper_2312_08053_amd as kimad
    z, rows = s["z"], s["rows"]
    out = {}
    if s["mode"] != "forward":
        out["grad"] = torch.empty(rows, s["vocab"], dtype=z.dtype, device=z.device)
    if s["mode"] == "backward":
        kimad.kimad_distill_grad(z, s["idx"], s["val"], s["T"], s["stats"], out["grad"], row_weight=s["weight"])
        return out
    out["loss"] = torch.empty(rows, device=z.device)
    out["stats"] = torch.empty(rows, 2, device=z.device)
    kimad.kimad_distill(z, s["idx"], s["val"], s["T"], out["loss"], stats=out["stats"], grad=out.get("grad"), row_weight=s["weight"])
    return out


_own = {"quantise": _own_quantise, "matmul": _own_matmul, "update": _own_update, "server": _own_server, "distill": _own_distill}


# ---- what a pass cannot do without -------------------------------------------------------------------------------------

def work(case):
    four = 4.25 / 8                      # bytes of an entry in 4 bits with its share of the scale
    if case["op"] == "quantise":
        # read once; per orientation written in 4 bits, read back and written in bfloat16
        n = case["rows"] * case["cols"]
        return {"bytes": n * (BYTES[case["type"]] + (2 if case["both"] else 1) * (2 * four + 2)), "flops": n * 4}
    if case["op"] == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": (M + N) * K * four + M * N * BYTES[case["type"]], "flops": 2 * M * N * K}
    if case["op"] == "update":
        # worker: g and h read, h and the update written; server: the update and its copy read, copy written, model read and written
        return {"bytes": sum(_sizes(case)) * (12 + four + four + 8 + 8), "flops": 8 * sum(_sizes(case))}
    if case["op"] == "server":
        return {"bytes": sum(_sizes(case)) * (case["workers"] * (8 + four) + 8), "flops": sum(_sizes(case)) * (4 * case["workers"] + 2)}
    n, small = case["rows"] * case["vocab"], case["rows"] * (8 * case["k"] + 16)
    return {"bytes": n * BYTES[case["type"]] * (1 if case["mode"] == "forward" else 2) + small, "flops": 6 * n}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def _power(n):
    """2^n in float64 for whole n, exactly (pow() may be off in the last place, which would decide ties)."""
    return (n.to(torch.int64) + 1023 << 52).view(torch.float64)


def _nearest(x):
    """The 4-bit values nearest to x [..., 32] (float64): halves, wholes and twos by magnitude, ties to the even multiple."""
    top = x.abs().amax(-1, keepdim=True)
    unit = _power(torch.where(top > 0, torch.frexp(top)[1] - 3, -127).clamp(min=-127))
    y = x / unit
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0)).double()
    return (torch.round(y / step) * step).clamp(-6, 6) * unit


def _nearest_rows(x):
    out = torch.zeros(x.shape[0], x.shape[1] + (-x.shape[1]) % 32, dtype=torch.float64, device=x.device)
    out[:, :x.shape[1]] = x
    return _nearest(out.view(x.shape[0], -1, 32)).view(x.shape[0], -1)[:, :x.shape[1]]


def _stored(codes, scales):
    """What a stored matrix stands for, float64: sign, exponent and mantissa bit of every code, times its block's scale."""
    words, rows = scales.shape
    c = torch.empty(rows, codes.shape[1], 2, dtype=torch.float64, device=codes.device)
    for half in (0, 1):
        n = (codes >> (4 * half)) & 15
        exponent, mantissa = ((n >> 1) & 3).double(), (n & 1).double()
        size = torch.where(exponent == 0, mantissa / 2, (1 + mantissa / 2) * _power(exponent - 1))
        c[..., half] = torch.where(n > 7, -size, size)
    at = torch.stack([(scales >> (8 * b)) & 255 for b in range(4)], -1)          # [W, R, 4]
    return c.view(rows, words, 4, 32) * _power(at.permute(1, 0, 2) - 127)[..., None]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantise":
        x = s["x"].double()
        return {"rows": _nearest_rows(x), "columns": _nearest_rows(x.t())} if case["both"] else {"rows": _nearest_rows(x)}
    if case["op"] == "matmul":
        a, b = (_stored(s[n], s[n + "_scales"]).view(s[n].shape[0], -1) for n in ("a", "b"))
        return a @ b.t()
    if case["op"] in ("update", "server"):
        bounds = [0]
        for n in s["sizes"]:
            bounds.append(bounds[-1] + n)
        pairs = list(zip(bounds[:-1], bounds[1:]))
        if case["op"] == "update":
            # (the operand and the sum are single 32-bit operations by definition)
            x = (s["g"] - s["h"]).double()
            sent = torch.cat([_nearest_rows(x[None, lo:hi])[0] for lo, hi in pairs])
            h, hat = (s["h"].double() + sent).float().double(), (s["hat"].double() + sent).float().double()
            return {"h": h, "hat": hat, "x": s["x"].double() - GAMMA * hat}
        hats, x = [], s["x"].double()
        for m, w in enumerate(s["weights"]):
            words = _stored(s["codes"][m], s["scales"][m][None]).reshape(-1)
            sent = torch.cat([words[128 * (lo // 128 + i):][:hi - lo] for i, (lo, hi) in enumerate(pairs)])
            hats.append((s["hats"][m].double() + sent).float().double())
            x = x - GAMMA * w * hats[-1]
        return {"hats": torch.stack(hats), "x": x}
    T, z, w = case["T"], s["z"].double() / case["T"], s["weight"].double()
    there = s["idx"] >= 0
    live = there.any(1) & (w != 0)
    p = torch.softmax(torch.where(there, s["val"].double() / T, -math.inf), 1).nan_to_num(0.0)
    lse = torch.logsumexp(z, 1, keepdim=True)
    out = {}
    if case["mode"] != "backward":
        log_q = z.gather(1, s["idx"].clamp(min=0).long()) - lse
        cross = torch.where(p > 0, p * (torch.log(p) - log_q), 0.0).sum(1)
        top = s["z"].double().amax(1)
        out["loss"] = torch.where(live, w * T * T * cross, 0.0)
        out["stats"] = torch.where(live[:, None], torch.stack([top, torch.exp(lse[:, 0] - top / T)], 1), 0.0)
    if case["mode"] != "forward":
        grad = torch.exp(z - lse)
        grad.scatter_add_(1, s["idx"].clamp(min=0).long(), -p)
        out["grad"] = torch.where(live[:, None], (w * T)[:, None] * grad, 0.0)
    return out

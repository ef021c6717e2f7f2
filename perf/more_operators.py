"""What the operators of language models in 8-bit floating point are measured on.

A case is a dict of plain values; `prepare` makes what a program holds before the call, `run` is one pass.  The format that all
share: codes e4m3 (torch.float8_e4m3fn, largest 448), one binary32 scale per 128 consecutive elements of a row of activations
(scales [ceil(K / 128)][rows]) and per block of 128 x 128 weights (scales [ceil(N / 128)][ceil(K / 128)]); a value is code * scale.
The kinds:

  quantize  rows as codes and scales:  v = x, or, gated, v = g / (1 + exp(-g)) * u with x = [g | u];
            s = max(max|v| over a row's block / 448, 2^-80), code = e4m3(v / s), nearest even
  norm      h = x, or x + residual rounded to x's type (returned then);  y = h / sqrt(mean h^2 + eps) * weight, as codes and
            scales of y; where asked for, y itself too
  matmul    y[m][n] = bias[n] + sum_k x[m][k] * w[n][k]
  moe       a layer of experts for a few tokens: the top_k largest of a token's logits choose its experts (ties: the lowest index),
            softmax over all logits weighs them, normalised again over the chosen;
            y[t] = sum_e weight[t][e] * down[e] (silu(gate[e] x[t]) * (up[e] x[t])), with gate and up as the halves of one array of rows

Codes come back as float8 tensors, their scales beside them: each is compared by its own type.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
BLOCK = 128
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# --------------------------------------------------------------------------- the cases

def listed():
    return [
        # one token between two layers: the smallest call, latency counts
        dict(name="norm_1x4096", kind="norm", M=1, K=4096, residual=True, with_y=False, type="bf16"),
        # rows that divide nothing, the first norm of a model (nothing to add)
        dict(name="norm_777x5003", kind="norm", M=777, K=5003, residual=False, with_y=True, type="f16"),
        # the prompts of a batch: memory bound
        dict(name="norm_16384x8192", kind="norm", M=16384, K=8192, residual=True, with_y=False, type="bf16"),
        # a decoding batch between the two products of a gated layer
        dict(name="gate_24x14336", kind="quantize", M=24, K=14336, gated=True, type="bf16"),
        # attention's output of a batch of prompts, before its projection; sizes that divide nothing
        dict(name="quantize_9001x4100", kind="quantize", M=9001, K=4100, gated=False, type="f16"),
        # one token through a square projection: the smallest product
        dict(name="matmul_1x4096x4096", kind="matmul", M=1, N=4096, K=4096, bias=False, type="bf16"),
        # a decoding batch through a wide projection: weight streaming
        dict(name="matmul_24x28672x8192", kind="matmul", M=24, N=28672, K=8192, bias=False, type="bf16"),
        # a short prompt, sizes that divide nothing, a bias, results in 32 bits
        dict(name="matmul_1021x1001x1027", kind="matmul", M=1021, N=1001, K=1027, bias=True, type="f32"),
        # a batch of prompts through a square projection: bound by the matrix units
        dict(name="matmul_8192x8192x8192", kind="matmul", M=8192, N=8192, K=8192, bias=False, type="bf16"),
        # one token through a layer of many experts: the weights of eight
        dict(name="moe_1_of_64x4096x1536", kind="moe", T=1, E=64, top_k=8, H=4096, I=1536, type="bf16"),
        # a few requests over few, odd experts
        dict(name="moe_5_of_10x2000x720", kind="moe", T=5, E=10, top_k=2, H=2000, I=720, type="f16"),
        # a decoding batch that reaches every expert
        dict(name="moe_64_of_64x4096x2048", kind="moe", T=64, E=64, top_k=6, H=4096, I=2048, type="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Whole blocks, whole pieces of 16 or any number."""
    to = rng.choice([128, 128, 16, 1])
    return max(to, _log(rng, lo, hi) // to * to)


def draw(rng):
    kind = rng.choice(["norm", "quantize", "matmul", "matmul", "moe", "moe"])
    if kind == "norm":
        M, K = _log(rng, 1, 16384), _size(rng, 64, 16384)
        while M * K > 16384 * 8192:
            M = M // 2
        residual = rng.random() < 0.6
        return dict(kind=kind, M=M, K=K, residual=residual, with_y=not residual and rng.random() < 0.5, type=rng.choice(["bf16", "f16"]))
    if kind == "quantize":
        M, K = _log(rng, 1, 16384), _size(rng, 64, 28672)
        while M * K > 9001 * 8192:
            M = M // 2
        return dict(kind=kind, M=M, K=K, gated=rng.random() < 0.5, type=rng.choice(["bf16", "f16"]))
    if kind == "matmul":
        M, K, N = _log(rng, 1, 8192), _size(rng, 64, 16384), _size(rng, 64, 28672)
        while M * N * K > 8192 ** 3 or N * K > 28672 * 8192:
            N = max(64, N // 2)
        return dict(kind=kind, M=M, N=N, K=K, bias=rng.random() < 0.3, type=rng.choice(["bf16", "bf16", "f16", "f32"]))
    T, E = _log(rng, 1, 64), rng.choice([4, 8, 16, 32, 64, 128])
    H, I = 16 * _log(rng, 16, 448), 16 * _log(rng, 8, 256)
    while E * H * I > 64 * 4096 * 2048:
        I = max(16, I // 32 * 16)
    return dict(kind=kind, T=T, E=E, top_k=rng.choice([1, 2, 4] if E < 8 else [1, 2, 4, 6, 8] if E < 64 else [2, 4, 6]), H=H, I=I, type=rng.choice(["bf16", "f16"]))


# --------------------------------------------------------------------------- what a program holds

def _blocks(n):
    return -(-n // BLOCK)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device=DEV, generator=g)  # noqa: E731
    uniform = lambda lo, hi, *shape: lo + (hi - lo) * torch.rand(*shape, device=DEV, generator=g)  # noqa: E731
    typ, s = TYPES[case["type"]], dict(case)

    def codes(*shape):  # as quantizing normal values leaves them: the largest of 128 is near 448
        c = torch.empty(*shape, dtype=torch.float8_e4m3fn, device=DEV)
        step = max(1, (1 << 27) // c[0].numel())
        for i in range(0, shape[0], step):
            c[i:i + step] = (normal(min(step, shape[0] - i), *shape[1:]) * 150.0).clamp_(-448, 448).to(torch.float8_e4m3fn)
        return c

    if case["kind"] in ("norm", "quantize"):
        M, K = case["M"], case["K"]
        if case["kind"] == "norm":
            # channels of different size, as the stream of activations between layers has
            s["x"] = (normal(M, K) * torch.exp(0.7 * normal(1, K))).to(typ)
            s["r"] = (3.0 * normal(M, K) * torch.exp(0.7 * normal(1, K))).to(typ) if case["residual"] else None
            s["g"] = uniform(0.5, 1.5, K).to(typ)
        else:
            s["x"] = (normal(M, K * (2 if case["gated"] else 1)) * 1.5).to(typ)
        return s
    s["typ"] = typ
    if case["kind"] == "matmul":
        M, N, K = (case[k] for k in ("M", "N", "K"))
        s["x"], s["xs"] = codes(M, K), uniform(0.5, 1.5, _blocks(K), M) / 150.0
        s["w"], s["ws"] = codes(N, K), uniform(0.5, 1.5, _blocks(N), _blocks(K)) * (0.02 / 150.0)
        s["b"] = normal(N).to(typ) if case["bias"] else None
        return s
    T, E, H, I = (case[k] for k in ("T", "E", "H", "I"))
    s["x"], s["xs"] = codes(T, H), uniform(0.5, 1.5, _blocks(H), T) / 150.0
    s["logits"] = normal(T, E)
    s["up"], s["ups"] = codes(E, 2 * I, H), uniform(0.5, 1.5, E, _blocks(2 * I), _blocks(H)) / (150.0 * math.sqrt(H))
    s["down"], s["downs"] = codes(E, H, I), uniform(0.5, 1.5, E, _blocks(H), _blocks(I)) / (150.0 * math.sqrt(I))
    return s


def run(s):
    if own:
        import paper_1806_08342_amd as qnn

        if s["kind"] == "quantize":
            return qnn.f8_quantize(s["x"], gated=s["gated"])
        if s["kind"] == "norm":
            return qnn.f8_rmsnorm(s["x"], s["g"], eps=EPS, residual=s["r"], with_y=s["with_y"])
        if s["kind"] == "matmul":
            return qnn.f8_matmul(s["x"], s["xs"], s["w"], s["ws"], bias=s["b"], dtype=s["typ"])
        return qnn.f8_moe(s["x"], s["xs"], s["logits"], s["up"], s["ups"], s["down"], s["downs"], s["top_k"], dtype=s["typ"])
    if s["kind"] == "quantize":
        return _plain_quantize(s)
    if s["kind"] == "norm":
        return _plain_norm(s)
    if s["kind"] == "matmul":
        return _plain_matmul(s)
    return _plain_moe(s)


# --------------------------------------------------------------------------- the plain forms

def _plain_codes(v):
    """(codes, scales) of rows in 32 bits."""
    M, K = v.shape
    v = torch.nn.functional.pad(v, (0, -K % BLOCK)).view(M, -1, BLOCK)
    size = torch.where(torch.isfinite(v), v.abs(), 0.0).amax(2, keepdim=True)
    scale = (size / 448.0).clamp(min=2.0 ** -80)
    c = (v / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return c.view(M, -1)[:, :K].contiguous(), scale[:, :, 0].t().contiguous()


def _plain_quantize(s):
    x = s["x"].float()
    if s["gated"]:
        gate, up = x[:, :s["K"]], x[:, s["K"]:]
        x = gate / (1.0 + torch.exp(-gate)) * up
    return _plain_codes(x)


def _plain_norm(s):
    h = s["x"] if s["r"] is None else (s["x"].float() + s["r"].float()).to(s["x"].dtype)
    v = h.float()
    y = v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS) * s["g"].float()
    return _plain_codes(y) + (() if s["r"] is None else (h,)) + ((y.to(h.dtype),) if s["with_y"] else ())


def _plain_weights(codes, scales):
    """[..., N, K] codes and [..., N / 128, K / 128] scales as values."""
    n, k = codes.shape[-2:]
    return codes.float() * scales.repeat_interleave(BLOCK, -2)[..., :n, :].repeat_interleave(BLOCK, -1)[..., :k]


def _plain_rows(codes, scales):
    return codes.float() * scales.t().repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]


def _plain_matmul(s):
    y = _plain_rows(s["x"], s["xs"]) @ _plain_weights(s["w"], s["ws"]).t()
    return (y if s["b"] is None else y + s["b"].float()).to(s["typ"])


def _plain_moe(s):
    x, k, I, T, E = _plain_rows(s["x"], s["xs"]), s["top_k"], s["I"], s["T"], s["E"]
    p = torch.exp(s["logits"].float() - s["logits"].float().amax(1, keepdim=True))
    order = torch.argsort(s["logits"].float(), dim=1, descending=True, stable=True)[:, :k]
    weight = torch.gather(p / p.sum(1, keepdim=True), 1, order)
    weight = weight / weight.sum(1, keepdim=True)
    if T * k < E:  # the weights of each choice
        at = order.flatten()
        x = x.repeat_interleave(k, 0)[:, :, None]
        h = _plain_weights(s["up"][at], s["ups"][at]) @ x
        h = h[:, :I] / (1.0 + torch.exp(-h[:, :I])) * h[:, I:]
        y = (_plain_weights(s["down"][at], s["downs"][at]) @ h).view(T, k, -1)
        y = (y * weight[:, :, None]).sum(1)
    else:  # all experts, for all tokens
        h = _plain_weights(s["up"], s["ups"]) @ x.t()[None]
        h = h[:, :I] / (1.0 + torch.exp(-h[:, :I])) * h[:, I:]
        y = _plain_weights(s["down"], s["downs"]) @ h
        share = torch.zeros(T, E, device=x.device).scatter_(1, order, weight)
        y = (y * share.t()[:, None, :]).sum(0).t()
    return y.to(s["typ"]).contiguous()


# --------------------------------------------------------------------------- the work, and 64 bits

def work(case):
    if case["kind"] in ("norm", "quantize"):
        M, K = case["M"], case["K"]
        each = 2 * (2 if case.get("gated") else 1) + 1 + (4 if case.get("residual") else 0) + (2 if case.get("with_y") else 0)
        return {"bytes": M * K * each + 4 * M * _blocks(K) + (2 * K if case["kind"] == "norm" else 0), "flops": 6 * M * K}
    out = 4 if case["type"] == "f32" else 2
    if case["kind"] == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": N * K + M * K + 4 * _blocks(K) * (M + _blocks(N)) + out * M * N + (out * N if case["bias"] else 0), "flops": 2 * M * N * K}
    T, E, k, H, I = (case[n] for n in ("T", "E", "top_k", "H", "I"))
    reached = E * (1.0 - (1.0 - k / E) ** T)  # experts that some token chooses, on the average
    return {"bytes": int(reached * 3 * H * I) + T * (H + 4 * _blocks(H) + 4 * E + out * H), "flops": 6 * T * k * H * I}


def _nearest_e4m3(v):
    """Nearest value that e4m3 has, ties to an even last bit: three bits after the first, steps of 2^-9 below 2^-6."""
    _, e = torch.frexp(v.abs().clamp(max=448.0))
    step = torch.exp2(torch.clamp(e - 1, min=-6).double() - 3.0)
    return torch.round(v / step).mul(step).clamp(-448.0, 448.0)


def _exact_codes(v):
    codes, scales = torch.empty_like(v), []
    for b in range(0, v.shape[1], BLOCK):
        part = v[:, b:b + BLOCK]
        s = torch.maximum(part.abs().max(1).values / 448.0, torch.tensor(2.0 ** -80, dtype=torch.float64, device=DEV))
        codes[:, b:b + BLOCK] = _nearest_e4m3(part / s[:, None])
        scales.append(s)
    return codes, torch.stack(scales)


def _exact_product(x, xs, w, ws):
    y = torch.zeros(x.shape[0], w.shape[0], dtype=torch.float64, device=DEV)
    for b in range(xs.shape[0]):
        part = x[:, b * BLOCK:(b + 1) * BLOCK].double() @ w[:, b * BLOCK:(b + 1) * BLOCK].double().t()
        of_rows = torch.repeat_interleave(ws[:, b].double(), BLOCK)[:w.shape[0]]
        y += part.mul_(xs[b].double()[:, None]).mul_(of_rows[None, :])
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "quantize":
        x = s["x"].double()
        return _exact_codes(torch.nn.functional.silu(x[:, :case["K"]]).mul_(x[:, case["K"]:]) if case["gated"] else x)
    if case["kind"] == "norm":
        h = s["x"] if s["r"] is None else (s["x"].double() + s["r"].double()).to(s["x"].dtype)  # (that rounding is the operator's)
        y = h.double()
        y = y / torch.sqrt(y.pow(2).sum(1, keepdim=True) / case["K"] + EPS) * s["g"].double()
        return _exact_codes(y) + (() if s["r"] is None else (h.double(),)) + ((y,) if case["with_y"] else ())
    if case["kind"] == "matmul":
        y = _exact_product(s["x"], s["xs"], s["w"], s["ws"])
        return y if s["b"] is None else y + s["b"].double()
    T, k, I = case["T"], case["top_k"], case["I"]
    y = torch.zeros(T, case["H"], dtype=torch.float64, device=DEV)
    logits = s["logits"].double().tolist()
    chosen = [sorted(range(case["E"]), key=lambda e: (-row[e], e))[:k] for row in logits]
    for e in sorted({e for c in chosen for e in c}):
        rows = [t for t in range(T) if e in chosen[t]]
        share = [1.0 / sum(math.exp(logits[t][o] - logits[t][e]) for o in chosen[t]) for t in rows]
        h = _exact_product(s["x"][rows], s["xs"][:, rows], s["up"][e], s["ups"][e])
        h = h[:, :I] * torch.sigmoid(h[:, :I]) * h[:, I:]
        w = s["down"][e].double() * s["downs"][e].double().repeat_interleave(BLOCK, 0)[:case["H"]].repeat_interleave(BLOCK, 1)[:, :I]
        y[rows] += (h @ w.t()) * torch.tensor(share, dtype=torch.float64, device=DEV)[:, None]
    return y

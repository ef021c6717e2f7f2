"""The operators of language models in 8-bit floating point in 64 bits, on the CPU, from their definitions, with what their rounding errors
scale with."""
import math

import torch

DEV = "cuda:0"
BLOCK = 128
F8 = torch.float8_e4m3fn
# The matrix unit on 8-bit codes aligns the products of 8 consecutive k to the largest and cuts each off below 2^-LOST_AT of it.
LOST_AT = 13


def blocks(n):
    return -(-n // BLOCK)


def wide(scales, n, dim):
    return scales.cpu().double().repeat_interleave(BLOCK, dim).narrow(dim, 0, n)


def values(codes, scales):
    """Rows [M,K] with scales [K/128,M]."""
    return codes.cpu().double() * wide(scales, codes.shape[1], 0).t()


def weights(codes, scales):
    return codes.cpu().double() * wide(wide(scales, codes.shape[-2], -2), codes.shape[-1], -1)


def step(v):
    """Distance of neighbouring values of e4m3 around v."""
    _, e = torch.frexp(v.abs().clamp(max=448.0))
    return torch.exp2((e - 1).clamp(min=-6).double() - 3)


def encode(v):
    """(codes, scales) of float32 rows as the definition has them, in binary32."""
    M, K = v.shape
    v = torch.nn.functional.pad(v, (0, -K % BLOCK)).view(M, -1, BLOCK)
    peak = torch.where(torch.isfinite(v), v.abs(), 0.0).amax(2, keepdim=True)
    scale = (peak / 448.0).clamp(min=2.0 ** -80)
    most = torch.maximum(peak, torch.tensor(448.0 * 2.0 ** -80))
    c = torch.where(v.isnan(), v, torch.minimum(torch.maximum(v, -most), most)) / scale
    return c.to(F8).view(M, -1)[:, :K], scale[:, :, 0].t()


def assert_codes(codes, scales, v, rel, what=""):
    """Codes and scales of values that are v up to a relative error of `rel`: the scale too, and a code is nearest to a
    quotient that is off by as much."""
    codes, scales = codes.cpu().double(), scales.cpu().double()
    M, K = v.shape
    want = torch.nn.functional.pad(v, (0, -K % BLOCK)).view(M, -1, BLOCK).abs().amax(2).t() / 448.0
    want = want.clamp(min=2.0 ** -80)
    assert codes.shape == v.shape and scales.shape == want.shape, what
    assert ((scales - want).abs() <= rel * want).all(), (what, ((scales - want).abs() / want).max())
    q = v / wide(scales, K, 0).t()
    off = (codes - q).abs() - (step(q) / 2 + 2 * rel * q.abs())
    assert (off <= 0).all(), (what, int((off > 0).sum()), off.max())


def product(x, xs, w, ws, narrow=True):
    """(y, its error's bound before it is rounded): x [M,K] and w [N,K] codes."""
    M, K = x.shape
    a, b, xs, ws = x.cpu().double(), w.cpu().double(), xs.cpu().double(), ws.cpu().double()
    y, off, size = (torch.zeros(M, w.shape[0]).double() for _ in range(3))
    for i in range(blocks(K)):
        p, q = a[:, i * BLOCK:(i + 1) * BLOCK], b[:, i * BLOCK:(i + 1) * BLOCK]
        scale = (xs[i][:, None] * wide(ws[:, i], w.shape[0], 0)[None]).abs()
        y += (p @ q.t()) * (xs[i][:, None] * wide(ws[:, i], w.shape[0], 0)[None])
        size += (p.abs() @ q.abs().t()) * scale
        if narrow:
            u, v = (torch.nn.functional.pad(t.abs(), (0, -t.shape[1] % 8)) for t in (p, q))
            largest = torch.stack([(row[None] * v).view(v.shape[0], -1, 8).amax(2).sum(1) for row in u]) if M else size
            off += 8 * largest * 2.0 ** -LOST_AT * scale
    # binary32: products of scales, one multiply-add per block, up to 128 additions in a block, the joining of up to 64 parts
    return y, off + size * (blocks(K) + 128 + 64 + 2) * 2.0 ** -24


def half_ulp(dtype):
    return {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}[dtype]


def choose(logits, k, renormalize=True):
    """[[(expert, weight)]] for each token."""
    got = []
    for row in logits.cpu().double().tolist():
        row = [min(v, 3.4028234663852886e38) if v == v else -math.inf for v in row]
        best = [e for e in sorted(range(len(row)), key=lambda e: (-row[e], e)) if row[e] > -math.inf][:k]
        of = best if renormalize else [e for e in range(len(row)) if row[e] > -math.inf]
        total = sum(math.exp(row[e] - row[best[0]]) for e in of) if best else 1.0
        got.append([(e, math.exp(row[e] - row[best[0]]) / total) for e in best])
    return got


def moe(x, xs, logits, up, ups, down, downs, k, renormalize=True):
    """(y, its error's bound before it is rounded)"""
    T, H = x.shape
    I = down.shape[2]
    y, off = torch.zeros(T, H).double(), torch.zeros(T, H).double()
    chosen = choose(logits, k, renormalize)
    for e in sorted({e for c in chosen for e, _ in c}):
        rows = [t for t in range(T) if any(e == o for o, _ in chosen[t])]
        share = torch.tensor([dict(chosen[t])[e] for t in rows]).double()[:, None]
        p, bad = product(x.cpu()[rows], xs.cpu()[:, rows], up[e].cpu(), ups[e].cpu())
        gate, lift = p[:, :I], p[:, I:]
        silu = gate * torch.sigmoid(gate)
        h = silu * lift
        # silu's slope is below 1.1, and it is below 1.1 times its argument; rounding of exp, quotient, products; two parts of 8 bits
        h_off = 1.1 * bad[:, :I] * (lift.abs() + bad[:, I:]) + silu.abs() * bad[:, I:] + h.abs() * (2.0 ** -16 + 16 * 2.0 ** -24) + 2.0 ** -126
        w = weights(down[e], downs[e])
        y[rows] += (h @ w.t()) * share
        size = (h.abs() + h_off) @ w.abs().t()
        off[rows] += share * (h_off @ w.abs().t() + size * (I + 64 + 16) * 2.0 ** -24)
    return y, off


def random_codes(g, *shape, size=150.0):
    return (torch.randn(*shape, generator=g) * size).clamp(-448, 448).to(F8)


def assert_close(got, want, allowed, what=""):
    got, off = got.cpu().double(), (got.cpu().double() - want).abs()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~(off <= allowed)
    if bad.any():
        i = int((off - allowed).nan_to_num(nan=math.inf).flatten().argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off; worst at {i}: {got.flatten()[i]} for {want.flatten()[i]}, allowed {allowed.flatten()[i]}")

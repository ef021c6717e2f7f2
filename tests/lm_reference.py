"""The operators of quantized language models in 64 bits, on the CPU, from their definitions; and inputs for their tests."""
import math

import torch

DEV = "cuda:0"


def unpack(codes):
    """uint8 [N,K/2] -> float64 [N,K], element 2j in the low nibble, two's complement."""
    c = codes.cpu().to(torch.int64)
    c = torch.stack((c % 16, c // 16), -1).flatten(1)
    return torch.where(c > 7, c - 16, c).double()


def w4(x, codes, scales, group, zeros=None, bias=None):
    """(y, what its rounding errors scale with: sum |x| (136 + |z|) s per output)"""
    x, c = x.cpu().double(), unpack(codes)
    at = torch.arange(c.shape[1]) // group
    s = scales.cpu().double()[at].t()
    z = zeros.cpu().double()[at].t() if zeros is not None else torch.zeros_like(c)
    y = x @ ((c - z) * s).t()
    if bias is not None:
        y = y + bias.cpu().double()
    return y, x.abs() @ ((136 + z.abs()) * s.abs()).t()


def round_away(x):
    return torch.sign(x) * torch.floor(x.abs() + 0.5)


def append(cache, k, v, cu, start, table):
    """The cache's four tensors (float32 scales, as the definition has them) after the call, on the CPU."""
    kc, ks, vc, vs = (t.cpu().clone() for t in cache)
    pages, heads, block, _ = kc.shape
    for r in range(table.shape[0]):
        a, b, at = int(cu[r]), int(cu[r + 1]), int(start[r])
        for j in range(at // block, -(-(at + b - a) // block) if b > a else 0):
            if j >= table.shape[1] or not 0 <= int(table[r, j]) < pages:
                continue
            p, lo, hi = int(table[r, j]), max(at, j * block) - j * block, min(at + b - a, (j + 1) * block) - j * block
            rows = slice(a + j * block + lo - at, a + j * block + hi - at)
            for x, codes, scale in ((k, kc[p], ks[p]), (v, vc[p].transpose(1, 2), vs[p])):
                x = x[rows].cpu().float().transpose(0, 1)  # [head][token][dim]
                peak = torch.where(torch.isfinite(x), x.abs(), 0.0).amax((1, 2))
                before = scale.clone() if lo else torch.zeros_like(scale)
                after = torch.maximum(before, peak / 127.0)
                by = torch.where(after > 0, after, 1.0)[:, None, None]
                held = codes[:, :lo].float()
                codes[:, :lo] = torch.where((after > before)[:, None, None], round_away((held * (before[:, None, None] / by)).double()).clamp(-127, 127), held.double()).to(torch.int8)
                q = torch.where(torch.isnan(x), 0.0, x / by)
                codes[:, lo:hi] = round_away(q.double()).clamp(-127, 127).to(torch.int8)
                scale.copy_(after)
    return kc, ks, vc, vs


def attend(cache, q, cu, lengths, table, scale=None, window=0):
    """(out, lse, sum of p |v| per output) in 64 bits"""
    kc, ks, vc, vs = (t.cpu().double() for t in cache)
    pages, heads, block, dim = kc.shape
    T, q_heads, _ = q.shape
    q, scale = q.cpu().double(), dim ** -0.5 if scale is None else scale
    out, spread, lse = torch.zeros(T, q_heads, dim).double(), torch.zeros(T, q_heads, dim).double(), torch.full((T, q_heads), -math.inf).double()
    for r in range(table.shape[0]):
        a, b, n_all = int(cu[r]), int(cu[r + 1]), int(lengths[r])
        if b <= a or n_all <= 0:
            continue
        page = table[r, :-(-n_all // block)].cpu().long()
        there = ((page >= 0) & (page < pages)).repeat_interleave(block)[:n_all]
        page = page.clamp(0, pages - 1)
        k = (kc[page] * ks[page][..., None, None]).permute(1, 0, 2, 3).reshape(heads, -1, dim)[:, :n_all]
        v = (vc[page] * vs[page][..., None, None]).permute(1, 0, 3, 2).reshape(heads, -1, dim)[:, :n_all]
        v = torch.where(there[:, None], v, 0.0)
        at, t = torch.arange(n_all - (b - a), n_all)[:, None], torch.arange(n_all)[None]
        sees = (t <= at) & there[None]
        if window:
            sees &= t > at - window
        for e in range(q_heads):
            h = e // (q_heads // heads)
            s = (q[a:b, e] @ k[h].t() * scale).masked_fill(~sees, -math.inf)
            lse[a:b, e] = torch.logsumexp(s, 1)
            p = torch.where(sees.any(1, keepdim=True), torch.softmax(s, 1), 0.0)
            out[a:b, e], spread[a:b, e] = p @ v[h], p @ v[h].abs()
    return out, lse, spread


def half_ulp(dtype):
    """Largest relative error of rounding to the type once: 2^-p for p significant bits."""
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11


def case(requests, heads, dim, block, dtype, seed, spare=2, q_heads=None, shuffle=True):
    """A filled cache for requests [(tokens in it, queries)], with garbage in the pages' unused places and no page in unused
    entries of the table."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // block) for n, _ in requests]
    pages = sum(need) + spare
    order = (torch.randperm(pages, generator=g) if shuffle else torch.arange(pages)).int()
    table = torch.full((len(requests), max(1, max(need))), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    codes = lambda *s: torch.randint(-127, 128, s, generator=g).to(torch.int8)  # noqa: E731
    cache = (codes(pages, heads, block, dim), 0.02 * torch.rand(pages, heads, generator=g) + 0.005, codes(pages, heads, dim, block),
             0.02 * torch.rand(pages, heads, generator=g) + 0.005)
    cu = torch.tensor([0] + [n for _, n in requests]).cumsum(0).int()
    q = torch.randn(int(cu[-1]), q_heads or heads, dim, generator=g).to(dtype)
    lengths = torch.tensor([n for n, _ in requests], dtype=torch.int32)
    return [t.to(DEV) for t in cache], q.to(DEV), cu.to(DEV), lengths.to(DEV), table.to(DEV)


def assert_close(got, want, allowed, what=""):
    got, off = got.cpu().double(), (got.cpu().double() - want).abs()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~(off <= allowed)
    if bad.any():
        i = int((off - allowed).nan_to_num(nan=math.inf).flatten().argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off; worst at {i}: {got.flatten()[i]} for {want.flatten()[i]}, allowed {allowed.flatten()[i]}")

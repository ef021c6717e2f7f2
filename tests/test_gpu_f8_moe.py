"""A layer of experts for a few tokens, against 64 bits."""
import math

import pytest
import torch

import f8_reference as ref
import paper_1806_08342_amd as qnn

pytestmark = pytest.mark.gpu
DEV = ref.DEV


def layer(T, E, H, I, seed=0):
    g = torch.Generator().manual_seed(seed + T + 11 * E + 101 * H + 1009 * I)
    spread = lambda *s: torch.exp(0.5 * torch.randn(*s, generator=g))  # noqa: E731
    return dict(x=ref.random_codes(g, T, H), xs=spread(ref.blocks(H), T) / 150, logits=torch.randn(T, E, generator=g), up=ref.random_codes(g, E, 2 * I, H),
                ups=spread(E, ref.blocks(2 * I), ref.blocks(H)) / (150 * H ** 0.5), down=ref.random_codes(g, E, H, I),
                downs=spread(E, ref.blocks(H), ref.blocks(I)) / (150 * I ** 0.5))


def on_gpu(c):
    return [c[n].to(DEV) for n in ("x", "xs", "logits", "up", "ups", "down", "downs")]


def check(c, k, got, dtype=torch.bfloat16, renormalize=True, what=""):
    want, off = ref.moe(*(c[n] for n in ("x", "xs", "logits", "up", "ups", "down", "downs")), k, renormalize)
    # (weights: exp, sums over the experts and a quotient)
    ref.assert_close(got, want, (1 + 2.0 ** -8) * off + (want.abs() + off) * (ref.half_ulp(dtype) + c["logits"].shape[1] * 2.0 ** -23) + torch.finfo(dtype).smallest_normal, what)


def check_choice(c, k, experts, weights, renormalize=True):
    for row, e, w in zip(ref.choose(c["logits"], k, renormalize), experts.cpu().tolist(), weights.cpu().tolist()):
        assert e == [o for o, _ in row] + [-1] * (k - len(row))
        assert all(abs(a - b) <= (16 + c["logits"].shape[1]) * 2.0 ** -24 for a, b in zip(w, [o for _, o in row] + [0.0] * (k - len(row)))), (w, row)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,E,k,H,I", [(1, 1, 1, 16, 16), (1, 4, 2, 128, 128), (1, 64, 8, 256, 384), (2, 3, 3, 48, 80), (5, 10, 2, 400, 144), (7, 100, 6, 272, 64), (16, 8, 2, 128, 272),
                                       (17, 8, 2, 144, 160), (33, 5, 1, 256, 128), (64, 4, 4, 128, 144), (65, 16, 3, 160, 96), (130, 6, 2, 64, 48)])
def test_sizes(T, E, k, H, I, dtype):
    c = layer(T, E, H, I)
    y, experts, weights = qnn.f8_moe(*on_gpu(c), k, dtype=dtype, with_choice=True)
    assert y.dtype == dtype
    check_choice(c, k, experts, weights)
    check(c, k, y, dtype, what=(T, E, k, H, I))
    assert torch.equal(qnn.f8_moe(*on_gpu(c), k, dtype=dtype), y)


@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
def test_types_of_logits_and_both_normalisations(kind, renormalize):
    c = layer(9, 70, 128, 64)
    c["logits"] = (3 * c["logits"]).to(kind)
    y, experts, weights = qnn.f8_moe(*on_gpu(c), 5, renormalize=renormalize, with_choice=True)
    check_choice(c, 5, experts, weights, renormalize)
    check(c, 5, y, renormalize=renormalize)


@pytest.mark.parametrize("E", [6, 64, 65, 1000])
def test_logits_that_are_equal_infinite_or_nan(E):
    k = 4
    c = layer(10, E, 64, 32)
    n = c["logits"]
    n[0] = 0.25
    n[1] = -math.inf
    n[2] = math.nan
    n[3] = -math.inf
    n[3, E - 2] = -5.0
    n[4, E - 1], n[4, 1] = math.inf, math.inf
    n[5] = torch.where(torch.arange(E) % 2 == 0, 0.0, -0.0)
    n[6] = torch.where(torch.arange(E) < 3, n[6], -math.inf)
    n[7] = torch.linspace(-3e38, 3e38, E)
    n[8] = torch.where(torch.arange(E) == 2, math.nan, n[8])
    for renormalize in (True, False):
        y, experts, weights = qnn.f8_moe(*on_gpu(c), k, renormalize=renormalize, with_choice=True)
        check_choice(c, k, experts, weights, renormalize)
        check(c, k, y, renormalize=renormalize)
        assert (y[1:3] == 0).all()


def test_experts_that_nobody_chose_are_not_read():
    c = layer(6, 12, 160, 96)
    c["logits"][:, 7] = -math.inf
    want = qnn.f8_moe(*on_gpu(c), 3)
    for name in ("up", "down"):
        c[name].view(torch.uint8)[7] = 0x7f
    assert torch.equal(qnn.f8_moe(*on_gpu(c), 3), want)
    # and a NaN in a chosen one reaches its tokens only
    c["up"].view(torch.uint8)[2, 5, 9] = 0x7f
    hit = (c["logits"].argsort(1, descending=True)[:, :3] == 2).any(1)
    got = qnn.f8_moe(*on_gpu(c), 3).cpu()
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], want.cpu()[~hit])


def test_all_tokens_to_one_expert():
    c = layer(64, 40, 272, 144)
    c["logits"][:, 31] = 50.0
    y = qnn.f8_moe(*on_gpu(c), 2)
    check(c, 2, y)


def test_spaced_rows_and_what_lies_between_them():
    T, E, H, I = 19, 9, 144, 80
    c = layer(T, E, H, I)
    x = torch.full((T, H + 21), 0x7f, dtype=torch.uint8, device=DEV)
    x[:, 7:7 + H] = c["x"].view(torch.uint8).to(DEV)
    xs = torch.full((ref.blocks(H), T + 4), math.nan, device=DEV)
    xs[:, 1:1 + T] = c["xs"].to(DEV)
    logits = torch.full((T, E + 3), math.inf, device=DEV)
    logits[:, 2:2 + E] = c["logits"].to(DEV)
    out = torch.full((T + 1, H + 5), 3.0, dtype=torch.bfloat16, device=DEV)
    a = on_gpu(c)
    y = qnn.f8_moe(x.view(ref.F8)[:, 7:7 + H], xs[:, 1:1 + T], logits[:, 2:2 + E], *a[3:], 3, out=out[:T, 2:2 + H])
    check(c, 3, y)
    rest = out.clone()
    rest[:T, 2:2 + H] = 3.0
    assert (rest == 3.0).all()


def test_no_tokens():
    c = layer(0, 4, 128, 64)
    y, experts, weights = qnn.f8_moe(*on_gpu(c), 2, with_choice=True)
    assert y.shape == (0, 128) and experts.shape == weights.shape == (0, 2)


@pytest.mark.parametrize("T", [1, 8, 40, 70])
def test_captured_and_replayed_with_other_tokens(T):
    c = layer(T, 16, 256, 128)
    a = on_gpu(c)
    qnn.f8_moe(*a, 4)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = qnn.f8_moe(*a, 4)
    for seed in range(3):
        other = layer(T, 16, 256, 128, seed + 1)
        a[0].view(torch.uint8).copy_(other["x"].view(torch.uint8))
        a[2].copy_(other["logits"])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, qnn.f8_moe(*a, 4))
        check({**c, "x": other["x"], "logits": other["logits"]}, 4, y)


def test_two_streams_at_once():
    cases = [layer(5, 12, 256, 128, s) for s in range(2)]
    args = [on_gpu(c) for c in cases]
    want = [qnn.f8_moe(*a, 3) for a in args]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in args], [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(qnn.f8_moe(*args[i], 3))
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for ys, w in zip(got, want) for y in ys)


def test_as_dense_layers_of_the_chosen_experts():
    # the same from the products of rows, expert by expert: h in 16 bits there, codes in between
    c = layer(4, 3, 256, 256)
    a = on_gpu(c)
    y = qnn.f8_moe(*a, 1, with_choice=True)
    for t in range(4):
        e = int(y[1][t, 0])
        both = qnn.f8_matmul(a[0][t:t + 1], a[1][:, t:t + 1], a[3][e], a[4][e])
        h, hs = qnn.f8_quantize(both, gated=True)
        dense = qnn.f8_matmul(h, hs, a[5][e], a[6][e])
        assert (dense.float() - y[0][t:t + 1].float()).norm() < 0.06 * y[0][t:t + 1].float().norm()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,E,k", [(3, 5, 1), (8, 70, 2), (12, 10, 2), (40, 6, 1), (64, 150, 4)])
def test_inner_values_up_to_the_end_of_binary32(T, E, k, dtype):
    # Gates of 2^64 (silu is exactly that) times ups of around 2^64.  bfloat16, whose two parts hold an inner value, rounds to infinity from 2^128 (1 - 2^-9) on:
    # that number, the one before it, one behind, binary32's largest, and one far from all of them.
    H = I = 128
    ups = [2.0 ** 64 * v for v in (1 - 2.0 ** -9, 1 - 2.0 ** -9 - 2.0 ** -24, 1 - 2.0 ** -10, 1 - 2.0 ** -24, 0.71875)]
    g = torch.Generator().manual_seed(T)
    sign = torch.where(torch.arange(I) % 3 == 1, -1.0, 1.0)
    one = torch.arange(E) % len(ups)
    c = layer(T, E, H, I)
    x, up, down = torch.randn(T, H, generator=g), torch.zeros(E, 2 * I, H), torch.zeros(E, H, I)
    x[:, 0], up[:, :I, 0], up[:, I:, 0] = 1.0, 1.0, sign
    n = torch.arange(H)
    down[:, n, n] = torch.where(n % 2 == 0, 1.0, 0.5)  # (whose sums with inner values stay within binary32)
    down[:, n[n % 2 == 1], (n[n % 2 == 1] + 5) % I] = -0.25
    c.update(x=x.to(ref.F8), xs=torch.ones(1, T), up=up.to(ref.F8), down=down.to(ref.F8), downs=torch.full((E, 1, 1), 2.0 ** -120))
    c["ups"] = torch.stack([torch.full((E,), 2.0 ** 64), torch.tensor(ups)[one]], 1)[:, :, None].contiguous()
    chosen = torch.arange(T) * 7 % E
    c["logits"] = torch.where(torch.arange(E)[None] == chosen[:, None], 0.5, -math.inf)
    y = qnn.f8_moe(*on_gpu(c), k, dtype=dtype)
    h = 2.0 ** 64 * torch.tensor(ups).double()[one[chosen]][:, None] * sign.double()
    w = down[0].double() * 2.0 ** -120
    want, size = h @ w.t(), h.abs() @ w.abs().t()
    # two parts of 8 bits, of which the second may be cut off rather than rounded, and a few roundings of binary32
    off = size * (2.0 ** -16 + 8 * 2.0 ** -24)
    ref.assert_close(y, want, off + (want.abs() + off) * ref.half_ulp(dtype), (T, E, k))

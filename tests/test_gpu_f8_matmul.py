"""Products of e4m3 rows and weights with a scale per 128 of a row and per 128 x 128 weights, against 64 bits."""
import math

import pytest
import torch

import f8_reference as ref
import paper_1806_08342_amd as qnn

pytestmark = pytest.mark.gpu
DEV = ref.DEV
KINDS = [torch.bfloat16, torch.float16, torch.float32]


def operands(M, N, K, seed=0, spread=1.0):
    g = torch.Generator().manual_seed(seed + M + 7 * N + 31 * K)
    scale = lambda *s: torch.exp(spread * torch.randn(*s, generator=g)) / 150  # noqa: E731
    return ref.random_codes(g, M, K), scale(ref.blocks(K), M), ref.random_codes(g, N, K), scale(ref.blocks(N), ref.blocks(K)), torch.randn(N, generator=g)


def check(x, xs, w, ws, bias, dtype, y, what):
    want, off = ref.product(x, xs, w, ws, narrow=dtype != torch.float32)
    if bias is not None:
        want = want + bias.to(dtype).double()
    ref.assert_close(y, want, (1 + 2.0 ** -8) * off + (want.abs() + off) * (ref.half_ulp(dtype) + 2.0 ** -24) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps, what)


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 5, 15), (2, 16, 16), (3, 17, 31), (1, 128, 128), (5, 130, 129), (16, 64, 256), (17, 257, 384), (1, 300, 4096), (33, 100, 1000),
                                   (64, 129, 640), (65, 128, 128), (100, 200, 1027), (130, 500, 2048), (257, 259, 513), (300, 1001, 272), (520, 384, 896)])
def test_sizes(M, N, K, dtype):
    x, xs, w, ws, b = operands(M, N, K)
    bias = b if (M + N) % 2 else None
    y = qnn.f8_matmul(x.to(DEV), xs.to(DEV), w.to(DEV), ws.to(DEV), bias=None if bias is None else bias.to(dtype).to(DEV), dtype=dtype)
    assert y.dtype == dtype
    check(x, xs, w, ws, bias, dtype, y, (M, N, K))


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("M,N,K", [(1, 256, 512), (40, 300, 300), (300, 300, 700)])
def test_whole_numbers_are_exact(M, N, K, dtype):
    # -1, 0 and 1 with scales of 1 and 2: neither the matrix unit nor binary32 rounds their sums
    g = torch.Generator().manual_seed(K)
    x, w = (torch.randint(-1, 2, s, generator=g).float().to(ref.F8) for s in ((M, K), (N, K)))
    xs, ws = (2.0 ** torch.randint(0, 2, s, generator=g) for s in ((ref.blocks(K), M), (ref.blocks(N), ref.blocks(K))))
    y = qnn.f8_matmul(x.to(DEV), xs.to(DEV), w.to(DEV), ws.to(DEV), dtype=dtype)
    want = ref.values(x, xs) @ ref.weights(w, ws).t()
    assert torch.equal(y.cpu(), want.float().to(dtype))


@pytest.mark.parametrize("dtype", KINDS)
def test_scales_far_apart(dtype):
    # (their products within the normal numbers of binary32)
    for M, N, K in ((3, 200, 1024), (150, 200, 1024)):
        x, xs, w, ws, _ = operands(M, N, K, spread=8.0)
        if dtype == torch.float16:
            xs, ws = xs.clamp(2.0 ** -30, 2.0 ** -9), ws.clamp(2.0 ** -30, 2.0 ** -9)
        y = qnn.f8_matmul(x.to(DEV), xs.to(DEV), w.to(DEV), ws.to(DEV), dtype=dtype)
        check(x, xs, w, ws, None, dtype, y, (M, N, K))


@pytest.mark.parametrize("M", [1, 20, 200])
def test_nan_codes_stay_in_their_rows_and_columns(M):
    N, K = 150, 300
    x, xs, w, ws, _ = operands(M, N, K)
    clean = qnn.f8_matmul(x.to(DEV), xs.to(DEV), w.to(DEV), ws.to(DEV)).cpu()
    x.view(torch.uint8)[M // 2, 299] = 0x7f
    w.view(torch.uint8)[149, 3] = 0xff
    y = qnn.f8_matmul(x.to(DEV), xs.to(DEV), w.to(DEV), ws.to(DEV)).cpu()
    bad = torch.zeros(M, N, dtype=torch.bool)
    bad[M // 2], bad[:, 149] = True, True
    assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], clean[~bad])


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("M,N,K", [(3, 70, 200), (40, 130, 144), (200, 260, 272), (300, 300, 1001)])
def test_spaced_rows_at_any_byte_and_what_lies_between_them(M, N, K, dtype):
    x, xs, w, ws, _ = operands(M, N, K)
    wide = torch.full((M + 2, K + 45), 0x7f, dtype=torch.uint8, device=DEV)  # NaN all around
    wide[1:1 + M, 13:13 + K] = x.view(torch.uint8).to(DEV)
    scales = torch.full((ref.blocks(K) + 2, M + 3), math.nan, device=DEV)
    scales[1:-1, 2:2 + M] = xs.to(DEV)
    near = torch.full((N * K + 64,), 0x7f, dtype=torch.uint8, device=DEV)
    near[17:17 + N * K] = w.view(torch.uint8).flatten().to(DEV)
    out = torch.full((M + 2, N + 9), 3.0, dtype=dtype, device=DEV)
    y = out[1:1 + M, 5:5 + N]
    back = qnn.f8_matmul(wide.view(ref.F8)[1:1 + M, 13:13 + K], scales[1:-1, 2:2 + M], near[17:17 + N * K].view(N, K).view(ref.F8), ws.to(DEV), dtype=dtype, out=y)
    assert back is y
    check(x, xs, w, ws, None, dtype, y, (M, N, K))
    rest = out.clone()
    rest[1:1 + M, 5:5 + N] = 3.0
    assert (rest == 3.0).all()


def test_no_rows():
    x, xs, w, ws, _ = operands(0, 200, 300)
    assert qnn.f8_matmul(x.to(DEV), xs.to(DEV), w.to(DEV), ws.to(DEV)).shape == (0, 200)


@pytest.mark.parametrize("M", [1, 48, 400])
def test_the_same_bits_again_and_from_a_graph_with_other_rows(M):
    N, K = 520, 1536
    x, xs, w, ws, _ = (t.to(DEV) for t in operands(M, N, K))
    want = qnn.f8_matmul(x, xs, w, ws)
    for _ in range(3):
        assert torch.equal(qnn.f8_matmul(x, xs, w, ws), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = qnn.f8_matmul(x, xs, w, ws)
    for seed in range(3):
        other = operands(M, N, K, seed + 1)
        x.view(torch.uint8).copy_(other[0].view(torch.uint8))
        xs.copy_(other[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, qnn.f8_matmul(x, xs, w, ws))


def test_rows_do_not_depend_on_the_others_of_their_launch():
    x, xs, w, ws, _ = (t.to(DEV) for t in operands(300, 260, 640))
    y = qnn.f8_matmul(x, xs, w, ws)
    turned = torch.randperm(300, generator=torch.Generator().manual_seed(1)).to(DEV)
    again = qnn.f8_matmul(x.view(torch.uint8)[turned].view(ref.F8), xs[:, turned].contiguous(), w, ws)
    assert torch.equal(again, y[turned])


def test_a_layer_as_it_is_used():
    # norm -> gate and up -> gated rows -> down, each step compared with the one before it as it came out
    g = torch.Generator().manual_seed(3)
    M, H, I = 37, 384, 200
    x, r = (torch.randn(M, H, generator=g).to(torch.bfloat16) for _ in range(2))
    up, ups = qnn.quantize_weights_blocks((torch.randn(2 * I, H, generator=g) / H ** 0.5).numpy())
    down, downs = qnn.quantize_weights_blocks((torch.randn(H, I, generator=g) / I ** 0.5).numpy())
    codes, scales, total = qnn.f8_rmsnorm(x.to(DEV), None, 1e-5, residual=r.to(DEV))
    both = qnn.f8_matmul(codes, scales, up.to(DEV), ups.to(DEV))
    check(codes, scales, up, ups, None, torch.bfloat16, both, "up")
    h, hs = qnn.f8_quantize(both, gated=True)
    v = both.cpu().double()
    ref.assert_codes(h, hs, torch.nn.functional.silu(v[:, :I]) * v[:, I:], 2.0 ** -20)
    y = qnn.f8_matmul(h, hs, down.to(DEV), downs.to(DEV))
    check(h, hs, down, downs, None, torch.bfloat16, y, "down")
    # and the whole against 64 bits without codes: e4m3 leaves an eighth of a step of relative error per factor, averaged over the sums
    t = total.cpu().double()
    t = t / torch.sqrt((t * t).mean(1, keepdim=True) + 1e-5)
    b = t @ ref.weights(up, ups).t()
    want = (torch.nn.functional.silu(b[:, :I]) * b[:, I:]) @ ref.weights(down, downs).t()
    assert (y.cpu().double() - want).norm() < 0.1 * want.norm()

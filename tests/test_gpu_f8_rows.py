"""Rows as e4m3 codes with a scale per 128 elements: plain (bit for bit), gated, behind a root-mean-square norm."""
import math

import pytest
import torch

import f8_reference as ref
import paper_1806_08342_amd as qnn

pytestmark = pytest.mark.gpu
DEV = ref.DEV
KINDS = [torch.bfloat16, torch.float16]
# binary32: exp, sum, quotient and product of silu are off by a few units of 2^-24 each
GATE = 2.0 ** -20
# sums of up to 64 squares in a lane, over lanes and waves (half of that counts behind the root), root, quotient, three products
NORM = 2.0 ** -18


def same_codes(got, want, what):
    got, want = got.cpu().view(torch.uint8), want.contiguous().view(torch.uint8)
    nan = (want & 127) == 127
    assert torch.equal((got & 127) == 127, nan), what
    assert torch.equal(got[~nan], want[~nan]), (what, int((got != want).sum()))


def rows(g, M, K, dtype, spread=1.0):
    return (torch.randn(M, K, generator=g) * torch.exp(spread * torch.randn(1, K, generator=g))).to(dtype)


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("M,K", [(1, 1), (3, 7), (2, 8), (1, 127), (5, 128), (4, 129), (1, 4096), (33, 1000), (700, 264), (130, 5003), (2, 40000)])
def test_plain_rows_are_the_definition_bit_for_bit(M, K, dtype):
    x = rows(torch.Generator().manual_seed(M * K), M, K, dtype)
    codes, scales = qnn.f8_quantize(x.to(DEV))
    want, want_scales = ref.encode(x.float())
    assert codes.dtype == ref.F8 and torch.equal(scales.cpu(), want_scales)
    same_codes(codes, want, (M, K))


@pytest.mark.parametrize("dtype", KINDS)
def test_rows_at_the_ends_of_the_range(dtype):
    g = torch.Generator().manual_seed(5)
    big, tiny = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    x = torch.stack([torch.zeros(256), torch.full((256,), big), torch.randn(256, generator=g) * tiny, torch.randn(256, generator=g) * tiny * 2.0 ** -6,
                     torch.where(torch.arange(256) % 7 == 0, math.inf, torch.randn(256, generator=g)), torch.full((256,), -math.inf),
                     torch.where(torch.arange(256) == 130, math.nan, torch.randn(256, generator=g)), torch.full((256,), math.nan),
                     torch.where(torch.arange(256) % 5 == 0, -math.inf, 0.0), torch.arange(256) - 128.0,
                     torch.where(torch.arange(256) % 2 == 0, big, tiny), torch.linspace(-3, 3, 256)]).to(dtype)
    codes, scales = qnn.f8_quantize(x.to(DEV))
    want, want_scales = ref.encode(x.float())
    assert torch.equal(scales.cpu(), want_scales) and (scales >= 2.0 ** -80).all()
    same_codes(codes, want, "ends")


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("M,K", [(1, 1), (2, 100), (1, 128), (24, 1408), (300, 515), (3, 14336)])
def test_gated_rows(M, K, dtype):
    x = (3 * rows(torch.Generator().manual_seed(K), M, 2 * K, dtype, 0.3)).to(dtype)
    codes, scales = qnn.f8_quantize(x.to(DEV), gated=True)
    v = x.double()
    ref.assert_codes(codes, scales, torch.nn.functional.silu(v[:, :K]) * v[:, K:], GATE, (M, K))


def test_gates_far_from_zero():
    x = torch.zeros(4, 512)
    x[:, 256:] = 2.0
    x[0, :256], x[1, :256], x[2, :256] = -1e4, 3e4, torch.linspace(-120, 120, 256)
    codes, scales = qnn.f8_quantize(x.to(torch.bfloat16).to(DEV), gated=True)
    v = x.to(torch.bfloat16).double()
    v = torch.nn.functional.silu(v[:, :256]) * v[:, 256:]
    got = ref.values(codes, scales)
    assert torch.isfinite(got).all() and (got[0] == 0).all() and (got[3] == 0).all()
    ref.assert_codes(codes[1:3], scales[:, 1:3], v[1:3], GATE)


def norm(x, residual, weight, eps):
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    v = h.double()
    v = v / torch.sqrt((v * v).mean(1, keepdim=True) + eps)
    return h, v if weight is None else v * weight.double()


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("residual,weighted", [(False, True), (True, True), (True, False)])
@pytest.mark.parametrize("M,K", [(1, 1), (3, 8), (5, 100), (9, 512), (6, 1000), (3, 2048), (1, 4096), (40, 2880), (2, 8192), (7, 9001), (2, 20000), (2, 33000), (1, 70001)])
def test_norm(M, K, residual, weighted, dtype):
    g = torch.Generator().manual_seed(M + K)
    x, r = rows(g, M, K, dtype, 0.7), rows(g, M, K, dtype, 0.7) if residual else None
    w = (0.5 + torch.rand(K, generator=g)).to(dtype) if weighted else None
    got = qnn.f8_rmsnorm(x.to(DEV), None if w is None else w.to(DEV), 1e-5, residual=None if r is None else r.to(DEV), with_y=True)
    h, v = norm(x, r, w, 1e-5)
    ref.assert_codes(got[0], got[1], v, NORM, (M, K))
    if residual:
        assert torch.equal(got[2].cpu(), h)
    ref.assert_close(got[-1], v, v.abs() * (ref.half_ulp(dtype) + 2 * NORM) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps, (M, K))
    assert len(got) == 3 + residual


@pytest.mark.parametrize("K", [64, 600, 3000, 40001])
@pytest.mark.parametrize("size,eps", [(1e30, 1e-5), (3e37, 0.0), (1e-25, 0.0), (1e-39, 0.0), (1e-25, 1e-5), (1e-12, 1e-24), (1e18, 1e-6)])
def test_norm_of_rows_whose_squares_leave_the_range(size, eps, K):
    g = torch.Generator().manual_seed(K)
    x = (torch.randn(3, K, generator=g).clamp(-4, 4) * size).to(torch.bfloat16)
    x[1] = 0
    got = qnn.f8_rmsnorm(x.to(DEV), None, eps)
    v = x.double()
    v = v / torch.sqrt((v * v).mean(1, keepdim=True) + (float(torch.tensor(eps)) or 1e-300))
    ref.assert_codes(got[0], got[1], v, NORM, (size, eps))


def test_norm_of_infinities_and_nan():
    x = torch.randn(5, 300).to(torch.bfloat16)
    x[1, 7], x[2, 200], x[3] = math.inf, math.nan, 0
    codes, scales, y = qnn.f8_rmsnorm(x.to(DEV), None, 1e-5, with_y=True)
    got, y = ref.values(codes, scales), y.cpu()
    assert torch.isfinite(got[[0, 3, 4]]).all() and torch.isnan(got[2]).all() and torch.isnan(got[1, 7]) and (got[1, torch.arange(300) != 7] == 0).all()
    assert torch.isnan(y[1, 7]) and (y[3] == 0).all()
    ref.assert_codes(codes[[0, 3, 4]], scales[:, [0, 3, 4]], norm(x[[0, 3, 4]], None, None, 1e-5)[1], NORM)


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("K", [72, 129, 640])
def test_spaced_rows_and_what_lies_between_them(K, dtype):
    M, pad = 21, 37
    g = torch.Generator().manual_seed(K)
    x, r = (rows(g, M, 2 * K + pad, dtype).to(DEV) for _ in range(2))
    codes, scales = torch.full((M, K + 11), 3, dtype=torch.uint8, device=DEV), torch.full((ref.blocks(K), M + 5), -7.0, device=DEV)
    out = (codes.view(ref.F8)[:, 3:3 + K], scales[:, 2:2 + M])
    total = torch.full((M, K + 9), 5.0, dtype=dtype, device=DEV)
    back = qnn.f8_rmsnorm(x[:, 5:5 + K], None, 1e-5, residual=r[:, 1:1 + K], total=total[:, 4:4 + K], out=out)
    assert back[0] is out[0] and back[1] is out[1]
    h, v = norm(x[:, 5:5 + K].cpu(), r[:, 1:1 + K].cpu(), None, 1e-5)
    ref.assert_codes(*out, v, NORM)
    assert torch.equal(total[:, 4:4 + K].cpu(), h) and (total[:, :4] == 5).all() and (total[:, 4 + K:] == 5).all()
    assert (codes[:, :3] == 3).all() and (codes[:, 3 + K:] == 3).all() and (scales[:, :2] == -7).all() and (scales[:, 2 + M:] == -7).all()
    for gated in (False, True):
        qnn.f8_quantize(x[:, 5:5 + K * (1 + gated)], gated, out=out)
        v = x[:, 5:5 + K * (1 + gated)].cpu().double()
        ref.assert_codes(*out, torch.nn.functional.silu(v[:, :K]) * v[:, K:] if gated else v, GATE)
        assert (codes[:, :3] == 3).all() and (codes[:, 3 + K:] == 3).all() and (scales[:, :2] == -7).all() and (scales[:, 2 + M:] == -7).all()


@pytest.mark.parametrize("K", [100, 1001, 4096, 50003])
def test_norm_in_place(K):
    g = torch.Generator().manual_seed(K)
    x, r = rows(g, 5, K, torch.bfloat16), rows(g, 5, K, torch.bfloat16)
    h, v = norm(x, r, None, 1e-5)
    for which in (0, 1):
        a, b = x.to(DEV), r.to(DEV)
        codes, scales, total = qnn.f8_rmsnorm(a, None, 1e-5, residual=b, total=(a, b)[which])
        assert total is (a, b)[which] and torch.equal(total.cpu(), h) and torch.equal((b, a)[which].cpu(), (r, x)[which])
        ref.assert_codes(codes, scales, v, NORM)


def test_no_rows():
    x = torch.empty(0, 256, dtype=torch.bfloat16, device=DEV)
    codes, scales = qnn.f8_quantize(x)
    assert codes.shape == (0, 256) and scales.shape == (2, 0)
    assert [t.shape[0] for t in qnn.f8_rmsnorm(x, residual=x)] == [0, 2, 0]


def test_captured_and_replayed_with_other_rows():
    x, r = (torch.randn(9, 1000, device=DEV).to(torch.bfloat16) for _ in range(2))
    qnn.f8_rmsnorm(x, residual=r), qnn.f8_quantize(x, True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = qnn.f8_rmsnorm(x, residual=r), qnn.f8_quantize(x, True)
    for seed in range(3):
        x.copy_(torch.randn(9, 1000, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(a + b, qnn.f8_rmsnorm(x, residual=r) + qnn.f8_quantize(x, True)):
            assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("M, K", [(1, 1), (3, 130), (257, 1000)])
def test_new_codes_and_scales_are_tensors_of_their_own(M, K):
    x = torch.randn(M, K, device=DEV).to(torch.bfloat16)
    codes, scales = qnn.f8_quantize(x)
    assert codes.is_contiguous() and scales.is_contiguous() and not codes.requires_grad and scales.data_ptr() % 256 == 0
    kept, copy = scales.clone(), codes.view(torch.uint8).clone()
    codes.view(torch.uint8).fill_(0x7f)
    assert torch.equal(scales, kept)
    scales.fill_(2.0)
    assert (codes.view(torch.uint8) == 0x7f).all()
    again, _ = qnn.f8_quantize(x)
    del codes, scales
    torch.empty(1 << 20, device=DEV).fill_(1.0)
    assert torch.equal(again.view(torch.uint8), copy)
    with torch.inference_mode():
        codes, scales = qnn.f8_quantize(x)
        assert torch.equal(codes.view(torch.uint8), copy) and torch.equal(scales, kept)


@pytest.mark.parametrize("size, weight", [(1e10, 1e30), (1e-10, 1e-30), (1.0, 3e37), (1e15, 1e-38), (1e-17, 1e38), (1e17, 1e20), (3e-3, 1e-22)])
@pytest.mark.parametrize("K", [200, 5003])
def test_norm_with_weights_at_the_ends_of_the_range(size, weight, K):
    # products of elements and weights that leave binary32 although what the norm makes of them does not, and scales near their bound
    g = torch.Generator().manual_seed(K)
    x, w = (torch.randn(3, K, generator=g) * size).to(torch.bfloat16), ((0.5 + torch.rand(K, generator=g)) * weight).to(torch.bfloat16)
    w[K // 2:] = 1.0
    codes, scales, y = qnn.f8_rmsnorm(x.to(DEV), w.to(DEV), 0.0, with_y=True)
    v = x.double()
    v = v / v.square().mean(1, keepdim=True).sqrt() * w.double()
    # v is held in binary32: what passes its largest number, 2^128 (1 - 2^-24), is infinite there (1.5e38 times a normal number over 2.3 is), which is
    # cut off at the largest finite one of its block
    passes = v.abs() > torch.finfo(torch.float32).max
    finite = torch.nn.functional.pad(torch.where(passes, 0.0, v.abs()), (0, -K % 128)).view(3, -1, 128)
    most = finite.amax(2, keepdim=True).expand(finite.shape).reshape(3, -1)[:, :K]
    for c, s in ((codes, scales), qnn.f8_rmsnorm(x.to(DEV), w.to(DEV), 0.0)):  # (without y codes come from the products with the weights)
        ref.assert_codes(c, s, torch.where(passes, most * v.sign(), v), 2.0 ** -20)
    # (a result is rounded to bfloat16 once, behind roundings in binary32; below its normal numbers to the last of their steps)
    ref.assert_close(torch.where(passes, 0.0, y.cpu().double()), torch.where(passes, 0.0, v), v.abs() * (ref.half_ulp(torch.bfloat16) + 2.0 ** -20) + 2.0 ** -133)
    assert (y.cpu()[passes].abs() == math.inf).all()


# Rows that a wave has alone with two pieces per lane, rows of four and of two waves with two and four pieces, whole pieces and not: forms that many
# rows, or lengths past 8192, take.
@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("residual,weighted", [(False, True), (True, False), (True, True)])
@pytest.mark.parametrize("M,K", [(600, 1000), (600, 1001), (600, 4096), (600, 5001), (600, 7001), (600, 12288), (4100, 1000), (4100, 2048), (3, 16384), (2, 16001), (2, 20001), (3, 32768)])
def test_norm_of_many_and_of_long_rows(M, K, residual, weighted, dtype):
    g = torch.Generator().manual_seed(M + K)
    x, r = rows(g, M, K, dtype, 0.7), rows(g, M, K, dtype, 0.7) if residual else None
    w = (0.5 + torch.rand(K, generator=g)).to(dtype) if weighted else None
    h, v = norm(x, r, w, 1e-5)
    x, r, w = (None if t is None else t.to(DEV) for t in (x, r, w))
    for with_y in (False, True):
        got = qnn.f8_rmsnorm(x, w, 1e-5, residual=r, with_y=with_y)
        assert len(got) == 2 + residual + with_y
        ref.assert_codes(got[0], got[1], v, NORM, (M, K, with_y))
        if residual:
            assert torch.equal(got[2].cpu(), h)
        if with_y:
            ref.assert_close(got[-1], v, v.abs() * (ref.half_ulp(dtype) + 2 * NORM) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps, (M, K))

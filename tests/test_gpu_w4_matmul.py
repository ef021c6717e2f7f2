"""Products with 4-bit weights and a scale per group against the definition in 64 bits."""
import pytest
import torch

import paper_1806_08342_amd as qnn
from lm_reference import DEV, assert_close, half_ulp, w4

pytestmark = pytest.mark.gpu


def make(M, N, K, group, dtype, zeros, bias, seed=0):
    g = torch.Generator().manual_seed(seed)
    groups = -(-K // group)
    x = torch.randn(M, K, generator=g).to(dtype)
    codes = torch.randint(0, 256, (N, K // 2), generator=g).to(torch.uint8)
    scales = (0.01 + 0.02 * torch.rand(groups, N, generator=g)).to(dtype)
    z = torch.randint(-8, 8, (groups, N), generator=g).to(torch.int8) if zeros else None
    b = torch.randn(N, generator=g).to(dtype) if bias else None
    return [t if t is None else t.to(DEV) for t in (x, codes, scales, z, b)]


def check(y, x, codes, scales, group, z, b, what):
    want, size = w4(x, codes, scales, group, z, b)
    K = x.shape[1]
    # one rounding to the type; sums in binary32: a handful of roundings in a group and one for each group, at most of the
    # size of the terms' absolute sum
    assert_close(y, want, half_ulp(x.dtype) * 1.01 * want.abs() + (8 + K / 32) * 2.0 ** -23 * size, what)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,N,K,group,zeros,bias", [
    (1, 1, 2, 32, False, False), (1, 16, 128, 128, False, True), (1, 100, 4096, 128, False, False), (2, 33, 1000, 64, True, False),
    (3, 257, 66, 32, True, True), (5, 130, 2890, 64, True, True), (7, 64, 254, 128, True, False), (16, 48, 640, 128, False, False),
    (17, 40, 384, 96, True, False), (24, 500, 512, 128, False, False), (31, 63, 130, 160, False, True), (33, 129, 1152, 64, True, True),
    (64, 96, 256, 32, False, False), (65, 200, 770, 128, True, False), (100, 300, 512, 1024, True, True), (128, 256, 1024, 128, False, False),
    (129, 130, 514, 64, False, True), (200, 513, 640, 32, True, False), (300, 1000, 384, 128, True, True)])
def test_against_the_definition(M, N, K, group, zeros, bias, dtype):
    x, codes, scales, z, b = make(M, N, K, group, dtype, zeros, bias)
    check(qnn.w4_matmul(x, codes, scales, group, z, b), x, codes, scales, group, z, b, (M, N, K, group))


@pytest.mark.parametrize("M", [1, 3, 40, 150])
def test_rows_spaced_apart_and_a_caller_s_output(M):
    x, codes, scales, z, b = make(M, 70, 320, 64, torch.bfloat16, True, True)
    wide = torch.full((M, 333), float("nan"), dtype=x.dtype, device=DEV)  # what lies between the rows must not be read
    wide[:, 5:325] = x
    out = torch.full((M, 81), 7.0, dtype=x.dtype, device=DEV)
    y = qnn.w4_matmul(wide[:, 5:325], codes, scales, 64, z, b, out=out[:, 3:73])
    check(y, x, codes, scales, 64, z, b, "spaced")
    assert (out[:, :3] == 7).all() and (out[:, 73:] == 7).all()


def test_all_codes_and_zero_points_are_exact():
    # one-hot rows: each output is one weight
    K, N, group = 128, 256, 32
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)[:, None].repeat(1, K // 2).to(DEV)
    for dtype in (torch.bfloat16, torch.float16):
        x = torch.eye(K, dtype=dtype, device=DEV)[:40].contiguous()
        scales = torch.full((4, N), 0.25, dtype=dtype, device=DEV)
        for zero in (-8, 0, 7):
            z = torch.full((4, N), zero, dtype=torch.int8, device=DEV)
            for m in (1, 16, 40):
                y = qnn.w4_matmul(x[:m], codes, scales, group, z)
                want, _ = w4(x[:m], codes, scales, group, z)
                assert torch.equal(y.cpu().double(), want)


def test_empty_and_zero_inputs():
    x, codes, scales, z, b = make(4, 20, 64, 32, torch.float16, True, True)
    assert qnn.w4_matmul(x[:0], codes, scales, 32, z, b).shape == (0, 20)
    assert torch.equal(qnn.w4_matmul(torch.zeros_like(x), codes, scales, 32, z, b), b.expand(4, 20))


def test_results_do_not_change_from_call_to_call_or_on_another_stream():
    for M in (1, 9, 50, 260):
        x, codes, scales, z, _ = make(M, 400, 2048, 128, torch.bfloat16, True, False)
        want = qnn.w4_matmul(x, codes, scales, 128, z)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = [qnn.w4_matmul(x, codes, scales, 128, z) for _ in range(5)]
        side.synchronize()
        assert all(torch.equal(want, y) for y in again)


def test_refusals():
    x, codes, scales, z, b = make(4, 20, 64, 32, torch.bfloat16, True, True)
    f = qnn.w4_matmul
    for bad in (lambda: f(x.float(), codes, scales, 32), lambda: f(x, codes.to(torch.int8), scales, 32), lambda: f(x, codes, scales.half(), 32),
                lambda: f(x.t(), codes, scales, 32), lambda: f(x[0], codes, scales, 32), lambda: f(x, codes, scales, 32, z.int()),
                lambda: f(x, codes, scales, 32, z, b.float()), lambda: f(x.cpu(), codes, scales, 32), lambda: f(x, codes, scales, 32, out=x.float())):
        with pytest.raises((TypeError, ValueError)):
            bad()
    for bad in (lambda: f(x, codes[:, :-1].contiguous(), scales, 32), lambda: f(x, codes, scales[:1], 32), lambda: f(x, codes, scales, 64), lambda: f(x, codes, scales, 32, z[:, :3].contiguous()),
                lambda: f(x, codes, scales, 32, z, b[:3]), lambda: f(x, codes, scales, 32, out=torch.empty(4, 21, dtype=x.dtype, device=DEV)),
                lambda: f(x, codes, scales, 0)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(qnn.QnnError, match="QNN_EINVAL"):
        f(x, codes, torch.cat([scales, scales]), 16)  # a group is a multiple of 32


# every kernel and form of one, at sizes that divide nothing
FORMS = {"few16x16/4": (3, 3, 30), "few16x32/8": (5, 17001, 330), "few16x16/8": (9, 4103, 514), "few16x16/16": (15, 1000, 1030), "tens32x64/4": (17, 1001, 386),
         "tens32x32/8": (65, 301, 1034), "tens32x128/4": (17, 17003, 770), "tens64x128/4": (33, 17001, 770), "tens64x128/2": (70, 9001, 514), "tens64x64/4": (40, 8203, 514),
         "many128x256": (201, 17003, 770)}


@pytest.mark.parametrize("group,zeros,dtype", [(128, False, torch.bfloat16), (64, True, torch.float16), (32, True, torch.bfloat16), (96, False, torch.float16)])
@pytest.mark.parametrize("form", FORMS)
def test_every_form(form, group, zeros, dtype):
    M, N, K = FORMS[form]
    with_group = "many64x256" if form == "many128x256" and group != 128 else form
    assert qnn.w4_matmul_plan(M, N, K, 128) == form and (form == "few16x16/4" or qnn.w4_matmul_plan(M, N, K, group) == with_group)
    if form == "few16x16/4" and group < 64:
        group = 32
    x, codes, scales, z, b = make(M, N, K, group, dtype, zeros, True)
    check(qnn.w4_matmul(x, codes, scales, group, z, b), x, codes, scales, group, z, b, form)


@pytest.mark.parametrize("M", [2, 30, 300])
@pytest.mark.parametrize("skip", [1, 2, 3])
def test_rows_of_codes_at_any_byte(M, skip):
    # rows of 65 bytes, the first of them `skip` bytes after a multiple of 4; guarded on both sides
    N, K = 260, 130
    x, codes, scales, z, _ = make(M, N, K, 32, torch.bfloat16, True, False)
    flat = torch.full((skip + codes.numel() + 8,), 0x77, dtype=torch.uint8, device=DEV)
    moved = flat[skip:skip + codes.numel()].view(N, K // 2)
    moved.copy_(codes)
    assert torch.equal(qnn.w4_matmul(x, moved, scales, 32, z), qnn.w4_matmul(x, codes, scales, 32, z))


@pytest.mark.parametrize("M", [4, 20, 50, 300])
def test_scales_far_apart_zero_and_negative(M):
    N, K, group = 300, 640, 64
    x, codes, scales, z, _ = make(M, N, K, group, torch.bfloat16, True, False)
    scales[0] *= 2.0 ** 30
    scales[3] *= 2.0 ** -30
    scales[4] = 0.0
    scales[5, ::2] = 0.0
    scales[0, 1::3] = 0.0
    scales[6] *= -1.0
    scales[9, 5] = 0.0
    check(qnn.w4_matmul(x, codes, scales, group, z), x, codes, scales, group, z, None, "apart")
    scales[:] = 0.0
    assert (qnn.w4_matmul(x, codes, scales, group, z) == 0).all()


@pytest.mark.parametrize("M", [3, 20, 300])
def test_sizes_of_rows_do_not_matter(M):
    # rows scaled by powers of two scale their results, up to the ends of the type's range
    x, codes, scales, z, _ = make(M, 260, 384, 128, torch.bfloat16, True, False)
    want = qnn.w4_matmul(x, codes, scales, 128, z)
    by = torch.tensor([2.0 ** (i % 9 * 20 - 80) for i in range(M)], device=DEV)[:, None].to(torch.bfloat16)
    got = qnn.w4_matmul(x * by, codes, scales, 128, z)
    assert torch.equal(got, want * by)
    x[1, 7] = float("nan")
    y = qnn.w4_matmul(x, codes, scales, 128, z)
    assert torch.isnan(y[1]).all() and torch.isfinite(y[0]).all() and torch.isfinite(y[2:]).all()


def test_long_rows():
    K = (1 << 21) + 258  # beyond the offsets of the kernels for many rows of x
    g = torch.Generator().manual_seed(0)
    x = torch.randn(18, K, generator=g).to(torch.bfloat16).to(DEV)
    codes = torch.randint(0, 256, (5, K // 2), generator=g).to(torch.uint8).to(DEV)
    scales = torch.full((-(-K // 1024), 5), 0.01, dtype=torch.bfloat16, device=DEV)
    assert qnn.w4_matmul_plan(18, 5, K, 1024).startswith("few")
    check(qnn.w4_matmul(x, codes, scales, 1024), x, codes, scales, 1024, None, None, "long")

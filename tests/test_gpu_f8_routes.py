"""Every kernel that the 8-bit floating point operators choose among, by its name, and tensors beyond 4 GiB; rows and columns picked from
large results against 64 bits."""
import math

import pytest
import torch

import f8_reference as ref
import paper_1806_08342_amd as qnn

pytestmark = pytest.mark.gpu
DEV = ref.DEV
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def codes(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV).mul_(150).clamp_(-448, 448).to(ref.F8)


def operands(M, N, K, seed=0):
    g = torch.Generator(DEV).manual_seed(seed + M + 7 * N + 31 * K)
    scale = lambda *s: torch.exp(torch.randn(*s, generator=g, device=DEV)) / 150  # noqa: E731
    return codes(g, M, K), scale(ref.blocks(K), M), codes(g, N, K), scale(ref.blocks(N), ref.blocks(K)), torch.randn(N, generator=g, device=DEV)


def some(n, most):
    """Both ends of n things, what lies around the middle's tiles, and others."""
    near = {0, 1, 15, 16, 63, 64, 127, 128, 255, 256, n // 2, n // 2 + 1, n - 65, n - 17, n - 16, n - 2, n - 1}
    g = torch.Generator().manual_seed(n)
    picked = sorted({i for i in near if 0 <= i < n})
    picked = sorted({*picked, *torch.randint(0, n, (max(0, most - len(picked)),), generator=g).tolist()})
    return torch.tensor(picked, device=DEV)


def rows_of(t, index):
    return t.view(torch.uint8)[index].view(ref.F8)


def check(x, xs, w, ws, bias, y, most_rows=20, most_columns=200, what=""):
    r, c = some(x.shape[0], most_rows), some(w.shape[0], most_columns)
    narrow = y.dtype != F32
    # (each column with the scales of its own block: weights' rows are picked one by one, so the scales are too)
    a, b, K = rows_of(x, r).cpu(), rows_of(w, c).cpu(), x.shape[1]
    sa, sb = xs[:, r].cpu(), ws[c // 128].cpu()
    want, off = torch.zeros(len(r), len(c)).double(), torch.zeros(len(r), len(c)).double()
    for i in range(ref.blocks(K)):
        p, q = a[:, i * 128:(i + 1) * 128], b[:, i * 128:(i + 1) * 128]
        one, bad = ref.product(p, torch.ones(1, len(r)), q, torch.ones(ref.blocks(len(c)), 1), narrow)
        scale = sa[i].double()[:, None] * sb[:, i].double()[None]
        size = (p.double().abs() @ q.double().abs().t()) * scale
        want, off = want + one * scale, off + bad * scale + size * (ref.blocks(K) + 64) * 2.0 ** -24
    if bias is not None:
        want = want + bias.cpu().double()[c.cpu()]
    got = y[r][:, c]
    ref.assert_close(got, want, (1 + 2.0 ** -8) * off + (want.abs() + off) * (ref.half_ulp(y.dtype) + 2.0 ** -24) + torch.finfo(y.dtype).smallest_normal * torch.finfo(y.dtype).eps, what)


@pytest.mark.parametrize("M,N,K,dtype,plan", [
    (1, 4096, 1024, BF16, "rows16x16"), (16, 1000, 2000, F32, "rows16x16"), (9, 9000, 512, BF16, "rows16x32"), (32, 500, 1040, F16, "rows32x16"), (20, 8200, 528, F32, "rows32x32"),
    (33, 600, 4096, BF16, "rows48x16"), (40, 600, 2047, F16, "rows48x16"), (48, 10000, 640, BF16, "rows48x32"), (64, 900, 2048, BF16, "rows64x16"), (50, 8192, 300, F32, "rows64x32"),
    (900, 1000, 512, BF16, "rows64x64"), (1021, 999, 1111, F32, "rows64x64"), (291, 1280, 692, F32, "rows64x64"), (130, 12000, 2048, BF16, "tile128x128/1"), (1000, 12288, 1040, F32, "tile128x128/1"),
    (1, 4100, 4095, BF16, "rows16x16"), (24, 2050, 1030, F16, "rows32x16"),
    (64, 1000, 1021, F32, "rows64x16"), (8, 600, 2049, F32, "rows16x16"), (300, 4096, 4096, BF16, "tile128x128/2"), (3970, 4090, 2047, BF16, "tile256x256/1"), (4096, 8192, 2048, F16, "tile256x256/1")])
def test_each_kernel(M, N, K, dtype, plan):
    assert qnn.f8_matmul_plan(M, N, K, dtype) == plan
    x, xs, w, ws, b = operands(M, N, K)
    y = qnn.f8_matmul(x, xs, w, ws, bias=b.to(dtype), dtype=dtype)
    check(x, xs, w, ws, b.to(dtype), y, what=plan)
    # x at an odd address and rows an odd distance apart: whichever kernel takes those, the same sums
    wide = torch.empty(M, K + 7, dtype=torch.uint8, device=DEV)
    wide[:, 3:3 + K] = x.view(torch.uint8)
    check(x, xs, w, ws, b.to(dtype), qnn.f8_matmul(wide.view(ref.F8)[:, 3:3 + K], xs, w, ws, bias=b.to(dtype), dtype=dtype), what=plan + " at any byte")


def test_x_beyond_4_gib():
    M, N, K = 600000, 64, 8192
    x, xs, w, ws, _ = operands(M, N, K)
    check(x, xs, w, ws, None, qnn.f8_matmul(x, xs, w, ws), most_rows=40)


def test_weights_beyond_4_gib():
    M, N, K = 3, 600000, 8192
    x, xs, w, ws, _ = operands(M, N, K)
    check(x, xs, w, ws, None, qnn.f8_matmul(x, xs, w, ws), most_columns=400)


@pytest.mark.parametrize("M,N", [(2, 4100), (4100, 20)])
def test_rows_longer_than_the_tiles_take(M, N):
    K = (1 << 20) + 16  # 4.3 GB of one operand
    assert qnn.f8_matmul_plan(M, N, K, BF16).startswith("rows")
    x, xs, w, ws, _ = operands(M, N, K)
    check(x, xs, w, ws, None, qnn.f8_matmul(x, xs, w, ws), most_rows=18, most_columns=40)


def test_weights_and_results_beyond_4_gib_in_tiles():
    M, N, K = 5000, 600000, 7184
    assert qnn.f8_matmul_plan(M, N, K, BF16).startswith("tile")
    x, xs, w, ws, _ = operands(M, N, K)
    check(x, xs, w, ws, None, qnn.f8_matmul(x, xs, w, ws), most_rows=30, most_columns=400)


def test_rows_beyond_4_gib_to_codes_and_normed():
    M, K = 270000, 8200
    g = torch.Generator(DEV).manual_seed(5)
    x = torch.empty(M, K, dtype=BF16, device=DEV)
    for part in x.split(10000):
        part.normal_(generator=g)
    r = some(M, 40)
    v = x[r].cpu()
    c, s = qnn.f8_quantize(x)
    ref.assert_codes(rows_of(c, r), s[:, r], v.double(), 2.0 ** -22)
    c, s = qnn.f8_quantize(x, gated=True)
    h = torch.nn.functional.silu(v[:, :K // 2].double()) * v[:, K // 2:].double()
    ref.assert_codes(rows_of(c, r), s[:, r], h, 2.0 ** -20)
    c, s, total = qnn.f8_rmsnorm(x, None, 1e-6, residual=x)
    v = total[r].cpu().double()
    assert torch.equal(total[r], (x[r].float() * 2).to(BF16))
    ref.assert_codes(rows_of(c, r), s[:, r], v / (v.square().mean(1, keepdim=True) + 1e-6).sqrt(), 2.0 ** -20)


def moe_layer(T, E, H, I, seed=0):
    g = torch.Generator(DEV).manual_seed(seed + T + 11 * E + 101 * H + 1009 * I)
    spread = lambda *s: torch.exp(0.5 * torch.randn(*s, generator=g, device=DEV))  # noqa: E731
    return dict(x=codes(g, T, H), xs=spread(ref.blocks(H), T) / 150, logits=torch.randn(T, E, generator=g, device=DEV), up=torch.empty(E, 2 * I, H, dtype=ref.F8, device=DEV),
                ups=spread(E, ref.blocks(2 * I), ref.blocks(H)) / (150 * H ** 0.5), down=torch.empty(E, H, I, dtype=ref.F8, device=DEV),
                downs=spread(E, ref.blocks(H), ref.blocks(I)) / (150 * I ** 0.5)), g


def filled(T, E, H, I, seed=0):
    c, g = moe_layer(T, E, H, I, seed)
    for e in range(E):
        c["up"].view(torch.uint8)[e] = codes(g, 2 * I, H).view(torch.uint8)
        c["down"].view(torch.uint8)[e] = codes(g, H, I).view(torch.uint8)
    return c


NAMES = ("x", "xs", "logits", "up", "ups", "down", "downs")


def check_moe(c, k, dtype=BF16, renormalize=True):
    """Against 64 bits, with the weights' rows of the chosen experts only."""
    y, experts, weights = qnn.f8_moe(*(c[n] for n in NAMES), k, renormalize=renormalize, dtype=dtype, with_choice=True)
    E = c["logits"].shape[1]
    for row, e, w in zip(ref.choose(c["logits"], k, renormalize), experts.cpu().tolist(), weights.cpu().tolist()):
        assert e == [o for o, _ in row] + [-1] * (k - len(row)), (e, row)
        assert all(abs(a - b) <= (16 + E) * 2.0 ** -24 for a, b in zip(w, [o for _, o in row] + [0.0] * (k - len(row)))), (w, row)
    want, off = ref.moe(*(c[n] for n in NAMES), k, renormalize)
    ref.assert_close(y, want, (1 + 2.0 ** -8) * off + (want.abs() + off) * (ref.half_ulp(dtype) + E * 2.0 ** -23) + torch.finfo(dtype).smallest_normal, (c["x"].shape, E, k))
    assert torch.equal(qnn.f8_moe(*(c[n] for n in NAMES), k, renormalize=renormalize, dtype=dtype), y)


# Tokens that choose for themselves and those routed before, experts past 64 and 256, more choices than 64 at once, an expert of 1, 8, 9, 16, 17
# and more tokens, an inner size in parts.
@pytest.mark.parametrize("T,E,k,H,I", [(8, 8, 8, 64, 48), (8, 64, 8, 144, 80), (9, 64, 8, 144, 80), (8, 65, 4, 64, 32), (3, 256, 8, 128, 64), (8, 257, 3, 96, 32), (40, 300, 5, 64, 48),
                                       (5, 1024, 32, 48, 32), (1, 1, 1, 32, 4096), (4, 32, 4, 272, 1968), (24, 2, 1, 528, 1040), (17, 1, 1, 144, 144), (33, 2, 2, 80, 272),
                                       (100, 3, 1, 256, 128), (300, 10, 6, 128, 96), (2, 4, 2, 4112, 16), (6, 5, 3, 16, 2064)])
def test_experts(T, E, k, H, I):
    for seed in range(2):
        check_moe(filled(T, E, H, I, seed), k, dtype=(BF16, F16)[seed], renormalize=seed == 0)


@pytest.mark.parametrize("T", [3, 5, 8, 9])
@pytest.mark.parametrize("E", [5, 64, 100, 256])
def test_few_tokens_with_logits_that_are_equal_infinite_or_nan(T, E):
    c = filled(T, E, 64, 32)
    n = c["logits"]
    n[0] = 0.25
    n[1] = -math.inf
    n[2, ::2] = math.nan
    if T > 3:
        n[3] = -math.inf
        n[3, E - 1] = -3e38
        n[4, 1], n[4, E - 1] = math.inf, math.inf
    for renormalize in (True, False):
        check_moe(c, 5, renormalize=renormalize)


def test_experts_beyond_4_gib():
    T, E, k, H, I = 12, 40, 3, 8192, 8192
    c, g = moe_layer(T, E, H, I)
    assert E * 2 * I * H > 1 << 32
    c["logits"].fill_(-math.inf)
    used = (0, 1, E // 2, E - 2, E - 1)
    for e in used:  # (the others are not chosen, so never read)
        c["up"].view(torch.uint8)[e] = codes(g, 2 * I, H).view(torch.uint8)
        c["down"].view(torch.uint8)[e] = codes(g, H, I).view(torch.uint8)
    c["logits"][:, list(used)] = torch.randn(T, len(used), generator=g, device=DEV)
    y, experts, weights = qnn.f8_moe(*(c[n] for n in NAMES), k, with_choice=True)
    # 64 bits of these sizes on the device, in parts, and what the bounds of smaller ones come to here: the norm of the difference
    total, chosen = torch.zeros(T, H, dtype=torch.float64, device=DEV), ref.choose(c["logits"], k)
    x = c["x"].double() * c["xs"].double().repeat_interleave(128, 0).t()
    for t, row in enumerate(chosen):
        assert experts[t].tolist() == [e for e, _ in row]
        for e, share in row:
            up = (c["up"][e].double() * c["ups"][e].double().repeat_interleave(128, 0).repeat_interleave(128, 1)) @ x[t]
            h = torch.nn.functional.silu(up[:I]) * up[I:]
            down = c["down"][e].double() * c["downs"][e].double().repeat_interleave(128, 0).repeat_interleave(128, 1)
            total[t] += (down @ h) * share
    # (the result's rounding is at most 2^-8 of a value; products are cut 13 bits below the largest of 8, 10^-4 of a sum's size and averaging)
    assert ((y.double() - total).norm(dim=1) <= 2.0 ** -8 * total.norm(dim=1)).all()


def test_infinite_products_between_the_experts_matrices():
    # up's sums pass binary32's largest in two tokens: h is infinite or NaN there, which reaches their rows and no others
    c = filled(6, 4, 128, 64)
    clean = qnn.f8_moe(*(c[n] for n in NAMES), 2)
    c["xs"][:, 1] = 3e38
    c["xs"][:, 4] = 3e38
    y = qnn.f8_moe(*(c[n] for n in NAMES), 2)
    keep = [0, 2, 3, 5]
    assert torch.equal(y[keep], clean[keep]) and not torch.isfinite(y[[1, 4]]).any()


@pytest.mark.parametrize("M,N,K,dtype", [(300, 4096, 4096, BF16), (1000, 1003, 1111, F32), (3970, 1030, 2047, BF16)])
def test_products_with_workspaces_on_two_streams_and_in_two_graphs_at_once(M, N, K, dtype):
    # parts of K and padded copies lie in memory of each call's, or graph's, own
    assert qnn.load_library().qnn_f8_matmul_workspace_bytes(M, N, K, 2 if dtype == F32 else 0) > 0
    args = [operands(M, N, K, seed)[:4] for seed in (1, 2)]
    want = [qnn.f8_matmul(*a, dtype=dtype) for a in args]
    torch.cuda.synchronize()
    streams, graphs, results = [torch.cuda.Stream() for _ in args], [], []
    got = [[], []]
    for _ in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(qnn.f8_matmul(*args[i], dtype=dtype))
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for ys, w in zip(got, want) for y in ys)
    for a in args:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            results.append(qnn.f8_matmul(*a, dtype=dtype))
    for _ in range(4):
        for y in results:
            y.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, w) for y, w in zip(results, want))


def test_a_workspace_of_the_callers_and_results_in_place_of_others():
    M, N, K = 300, 4096, 4096
    x, xs, w, ws, _ = operands(M, N, K)
    want = qnn.f8_matmul(x, xs, w, ws)
    space = torch.full((qnn.load_library().qnn_f8_matmul_workspace_bytes(M, N, K, 0) + 256,), 0xff, dtype=torch.uint8, device=DEV)
    out = torch.full((M, N), math.nan, dtype=BF16, device=DEV)
    assert qnn.f8_matmul(x, xs, w, ws, out=out, workspace=space[:-256]) is out and torch.equal(out, want) and (space[-256:] == 0xff).all()
    with pytest.raises(Exception):
        qnn.f8_matmul(x, xs, w, ws, workspace=space[:1024])
    c = filled(20, 8, 144, 96)
    want = qnn.f8_moe(*(c[n] for n in NAMES), 3)
    space = torch.full((qnn.load_library().qnn_f8_moe_workspace_bytes(20, 8, 3, 144, 96) + 256,), 0xff, dtype=torch.uint8, device=DEV)
    assert torch.equal(qnn.f8_moe(*(c[n] for n in NAMES), 3, workspace=space[:-256]), want) and (space[-256:] == 0xff).all()
    with pytest.raises(Exception):
        qnn.f8_moe(*(c[n] for n in NAMES), 3, workspace=space[:256])


def test_tensors_that_require_grad_are_refused():
    x, xs, w, ws, b = operands(4, 128, 128)
    rows = torch.randn(4, 128, device=DEV, dtype=BF16, requires_grad=True)
    scales = xs.clone().requires_grad_()
    for call in (lambda: qnn.f8_quantize(rows), lambda: qnn.f8_rmsnorm(rows), lambda: qnn.f8_rmsnorm(rows.detach(), residual=rows), lambda: qnn.f8_matmul(x, scales, w, ws)):
        with pytest.raises(Exception):
            call()
        with torch.no_grad():
            call()


@pytest.mark.parametrize("T,E,k,H,I", [(64, 40, 2, 64, 480), (17, 128, 3, 144, 336), (50, 33, 8, 272, 512)])
def test_many_experts_some_of_many_tokens(T, E, k, H, I):
    # 16 tokens of an expert at a time, and up to all of them in one
    c = filled(T, E, H, I)
    check_moe(c, k)
    c["logits"][:, E - 2] = 50.0
    c["logits"][: T // 2 + 1, 1] = 49.0
    check_moe(c, k, dtype=F16)


@pytest.mark.parametrize("T,E,k,H,I", [(17, 3, 3, 4112, 4112), (40, 2, 2, 3600, 4112), (70, 2, 2, 4096, 3696)])
def test_large_experts_for_many_tokens(T, E, k, H, I):
    # 128 columns of the second product for a workgroup, the last of them not whole, odd numbers of blocks, parts that begin within an expert
    c = filled(T, E, H, I)
    c["logits"][3] = -math.inf
    c["logits"][5, 1] = -math.inf
    check_moe(c, k)
    a = [c[n] for n in NAMES]
    want = qnn.f8_moe(*a, k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = qnn.f8_moe(*a, k)
    for _ in range(3):
        y.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


@pytest.mark.parametrize("M,N,K,dtype,plan", [
    (257, 1000, 4096, F16, "tile128x128/8"), (257, 1000, 4111, BF16, "tile128x128/7"), (1500, 2986, 6144, BF16, "tile256x256/3"), (1500, 2986, 6147, F16, "tile256x256/3"),
    (129, 9000, 6147, BF16, "tile256x256/7"), (130, 2051, 6144, F32, "tile128x128/7"), (129, 2047, 4111, F32, "tile128x128/7"), (257, 4099, 4096, F32, "tile128x128/2")])
def test_tiles_in_parts(M, N, K, dtype, plan):
    # with K of whole pieces, and of others, whose copies lie in the workspace before the parts' sums
    assert qnn.f8_matmul_plan(M, N, K, dtype) == plan
    x, xs, w, ws, b = operands(M, N, K)
    space = torch.full((qnn.load_library().qnn_f8_matmul_workspace_bytes(M, N, K, {BF16: 0, F16: 1, F32: 2}[dtype]) + 256,), 0xff, dtype=torch.uint8, device=DEV)
    for bias in (None, b.to(dtype)):
        y = qnn.f8_matmul(x, xs, w, ws, bias=bias, dtype=dtype, workspace=space[:-256])
        check(x, xs, w, ws, bias, y, what=plan)
        assert (space[-256:] == 0xff).all()

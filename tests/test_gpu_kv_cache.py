"""Appending to the 8-bit cache and reading it back: codes bit for bit against the definition."""
import pytest
import torch

import paper_1806_08342_amd as qnn
from lm_reference import DEV, append, case

pytestmark = pytest.mark.gpu


def fresh(requests, heads, dim, block, dtype, seed=0, scale=1.0):
    """A filled cache of `start` tokens per request, tables with room, and new rows."""
    total = [(s + n, n) for s, n in requests]
    cache, _, cu, _, table = case(total, heads, dim, block, dtype, seed)
    g = torch.Generator().manual_seed(seed + 1)
    kv = (scale * torch.randn(int(cu[-1]), 2, heads, dim, generator=g)).to(dtype).to(DEV)
    return cache, kv[:, 0], kv[:, 1], cu, torch.tensor([s for s, _ in requests], dtype=torch.int32, device=DEV), table


def check(cache, k, v, cu, start, table, what):
    want = append(cache, k, v, cu.cpu(), start.cpu(), table.cpu())
    qnn.kv_append(cache, k, v, cu, start, table)
    torch.cuda.synchronize()
    for got, ref, name in zip(cache, want, ("k_codes", "k_scales", "v_codes", "v_scales")):
        assert torch.equal(got.cpu(), ref), (what, name, int((got.cpu() != ref).sum()))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("requests,heads,dim,block", [
    ([(0, 1)], 1, 64, 32), ([(5, 1), (63, 1), (64, 1), (0, 0), (127, 1)], 2, 128, 64), ([(0, 300), (17, 100), (64, 64), (0, 0), (31, 33), (1, 0)], 3, 96, 64),
    ([(30, 5), (32, 31), (0, 32), (100, 1)], 2, 192, 32), ([(0, 129), (127, 2), (200, 57)], 1, 256, 128), ([(10, 200), (0, 700)], 2, 64, 256),
    ([(7, 90)], 2, 128, 96), ([(i * 7 % 50, i % 4) for i in range(150)], 1, 64, 32),
    ([(i, 1) for i in range(70)] + [(3, 300), (250, 90)], 3, 96, 256)])
def test_append_bit_for_bit(requests, heads, dim, block, dtype):
    # small, like and large against what the pages hold: scales stay, or grow and the codes held are rescaled
    for scale in (0.01, 0.6, 5.0):
        check(*fresh(requests, heads, dim, block, dtype, scale=scale), (requests, scale))


def test_values_that_are_no_numbers_and_pages_of_zeros():
    cache, k, v, cu, start, table = fresh([(40, 3), (0, 70), (64, 2)], 2, 64, 64, torch.bfloat16)
    k[0, 0, :5] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38, 1e-40])
    v[5, 1, 7] = float("-inf")
    k[3:73, 1] = 0.0
    v[73:, 0] = float("nan")
    check(cache, k, v, cu, start, table, "no numbers")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("held, new", [(0, 64), (63, 1), (40, 20)])
def test_infinities_beside_ordinary_values(held, new, dtype):
    cache, k, v, cu, start, table = fresh([(held, new)], 2, 128, 64, dtype)
    for x in (k, v):
        x[0, 0, 3], x[0, 0, 77], x[new - 1, 1, 64] = float("inf"), float("-inf"), float("nan")
        x[new - 1, 1, 127] = float("inf")
    check(cache, k, v, cu, start, table, "infinite")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_quotients_at_the_ends_of_codes(dtype):
    # each page's scale is (its largest element) / 127: all values of the type up to it, for largest elements whose scales lie on,
    # beside and away from multiples of 2^17 of their last place, and ones far from 1
    tops = [127.0, 63.5, 1.0, 1.9921875, 129.0, 100.0, 3.0, 0.3, 2.0 ** -14] + ([1e-37, 1e30, 3e38] if dtype is torch.bfloat16 else [65504.0])
    n, dim, block = len(tops), 128, 64
    kinds = torch.float64
    top = torch.tensor(tops, dtype=kinds).to(dtype).to(kinds)
    steps = (torch.arange(block * dim, dtype=kinds).reshape(block, dim) + 0.5) / (block * dim)
    x = top[:, None, None] * steps[None]  # within a code's half of every multiple
    half = (torch.arange(256 * 32, dtype=torch.int64).reshape(block, dim) % 255 - 127).to(kinds) + 0.5
    y = (top[:, None, None] / 127 * half).clamp(-top[:, None, None], top[:, None, None])  # at the ends of codes, rounded to the type
    y[:, 0, 0] = top
    x[:, 0, 0] = -top
    cache, _, _, cu, start, table = fresh([(0, block)] * n, 1, dim, block, dtype)
    rows = lambda a: a.reshape(n * block, 1, dim).to(dtype).to(DEV)  # noqa: E731
    check(cache, rows(x), rows(y), cu, start, table, "ends")


def test_strided_views_missing_pages_and_positions_past_the_table():
    cache, k, v, cu, start, table = fresh([(40, 30), (0, 130)], 2, 64, 64, torch.float16)
    rows = torch.full((k.shape[0], 7, 2, 80), float("nan"), dtype=k.dtype, device=DEV)
    rows[:, 2, :, 3:67], rows[:, 5, :, 9:73] = k, v
    table[1, 1] = -1
    table[0, 1] = cache[0].shape[0]
    check(cache, rows[:, 2, :, 3:67], rows[:, 5, :, 9:73], cu, start, table, "missing")
    check(cache, k, v, cu, start, table[:, :2].contiguous(), "past the table")


def test_token_by_token_reaches_the_whole_cache_once():
    # each step appends one token to each request; another order of the same pages gives the same codes
    cache, k, v, cu, start, table = fresh([(0, 70), (0, 70), (0, 70)], 2, 64, 32, torch.bfloat16)
    step = torch.arange(4, dtype=torch.int32, device=DEV)
    want = cache
    for i in range(70):
        rows = torch.tensor([i, 70 + i, 140 + i], device=DEV)
        at = torch.full((3,), i, dtype=torch.int32, device=DEV)
        kk, vv = k[rows], v[rows]
        want = append(want, kk, vv, step.cpu(), at.cpu(), table.cpu())
        qnn.kv_append(cache, kk, vv, step, at, table)
    assert all(torch.equal(a.cpu(), b) for a, b in zip(cache, want))
    # what is read back is within half a step of the last scale, and one more for each time that a block was rescaled
    back, _ = qnn.kv_gather(cache, cu, start, table, 210, torch.float16)
    assert (back.float() - k.float()).abs().max() < 4 * cache[1].max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,block", [(64, 32), (96, 96), (128, 64), (192, 128), (256, 256)])
def test_gather(dim, block, dtype):
    requests = [(300, 0), (5, 0), (0, 0), (block, 0), (2 * block + 1, 0)]
    cache, _, _, lengths, table = case(requests, 2, dim, block, dtype, 3)
    first = torch.tensor([37, 0, 0, block - 1, 0], dtype=torch.int32, device=DEV)
    counts = (lengths - first).clamp(min=0)
    cu = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()
    T = int(cu[-1])
    k, v = qnn.kv_gather(cache, cu, first, table, T, dtype)
    for r in range(len(requests)):
        for i in range(int(counts[r])):
            t = int(first[r]) + i
            p = int(table[r, t // block])
            row = int(cu[r]) + i
            if i in (0, 1, int(counts[r]) // 2, int(counts[r]) - 1):
                assert torch.equal(k[row], (cache[0][p, :, t % block].float() * cache[1][p][:, None]).to(dtype))
                assert torch.equal(v[row], (cache[2][p, :, :, t % block].float() * cache[3][p][:, None]).to(dtype))
    table[0, 0] = 1 << 30  # no such page: zeros
    k, _ = qnn.kv_gather(cache, cu, first, table, T, dtype)
    assert (k[: max(0, min(int(counts[0]), block - 37))] == 0).all()


def test_refusals():
    cache, k, v, cu, start, table = fresh([(3, 2)], 2, 64, 32, torch.bfloat16)
    f = qnn.kv_append
    for bad in (lambda: f(cache[:3], k, v, cu, start, table), lambda: f(cache, k.float(), v, cu, start, table), lambda: f(cache, k, v.half(), cu, start, table),
                lambda: f(cache, k, v, cu.long(), start, table), lambda: f(cache, k[:, :1], v, cu, start, table), lambda: f(cache, k, v[:1], cu, start, table),
                lambda: f(cache, k, v, cu[:1], start, table), lambda: f(cache, k, v, cu, start, table[0]), lambda: f(3, k, v, cu, start, table),
                lambda: f((cache[0].float(), *cache[1:]), k, v, cu, start, table), lambda: f((cache[0], cache[1], cache[0], cache[3]), k, v, cu, start, table),
                lambda: f(cache, k.transpose(1, 2), v, cu, start, table), lambda: f(cache, k, v, cu.cpu(), start, table),
                lambda: qnn.kv_gather(cache, cu, start, table, -1, torch.float16), lambda: qnn.kv_gather(cache, cu, start, table, 3, torch.float32)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    odd = qnn.new_kv_cache(2, 2, 80, 32)
    z = torch.zeros(2, 2, 80, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(qnn.QnnError, match="QNN_EINVAL"):
        f(odd, z, z, cu, start, table)  # a head size that the kernels do not have
    odd = qnn.new_kv_cache(2, 2, 64, 16)
    with pytest.raises(qnn.QnnError, match="QNN_EINVAL"):
        f(odd, k, v, cu, start, table)  # a page of 16 tokens
    f(cache, k[:0], v[:0], torch.zeros_like(cu), start, table)

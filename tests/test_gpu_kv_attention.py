"""Attention over the 8-bit cache against the definition in 64 bits."""
import math

import pytest
import torch

import paper_1806_08342_amd as qnn
from lm_reference import DEV, append, assert_close, attend, case, half_ulp

pytestmark = pytest.mark.gpu


def check(cache, q, cu, lengths, table, what="", **kw):
    out, lse = qnn.kv_attention(cache, q, cu, lengths, table, with_lse=True, **kw)
    kw.pop("max_queries", None)
    want, want_lse, spread = attend(cache, q, cu.cpu(), lengths.cpu(), table.cpu(), **kw)
    # one rounding of the result; each probability rounded to binary16 (2^-11); scores of size up to 100 in binary32 and the
    # exponential and the sum give another 2^-14 of what is averaged; channels that average to little: 2^-30; binary16's last step
    # is 2^-24
    last = 2.0 ** -25 if q.dtype == torch.float16 else 0.0
    assert_close(out, want, 1.01 * half_ulp(q.dtype) * want.abs() + (2.0 ** -11 + 2.0 ** -13) * spread + 2.0 ** -30 + last, what)
    rows = int(cu[-1])
    seen = torch.isfinite(want_lse[:rows])
    assert torch.equal(torch.isfinite(lse[:rows].cpu()), seen) and (lse[:rows].cpu()[~seen] == -math.inf).all()
    assert ((lse[:rows].cpu().double() - want_lse[:rows])[seen].abs() < 1e-4).all()
    return out


LENGTHS = [(1, 1), (2, 1), (31, 1), (32, 1), (33, 1), (63, 1), (64, 1), (65, 1), (0, 0), (255, 1), (256, 1), (257, 1), (700, 1)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("block", [32, 64, 96, 128])
def test_single_tokens(dim, block, dtype):
    check(*case(LENGTHS, 2, dim, block, dtype, dim + block, q_heads=6), (dim, block), max_queries=1)


@pytest.mark.parametrize("group", [1, 2, 3, 5, 7, 8, 12, 16, 17, 33, 64, 70])
def test_groups_of_heads(group):
    for dim in (64, 128, 256):
        check(*case([(100, 1), (300, 1), (513, 1), (64, 1)], 1, dim, 64, torch.bfloat16, group, q_heads=group), (group, dim), max_queries=1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,block", [(64, 32), (96, 64), (128, 64), (128, 32), (192, 128), (256, 64), (256, 32)])
def test_prompts_and_drafts(dim, block, dtype):
    requests = [(1, 1), (7, 7), (64, 64), (65, 65), (200, 200), (0, 0), (333, 40), (500, 4), (129, 128), (90, 1)]
    check(*case(requests, 2, dim, block, dtype, 5, q_heads=4), (dim, block), max_queries=200)


@pytest.mark.parametrize("window", [1, 2, 31, 64, 100, 1000])
def test_windows(window):
    for dim, block, group in ((64, 32, 7), (128, 64, 2), (256, 64, 3)):
        args = case([(700, 1), (65, 4), (300, 300), (3, 3), (0, 0), (128, 9), (129, 70)], 2, dim, block, torch.bfloat16, window, q_heads=2 * group)
        check(*args, (window, dim), window=window, max_queries=300)
        few = case([(700, 1), (65, 4), (3, 3), (0, 0), (128, 4)], 2, dim, block, torch.bfloat16, window, q_heads=2 * group)
        check(*few, (window, dim, "few"), window=window, max_queries=4)


@pytest.mark.parametrize("n,length", [(1, 5000), (3, 9001), (1, 40000)])
def test_contexts_divided_over_workgroups(n, length):
    check(*case([(length, n), (length // 3, n), (n, n)], 2, 128, 64, torch.bfloat16, 9, q_heads=10), (n, length), max_queries=n)
    check(*case([(length, n)], 1, 64, 32, torch.float16, 9, q_heads=16), (n, length), max_queries=n, window=length // 2)


def test_fewer_keys_than_queries_and_missing_pages():
    # queries that stand before the first token see nothing; so do those whose pages are not there
    cache, q, cu, lengths, table = case([(100, 40), (50, 50), (200, 3)], 2, 64, 64, torch.bfloat16, 1, q_heads=4)
    lengths[0] = 10
    lengths[1] = 0
    out = check(cache, q, cu, lengths, table, "short", max_queries=50)
    assert (out[:30] == 0).all() and (out[40:90] == 0).all()
    table[2, 1], table[2, 3], table[0, 0] = -1, 1 << 30, -7
    check(cache, q, cu, lengths, table, "missing", max_queries=50)


def test_unused_places_may_hold_anything():
    # scales of other pages NaN, places past a request's end with the largest codes
    cache, q, cu, lengths, table = case([(70, 1), (5, 5), (200, 130)], 2, 128, 64, torch.bfloat16, 2, q_heads=8)
    used = torch.unique(table[table >= 0]).long()
    rest = torch.ones(cache[0].shape[0], dtype=torch.bool, device=DEV)
    rest[used] = False
    cache[1][rest], cache[3][rest] = float("nan"), float("inf")
    want = qnn.kv_attention(cache, q, cu, lengths, table)
    for r, n in enumerate(lengths.tolist()):
        if n % 64:
            p = int(table[r, n // 64])
            cache[0][p, :, n % 64:], cache[2][p, :, :, n % 64:] = -128, 127
    assert torch.isfinite(want).all() and torch.equal(want, qnn.kv_attention(cache, q, cu, lengths, table))


def test_large_small_and_no_numbers_in_queries():
    cache, q, cu, lengths, table = case([(300, 2), (64, 3)], 1, 64, 32, torch.bfloat16, 3, q_heads=2)
    q[0] *= 1e30
    q[1] *= 1e-30
    q[2, 0] = 0.0
    q[3, 0, 5] = float("nan")
    out = qnn.kv_attention(cache, q, cu, lengths, table, max_queries=3)
    assert torch.isnan(out[3, 0]).all() and torch.isfinite(out[3, 1]).all()
    ok = torch.tensor([1, 2, 4], device=DEV)
    want, _, spread = attend(cache, q, cu.cpu(), lengths.cpu(), table.cpu())
    assert_close(out[ok], want[ok.cpu()], 1.01 * 2.0 ** -8 * want[ok.cpu()].abs() + 2.0 ** -10 * spread[ok.cpu()], "sizes")
    # scores of 1e30: the largest takes all
    assert_close(out[0], want[0], 1.01 * 2.0 ** -8 * want[0].abs() + 1e-6, "one takes all")


def test_strides_scale_outputs_and_more_queries_than_told():
    cache, q, cu, lengths, table = case([(90, 20), (200, 1), (333, 90)], 2, 128, 64, torch.float16, 4, q_heads=6)
    rows = torch.full((q.shape[0], 11, 140), float("nan"), dtype=q.dtype, device=DEV)
    rows[:, 2:8, 7:135] = q
    out = torch.empty_like(q)
    want = check(cache, q, cu, lengths, table, "scale", scale=0.3, max_queries=90)
    assert qnn.kv_attention(cache, rows[:, 2:8, 7:135], cu, lengths, table, scale=0.3, max_queries=90, out=out) is out and torch.equal(out, want)
    for told in (1, 4, None):
        got, more = qnn.kv_attention(cache, q, cu, lengths, table, scale=0.3, max_queries=told), qnn.kv_attention(cache, q, cu, lengths, table, window=50, max_queries=told)
        ref, _, spread = attend(cache, q, cu.cpu(), lengths.cpu(), table.cpu(), scale=0.3)
        assert_close(got, ref, 1.01 * 2.0 ** -11 * ref.abs() + 2.0 ** -10 * spread, told)
        ref, _, spread = attend(cache, q, cu.cpu(), lengths.cpu(), table.cpu(), window=50)
        assert_close(more, ref, 1.01 * 2.0 ** -11 * ref.abs() + 2.0 ** -10 * spread, told)


def test_parts_of_a_context_join_by_their_sums():
    cache, q, cu, lengths, table = case([(300, 1)], 2, 64, 64, torch.bfloat16, 6, q_heads=4)
    whole, total = qnn.kv_attention(cache, q, cu, lengths, table, with_lse=True)
    a, la = qnn.kv_attention(cache, q, cu, torch.full_like(lengths, 128), table, with_lse=True)
    b, lb = qnn.kv_attention(cache, q, cu, lengths - 128, table[:, 2:].contiguous(), with_lse=True)
    assert ((torch.logaddexp(la, lb) - total).abs() < 1e-4).all()
    joined = a.float() * torch.exp(la - total)[..., None] + b.float() * torch.exp(lb - total)[..., None]
    assert (joined - whole.float()).abs().max() < 2.0 ** -7 * whole.float().abs().max()


def test_results_repeat_on_any_stream_and_in_a_graph():
    for requests, most in (([(5000, 1), (17, 1), (900, 1)], 1), ([(300, 300), (70, 5)], 300)):
        cache, q, cu, lengths, table = case(requests, 2, 128, 64, torch.bfloat16, 8, q_heads=8)
        want = qnn.kv_attention(cache, q, cu, lengths, table, max_queries=most)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = [qnn.kv_attention(cache, q, cu, lengths, table, max_queries=most) for _ in range(3)]
        side.synchronize()
        assert all(torch.equal(want, y) for y in again)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = qnn.kv_attention(cache, q, cu, lengths, table, max_queries=most)
        for i in range(3):
            q.mul_(-1.0)
            lengths.sub_(1)
            want = qnn.kv_attention(cache, q, cu, lengths, table, max_queries=most)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), i


def test_the_cache_that_append_writes():
    # a prompt, then single tokens, against attention over what the definition of the cache holds
    cache, _, cu, lengths, table = case([(150, 140)], 2, 64, 32, torch.bfloat16, 10)
    g = torch.Generator().manual_seed(1)
    kv = torch.randn(150, 2, 2, 64, generator=g).to(torch.bfloat16).to(DEV)
    zero = torch.zeros(1, dtype=torch.int32, device=DEV)
    want = append(cache, kv[:140, 0], kv[:140, 1], cu.cpu(), zero.cpu(), table.cpu())
    qnn.kv_append(cache, kv[:140, 0], kv[:140, 1], cu, zero, table)
    one = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    for i in range(140, 150):
        want = append(want, kv[i:i + 1, 0], kv[i:i + 1, 1], one.cpu(), zero.cpu() + i, table.cpu())
        qnn.kv_append(cache, kv[i:i + 1, 0], kv[i:i + 1, 1], one, zero + i, table)
        q = torch.randn(1, 6, 64, generator=g).to(torch.bfloat16).to(DEV)
        out = check(cache, q, one, zero + i + 1, table, i, max_queries=1)
        ref, _, spread = attend(want, q, one.cpu(), zero.cpu() + i + 1, table.cpu())
        assert_close(out, ref, 1.01 * 2.0 ** -8 * ref.abs() + 2.0 ** -10 * spread, "definition's cache")


def test_offsets_past_32_bits():
    # pages whose codes lie more than 2^32 bytes into the arrays
    heads, dim, block, pages = 8, 256, 256, 8300
    cache = qnn.new_kv_cache(pages, heads, dim, block)
    assert cache[0].numel() > 1 << 32
    g = torch.Generator().manual_seed(0)
    zero, start = torch.zeros(1, dtype=torch.int32, device=DEV), torch.tensor([0, 300], dtype=torch.int32, device=DEV)
    kv = torch.randn(300, 2, heads, dim, generator=g).to(torch.bfloat16).to(DEV)
    high, low = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device=DEV), torch.tensor([[1, 0]], dtype=torch.int32, device=DEV)
    outs = []
    for table in (high, low):
        qnn.kv_append(cache, kv[:, 0], kv[:, 1], start, zero, table)
        q = kv[:, 0, :, :].contiguous()
        outs.append((qnn.kv_attention(cache, q[-1:], start.clamp(max=1), zero + 300, table, max_queries=1),
                     qnn.kv_attention(cache, q, start, zero + 300, table, max_queries=300), *qnn.kv_gather(cache, start, zero, table, 300, torch.bfloat16)))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert int(cache[0][2:-2].count_nonzero()) == 0  # nothing else was written


def test_refusals():
    cache, q, cu, lengths, table = case([(70, 2)], 2, 64, 32, torch.bfloat16, 0, q_heads=4)
    f = qnn.kv_attention
    for bad in (lambda: f(cache, q.float(), cu, lengths, table), lambda: f(cache, q[0], cu, lengths, table), lambda: f(cache, q[..., :32], cu, lengths, table),
                lambda: f(cache, q, cu.long(), lengths, table), lambda: f(cache, q, cu, lengths[:0], table), lambda: f(cache, q, cu, lengths, table.float()),
                lambda: f(cache, q.cpu(), cu, lengths, table), lambda: f(cache, q, cu, lengths, table, out=q.half()), lambda: f(cache, q, cu, lengths, table, out=q[:1]),
                lambda: f(cache, q, cu, lengths, table, scale="x")):
        with pytest.raises((TypeError, ValueError)):
            bad()
    for bad in (lambda: f(cache, q[:, :3].contiguous(), cu, lengths, table), lambda: f(cache, q, cu, lengths, table, window=-1),
                lambda: f(cache, q, cu, lengths, table, scale=float("nan"))):
        with pytest.raises(qnn.QnnError, match="QNN_EINVAL"):
            bad()
    assert f(cache, q[:0], torch.zeros_like(cu), lengths, table).shape == (0, 4, 64)
    long = case([(9000, 1)], 1, 64, 64, torch.bfloat16, 0, q_heads=1)
    with pytest.raises(qnn.QnnError, match="QNN_EINVAL"):
        f(*long, max_queries=1, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))  # too little scratch


@pytest.mark.parametrize("dim", [64, 96, 128])
def test_many_prompts_at_once(dim):
    # rows enough for workgroups of eight waves; requests with few rows among them go to the other kernel
    requests = [(70 + i % 13, 70 + i % 13) if i % 7 else (90 + i, 1 + i % 3) for i in range(36)] + [(0, 0), (500, 20)]
    check(*case(requests, 8, dim, 64, torch.bfloat16, dim, q_heads=32), dim, max_queries=82)


@pytest.mark.parametrize("dim,group", [(64, 8), (128, 4), (256, 3)])
def test_hundreds_of_rows_over_a_long_context(dim, group):
    # one context is divided over workgroups and joined, with the kernels for many rows too
    args = case([(9001, 40), (700, 33), (3000, 1)], 1, dim, 64, torch.bfloat16, 7, q_heads=group)
    check(*args, (dim, group), max_queries=40)
    check(*args, (dim, group, "window"), max_queries=40, window=3000)


@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("dim", [64, 256])
def test_value_scales_far_apart_and_zero(dim, block):
    # accumulators stand in units of a page's value scale: rows that see small pages only stay exact, pages of zeros count in the sum
    for requests, most in (([(300, 300), (200, 150)], 300), ([(300, 1), (200, 3)], 3)):
        cache, q, cu, lengths, table = case(requests, 2, dim, block, torch.float16, block, q_heads=4)
        for r in range(2):
            for j, by in enumerate((1e-4, 1.0, 300.0, 0.0, 1e-3, 1.0, 1e-2)):
                if j < table.shape[1] and table[r, j] >= 0:
                    cache[3][int(table[r, j])] *= by
        check(cache, q, cu, lengths, table, (dim, block, most), max_queries=most)
        cache[1][:] = 0.0  # all scores equal
        check(cache, q, cu, lengths, table, (dim, block, most, "keys"), max_queries=most)


def test_negative_scale_factor_and_large_scores():
    for requests, most in (([(300, 300)], 300), ([(300, 2)], 2)):
        args = case(requests, 1, 64, 64, torch.bfloat16, 4, q_heads=2)
        check(*args, most, max_queries=most, scale=-0.2)
        args[0][1].mul_(20.0)  # scores of hundreds: the running maximum moves on and on
        out = qnn.kv_attention(*args, max_queries=most)
        want, _, spread = attend(args[0], args[1], *(t.cpu() for t in args[2:]))
        # scores of size 400 in binary32: an error of 400 * 2^-22 in the exponent is one of 1e-4 of what is averaged.  Where one
        # token takes nearly all, the others' probabilities are below binary16's normal numbers: 2^-25 of the 2^2 that 1 is at least
        # held as, for each of 300 values of at most 127 * 0.025
        assert_close(out, want, 1.01 * 2.0 ** -8 * want.abs() + (2.0 ** -11 + 4e-4) * spread + 300 * 127 * 0.025 * 2.0 ** -27, "large")

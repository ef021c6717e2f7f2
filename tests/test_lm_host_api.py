"""Operators of quantized language models: what the host checks and computes, without a GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_1806_08342_amd as qnn
from lm_reference import unpack

EINVAL = 1


@pytest.fixture(scope="module")
def lib():
    return qnn.load_library()


class Cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("ks", C.c_void_p), ("v", C.c_void_p), ("vs", C.c_void_p), ("pages", C.c_int64), ("heads", C.c_int32), ("dim", C.c_int32),
                ("block", C.c_int32)]


def cache(**kw):
    return Cache(**{**dict(k=4096, ks=4096, v=4096, vs=4096, pages=10, heads=2, dim=64, block=64), **kw})


def test_bad_arguments_are_refused_before_anything_is_launched(lib):
    p, null = C.c_void_p(4096), C.c_void_p(0)  # never dereferenced
    w4 = lambda **kw: lib.qnn_w4_matmul(*[kw.get(k, d) for k, d in [  # noqa: E731
        ("x", p), ("ldx", 128), ("codes", p), ("scales", p), ("zeros", null), ("bias", null), ("M", 4), ("N", 8), ("K", 128), ("group", 128), ("type", 0),
        ("y", p), ("ldy", 8), ("ws", null), ("wsb", 0), ("stream", None)]])
    for bad in (dict(M=-1), dict(N=0), dict(K=127), dict(K=0), dict(group=16), dict(group=0), dict(group=-32), dict(type=2), dict(x=null), dict(codes=null),
                dict(scales=null), dict(y=null), dict(ldx=127), dict(ldy=7)):
        assert w4(**bad) == EINVAL, bad
    assert w4(M=0, x=null, y=null) == 0
    c = cache()
    app = lambda **kw: lib.qnn_kv_append(*[kw.get(k, d) for k, d in [  # noqa: E731
        ("cache", C.byref(c)), ("k", p), ("kt", 128), ("kh", 64), ("v", p), ("vt", 128), ("vh", 64), ("type", 0), ("cu", p), ("start", p), ("table", p), ("width", 4),
        ("requests", 3), ("tokens", 3), ("stream", None)]])
    broken = [cache(dim=80), cache(dim=512), cache(block=16), cache(block=288), cache(block=0), cache(heads=0), cache(pages=-1), cache(k=None), cache(vs=4100)]
    for bad in [dict(type=3), dict(k=null), dict(v=null), dict(cu=null), dict(start=null), dict(table=null), dict(width=-1), dict(requests=-1), dict(tokens=-1),
                dict(cache=None)] + [dict(cache=C.byref(b)) for b in broken]:
        assert app(**bad) == EINVAL, bad
    assert app(tokens=0, k=null, v=null) == 0 and app(requests=0, cu=null) == 0
    gat = lambda **kw: lib.qnn_kv_gather(*[kw.get(k, d) for k, d in [  # noqa: E731
        ("cache", C.byref(c)), ("cu", p), ("first", p), ("table", p), ("width", 4), ("requests", 3), ("tokens", 3), ("type", 1), ("k", p), ("v", p), ("stream", None)]])
    for bad in [dict(type=-1), dict(k=null), dict(v=null), dict(first=null), dict(tokens=-5)] + [dict(cache=C.byref(b)) for b in broken]:
        assert gat(**bad) == EINVAL, bad
    att = lambda **kw: lib.qnn_kv_attention(*[kw.get(k, d) for k, d in [  # noqa: E731
        ("cache", C.byref(c)), ("q", p), ("qt", 256), ("qh", 64), ("heads", 4), ("type", 0), ("cu", p), ("lengths", p), ("table", p), ("width", 4), ("requests", 3),
        ("tokens", 3), ("scale", 0.1), ("window", 0), ("most", 1), ("out", p), ("lse", null), ("ws", null), ("wsb", 0), ("stream", None)]])
    for bad in [dict(heads=3), dict(heads=0), dict(type=2), dict(q=null), dict(out=null), dict(lengths=null), dict(cu=null), dict(window=-1), dict(scale=float("inf")),
                dict(requests=-2), dict(tokens=-1), dict(out=C.c_void_p(4098)), dict(width=1 << 40)] + [dict(cache=C.byref(b)) for b in broken]:
        assert att(**bad) == EINVAL, bad
    assert att(tokens=0, q=null, out=null) == 0
    wide = 1000  # a long context of few heads is divided, which takes scratch
    assert lib.qnn_kv_attention_workspace_bytes(C.byref(c), 4, wide, 3, 3, 0, 1) > 0
    assert att(width=wide) == EINVAL and lib.qnn_kv_attention_workspace_bytes(C.byref(c), 3, wide, 3, 3, 0, 1) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("asymmetric", [False, True])
@pytest.mark.parametrize("rows,cols,group", [(3, 64, 32), (5, 250, 64), (1, 2, 32), (4, 100, 128)])
def test_grouped_quantizer(rows, cols, group, asymmetric, dtype):
    rng = np.random.default_rng(rows + cols)
    w = (rng.normal(0.02, 0.1, (rows, cols)) * rng.uniform(0.2, 3.0, (rows, 1))).astype(np.float32)
    w[0, :32] = 0.0
    codes, scales, zeros = qnn.quantize_weights_grouped(w, group, dtype, asymmetric)
    groups = -(-cols // group)
    assert codes.shape == (rows, cols // 2) and scales.shape == (groups, rows) and scales.dtype == dtype and (zeros is not None) == asymmetric
    c, at = unpack(codes), torch.arange(cols) // group
    s = scales.double()[at].t()
    z = zeros.double()[at].t() if asymmetric else 0.0
    assert c.min() >= (-8 if asymmetric else -7) and c.max() <= 7
    # half a step, and what the ends of the range lose by the scale's own rounding (2^-9 of 15 steps) and the zero-point's (half a step)
    off = ((c - z) * s - torch.from_numpy(w).double()).abs()
    assert (off <= s * (0.5 + 15 * 2.0 ** -9 + (0.5 if asymmetric else 0.0))).all()
    if not asymmetric:
        for g in range(groups):
            part = torch.from_numpy(w[:, g * group:(g + 1) * group])
            peak = part.abs().amax(1)
            want = torch.where(peak > 0, (peak.double() / 7.0).float(), 1.0).to(dtype)
            assert torch.equal(scales[g], want)


def test_grouped_quantizer_refuses():
    w = np.ones((4, 64), np.float32)
    for bad in (lambda: qnn.quantize_weights_grouped(w, 16), lambda: qnn.quantize_weights_grouped(w, 0), lambda: qnn.quantize_weights_grouped(w[:, :63], 32),
                lambda: qnn.quantize_weights_grouped(w * np.nan, 32), lambda: qnn.quantize_weights_grouped(w * 1e9, 32, torch.float16)):
        with pytest.raises(qnn.QnnError):
            bad()
    for bad in (lambda: qnn.quantize_weights_grouped(w[0], 32), lambda: qnn.quantize_weights_grouped(w, 32, torch.float32)):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("bad", [None, 3, torch.zeros(4, 64), torch.zeros(4, 64, dtype=torch.bfloat16)])
def test_tensors_of_the_wrong_kind(bad):
    with pytest.raises((TypeError, ValueError)):
        qnn.w4_matmul(bad, bad, bad, 32)
    with pytest.raises((TypeError, ValueError)):
        qnn.kv_append((bad,) * 4, bad, bad, bad, bad, bad)
    with pytest.raises((TypeError, ValueError)):
        qnn.kv_attention((bad,) * 4, bad, bad, bad, bad, scale=1.0)

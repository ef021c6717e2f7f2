"""Limits of the operators of quantized language models, checked on the host before anything is launched."""
import ctypes as C

import pytest
import torch

import paper_1806_08342_amd as qnn
from test_lm_host_api import EINVAL, cache


@pytest.mark.parametrize("block,tokens,requests", [(32, 1 << 29, 1), (32, (1 << 29) - 32, 8), (256, 1 << 30, 1), (64, 1 << 29, 1 << 22)])
def test_calls_of_more_pages_than_a_launch_takes_are_refused(block, tokens, requests):
    lib, p, c = qnn.load_library(), C.c_void_p(4096), cache(block=block)
    assert lib.qnn_kv_append(C.byref(c), p, 128, 64, p, 128, 64, 0, p, p, p, 4, requests, tokens, None) == EINVAL
    assert lib.qnn_kv_gather(C.byref(c), p, p, p, 4, requests, tokens, 0, p, p, None) == EINVAL


def test_products_of_more_rows_than_a_launch_takes_are_refused():
    lib, p = qnn.load_library(), C.c_void_p(4096)
    most = (1 << 28) - 32
    assert qnn.w4_matmul_plan(1, most, 64) and not qnn.w4_matmul_plan(1, most + 1, 64)
    assert lib.qnn_w4_matmul(p, 64, p, p, None, None, 1, most + 1, 64, 128, 0, p, most + 1, None, 0, None) == EINVAL


def test_tensors_that_require_grad_are_refused():
    # there is no backward pass: a result cut off from its inputs would go unnoticed
    x = torch.zeros(4, 64, dtype=torch.bfloat16, requires_grad=True)
    kv = torch.zeros(4, 2, 64, dtype=torch.bfloat16, requires_grad=True)
    calls = (lambda: qnn.w4_matmul(x, x, x, 32), lambda: qnn.kv_append((kv,) * 4, kv, kv, kv, kv, kv), lambda: qnn.kv_attention((kv,) * 4, kv, kv, kv, kv))
    for call in calls:
        with pytest.raises(RuntimeError, match="no backward pass"):
            call()
        with torch.no_grad(), pytest.raises(TypeError):  # (no device tensors)
            call()

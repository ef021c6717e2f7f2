"""The example of a decoder in 8-bit floating point: norms, products, cache, attention and experts as one program runs them."""

import importlib.util
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    folder = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")
    spec = importlib.util.spec_from_file_location("experts_step", os.path.join(folder, "experts_step.py"))
    module = importlib.util.module_from_spec(spec)
    before = list(sys.path)
    spec.loader.exec_module(module)
    sys.path[:] = before
    return module


PROMPTS = [[5], list(range(40)), list(range(100, 163))]


@pytest.mark.parametrize("width, heads, kv_heads, experts, inner", [(1024, 8, 2, 8, 384), (576, 3, 1, 5, 80)])
def test_replayed_steps_equal_launched_ones(example, width, heads, kv_heads, experts, inner):
    make = lambda: example.Decoder(2, width, heads, kv_heads, experts, inner, capacity=96, requests=3)  # noqa: E731
    first = example.generate(make(), PROMPTS, 20, graph=True)
    second = example.generate(make(), PROMPTS, 20, graph=False)
    assert first[0].shape == (3, 21) and torch.isfinite(first[1]).all()
    assert torch.equal(first[0], second[0]) and torch.equal(first[1], second[1])


def test_requests_together_equal_those_alone(example):
    # Every product of up to 16 rows goes through the same kernel, a row of it by itself; the caches of the two start out the same.
    whole = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    model = example.Decoder(1, 1024, capacity=64, requests=2)
    both = model.rows(whole([7, 9]), whole([0, 1, 2]), whole([0, 0]), whole([1, 1]), 1)
    model = example.Decoder(1, 1024, capacity=64, requests=2)
    alone = [model.rows(whole([t]), whole([0, 1, 1] if r == 0 else [0, 0, 1]), whole([0, 0]), whole([1, 0] if r == 0 else [0, 1]), 1) for r, t in enumerate((7, 9))]
    assert torch.equal(both, torch.cat(alone))


def test_logits_are_near_those_of_float32_without_a_cache(example):
    # Two experts of which both are taken, so that no token's router can choose others.  A code is off by at most 1/16 of its value, evenly
    # within a step: (1/16) / sqrt(3) = 3.6 % at the lower end of a power of two and half that at the upper, 2.7 % in the mean square.
    # Six products take codes one after the other (qkv, out, router, up, down, head), and up's error counts twice (both halves): under
    # sqrt(7) * 2.7 = 7 % were nothing carried past them; the stream carries most of a row past each of them, while the softmax of the
    # attention and the router may enlarge an error of theirs.  The cache's 1 % of decode_step and bfloat16's 0.2 % are small beside it.
    model = example.Decoder(2, 1024, experts=2, capacity=128, requests=3)
    tokens, logits = example.generate(model, PROMPTS, 12)
    for r in range(3):
        plain = model.plain_logits(torch.tensor(PROMPTS[r] + tokens[r, :-1].tolist()))
        assert (logits[r] - plain).norm() <= 0.1 * plain.norm()

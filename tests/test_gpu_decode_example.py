"""The decoding example: 4-bit products, cache and attention as one program runs them."""

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_step.py")
    spec = importlib.util.spec_from_file_location("decode_step", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("width, heads, kv_heads", [(1024, 8, 2), (768, 8, 8), (576, 3, 1)])
def test_generated_logits_are_near_those_of_float32_without_a_cache(example, width, heads, kv_heads):
    # Against the same 4-bit weights: 8-bit keys and values (a block's largest of 32 * dim normal numbers is about 4.3 of their
    # standard deviations: steps of 4.3 / 127, errors of 4.3 / 127 / sqrt(12) = 1 % of a value), and some ten roundings to bfloat16
    # (0.2 % each).  Two layers of both on top of each other: about 2 %; the bound allows twice that and some.
    model = example.Decoder(2, width, heads, kv_heads, capacity=128, requests=3)
    prompts = [[(31 * i * i + 17 * r) % example.VOCABULARY for i in range(n)] for r, n in enumerate((1, 45, 96))]
    tokens, logits = example.generate(model, prompts, 12)
    assert tokens.shape == (3, 13)
    for r in range(3):
        plain = model.plain_logits(torch.tensor(prompts[r] + tokens[r, :-1].tolist()))
        assert (logits[r] - plain).norm() <= 0.05 * plain.norm()


def test_replayed_steps_equal_launched_ones(example):
    prompts = [[5], list(range(40)), list(range(100, 163))]
    first = example.generate(example.Decoder(2, 1024, capacity=96, requests=3), prompts, 20, graph=True)
    second = example.generate(example.Decoder(2, 1024, capacity=96, requests=3), prompts, 20, graph=False)
    assert torch.equal(first[0], second[0]) and torch.equal(first[1], second[1])

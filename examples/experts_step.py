"""Text generation with 8-bit floating point on both sides of every product, and experts: a small decoder whose weights are random.

    python examples/experts_step.py [--layers 2] [--width 1024] [--heads 8] [--kv_heads 2] [--experts 8] [--inner 384] [--requests 3] [--tokens 16]

The prompts and the steps run as in decode_step.py, the steps from a captured graph.  A layer is

    f8_rmsnorm -> f8_matmul (queries, keys and values) -> kv_append -> kv_attention -> f8_quantize -> f8_matmul
    -> f8_rmsnorm (which adds) -> f8_matmul (the router, in float32) -> f8_moe

and torch does nothing between.  What is printed at the end are the tokens, the time of a step launched one kernel after the other and
replayed, and how far the logits of the last step are from those of the same weights in float32 without a cache (8-bit activations are
3 % off each, and a token whose router hesitates may go to another expert)."""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1806_08342_amd as qnn  # noqa: E402
from decode_step import BLOCK, DTYPE, VOCABULARY, generate, norm, step_time  # noqa: E402

TOP_K, EPS = 2, 1e-6


class Weights:
    """Matrices [..., outputs, inputs], quantized on the host; `plain` is what their codes stand for."""

    def __init__(self, *shape, seed):
        w = torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * shape[-1] ** -0.5
        codes, scales = qnn.quantize_weights_blocks(w.numpy())
        self.plain = codes.float() * scales.repeat_interleave(128, -2)[..., :shape[-2], :].repeat_interleave(128, -1)[..., :shape[-1]]
        self.parts = codes.cuda(), scales.cuda()

    def __call__(self, codes, scales, dtype=DTYPE):
        return qnn.f8_matmul(codes, scales, *self.parts, dtype=dtype)


class Decoder:
    def __init__(self, layers=2, width=1024, heads=8, kv_heads=2, experts=8, inner=384, capacity=512, requests=3):
        self.dim, self.heads, self.kv_heads, self.inner = width // heads, heads, kv_heads, inner
        self.embedding = torch.randn(VOCABULARY, width, generator=torch.Generator().manual_seed(0)).to(DTYPE).cuda()
        self.layers = [{"qkv": Weights((heads + 2 * kv_heads) * self.dim, width, seed=10 * i + 1), "out": Weights(width, width, seed=10 * i + 2),
                        "router": Weights(experts, width, seed=10 * i + 3), "up": Weights(experts, 2 * inner, width, seed=10 * i + 4),
                        "down": Weights(experts, width, inner, seed=10 * i + 5)} for i in range(layers)]
        self.head = Weights(VOCABULARY, width, seed=9)
        pages = -(-capacity // BLOCK)  # of each request; dealt out in turn, so that a request's lie apart
        self.caches = [qnn.new_kv_cache(pages * requests, kv_heads, self.dim, BLOCK) for _ in range(layers)]
        self.table = torch.arange(pages * requests, dtype=torch.int32).reshape(pages, requests).t().contiguous().cuda()
        self.capacity = capacity

    def rows(self, tokens, cu, start, lengths, max_queries):
        """The last layer's rows for `tokens` (cu[r]:cu[r+1] are request r's), which the cache holds afterwards."""
        stream, more = self.embedding[tokens], None
        for layer, cache in zip(self.layers, self.caches):
            if more is None:
                codes, scales = qnn.f8_rmsnorm(stream, None, EPS)
            else:
                codes, scales, stream = qnn.f8_rmsnorm(more, None, EPS, residual=stream)
            qkv = layer["qkv"](codes, scales).view(len(tokens), -1, self.dim)  # views of one product, no copies
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
            qnn.kv_append(cache, k, v, cu, start, self.table)
            seen = qnn.kv_attention(cache, q, cu, lengths, self.table, max_queries=max_queries)
            more = layer["out"](*qnn.f8_quantize(seen.view(len(tokens), -1)))
            codes, scales, stream = qnn.f8_rmsnorm(more, None, EPS, residual=stream)
            logits = layer["router"](codes, scales, torch.float32)
            more = qnn.f8_moe(codes, scales, logits, *layer["up"].parts, *layer["down"].parts, TOP_K)
        return stream + more

    def logits(self, x):
        return self.head(*qnn.f8_rmsnorm(x, None, EPS))

    def plain_logits(self, tokens):
        """Logits of one request's last token: the same weights, in float32, nothing cached."""
        x, n = self.embedding[tokens].float().cpu(), len(tokens)
        hidden = torch.ones(n, n, dtype=torch.bool).triu(1)
        for layer in self.layers:
            qkv = (norm(x) @ layer["qkv"].plain.t()).view(n, -1, self.dim).transpose(0, 1)
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 0)
            k, v = (part.repeat_interleave(self.heads // self.kv_heads, 0) for part in (k, v))
            p = (q @ k.transpose(1, 2) * self.dim ** -0.5).masked_fill(hidden, -torch.inf).softmax(-1)
            x = x + (p @ v).transpose(0, 1).reshape(n, -1) @ layer["out"].plain.t()
            y = norm(x)
            best = (y @ layer["router"].plain.t()).topk(TOP_K)
            both = torch.einsum("th,enh->ten", y, layer["up"].plain)
            of_each = torch.einsum("tei,ehi->teh", torch.nn.functional.silu(both[..., :self.inner]) * both[..., self.inner:], layer["down"].plain)
            x = x + (of_each[torch.arange(n)[:, None], best.indices] * best.values.softmax(-1)[..., None]).sum(1)
        return norm(x[-1]) @ self.head.plain.t()


def main():
    parser = argparse.ArgumentParser()
    for name, value in (("layers", 2), ("width", 1024), ("heads", 8), ("kv_heads", 2), ("experts", 8), ("inner", 384), ("requests", 3), ("tokens", 16)):
        parser.add_argument("--" + name, type=int, default=value)
    args = parser.parse_args()
    model = Decoder(args.layers, args.width, args.heads, args.kv_heads, args.experts, args.inner, requests=args.requests)
    prompts = [[(31 * i * i + 17 * r) % VOCABULARY for i in range(5 + 40 * r)] for r in range(args.requests)]
    tokens, logits = generate(model, prompts, args.tokens)
    for r, row in enumerate(tokens.tolist()):
        plain = model.plain_logits(torch.tensor(prompts[r] + row[:-1]))
        error = ((logits[r] - plain).norm() / plain.norm()).item()
        print(f"request {r}: {len(prompts[r])} tokens, then {row}; last logits {100 * error:.1f} % from float32's")
    print(f"a step: {step_time(model, args.requests, False):.0f} us launched, {step_time(model, args.requests, True):.0f} us replayed")


if __name__ == "__main__":
    main()

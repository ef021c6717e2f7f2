"""Text generation with 4-bit weights and an 8-bit cache: a small decoder whose weights are random.

    python examples/decode_step.py [--layers 2] [--width 1024] [--heads 8] [--kv_heads 2] [--requests 3] [--tokens 16]

A prompt of each request goes through the layers at once, then the requests advance together, a token a step.  A layer is

    w4_matmul (queries, keys and values in one product) -> kv_append -> kv_attention -> w4_matmul -> two more for the MLP

and torch does what lies between (norms, sums, the activation).  The step of single tokens is captured into a graph: all that
changes from step to step (tokens, lengths, pages) is in device tensors.  What is printed at the end are the tokens, the time of a step launched
one kernel after the other and replayed, and how far the logits of the last step are from those of the same weights
in float32 without a cache."""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1806_08342_amd as qnn  # noqa: E402

DTYPE, GROUP, BLOCK, VOCABULARY = torch.bfloat16, 64, 32, 1000


def norm(x):
    x32 = x.float()
    return (x32 * torch.rsqrt(x32.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


class Linear:
    """A matrix [outputs, inputs], quantized on the host; `plain` is what its codes stand for."""

    def __init__(self, outputs, inputs, seed):
        w = torch.randn(outputs, inputs, generator=torch.Generator().manual_seed(seed)) * inputs ** -0.5
        codes, scales, zeros = qnn.quantize_weights_grouped(w, GROUP, DTYPE, asymmetric=True)
        low, high = (codes & 15).to(torch.int32), (codes >> 4).to(torch.int32)
        whole = torch.stack([low, high], -1).reshape(outputs, inputs)
        whole = torch.where(whole > 7, whole - 16, whole)
        spread = lambda per_group: per_group.float().t().repeat_interleave(GROUP, 1)[:, :inputs]  # noqa: E731
        self.plain = (whole - spread(zeros)) * spread(scales)
        self.parts = [part.cuda() for part in (codes, scales, zeros)]

    def __call__(self, x):
        codes, scales, zeros = self.parts
        return qnn.w4_matmul(x, codes, scales, GROUP, zeros)


class Decoder:
    def __init__(self, layers=2, width=1024, heads=8, kv_heads=2, capacity=512, requests=3):
        self.dim, self.heads, self.kv_heads, self.width = width // heads, heads, kv_heads, width
        self.embedding = torch.randn(VOCABULARY, width, generator=torch.Generator().manual_seed(0)).to(DTYPE).cuda()
        self.layers = [{"qkv": Linear((heads + 2 * kv_heads) * self.dim, width, 10 * i + 1), "out": Linear(width, width, 10 * i + 2),
                        "up": Linear(2 * width, width, 10 * i + 3), "down": Linear(width, 2 * width, 10 * i + 4)} for i in range(layers)]
        self.head = Linear(VOCABULARY, width, 9)
        pages = -(-capacity // BLOCK)  # of each request; dealt out in turn, so that a request's lie apart
        self.caches = [qnn.new_kv_cache(pages * requests, kv_heads, self.dim, BLOCK) for _ in range(layers)]
        self.table = torch.arange(pages * requests, dtype=torch.int32).reshape(pages, requests).t().contiguous().cuda()
        self.capacity = capacity

    def rows(self, tokens, cu, start, lengths, max_queries):
        """The last layer's rows for `tokens` (cu[r]:cu[r+1] are request r's), which the cache holds afterwards."""
        x, split = self.embedding[tokens], self.heads * self.dim
        for layer, cache in zip(self.layers, self.caches):
            qkv = layer["qkv"](norm(x)).view(len(tokens), -1, self.dim)  # views of one product, no copies
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
            qnn.kv_append(cache, k, v, cu, start, self.table)
            seen = qnn.kv_attention(cache, q, cu, lengths, self.table, max_queries=max_queries)
            x = x + layer["out"](seen.view(len(tokens), split))
            x = x + layer["down"](torch.nn.functional.silu(layer["up"](norm(x))))
        return x

    def logits(self, x):
        return self.head(norm(x))

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
            x = x + torch.nn.functional.silu(norm(x) @ layer["up"].plain.t()) @ layer["down"].plain.t()
        return norm(x[-1]) @ self.head.plain.t()


def generate(model, prompts, steps, graph=True):
    """Greedy tokens [requests, steps + 1] after `prompts` (lists of numbers), and the logits of the last step."""
    requests = len(prompts)
    assert max(map(len, prompts)) + steps <= model.capacity
    whole = lambda values: torch.tensor(values, dtype=torch.int32, device="cuda")  # noqa: E731
    ends = [0]
    for prompt in prompts:
        ends.append(ends[-1] + len(prompt))
    lengths = whole([len(prompt) for prompt in prompts])
    x = model.rows(whole(sum(prompts, [])), whole(ends), torch.zeros_like(lengths), lengths, max(map(len, prompts)))
    logits = model.logits(x[whole(ends[1:]) - 1])
    latest, cu = logits.argmax(-1).to(torch.int32), torch.arange(requests + 1, dtype=torch.int32, device="cuda")
    start = lengths.clone()

    def step():
        lengths.copy_(start + 1)
        out = model.logits(model.rows(latest, cu, start, lengths, 1))
        latest.copy_(out.argmax(-1))
        start.add_(1)
        return out

    tokens, replay, left = [latest.clone()], step, steps
    if graph and steps:
        side = torch.cuda.Stream()  # the first step, on a stream of its own, also loads the kernels
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            logits = step()
        torch.cuda.current_stream().wait_stream(side)
        tokens.append(latest.clone())
        captured, left = torch.cuda.CUDAGraph(), steps - 1
        with torch.cuda.graph(captured):
            held = step()

        def replay():
            captured.replay()
            return held

    for _ in range(left):
        logits = replay()
        tokens.append(latest.clone())
    return torch.stack(tokens, 1).cpu(), logits.float().cpu()


def step_time(model, requests, graph, steps=50):
    """Microseconds of a step behind a prompt of 64 tokens."""
    prompts = [[(7 * i + r) % VOCABULARY for i in range(64)] for r in range(requests)]
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    short, long = steps, 3 * steps
    took = []
    for count in (short, long):
        generate(model, prompts, 3, graph)
        begin.record()
        generate(model, prompts, count, graph)
        end.record()
        torch.cuda.synchronize()
        took.append(begin.elapsed_time(end))
    return 1e3 * (took[1] - took[0]) / (long - short)


def main():
    parser = argparse.ArgumentParser()
    for name, value in (("layers", 2), ("width", 1024), ("heads", 8), ("kv_heads", 2), ("requests", 3), ("tokens", 16)):
        parser.add_argument("--" + name, type=int, default=value)
    args = parser.parse_args()
    model = Decoder(args.layers, args.width, args.heads, args.kv_heads, requests=args.requests)
    prompts = [[(31 * i * i + 17 * r) % VOCABULARY for i in range(5 + 40 * r)] for r in range(args.requests)]
    tokens, logits = generate(model, prompts, args.tokens)
    for r, row in enumerate(tokens.tolist()):
        plain = model.plain_logits(torch.tensor(prompts[r] + row[:-1]))
        error = ((logits[r] - plain).norm() / plain.norm()).item()
        print(f"request {r}: {len(prompts[r])} tokens, then {row}; last logits {100 * error:.1f} % from float32's")
    print(f"a step: {step_time(model, args.requests, False):.0f} us launched, {step_time(model, args.requests, True):.0f} us replayed")


if __name__ == "__main__":
    main()

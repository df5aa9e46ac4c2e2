"""A small decoder-only language model on the library's decoder operators: linear layers with fused epilogues, the norm
and rotation of heads, the 8-bit paged cache and attention over it.  Weights are random, so its words mean nothing; what
it shows is how the operators fit together: a prompt of every sequence in one call, then one token of each a step, with
the step's kernels captured in a HIP graph.

With ``--weights int8`` every layer's weights are held as 8-bit codes; with ``--direct`` prompts attend to their keys and
values themselves, not to the cache's codes of them; ``--repetition`` and ``--frequency`` hold back tokens that a sequence
has seen.

    python examples/decoder.py [--fmt int8|fp8] [--layers N] [--prompts 100,37,256] [--new 32] [--weights int8] [--direct]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2410_08300_amd as cs  # noqa: E402


def rms(x, weight):
    z = x.float()
    return (z * torch.rsqrt(z.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype) * weight


class Decoder:
    """``layers`` layers of ``q_heads`` query and ``kv_heads`` key heads of width ``dim``; ``pages`` cache pages each."""

    def __init__(self, layers=4, hidden=1024, q_heads=16, kv_heads=4, dim=64, mlp=4096, vocab=8000, positions=4096,
                 pages=512, page_size=64, fmt="int8", dtype=torch.bfloat16, device="cuda", seed=0, weights=None,
                 direct=False):
        if weights not in (None, "int8"):
            raise ValueError("unknown weights %r (None or int8)" % (weights,))
        g = torch.Generator(device=device).manual_seed(seed)
        self.direct = direct

        def weight(out, inner):
            w = (torch.randn(out, inner, generator=g, device=device) / inner ** 0.5).to(dtype)
            return cs.quantize_rows(w) if weights == "int8" else w

        self.q_heads, self.kv_heads, self.dim = q_heads, kv_heads, dim
        ones = torch.ones(hidden, dtype=dtype, device=device)
        one_head = torch.ones(dim, dtype=dtype, device=device)
        self.embed = torch.randn(vocab, hidden, generator=g, device=device).to(dtype)
        self.layers = [dict(norm=ones, qkv=weight((q_heads + 2 * kv_heads) * dim, hidden), q_norm=one_head,
                            k_norm=one_head, proj=weight(hidden, q_heads * dim), mlp_norm=ones,
                            up=weight(mlp, hidden), up_bias=torch.zeros(mlp, dtype=dtype, device=device),
                            down=weight(hidden, mlp)) for _ in range(layers)]
        self.norm, self.head = ones, weight(vocab, hidden)
        self.caches = [cs.KVCache(pages, kv_heads, dim, page_size, fmt, device) for _ in range(layers)]
        angle = (torch.arange(positions, device=device)[:, None]
                 * 10000.0 ** (-torch.arange(0, dim, 2, device=device) / dim)[None])
        self.cos, self.sin = angle.cos().float(), angle.sin().float()

    @staticmethod
    def product(x, w, b=None, act="none", residual=None):
        """A linear layer, whose weights are numbers or (codes, scales)."""
        if isinstance(w, tuple):
            return cs.linear_int8(x, *w, b, act=act, residual=residual)
        return cs.linear(x, w, b, act=act, residual=residual)

    def forward(self, tokens, positions, table, starts, lengths, offsets, fresh=False):
        """Logits of the packed ``tokens`` (offsets[b] .. offsets[b + 1] are sequence b's), whose sequences held
        ``starts[b]`` tokens before and hold ``lengths[b]`` with them; ``fresh``: they held none, and the new tokens
        attend to each other without the cache."""
        q_end, k_end = self.q_heads, self.q_heads + self.kv_heads
        x = self.embed[tokens]
        n = x.shape[0]
        for layer, cache in zip(self.layers, self.caches):
            heads = self.product(rms(x, layer["norm"]), layer["qkv"]).view(n, -1, self.dim)
            # Queries and keys turn in place: they are views of the projection.
            q, k, v = heads[:, :q_end], heads[:, q_end:k_end], heads[:, k_end:]
            cs.qk_norm_rope(q, k, positions, self.cos, self.sin, layer["q_norm"], layer["k_norm"], q_out=q, k_out=k)
            cache.write(k, v, table, starts, offsets)
            a = (cs.prompt_attention(q, k, v, offsets) if fresh
                 else cs.cached_attention(q, cache, table, lengths, offsets))
            x = self.product(a.view(n, -1), layer["proj"], residual=x)
            h = self.product(rms(x, layer["mlp_norm"]), layer["up"], layer["up_bias"], act="gelu_tanh")
            x = self.product(h, layer["down"], residual=x)
        return self.product(rms(x, self.norm), self.head)

    def generate(self, prompts, new, graph=True, repetition=1.0, frequency=0.0):
        """``new`` greedy tokens for each of ``prompts`` (lists of tokens), as a tensor [prompts][new], and the seconds
        that a step took.  ``repetition`` divides the logits of tokens that the sequence holds (multiplies negative
        ones), ``frequency`` is taken off for each time that one was generated."""
        if new < 1 or not prompts or not all(prompts):
            raise ValueError("generate: prompts of a token at least, and a token at least to add to them")
        device = self.embed.device
        size = self.caches[0].page_size
        each = max((len(p) + new + size - 1) // size for p in prompts)
        if each * len(prompts) > self.caches[0].pages or max(map(len, prompts)) + new > self.cos.shape[0]:
            raise ValueError("generate: the cache or the position tables are too small for these sequences")

        def ints(values):
            return torch.tensor(values, dtype=torch.int32, device=device)

        table = torch.arange(each * len(prompts), dtype=torch.int32, device=device).view(len(prompts), each)
        lengths = ints([len(p) for p in prompts])
        offsets = [0]
        for p in prompts:
            offsets.append(offsets[-1] + len(p))
        places = ints([i for p in prompts for i in range(len(p))])
        # What a sequence holds, a row of fixed length each: -1 is no token.
        held = torch.full((len(prompts), max(map(len, prompts)) + new), -1, dtype=torch.int32, device=device)
        for row, p in zip(held, prompts):
            row[:len(p)] = ints(p)
        rows = torch.arange(len(prompts), device=device)
        held_at = ints([i * held.shape[1] for i in range(len(prompts) + 1)])
        penalties = [torch.full((len(prompts),), v, dtype=torch.float32, device=device) for v in (repetition, frequency)]
        prompt_lengths = lengths.clone()

        def adjusted(logits):
            if repetition == 1.0 and frequency == 0.0:
                return logits
            return cs.adjust_logits(logits, held.view(-1), held_at, prompt_lengths, repetition=penalties[0],
                                    frequency=penalties[1])

        logits = self.forward(torch.tensor(sum(prompts, []), device=device), places, table, torch.zeros_like(lengths),
                              lengths, ints(offsets), fresh=self.direct)
        token = adjusted(logits[torch.tensor(offsets[1:], device=device) - 1]).argmax(-1)
        found = torch.empty(len(prompts), new, dtype=torch.long, device=device)
        found[:, 0] = token
        starts, single = lengths.clone(), ints(range(len(prompts) + 1))

        logits = None

        def step():
            nonlocal logits
            held[rows, starts.long()] = token.int()
            logits = adjusted(self.forward(token, starts, table, starts, lengths, single))

        run, seconds = step, []
        for i in range(1, new):
            lengths.add_(1)
            if graph and i == 2:  # the first step has warmed the library up
                recorded = torch.cuda.CUDAGraph()
                with torch.cuda.graph(recorded):
                    step()
                run = recorded.replay
            torch.cuda.synchronize()
            t0 = time.perf_counter()
            run()
            token.copy_(logits.argmax(-1))
            torch.cuda.synchronize()
            seconds.append(time.perf_counter() - t0)
            starts.add_(1)
            found[:, i] = token
        return found, min(seconds) if seconds else 0.0


def main():
    p = argparse.ArgumentParser(description="greedy decoding with random weights")
    p.add_argument("--fmt", choices=cs.FORMATS, default="int8")
    p.add_argument("--layers", type=int, default=4)
    p.add_argument("--prompts", default="100,37,256", help="lengths of the prompts")
    p.add_argument("--new", type=int, default=32, help="tokens to add to each")
    p.add_argument("--weights", choices=["int8"], help="hold weights as 8-bit codes")
    p.add_argument("--direct", action="store_true", help="prompts attend without the cache")
    p.add_argument("--repetition", type=float, default=1.0)
    p.add_argument("--frequency", type=float, default=0.0)
    p.add_argument("--eager", action="store_true", help="launch every step's kernels instead of replaying a graph")
    a = p.parse_args()
    model = Decoder(layers=a.layers, fmt=a.fmt, weights=a.weights, direct=a.direct)
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, 8000, (int(n),), generator=g).tolist() for n in a.prompts.split(",")]
    found, seconds = model.generate(prompts, a.new, not a.eager, a.repetition, a.frequency)
    for n, row in zip(a.prompts.split(","), found.tolist()):
        print("prompt of %s: %s" % (n, " ".join(map(str, row))))
    print("%d sequences, %d layers, %s cache: %.0f us a step, %.0f tokens/s"
          % (len(prompts), a.layers, a.fmt, seconds * 1e6, len(prompts) / seconds if seconds else 0))


if __name__ == "__main__":
    main()

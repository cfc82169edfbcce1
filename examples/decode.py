"""A small LLaMA-shaped decoder with PEQA linears that reads prompts, writes, and scores what it wrote.

    python examples/decode.py [--layers 4] [--dim 1024] [--fp8]

Every layer is: normalisation, one stacked PEQA linear for queries, keys and values, peqa_rope_append into the layer's paged
cache, peqa_paged_attention, PEQA linears for the output projection and the MLP.  peqa_token_logprobs gives the next words (the
largest alternative) and, for the text as a whole, its perplexity; peqa_token_logprobs_bwd the loss's gradient with respect
to the logits.  Weights are random: the numbers mean nothing, the calls are those of a program with a checkpoint.
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2305_14152_amd import peqa  # noqa: E402


class Linear:
    """A PEQA layer of the given fp32 weight [N, K], quantized on the GPU."""

    def __init__(self, W, bits=4, group=128):
        self.L = peqa.layout(W.shape[0], W.shape[1], bits, group)
        self.packed = torch.empty(peqa.packed_words(self.L), dtype=torch.int32, device="cuda")
        self.s0 = torch.empty((W.shape[0], self.L.groups), device="cuda")
        self.z0 = torch.empty((W.shape[0], self.L.groups), dtype=torch.uint8, device="cuda")
        peqa.quantize(self.L, W.contiguous(), self.packed, self.s0, self.z0)

    def __call__(self, X):
        T = X.shape[0]
        Y = torch.empty((T, self.L.n_out), dtype=torch.bfloat16, device="cuda")
        room = peqa.workspace_bytes(self.L, T, peqa.PEQA_OP_FWD)
        peqa.linear_fwd(self.L, self.packed, self.s0, None, self.z0, X, T, Y, torch.empty(room, dtype=torch.uint8, device="cuda"), room)
        return Y


class Decoder:
    def __init__(self, layers=4, dim=1024, mlp=2816, heads=8, kv_heads=2, vocab=32000, seqs=4, positions=1024, page=64, fp8=False, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *shape, std=1.0: torch.randn(shape, device="cuda", generator=gen) * std  # noqa: E731
        self.dim, self.heads, self.kv_heads, self.head_dim, self.vocab = dim, heads, kv_heads, dim // heads, vocab
        self.embedding = normal(vocab, dim).bfloat16()
        self.head = normal(vocab, dim, std=2.0 / math.sqrt(dim)).bfloat16()
        self.weights = []                                       # what was quantized, for whoever wants to compare
        self.layers = []
        qkv = (heads + 2 * kv_heads) * self.head_dim
        std = 1.0 / math.sqrt(dim)
        for _ in range(layers):
            W = {"qkv": normal(qkv, dim, std=std), "o": normal(dim, heads * self.head_dim, std=std), "up": normal(2 * mlp, dim, std=std),
                 "down": normal(dim, mlp, std=1.0 / math.sqrt(mlp))}
            self.weights.append(W)
            self.layers.append({n: Linear(w) for n, w in W.items()})
        # one table for all layers; every sequence owns the pages of its row
        blocks = -(-positions // page)
        table = torch.randperm(seqs * blocks, device="cuda", generator=gen).to(torch.int32).view(seqs, blocks)
        kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
        scale = torch.full((kv_heads,), 1 / 32, device="cuda") if fp8 else None
        shape = (seqs * blocks, kv_heads, page, self.head_dim)
        self.caches = [peqa.kv_cache(torch.zeros(shape, device="cuda").to(kind), torch.zeros(shape, device="cuda").to(kind), table, scale, scale)
                       for _ in range(layers)]
        angle = torch.outer(torch.arange(positions, device="cuda", dtype=torch.float64),
                            10000.0 ** (-torch.arange(0, self.head_dim, 2, device="cuda", dtype=torch.float64) / self.head_dim))
        self.cos, self.sin = angle.cos().float(), angle.sin().float()

    @staticmethod
    def norm(x):
        return (x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-5)).bfloat16()

    def logits(self, tokens, seq, pos, longest):
        """Logits [T, vocab] after tokens [T] at positions pos of sequences seq, none past position longest - 1: a prompt's tokens all
        at once, or the next token of every sequence."""
        T, D = tokens.shape[0], self.head_dim
        x = self.embedding[tokens.long()].float()
        lens = pos + 1                                          # a token sees itself and what was before it
        room = peqa.paged_attention_workspace_bytes(self.caches[0], self.heads, T, longest)
        ws = torch.empty(room, dtype=torch.uint8, device="cuda")
        q_out, out = (torch.empty((T, self.heads, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for linear, cache in zip(self.layers, self.caches):
            qkv = linear["qkv"](self.norm(x)).unflatten(1, (-1, D))
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
            peqa.rope_append(cache, q, k, v, pos, self.cos, self.sin, q_out, seq=seq)
            peqa.paged_attention(cache, q_out, lens, longest, D ** -0.5, out, ws, room, seq=seq)
            x = x + linear["o"](out.view(T, -1)).float()
            gate, up = linear["up"](self.norm(x)).float().chunk(2, 1)
            x = x + linear["down"]((torch.nn.functional.silu(gate) * up).bfloat16()).float()
        return self.norm(x) @ self.head.T


def score(logits, targets, top=0):
    """(log probabilities, entropy, log-sum-exp, alternatives' log probabilities, alternatives) of every row."""
    T, V = logits.shape
    logp, entropy, lse = (torch.empty(T, device="cuda") for _ in range(3))
    best, ids = (torch.empty((T, top), device="cuda"), torch.empty((T, top), dtype=torch.int32, device="cuda")) if top else (None, None)
    room = peqa.token_logprobs_workspace_bytes(T, V, top)
    peqa.token_logprobs(logits, targets, logp if targets is not None else None, entropy, lse, best, ids,
                        torch.empty(room, dtype=torch.uint8, device="cuda"), room)
    return logp, entropy, lse, best, ids


def generate(model, prompts, steps, top=5):
    """Reads the prompts (a list of lists of words) and writes `steps` words after each; texts, and every written word's alternatives."""
    int32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    lens = [len(p) for p in prompts]
    logits = model.logits(int32(sum(prompts, [])), int32([s for s, n in enumerate(lens) for _ in range(n)]),
                          int32([i for n in lens for i in range(n)]), max(lens))
    last = torch.tensor(lens, device="cuda").cumsum(0) - 1
    logits, seq, pos = logits[last], int32(list(range(len(prompts)))), int32(lens)
    words, alternatives = [], []
    for i in range(steps):
        _, _, _, best, ids = score(logits, None, top)
        words.append(ids[:, 0].contiguous())
        alternatives.append((best, ids))
        if i + 1 < steps:
            logits = model.logits(words[-1], seq, pos, max(lens) + i + 1)
            pos = pos + 1
    return [p + torch.stack(words, 1)[s].tolist() for s, p in enumerate(prompts)], alternatives


def evaluate(model, text):
    """(mean loss, its gradient with respect to the logits) of a text, read at once into sequence 0."""
    T = len(text)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    logits = model.logits(torch.tensor(text, dtype=torch.int32, device="cuda"), torch.zeros_like(pos), pos, T)
    targets = torch.tensor(text[1:] + [-100], dtype=torch.int32, device="cuda")          # nothing to foresee after the last word
    logp, _, lse, _, _ = score(logits, targets)
    d_logits = torch.empty_like(logits)
    peqa.token_logprobs_bwd(logits, targets, lse, None, torch.full((T,), -1.0 / (T - 1), device="cuda"), None, d_logits)
    return -logp.sum() / (T - 1), d_logits


def main():
    ap = argparse.ArgumentParser()
    for name, value in (("layers", 4), ("dim", 1024), ("steps", 64), ("prompt", 200)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--fp8", action="store_true", help="8-bit cache")
    a = ap.parse_args()
    model = Decoder(layers=a.layers, dim=a.dim, mlp=-(-a.dim * 11 // 4 // 128) * 128, heads=a.dim // 128, kv_heads=max(1, a.dim // 512), fp8=a.fp8)
    gen = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, model.vocab, (max(1, a.prompt - 37 * s),), generator=gen).tolist() for s in range(4)]
    generate(model, prompts, 3)
    torch.cuda.synchronize()
    began = time.perf_counter()
    texts, _ = generate(model, prompts, a.steps)
    torch.cuda.synchronize()
    spent = time.perf_counter() - began
    loss, d_logits = evaluate(model, texts[0])
    print("%d sequences, prompts of %s words, %d words each in %.1f ms; loss of the first %.3f (uniform: %.3f), gradient's norm %.4f" % (
        len(texts), [len(p) for p in prompts], a.steps, 1e3 * spent, float(loss), math.log(model.vocab), float(d_logits.float().norm())))


if __name__ == "__main__":
    main()

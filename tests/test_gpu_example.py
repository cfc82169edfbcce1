"""The decoding example against a plain decoder in 64 bits on the same quantized weights: prompt and written words through the paged
cache, and the loss and its gradient.

Tolerance.  Activations are rounded to bf16 (2^-8 each) some ten times a layer over two layers, and the logits (of the order of 2) once:
0.05 for single log probabilities' typical and 0.3 for the worst of them, several times what independent roundings add up to."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def plain(model, text, oracle):
    """Log probabilities [T, vocab] of the next word after every word of a text."""
    T, D = len(text), model.head_dim
    x = model.embedding[text].double().cpu().numpy()
    norm = lambda a: a / np.sqrt((a * a).mean(1, keepdims=True) + 1e-5)  # noqa: E731
    cos, sin = model.cos[:T].double().cpu().numpy(), model.sin[:T].double().cpu().numpy()

    def rotate(a):                                                 # [T, heads, D]
        h = D // 2
        c, s = cos[:, None], sin[:, None]
        return np.concatenate((a[..., :h] * c - a[..., h:] * s, a[..., :h] * s + a[..., h:] * c), -1)

    for W in model.weights:
        def linear(a, name):
            w = W[name].cpu().numpy()
            codes, s0, z0 = oracle.quantize(w, 4, 128)
            s, z = s0.astype(np.float64).repeat(128, 1), z0.astype(np.float64).repeat(128, 1)
            return a @ (s * (codes.astype(np.float64) - z)).T
        qkv = linear(norm(x), "qkv").reshape(T, -1, D)
        q, k, v = rotate(qkv[:, :model.heads]), rotate(qkv[:, model.heads:model.heads + model.kv_heads]), qkv[:, model.heads + model.kv_heads:]
        out = np.zeros((T, model.heads, D))
        for h in range(model.heads):
            g = h // (model.heads // model.kv_heads)
            z = q[:, h] @ k[:, g].T / np.sqrt(D)
            z[np.triu_indices(T, 1)] = -np.inf
            p = np.exp(z - z.max(1, keepdims=True))
            out[:, h] = p / p.sum(1, keepdims=True) @ v[:, g]
        x = x + linear(out.reshape(T, -1), "o")
        gate, up = np.split(linear(norm(x), "up"), 2, 1)
        x = x + linear(gate / (1 + np.exp(-gate)) * up, "down")
    logits = norm(x) @ model.head.double().cpu().numpy().T
    m = logits.max(1, keepdims=True)
    return logits - m - np.log(np.exp(logits - m).sum(1, keepdims=True))


def test_example(oracle):
    import torch
    assert torch.cuda.is_available()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import decode
    model = decode.Decoder(layers=2, dim=512, mlp=768, heads=4, kv_heads=2, vocab=1000, seqs=3, positions=128, page=16)
    gen = torch.Generator().manual_seed(0)
    prompts = [torch.randint(0, 1000, (n,), generator=gen).tolist() for n in (21, 1, 40)]
    texts, alternatives = decode.generate(model, prompts, 6)
    for s, (prompt, text) in enumerate(zip(prompts, texts)):
        assert text[:len(prompt)] == prompt and len(text) == len(prompt) + 6
        want = plain(model, text, oracle)
        for i in range(6):
            at = len(prompt) + i - 1                              # the word that the i-th written one follows
            best, ids = alternatives[i][0][s].cpu().numpy(), alternatives[i][1][s].cpu().numpy()
            off = np.abs(best - want[at, ids])
            assert off.max() <= 0.3, (s, i, off)
            # no alternative is far behind what the plain decoder would have taken in its place
            assert (np.sort(want[at])[::-1][:5] - np.sort(want[at, ids])[::-1]).max() <= 0.3
    loss, d_logits = decode.evaluate(model, texts[2])
    want = plain(model, texts[2], oracle)
    T = len(texts[2])
    nll = -want[np.arange(T - 1), texts[2][1:]]
    assert abs(float(loss) - nll.mean()) <= 0.05
    p = np.exp(want)
    grad = p.copy()
    grad[np.arange(T - 1), texts[2][1:]] -= 1
    grad[T - 1] = 0
    grad /= T - 1
    got = d_logits.double().cpu().numpy()
    assert np.linalg.norm(got - grad) <= 0.05 * np.linalg.norm(grad)
    assert (got[T - 1] == 0).all()


def test_example_with_an_8_bit_cache():
    """The same text through both caches: 8-bit keys and values are off by up to 2^-4 each, averaged over positions."""
    import torch
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import decode
    gen = torch.Generator().manual_seed(3)
    text = torch.randint(0, 1000, (50,), generator=gen).tolist()
    loss = []
    for fp8 in (False, True):
        model = decode.Decoder(layers=2, dim=512, mlp=768, heads=4, kv_heads=2, vocab=1000, seqs=3, positions=128, page=16, fp8=fp8)
        value, d = decode.evaluate(model, text)
        assert bool(d.isfinite().all())
        loss.append(float(value))
    assert abs(loss[0] - loss[1]) <= 0.1

"""The calls around a decoder layer's cache together, as a program that keeps a bounded cache makes them: normalised heads to places of their
own, attention that adds up what positions are given, eviction, and on; several answers behind one prompt; the decoding example with all
of them.

Tolerance of the runs.  Stored keys, values and queries are rounded to bf16 (2^-8 each at most): heads are of size sqrt(head_dim) (norms'
weights near 1), so a score is off by 2^-7 sqrt(head_dim) at most and, as its rounding errors are independent, by about 2^-7 of its typical size
1: weights by under 2^-5 of themselves, outputs by twice that of sum w |v|."""
import math
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EPS = 1e-6


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_2305_14152_amd import peqa
    peqa.lib()
    return torch, peqa


def test_bounded_cache(env):
    torch, peqa = env
    gen = torch.Generator().manual_seed(11)
    S, heads, kv, dim, page, keep, slack, steps, cap = 3, 6, 2, 64, 16, 40, 8, 150, 48
    group, scale = heads // kv, dim ** -0.5
    table = torch.randperm(S * cap // page, generator=gen).to(torch.int32).view(S, -1).cuda()
    cache = peqa.kv_cache(*(torch.full((S * cap // page, kv, page, dim), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)), table)
    angle = torch.outer(torch.arange(steps, dtype=torch.float64), 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim))
    cos, sin = angle.cos().float().cuda(), angle.sin().float().cuda()
    wq, wk = ((1 + 0.2 * torch.randn(dim, generator=gen)).cuda() for _ in range(2))
    given = torch.zeros((S, kv, cap), device="cuda")
    out, q_out = (torch.empty((S, heads, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kept, left = torch.empty((S, kv, keep), dtype=torch.int32, device="cuda"), torch.empty(S, dtype=torch.int32, device="cuda")
    r1, r2 = peqa.paged_attention_weights_workspace_bytes(cache, heads, S, cap), peqa.cache_evict_workspace_bytes(cache, S, cap, keep)
    ws1, ws2 = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in (r1, r2))
    f64 = lambda t: t.float().cpu().double().numpy()  # noqa: E731
    c64, s64 = angle.cos().numpy(), angle.sin().numpy()

    def head(x, w, p):
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS) * f64(w)
        a, b = x[..., :dim // 2], x[..., dim // 2:]
        return np.concatenate((a * c64[p] - b * s64[p], a * s64[p] + b * c64[p]), -1)

    memory = [[([], [], []) for _ in range(kv)] for _ in range(S)]      # keys, values and what they were given, of every sequence and head
    place, evictions = torch.zeros(S, dtype=torch.int32, device="cuda"), 0
    for p in range(steps):
        qkv = torch.randn((S, (heads + 2 * kv) * dim), generator=gen).to(torch.bfloat16).cuda().unflatten(1, (-1, dim))
        q, k, v = qkv.split([heads, kv, kv], 1)
        pos = torch.full((S,), p, dtype=torch.int32, device="cuda")
        peqa.norm_rope_append(cache, q, k, v, pos, cos, sin, wq, wk, EPS, q_out, place=place)
        place = place + 1
        peqa.paged_attention_weights(cache, q_out, place, cap, scale, out, given, given, ws1, r1)
        got, Q, K, V = f64(out), head(f64(q), wq, p), head(f64(k), wk, p), f64(v)
        for s in range(S):
            for h in range(kv):
                keys, values, sums = memory[s][h]
                keys.append(K[s, h])
                values.append(V[s, h])
                sums.append(0.0)
                kk, vv = np.array(keys), np.array(values)
                total = np.zeros(len(keys))
                for i in range(h * group, (h + 1) * group):
                    z = kk @ Q[s, i] * scale
                    w = np.exp(z - z.max())
                    w /= w.sum()
                    total += w
                    assert (np.abs(got[s, i] - w @ vv) <= 2.0 ** -4 * (w @ np.abs(vv)) + 1e-3).all(), (p, s, i)
                memory[s][h] = (keys, values, list(np.array(sums) + total))
        if (p + 1) % slack == 0 and int(place[0]) >= keep + slack:
            before = given.clone()
            peqa.cache_evict(cache, place, cap, given, given, keep, 2, 10, kept, left, ws2, r2)
            assert left.tolist() == [keep] * S
            n, b, chosen = int(place[0]), before.cpu().numpy(), kept.cpu().numpy()
            for s in range(S):
                for h in range(kv):
                    mid = np.argsort(-b[s, h, 2:n - 10], kind="stable")[:keep - 12] + 2
                    assert (chosen[s, h] == np.sort(np.concatenate((np.arange(2), mid, np.arange(n - 10, n))))).all()
                    keys, values, sums = memory[s][h]
                    assert (np.abs(b[s, h, :n] - sums) <= 2.0 ** -4 * np.array(sums)).all()
                    memory[s][h] = tuple([x[j] for j in chosen[s, h]] for x in (keys, values, sums))
            place, evictions = left.clone(), evictions + 1
    assert evictions > 10


def plain(model, texts, oracle):
    """Log probabilities [T, vocab] of the next word after every word of each text, in 64 bits, with the heads' norms."""
    results = []
    D, W64 = model.head_dim, []
    for W in model.weights:
        one = {}
        for name, w in W.items():
            codes, s0, z0 = oracle.quantize(w.cpu().numpy(), 4, 128)
            s, z = s0.astype(np.float64).repeat(128, 1), z0.astype(np.float64).repeat(128, 1)
            one[name] = s * (codes.astype(np.float64) - z)
        W64.append(one)
    for text in texts:
        T = len(text)
        x = model.embedding[text].double().cpu().numpy()
        rms = lambda a, eps=1e-5: a / np.sqrt((a * a).mean(-1, keepdims=True) + eps)  # noqa: E731
        cos, sin = model.cos[:T].double().cpu().numpy()[:, None], model.sin[:T].double().cpu().numpy()[:, None]

        def rotate(a):
            h = D // 2
            return np.concatenate((a[..., :h] * cos - a[..., h:] * sin, a[..., :h] * sin + a[..., h:] * cos), -1)
        for n, W in enumerate(W64):
            qkv = (rms(x) @ W["qkv"].T).reshape(T, -1, D)
            q, k, v = np.split(qkv, [model.heads, model.heads + model.kv_heads], 1)
            if model.norms is not None:
                q, k = (rms(a, 1e-6) * w.double().cpu().numpy() for a, w in zip((q, k), model.norms[n]))
            q, k = rotate(q), rotate(k)
            out = np.zeros((T, model.heads, D))
            for h in range(model.heads):
                g = h // (model.heads // model.kv_heads)
                z = q[:, h] @ k[:, g].T / np.sqrt(D)
                z[np.triu_indices(T, 1)] = -np.inf
                p = np.exp(z - z.max(1, keepdims=True))
                out[:, h] = p / p.sum(1, keepdims=True) @ v[:, g]
            x = x + out.reshape(T, -1) @ W["o"].T
            gate, up = np.split(rms(x) @ W["up"].T, 2, 1)
            x = x + (gate / (1 + np.exp(-gate)) * up) @ W["down"].T
        logits = rms(x) @ model.head.double().cpu().numpy().T
        m = logits.max(1, keepdims=True)
        results.append(logits - m - np.log(np.exp(logits - m).sum(1, keepdims=True)))
    return results


def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import decode
    return decode


@pytest.mark.parametrize("norms", [False, True])
def test_answers_behind_one_prompt(env, oracle, norms):
    """Tolerance as in the test of the example: 0.3 for a single log probability."""
    torch, _ = env
    decode = example()
    model = decode.Decoder(layers=2, dim=512, mlp=768, heads=4, kv_heads=2, vocab=1000, seqs=4, positions=128, page=16, norms=norms)
    prompt = torch.randint(0, 1000, (37,), generator=torch.Generator().manual_seed(2)).tolist()
    texts, logps = decode.answers(model, prompt, 3, 6)
    assert len({t[37] for t in texts}) == 3
    for text, logp, want in zip(texts, logps.cpu().numpy(), plain(model, texts, oracle)):
        assert text[:37] == prompt and len(text) == 43
        assert max(abs(logp[i] - want[36 + i, text[37 + i]]) for i in range(6)) <= 0.3


def test_generation_with_a_bounded_cache(env, oracle):
    """As long as nothing has left, the words' log probabilities are those of a whole cache; afterwards everything stays finite, and the sequences go on."""
    torch, _ = env
    decode = example()
    model = decode.Decoder(layers=2, dim=512, mlp=768, heads=4, kv_heads=2, vocab=1000, seqs=3, positions=256, page=16, norms=True)
    gen = torch.Generator().manual_seed(5)
    prompts = [torch.randint(0, 1000, (n,), generator=gen).tolist() for n in (21, 1, 40)]
    texts, alternatives = decode.generate(model, prompts, 60, keep=32, slack=16)
    assert [len(t) for t in texts] == [81, 61, 100]
    want = plain(model, texts, oracle)
    for s, (prompt, text) in enumerate(zip(prompts, texts)):
        for i in range(60):
            best, ids = alternatives[i][0][s].cpu().numpy(), alternatives[i][1][s].cpu().numpy()
            assert np.isfinite(best).all() and (best <= 0).all()
            if i < 8:                                         # (the longest has 48 positions after eight words)
                assert np.abs(best - want[s][len(prompt) + i - 1, ids]).max() <= 0.3, (s, i)
    whole, others = decode.generate(model, prompts, 8)
    for s in range(3):
        for i in range(8):
            a, b = alternatives[i], others[i]
            if texts[s][:len(prompts[s]) + i] == whole[s][:len(prompts[s]) + i]:
                assert float((a[0][s] - b[0][s]).abs().max()) <= 0.3
    assert math.isfinite(float(decode.evaluate(model, texts[0])[0]))

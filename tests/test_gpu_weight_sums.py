"""What positions are given where a row's scores are far from zero (peqa_paged_attention_weights), against 64 bits.

Scores are, in powers of two, base + r exactly, base up to 2^14 in size and r a whole number from -6 to 0: products of whole numbers, and a scale whose fp32
product with log2 e is 1.  So nothing but the weights' own arithmetic rounds: powers of two (2^-22), a row's sum of up to 20000 of them
(fp32 sums of at most 640 numbers each before they are joined, 2^-24 sqrt(640) of it typically, 2^-19 taken), its reciprocal and the product (2^-24 each), and
sums over up to 20 heads and rows: 2^-17 of what a position is given, in every form of the call.  A sum kept as its logarithm would be off by 2^-11."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_2305_14152_amd import peqa
    peqa.lib()
    return torch, peqa


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("base", [2.0 ** 14, -2.0 ** 14, 1024.0])
@pytest.mark.parametrize("lens,kv,group,seq", [([333], 4, 1, None), ([700, 90, 1], 2, 4, None), ([20000], 1, 3, None), ([300, 299, 40], 2, 4, [0, 0, 1]),
                                               ([2500, 1200] * 3, 3, 3, None)])
def test_far_scores(env, lens, kv, group, seq, base, fp8):
    torch, peqa = env
    scale = float(np.float32(math.log(2.0)))
    assert np.float32(scale) * np.float32(1.44269504088896341) == 1
    gen = torch.Generator().manual_seed(len(lens) + kv)
    page, dim, most, seqs = 16, 64, max(lens), 1 + max(seq or range(len(lens)))
    blocks = -(-most // page)
    r = torch.randint(-6, 1, (seqs, blocks, kv, page), generator=gen).float()
    k = torch.zeros((seqs, blocks, kv, page, dim))
    k[..., 0], k[..., 1] = math.copysign(1.0, base), r
    kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
    pools = [x.flatten(0, 1).to(kind).cuda() for x in (k, torch.randn(k.shape, generator=gen))]
    cache = peqa.kv_cache(*pools, torch.arange(seqs * blocks, dtype=torch.int32, device="cuda").view(seqs, blocks))
    rows, heads = len(lens), kv * group
    q = torch.zeros((rows, heads, dim))
    q[..., 0], q[..., 1] = abs(base), 1.0
    q = q.to(torch.bfloat16).cuda()
    room = peqa.paged_attention_weights_workspace_bytes(cache, heads, rows, most)
    ws, out = torch.full((room,), 255, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
    got = torch.zeros((seqs, kv, -(-most // 4) * 4), device="cuda")
    index = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    peqa.paged_attention_weights(cache, q, index(lens), most, scale, out, None, got, ws, room, seq=index(seq))
    want = np.zeros(got.shape)
    x = r.permute(0, 2, 1, 3).flatten(2).double().numpy() * (scale / math.log(2.0))
    for i, n in enumerate(lens):
        s = i if seq is None else seq[i]
        w = np.exp2(x[s, :, :n])
        want[s, :, :n] += group * w / w.sum(1, keepdims=True)
    off = np.abs(got.cpu().double().numpy() - want) / np.maximum(want, 1e-30)
    assert off.max() <= 2.0 ** -17, off.max()

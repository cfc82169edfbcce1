"""Attention over values that are not finite, against 64 bits: an infinite value at a position that counts makes its element of the result
infinite, of the same sign, for every head that attends to it, values of both signs or NaN make it NaN, and neither reaches another
element, position or head.  The finite elements have the tolerance of tests/test_gpu_decode.py, 2^-14 of sum w |v| and bf16's half unit."""
import math

import numpy as np
import pytest

from test_gpu_decode import make_cache, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_2305_14152_amd import peqa
    peqa.lib()
    return torch, peqa


@pytest.mark.parametrize("heads,kv_heads,dim,lens", [
    (4, 1, 128, [64]), (8, 8, 128, [300, 33, 5]), (12, 1, 128, [40, 70]), (16, 2, 64, [500, 129]), (3, 3, 256, [100]), (24, 2, 256, [300, 50]),
    (4, 4, 128, [60] * 140), (8, 1, 128, [9000, 100]), (2, 1, 256, [7000]), (8, 8, 64, [3001] + [40] * 23),
])
def test_infinite_values(env, heads, kv_heads, dim, lens):
    torch, peqa = env
    print("infinite", heads, kv_heads, dim, len(lens), lens[0], flush=True)
    gen = torch.Generator().manual_seed(heads + dim)
    cache = make_cache(torch, peqa, gen, lens, kv_heads, dim, 16)
    v, table = cache.tensors[1], cache.tensors[2].cpu()
    for r, n in enumerate(lens):
        h = r % kv_heads
        for at, d, value in ((n // 2, 3, math.inf), (n - 1, 4, -math.inf), (0, dim - 1, math.inf), (n // 3, 17, math.inf), (n // 2, 17, -math.inf),
                             (n - 1, 20, math.nan), (0, 33, math.inf), (n - 1, 33, math.inf)):
            v[int(table[r, at // 16]), h, at % 16, d] = value
    q = torch.randn((len(lens), heads, dim), generator=gen).to(torch.bfloat16).cuda()
    scale = 0.2 * dim ** -0.5                                    # scores of the order of one: no weight vanishes
    out = torch.empty_like(q)
    lse = torch.empty((len(lens), heads), device="cuda")
    room = peqa.paged_attention_workspace_bytes(cache, heads, len(lens), max(lens))
    peqa.paged_attention(cache, q, torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens), scale, out,
                         torch.full((room,), 0xFF, dtype=torch.uint8, device="cuda"), room, lse=lse)
    with np.errstate(invalid="ignore"):
        want, want_lse, size = reference(cache, q, lens, max(lens), scale)
    got = out.float().cpu().double().numpy()
    assert np.isinf(want).any() and np.isnan(want).any()
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    infinite = np.isinf(want)
    np.testing.assert_array_equal(got[infinite], want[infinite])
    fine = np.isfinite(want)
    assert (np.abs(got[fine] - want[fine]) <= 2.0 ** -8 * np.abs(want[fine]) * 1.01 + 2.0 ** -14 * size[fine]).all()
    assert np.abs(lse.cpu().double().numpy() - want_lse).max() <= 2.0 ** -14 * (1 + np.abs(want_lse).max())

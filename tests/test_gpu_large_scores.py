"""Attention whose scores are finite but so large that an fp32 number of their size is no multiple of one (2^22 to 2^40 and both signs): the
result is that of the positions with the largest score, and log-sum-exp is that score, in the attention behind shared positions as in the paged one.

Keys and queries have one element that is not 0, so that products are exact, and different scores of a row are a fifteenth of the largest
apart or equal: of everything but the largest ones the weight is 0.  The tolerances are those of tests/test_gpu_shared.py; of the rows with scores
of ordinary size beside them, whose products are exact too, the same ones."""
import numpy as np
import pytest

from test_gpu_decode import check_attention
from test_gpu_shared import both, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_2305_14152_amd import peqa
    peqa.lib()
    return torch, peqa


def keys_of_one_element(torch, gen, cache):
    """Every stored key gets whole numbers from -15 to 15 in its first element, of few positions the largest, and zeros in the others."""
    k = cache.tensors[0]
    whole = torch.randint(-14, 15, k.shape[:3], generator=gen)
    rare = torch.rand(k.shape[:3], generator=gen)
    whole[rare < 0.02] = 15
    whole[rare > 0.98] = -15
    x = torch.zeros(k.shape)
    x[..., 0] = whole.float()
    hole = k.float().isnan()
    k.copy_(x.cuda().to(k.dtype))
    (k.view(torch.uint8) if k.dtype != torch.bfloat16 else k.view(torch.int16)).masked_fill_(hole, 0x7F if k.dtype != torch.bfloat16 else 0x7FC0)


def queries(torch, gen, rows, heads, dim, size):
    """Of sizes `size` to twice that; every third one ordinary."""
    q = torch.zeros((rows, heads, dim))
    q[..., 0] = (1 + torch.rand((rows, heads), generator=gen)) * size
    q.view(rows * heads, dim)[::3, 0] *= 0.25 / size
    return q.to(torch.bfloat16).cuda()


# rows, heads of a key head, key heads, shared positions: columns in every wave (16, 32, 64), waves' own columns, once and twice
FORMS = [(2, 3, 2, 300), (6, 4, 1, 300), (12, 4, 2, 700), (9, 12, 1, 1111), (32, 8, 8, 8200)]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("rows,group,kv,shared", FORMS)
def test_behind_shared_positions(env, rows, group, kv, shared, fp8):
    torch, peqa = env
    gen = torch.Generator().manual_seed(rows + shared)
    own = [int(n) for n in torch.randint(0, 200, (rows,), generator=gen)]
    cache = both(torch, peqa, gen, shared, own, kv, 64, 32, fp8)
    keys_of_one_element(torch, gen, cache)
    lens = [shared + n for n in own]
    for power in (22, 25, 27, 29, 31, 34, 40) if shared < 8000 else (29, 34):
        q = queries(torch, gen, rows, kv * group, 64, 2.0 ** power / 15)
        print("shared", rows, group, kv, shared, fp8, power, flush=True)
        for scale in (1.0, -0.7) if shared < 8000 else (0.9,):
            # (the cache's scales are part of an 8-bit cache's scores)
            check(torch, peqa, cache, q, lens, max(lens), rows, shared, scale=scale * (25 if fp8 else 1))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("group,lens", [(3, [40, 333]), (12, [700, 9])])
def test_paged(env, group, lens, fp8):
    torch, peqa = env
    from test_gpu_decode import make_cache
    gen = torch.Generator().manual_seed(group)
    cache = make_cache(torch, peqa, gen, lens, 2, 64, 32, fp8=fp8)
    keys_of_one_element(torch, gen, cache)
    for power in (22, 25, 27, 29, 31, 34, 40):
        q = queries(torch, gen, len(lens), 2 * group, 64, 2.0 ** power / 15)
        print("paged", group, lens, fp8, power, flush=True)
        for scale in (1.0, -0.7):
            check_attention(torch, peqa, cache, q, lens, max(lens), scale=scale * (25 if fp8 else 1), fp8=fp8)

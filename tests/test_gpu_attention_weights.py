"""How exactly softmax weights are kept against 8-bit values: rows whose result is a small difference of large sums.

Half of a row's positions have the score d and the value c, the others the score 0 and the value -c: the result is c tanh(d / 2).  With d
around 2^-12 it is made of the last bits of the weights; a relative error of at most E of every weight moves it by E c at most.  Scores
are exact here, the exponentials of differences under 2^-10 are off by 2^-20: 2^-14 c, as against bf16 values, where up to eight heads
share a key head, and bf16's half unit of the result.  More heads have weights of 11 bits: 2^-10 c."""

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_2305_14152_amd import peqa
    peqa.lib()
    return torch, peqa


@pytest.mark.parametrize("dim,kv_heads,group", [(64, 2, 8), (128, 4, 1), (128, 2, 5), (128, 1, 8), (256, 2, 8), (256, 1, 3), (64, 1, 9), (128, 1, 20), (256, 1, 16)])
@pytest.mark.parametrize("lens", [[2, 30, 100], [400, 2], [200] * 300 + [2] * 300, [9000, 10], [2048, 16000, 64, 4444] * 16])
def test_small_differences(env, dim, kv_heads, group, lens):
    torch, peqa = env
    print("weights", dim, kv_heads, group, len(lens), lens[0], flush=True)
    c, heads, page = 448.0, kv_heads * group, 16
    # every row attends to the same sequence, whose even positions have the score d
    pages = max(lens) // page + 1
    k, v = (torch.zeros((pages, kv_heads, page, dim), device="cuda") for _ in range(2))
    k[:, :, ::2, 0] = 1.0
    v[:, :, ::2], v[:, :, 1::2] = c, -c
    e4m3 = torch.float8_e4m3fn
    cache = peqa.kv_cache(k.to(e4m3), v.to(e4m3), torch.arange(pages, dtype=torch.int32, device="cuda")[None])
    rows = len(lens)
    q = torch.zeros((rows, heads, dim), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = torch.rand((rows, heads), generator=torch.Generator().manual_seed(rows + dim)).to(torch.bfloat16).cuda() * 2.0 ** -11
    q[:, 0, 0] = 0.99 * 2.0 ** -12                               # (lost in a single fp16 number)
    out = torch.empty_like(q)
    room = peqa.paged_attention_workspace_bytes(cache, heads, rows, max(lens))
    peqa.paged_attention(cache, q, torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens), 1.0, out,
                         torch.full((room,), 0xFF, dtype=torch.uint8, device="cuda"), room, seq=torch.zeros(rows, dtype=torch.int32, device="cuda"))
    want = c * torch.tanh(q[..., :1].double() / 2).expand(rows, heads, dim)
    assert float(want[:, 0].min()) > 2.0 ** -14 * c * 1.5
    bound = 2.0 ** -8 * 1.01 * want.abs() + 2.0 ** (-14 if group <= 8 else -10) * c
    assert bool(((out.double() - want).abs() <= bound).all()), float((out.double() - want).abs().max() / c)

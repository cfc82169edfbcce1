"""Attention behind shared positions (peqa_shared_attention) against a plain implementation in 64 bits, and against the paged attention.

Tolerances.  As in the tests of the paged attention: a relative error of every weight of at most E moves the output by 2 E sum w |v|.  E adds the
scores' fp32 rounding (under 2^-16 for the scores of these inputs), the exponential's (2^-20) and that of the weights: 2^-16 in two bf16
parts of which the first is cut, 2^-12 as fp16; taken are 2^-14 and 2^-10 of sum w |v| in all, and bf16's 2^-8 of the output.
lse: 2^-14, and 2^-21 of itself, for the roundings (2^-24 each) of scale log2 e, of the reference, of the sum and of its product with log 2."""
import math

import numpy as np
import pytest

from test_gpu_decode import make_cache, read

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_2305_14152_amd import peqa
    peqa.lib()
    return torch, peqa


def reference(cache, q, lens, max_len, prefix, shared, scale, seq=None):
    rows, heads, dim = q.shape
    q, group = q.float().cpu().double().numpy(), heads // cache.kv_heads
    out, lse, size = np.zeros(q.shape), np.full((rows, heads), -math.inf), np.zeros(q.shape)
    whole = {}
    for r in range(rows):
        s, n = r if seq is None else seq[r], min(lens[r], max_len)
        if n <= 0 or not 0 <= s < cache.n_seqs:
            continue
        m = min(n, shared)
        for h in range(cache.kv_heads):
            if h not in whole:
                whole[h] = [read(cache, w, prefix, h, shared) for w in (0, 1)] if shared else [(np.zeros((0, dim)), np.zeros(0, bool))] * 2
            (k, there), (v, _) = whole[h]
            k, v, there = k[:m], v[:m], there[:m]
            if n > shared:
                (mk, mine), (mv, _) = read(cache, 0, s, h, n), read(cache, 1, s, h, n)
                k, v, there = np.concatenate((k, mk[shared:])), np.concatenate((v, mv[shared:])), np.concatenate((there, mine[shared:]))
            if not there.any():
                continue
            k, v = k[there], v[there]
            for i in range(h * group, (h + 1) * group):
                z = k @ q[r, i] * scale
                w = np.exp(z - z.max())
                lse[r, i] = z.max() + math.log(w.sum())
                w /= w.sum()
                out[r, i], size[r, i] = w @ v, w @ np.abs(v)
    return out, lse, size


def call(torch, peqa, cache, q, lens, max_len, prefix, shared, scale, seq=None, lse=True):
    rows, heads, dim = q.shape
    index = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    room = peqa.shared_attention_workspace_bytes(cache, heads, rows, max_len, shared)
    ws = torch.full((room,), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((rows, heads * dim + 8), float("nan"), dtype=torch.bfloat16, device="cuda")[:, :heads * dim].unflatten(1, (heads, dim))
    sums = torch.full((rows, heads), float("nan"), device="cuda") if lse else None
    peqa.shared_attention(cache, q, index(lens), max_len, prefix, shared, scale, out, ws, room, lse=sums, seq=index(seq))
    return out, sums


def check(torch, peqa, cache, q, lens, max_len, prefix, shared, seq=None, scale=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    out, lse = call(torch, peqa, cache, q, lens, max_len, prefix, shared, scale, seq)
    want, sums, size = reference(cache, q, lens, max_len, prefix, shared, scale, seq)
    got = out.float().cpu().double().numpy()
    assert np.isfinite(got).all()
    off = np.abs(got - want) - (2.0 ** -8 * np.abs(want) + 2.0 ** (-10 if cache.dtype else -14) * size)
    assert off.max() <= 0, (off.max(), np.unravel_index(off.argmax(), off.shape))
    got, none = lse.cpu().double().numpy(), np.isinf(sums)
    assert (got[none] == -math.inf).all() and (np.abs(got[~none] - sums[~none]) <= 2.0 ** -14 + 2.0 ** -21 * np.abs(sums[~none])).all()
    again, _ = call(torch, peqa, cache, q, lens, max_len, prefix, shared, scale, seq, lse=False)
    assert torch.equal(again, out)
    return out, lse


def both(torch, peqa, gen, shared, own, kv, dim, page, fp8, layout="heads"):
    """A cache whose last sequence has the shared positions and whose others have `own` more each, with nothing in front of them."""
    caps = [shared + n if n >= 0 else 0 for n in own] + [shared]
    cache = make_cache(torch, peqa, gen, caps, kv, dim, page, fp8=fp8, layout=layout)
    table = cache.tensors[2]
    table[:-1, :shared // page] = torch.randint(-2 ** 31, 2 ** 31 - 1, (len(own), shared // page), generator=gen, dtype=torch.int64).to(torch.int32).cuda()
    return cache


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("shared,own,kv,group,dim,page,layout", [
    (1, [1], 1, 1, 64, 8, "heads"), (1, [0, 0], 1, 1, 128, 8, "heads"), (33, [1, 5, 0], 2, 2, 64, 8, "slots"), (555, [77, 3, 40], 4, 1, 128, 16, "both"),
    (128, [128] * 17, 2, 1, 64, 32, "heads"), (100, [300, 1, 31, 32, 33], 1, 16, 128, 64, "heads"), (257, [65] * 9, 2, 8, 128, 16, "slots"),
    (1000, [20, 30], 1, 40, 64, 8, "heads"), (700, [9, 90] * 20, 1, 4, 256, 128, "heads"), (31, [1500, 2], 2, 3, 256, 16, "both"),
    (5000, [64] * 3, 1, 12, 128, 16, "heads"), (2050, [130] * 33, 1, 8, 64, 8, "heads"), (0, [40, 1, 0], 2, 4, 128, 16, "heads"),
    (1100, [33] * 20, 2, 8, 128, 16, "both"), (3001, [5, 600] * 20, 1, 14, 128, 8, "slots"), (130, [1, 2] * 40, 1, 1, 64, 64, "heads"), (97, [40] * 70, 3, 2, 128, 32, "heads")])
def test_shared(env, shared, own, kv, group, dim, page, layout, fp8):
    torch, peqa = env
    gen = torch.Generator().manual_seed(shared + sum(own) + dim)
    cache = both(torch, peqa, gen, shared, own, kv, dim, page, fp8, layout)
    rows = len(own)
    q = torch.randn((rows, (kv * group + 1) * dim), generator=gen).to(torch.bfloat16).cuda()[:, :kv * group * dim].unflatten(1, (kv * group, dim))
    lens = [shared + n for n in own]
    check(torch, peqa, cache, q, lens, max(lens), rows, shared)
    check(torch, peqa, cache, q, lens, max(lens) - 1, rows, shared, scale=-0.2)
    # rows that end among the shared positions, that are empty, that are none
    lens = [n if r % 3 else [0, shared // 2, -7, min(1, shared), max(0, shared - 1)][r // 3 % 5] for r, n in enumerate(lens)]
    seq = [r if r % 4 != 2 else [-1, rows + 1][r // 4 % 2] for r in range(rows)]
    check(torch, peqa, cache, q, lens, max(1, max(lens)), rows, shared, seq=seq)
    check(torch, peqa, cache, q, lens, max(0, min(shared - 1, max(lens))), rows, shared)


def test_rows_in_any_order_and_twice(env):
    """Several new tokens of a sequence, the prefix's own sequence as a row's, pages that are not there."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(2)
    cache = both(torch, peqa, gen, 300, [40, 50, 60], 2, 128, 16, False)
    cache.tensors[2][3, 4] = -1
    cache.tensors[2][1, 20] = cache.n_pages
    q = torch.randn((8, 6, 128), generator=gen).to(torch.bfloat16).cuda()
    check(torch, peqa, cache, q, [340, 339, 338, 350, 300, 20, 360, 350], 360, 3, 300, seq=[0, 0, 0, 1, 3, 3, 2, 1])
    cache.tensors[2][3, :] = -1
    check(torch, peqa, cache, q, [340, 339, 338, 350, 300, 20, 360, 350], 360, 3, 300, seq=[0, 0, 0, 1, 3, 3, 2, 1])


@pytest.mark.parametrize("fp8", [False, True])
def test_against_paged_attention(env, fp8):
    """Tables that share whole pages: the same attention by both calls."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(6)
    shared, own, page = 1024, [100, 200, 1, 0, 64, 33], 32
    cache = both(torch, peqa, gen, shared, own, 2, 128, page, fp8)
    cache.tensors[2][:-1, :shared // page] = cache.tensors[2][-1:, :shared // page]
    q = torch.randn((6, 16, 128), generator=gen).to(torch.bfloat16).cuda()
    lens = [shared + n for n in own]
    a, la = call(torch, peqa, cache, q, lens, max(lens), 6, shared, 0.09)
    b, lb = torch.empty_like(q), torch.empty((6, 16), device="cuda")
    room = peqa.paged_attention_workspace_bytes(cache, 16, 6, max(lens))
    peqa.paged_attention(cache, q, torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens), 0.09, b, torch.empty(room, dtype=torch.uint8, device="cuda"),
                         room, lse=lb)
    _, _, size = reference(cache, q, lens, max(lens), 6, shared, 0.09)
    off = (a.double() - b.double()).abs().cpu().numpy() - 2.0 ** -8 * a.double().abs().cpu().numpy() - 2.0 ** -9 * size
    assert off.max() <= 0 and float((la - lb).abs().max()) <= 2.0 ** -13


@pytest.mark.parametrize("group", [1, 8])
def test_what_scores_can_be(env, group):
    """Scores that rise along the positions by hundreds, all alike, a scale of 0, values that are infinite or far apart in size."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(7)
    shared, own, dim = 600, [50, 300, 7], 64
    cache = both(torch, peqa, gen, shared, own, 1, dim, 16, False)
    lens = [shared + n for n in own]
    q = torch.randn((3, group, dim), generator=gen).to(torch.bfloat16).cuda()
    k, table = cache.tensors[0], cache.tensors[2].cpu()
    for s, n in ((3, shared), (0, 650), (1, 900), (2, 607)):
        for b in range(0 if s == 3 else shared // 16, -(-n // 16)):
            slope = torch.linspace(0.5 * b, 0.5 * b + 0.47, 16)[None, :, None]
            k[int(table[s, b])] = (torch.ones((1, 16, dim)) * slope).to(torch.bfloat16).cuda()
    q.fill_(1.0)
    for scale in (0.25, -0.25, 0.0, 1e-3, 40.0):
        check(torch, peqa, cache, q, lens, max(lens), 3, shared, scale=scale)
    v = cache.tensors[1]
    v[int(table[3, 2]), 0, 3, 5] = float("inf")
    v[int(table[3, 2]), 0, 3, 6] = -float("inf")
    v[int(table[0, 39]), 0, 1, 7] = float("inf")
    out, _ = call(torch, peqa, cache, q, lens, max(lens), 3, shared, 1e-3)
    got = out.float().cpu()
    assert bool((got[:, :, 5] == math.inf).all()) and bool((got[:, :, 6] == -math.inf).all()) and bool((got[0, :, 7] == math.inf).all())
    got[:, :, 5:7] = 0
    got[0, :, 7] = 0
    assert bool(got.isfinite().all())


def test_far_places(env):
    """Pages past 2^31 elements of a pool, two workspaces, streams of their own."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(9)
    page, dim, pages = 256, 128, 40000                          # 2.6 GB a pool
    k, v = (torch.zeros((pages, 2, page, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.tensor([[1, 39990], [2, 39991], [39999, 7]], dtype=torch.int32, device="cuda")
    for p in table.flatten().tolist():
        k[p], v[p] = (torch.randn((2, page, dim), generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    cache = peqa.kv_cache(k, v, table)
    q = torch.randn((2, 4, dim), generator=gen).to(torch.bfloat16).cuda()
    check(torch, peqa, cache, q, [400, 512], 512, 2, 300)
    want = [call(torch, peqa, cache, q * f, [400, 512], 512, 2, 300, 0.1)[0] for f in (1.0, 2.0)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for s, f in zip(streams, (1.0, 2.0)):
        with torch.cuda.stream(s):
            got.append(call(torch, peqa, cache, q * f, [400, 512], 512, 2, 300, 0.1)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_replayed(env):
    """A captured call, replayed over new queries, contents and lengths, against eager calls."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(10)
    shared, own, dim, heads = 500, [200] * 5, 128, 8
    cache = both(torch, peqa, gen, shared, own, 2, dim, 16, False)
    q = torch.randn((5, heads, dim), generator=gen).to(torch.bfloat16).cuda()
    lens = torch.tensor([700] * 5, dtype=torch.int32, device="cuda")
    room = peqa.shared_attention_workspace_bytes(cache, heads, 5, 700, shared)
    got, sums, ws = torch.empty_like(q), torch.empty((5, heads), device="cuda"), torch.empty(room, dtype=torch.uint8, device="cuda")
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        peqa.shared_attention(cache, q, lens, 700, 5, shared, 0.09, got, ws, room, lse=sums)
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            peqa.shared_attention(cache, q, lens, 700, 5, shared, 0.09, got, ws, room, lse=sums)
    for i in range(4):
        q.copy_(torch.randn(q.shape, generator=gen).to(torch.bfloat16))
        lens.copy_(torch.randint(0, 701, (5,), generator=gen, dtype=torch.int32))
        out, lse = call(torch, peqa, cache, q, lens.tolist(), 700, 5, shared, 0.09)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(sums, lse), i

"""Attention that adds up what positions were given (peqa_paged_attention_weights) and eviction by it (peqa_cache_evict) against plain
implementations.

Tolerances.  What a position is given is exp(x - lse): the scores' fp32 rounding (under 2^-16 for the scores of these inputs), that of lse and the
exponential's, 2^-20 each, so 2^-14 of what is added, and fp32 sums of up to 70 numbers, 2^-17 of it and of what was there before.  Which
positions stay, and what is moved, is exact."""
import numpy as np
import pytest

from test_gpu_decode import make_cache, read, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_2305_14152_amd import peqa
    peqa.lib()
    return torch, peqa


def given(cache, q, lse, lens, max_len, scale, window=0, seq=None):
    """What the positions of every sequence and key head are given, and how many positions of a sequence there are."""
    rows, heads, dim = q.shape
    q, group = q.float().cpu().double().numpy(), heads // cache.kv_heads
    w, longest = np.zeros((cache.n_seqs, cache.kv_heads, max(1, max_len))), np.zeros(cache.n_seqs, int)
    for r in range(rows):
        s, n = r if seq is None else seq[r], min(lens[r], max_len)
        if n <= 0 or not 0 <= s < cache.n_seqs:
            continue
        longest[s] = max(longest[s], n)
        for h in range(cache.kv_heads):
            k, there = read(cache, 0, s, h, n)
            take = there & (np.arange(n) >= (max(0, n - window) if window else 0))
            for i in range(h * group, (h + 1) * group):
                if take.any():
                    w[s, h, :n][take] += np.exp(k[take] @ q[r, i] * scale - lse[r, i])
    return w, longest


def check_weights(torch, peqa, gen, cache, q, lens, max_len, window=0, seq=None, first=True):
    rows, heads, dim = q.shape
    scale = dim ** -0.5
    out, lse = (torch.empty_like(q) for _ in range(2)), (torch.empty((rows, heads), device="cuda") for _ in range(2))
    (a, b), (la, lb) = out, lse
    index = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    room = peqa.paged_attention_workspace_bytes(cache, heads, rows, max_len, window)
    peqa.paged_attention(cache, q, index(lens), max_len, scale, a, torch.empty(room, dtype=torch.uint8, device="cuda"), room, lse=la, seq=index(seq),
                         window=window)
    room = peqa.paged_attention_weights_workspace_bytes(cache, heads, rows, max_len, window)
    ws = torch.full((room,), 255, dtype=torch.uint8, device="cuda")
    before = torch.rand((cache.n_seqs, cache.kv_heads, -(-max(1, max_len) // 4) * 4 + 8), generator=gen).cuda()
    after = torch.full_like(before, -7.0)
    args = (cache, q, index(lens), max_len, scale, b)
    peqa.paged_attention_weights(*args, before, after, ws, room, lse=lb, seq=index(seq), window=window)
    assert torch.equal(a, b) and torch.equal(la, lb)
    _, exact_lse, _ = reference(cache, q, lens, max_len, scale, window, seq)
    want, longest = given(cache, q, exact_lse, lens, max_len, scale, window, seq)
    got, old = after.cpu().double().numpy(), before.cpu().double().numpy()
    for s in range(cache.n_seqs):
        n = longest[s]
        assert (got[s, :, n:] == -7.0).all()
        off = np.abs(got[s, :, :n] - old[s, :, :n] - want[s, :, :n]) - 2.0 ** -14 * want[s, :, :n] - 2.0 ** -17 * (old[s, :, :n] + want[s, :, :n])
        assert n == 0 or off.max() <= 0, (s, off.max())
    # in place, without what was there before, without lse: the same sums
    same = before.clone()
    peqa.paged_attention_weights(*args, same, same, ws, room, seq=index(seq), window=window)
    new = torch.full_like(before, -7.0)
    peqa.paged_attention_weights(*args, None, new, ws, room, seq=index(seq), window=window)
    for s in range(cache.n_seqs):
        n = longest[s]
        assert torch.equal(same[s, :, :n], after[s, :, :n]) and torch.equal(same[s, :, n:], before[s, :, n:])
        assert torch.equal(new[s, :, :n] + before[s, :, :n], after[s, :, :n]) and bool((new[s, :, n:] == -7.0).all())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,kv,group,dim,page,window", [
    ([1], 1, 1, 64, 8, 0), ([333], 8, 1, 128, 16, 0), ([5, 0, 64, 65, 31, -3], 2, 4, 64, 8, 0), ([700, 1, 33], 2, 8, 128, 32, 100), ([200] * 4, 1, 12, 128, 64, 0),
    ([100, 257], 3, 16, 256, 16, 0), ([9000], 2, 2, 64, 128, 0), ([50] * 40, 16, 1, 64, 16, 7), ([4000, 2500, 17], 4, 3, 128, 16, 0), ([1500] * 3, 2, 20, 64, 8, 999)])
def test_weights(env, lens, kv, group, dim, page, window, fp8):
    torch, peqa = env
    gen = torch.Generator().manual_seed(sum(lens) + dim)
    cache = make_cache(torch, peqa, gen, [max(0, n) for n in lens], kv, dim, page, fp8=fp8)
    q = torch.randn((len(lens), kv * group, dim), generator=gen).to(torch.bfloat16).cuda()
    check_weights(torch, peqa, gen, cache, q, lens, max(lens), window)
    if max(lens) > 50:
        check_weights(torch, peqa, gen, cache, q, lens, max(lens) - 3, window)


def test_weights_of_rows_of_one_sequence(env):
    """Several new tokens of a sequence, rows whose sequence is none, pages that are not there: sums in the rows' order."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(1)
    cache = make_cache(torch, peqa, gen, [600, 40, 300], 2, 64, 16)
    cache.tensors[2][0, 3] = -1
    cache.tensors[2][2, :] = cache.n_pages
    seq, lens = [0] * 70 + [1, 5, 0, 2, -1, 1], list(range(500, 570)) + [40, 30, 3, 300, 20, 39]
    q = torch.randn((len(seq), 6, 64), generator=gen).to(torch.bfloat16).cuda()
    check_weights(torch, peqa, gen, cache, q, lens, 600, 0, seq)


def evicted(w, n, keep, sinks, recent):
    """The positions of one head that stay."""
    if n <= keep:
        return np.arange(n)
    mid = np.arange(sinks, n - recent)
    key = np.where(np.isnan(w[mid]), -np.inf, w[mid])
    order = np.lexsort((mid, -key, np.isnan(w[mid])))          # NaN behind -inf
    return np.sort(np.concatenate((np.arange(sinks), mid[order[:keep - sinks - recent]], np.arange(n - recent, n))))


def check_evict(torch, peqa, gen, cache, lens, max_len, keep, sinks, recent, weights, seq=None, to=None, page=None):
    n, kv, bits = len(lens), cache.kv_heads, torch.int16 if cache.dtype == 0 else torch.uint8
    target = cache if to is None else to
    old = [p.view(bits).cpu().numpy().copy() for p in cache.tensors[:2]]
    want = [p.view(bits).cpu().numpy().copy() for p in target.tensors[:2]]
    w = weights.cpu().numpy()
    after = torch.full_like(weights, -7.0)
    expect_after = after.cpu().numpy().copy()
    kept = torch.full((n, kv, keep), 77, dtype=torch.int32, device="cuda")
    new_lens = torch.full((n,), 77, dtype=torch.int32, device="cuda")
    expect, expect_lens = np.full((n, kv, keep), -1), np.zeros(n, int)
    table, goals = cache.tensors[2].cpu().numpy(), target.tensors[2].cpu().numpy()
    seen = {}
    for i in range(n):
        s = i if seq is None else seq[i]
        if not 0 <= s < cache.n_seqs:
            continue
        if s in seen:
            expect_lens[i] = expect_lens[seen[s]]
            continue
        seen[s] = i
        m = max(0, min(lens[i], max_len))
        expect_lens[i] = min(m, keep)
        if m == 0:
            continue
        for h in range(kv):
            stay = evicted(w[s, h], m, keep, sinks, recent)
            expect[i, h, :len(stay)] = stay
            expect_after[s, h, :max_len] = 0
            expect_after[s, h, :len(stay)] = w[s, h, stay]
            for j, p in enumerate(stay):
                if to is None and j == p:
                    continue
                a, b = table[s, p // cache.page_size], goals[s, j // target.page_size]
                if 0 <= b < target.n_pages:
                    for x, y in zip(old, want):
                        y[b, h, j % target.page_size] = x[a, h, p % cache.page_size] if 0 <= a < cache.n_pages else 0
    index = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    room = peqa.cache_evict_workspace_bytes(cache, n, max_len, keep)
    ws = torch.full((room,), 255, dtype=torch.uint8, device="cuda")
    start = [p.view(bits).clone() for p in cache.tensors[:2]]
    peqa.cache_evict(cache, index(lens), max_len, weights, after, keep, sinks, recent, kept, new_lens, ws, room, seq=index(seq), to=to)
    assert (kept.cpu().numpy() == expect).all()
    assert (new_lens.cpu().numpy() == expect_lens).all()
    assert np.array_equal(after.cpu().numpy(), expect_after, equal_nan=True)
    for p, y in zip(target.tensors[:2], want):
        assert (p.view(bits).cpu().numpy() == y).all()
    # weights in their own place, nothing asked for beside: the same
    if to is None:
        for p, o in zip(cache.tensors[:2], start):
            p.view(bits).copy_(o)
    both = weights.clone()
    peqa.cache_evict(cache, index(lens), max_len, both, both, keep, sinks, recent, None, None, ws, room, seq=index(seq), to=to)
    done = after != -7.0
    assert torch.equal(both[done].nan_to_num(5e4), after[done].nan_to_num(5e4)) and torch.equal(both[~done].nan_to_num(5e4), weights[~done].nan_to_num(5e4))
    for p, y in zip(target.tensors[:2], want):
        assert (p.view(bits).cpu().numpy() == y).all()


def some_weights(torch, gen, cache, room, kind):
    w = torch.randn((cache.n_seqs, cache.kv_heads, -(-room // 4) * 4), generator=gen)
    if kind == "heavy":
        w = torch.exp(3 * w)
    elif kind == "ties":
        w = torch.randint(0, 3, w.shape, generator=gen).float() - 0.0
        w[w == 0] = torch.where(torch.rand(int((w == 0).sum()), generator=gen) < 0.5, 0.0, -0.0)
    elif kind == "same":
        w = torch.full_like(w, 0.25)
    elif kind == "odd":                                       # infinities, NaN of both signs, the least numbers
        odd = torch.tensor([float("inf"), -float("inf"), float("nan"), -float("nan"), 1e-45, -1e-45, 0.0, 3.4e38])
        w = odd[torch.randint(0, 8, w.shape, generator=gen)]
    return w.cuda()


EVICT = [([1], 1, 64, 8, 1, 0, 0), ([2], 1, 64, 8, 1, 0, 0), ([2], 1, 64, 8, 1, 0, 1), ([333], 2, 128, 16, 100, 4, 30), ([100, 0, 50, 51, 700, -2], 3, 64, 32, 50, 1, 9),
         ([1500] * 2, 2, 256, 64, 1499, 0, 0), ([2500, 1025, 1024, 1023], 1, 64, 16, 1024, 1000, 24), ([5000], 1, 64, 128, 17, 0, 16), ([3000, 2047], 2, 128, 16, 1900, 16, 900),
         ([64] * 300, 1, 64, 8, 33, 1, 7)]


@pytest.mark.parametrize("lens,kv,dim,page,keep,sinks,recent", EVICT)
@pytest.mark.parametrize("fp8,kind,layout", [(False, "heavy", "heads"), (True, "ties", "slots"), (False, "odd", "both"), (True, "same", "heads"), (False, "any", "slots")])
def test_evict(env, lens, kv, dim, page, keep, sinks, recent, fp8, kind, layout):
    torch, peqa = env
    gen = torch.Generator().manual_seed(sum(lens) + keep)
    caps = [max(0, n) for n in lens]
    cache = make_cache(torch, peqa, gen, caps, kv, dim, page, fp8=fp8, layout=layout, scales=False)
    weights = some_weights(torch, gen, cache, max(lens) + 5, kind)
    # to a cache with pages of another size, then (this one is as it was) in place
    to = make_cache(torch, peqa, gen, [min(n, keep) for n in caps], kv, dim, 16 if page != 16 else 8, fp8=fp8, scales=False)
    check_evict(torch, peqa, gen, cache, lens, max(lens), keep, sinks, recent, weights, to=to)
    check_evict(torch, peqa, gen, cache, lens, max(lens), keep, sinks, recent, weights)


@pytest.mark.parametrize("in_place", [True, False])
def test_evict_entries(env, in_place):
    """Sequences in any order, one twice, some that are none; pages that are not there; lengths past the bound."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(3)
    caps = [200, 150, 90, 300, 40]
    cache = make_cache(torch, peqa, gen, caps, 2, 64, 16)
    cache.tensors[2][1, 2] = -1
    cache.tensors[2][3, 0] = 2 ** 31 - 1
    to = None
    if not in_place:
        to = make_cache(torch, peqa, gen, [60] * 5, 2, 64, 32)
        to.tensors[2][3, 1] = -5
    weights = some_weights(torch, gen, cache, 300, "heavy")
    check_evict(torch, peqa, gen, cache, [300, 90, 70, 150, 12, 33, 400], 280, 60, 3, 10, weights, seq=[3, 2, 3, 1, -1, 5, 0], to=to)


def test_evict_replayed(env):
    """A captured eviction and the attention behind it, replayed over new contents and lengths, against eager calls."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(4)
    cap, keep, kv, heads, dim = 500, 200, 2, 8, 64
    cache = make_cache(torch, peqa, gen, [cap] * 3, kv, dim, 16, poison=False)
    q = torch.randn((3, heads, dim), generator=gen).to(torch.bfloat16).cuda()
    lens = torch.zeros(3, dtype=torch.int32, device="cuda")
    weights = torch.zeros((3, kv, cap), device="cuda")
    r1, r2 = peqa.paged_attention_weights_workspace_bytes(cache, heads, 3, cap), peqa.cache_evict_workspace_bytes(cache, 3, cap, keep)

    def step(state, wa, wb):
        out, kept, new_lens = state
        peqa.paged_attention_weights(cache, q, lens, cap, 0.125, out, weights, weights, wa, r1)
        peqa.cache_evict(cache, lens, cap, weights, weights, keep, 2, 50, kept, new_lens, wb, r2)
        peqa.paged_attention_weights(cache, q, new_lens, keep, 0.125, out, weights, weights, wa, r1)

    def fresh():
        return [torch.empty_like(q), torch.empty((3, kv, keep), dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")]

    def rooms():
        return [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (r1, r2)]
    got, ws = fresh(), rooms()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step(got, *ws)
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step(got, *ws)
    for i in range(4):
        for p in cache.tensors[:2]:
            p.copy_(torch.randn(p.shape, generator=gen).to(torch.bfloat16))
        lens.copy_(torch.randint(1, cap + 1, (3,), generator=gen, dtype=torch.int32))
        weights.copy_(torch.rand(weights.shape, generator=gen))
        start = [weights.clone()] + [p.clone() for p in cache.tensors[:2]]
        want = fresh()
        step(want, *rooms())
        ends = [weights.clone()] + [p.clone() for p in cache.tensors[:2]]
        for t, o in zip([weights, *cache.tensors[:2]], start):
            t.copy_(o)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        assert all(torch.equal(a, b) for a, b in zip([weights, *cache.tensors[:2]], ends)), i


@pytest.mark.parametrize("fp8", [False, True])
def test_far_places(env, fp8):
    """Pages past 2^31 elements of a pool: appended to, attended to and evicted as in a small pool, on two streams at once."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(12)
    page, dim, kv, heads, keep = 256, 128, 2, 4, 200
    dtype, bits = (torch.float8_e4m3fn, torch.uint8) if fp8 else (torch.bfloat16, torch.int16)
    near, far = [0, 1, 2, 3], [1, 39990, 39999, 2]
    pools = [[torch.zeros((n, kv, page, dim), dtype=dtype, device="cuda") for _ in range(4)] for n in (4, 40000)]
    for which in range(2):
        data = torch.randn((4, kv, page, dim), generator=gen).to(dtype).cuda()
        pools[0][which].view(bits).copy_(data.view(bits))
        for a, b in zip(near, far):
            pools[1][which].view(bits)[b] = data.view(bits)[a]
    scales = [torch.full((kv,), 0.5, device="cuda") for _ in range(2)] if fp8 else [None, None]
    lens = torch.tensor([400, 511], dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn((2, n, dim), generator=gen).to(torch.bfloat16).cuda() for n in (heads, kv, kv))
    weights = torch.rand((2, kv, 512), generator=gen).cuda()
    start, results = torch.cuda.Event(), []
    streams = [torch.cuda.Stream() for _ in range(2)]
    caches = []
    for pool, pages in zip(pools, (near, far)):
        table = torch.tensor(pages, dtype=torch.int32, device="cuda").view(2, 2)
        caches.append([peqa.kv_cache(pool[i], pool[i + 1], table, *scales) for i in (0, 2)])
    torch.cuda.synchronize()
    start.record()
    for stream, (cache, to) in zip(streams, caches):
        with torch.cuda.stream(stream):
            stream.wait_event(start)
            qo, out, w = torch.empty_like(q), torch.empty_like(q), weights.clone()
            kept, left = torch.empty((2, kv, keep), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
            peqa.norm_rope_append(cache, q, k, v, lens, None, None, None, None, 1e-6, qo, place=lens)
            r1, r2 = peqa.paged_attention_weights_workspace_bytes(cache, heads, 2, 512), peqa.cache_evict_workspace_bytes(cache, 2, 512, keep)
            w1, w2 = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in (r1, r2))
            peqa.paged_attention_weights(cache, qo, lens, 512, 0.1, out, w, w, w1, r1)
            elsewhere = torch.zeros_like(w)
            peqa.cache_evict(cache, lens, 512, w, elsewhere, keep, 3, 20, kept, left, w2, r2, to=to)
            peqa.cache_evict(cache, lens, 512, w, w, keep, 3, 20, kept, left, w2, r2)
            results.append([qo, out, w, elsewhere, kept, left])
    torch.cuda.synchronize()
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert torch.equal(results[0][2], results[0][3]) and results[0][5].tolist() == [keep] * 2
    for small, big in zip(*pools):
        for a, b in zip(near, far):
            assert torch.equal(small.view(bits)[a], big.view(bits)[b])


def test_in_place_by_name(env):
    """The cache itself as the one that positions go to, and another descriptor of the same pools: in place.  Its own spare pages: elsewhere."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(13)
    lens, results = [300, 77, 450], []
    for name in ("none", "itself", "alike", "spare"):
        gen.manual_seed(13)
        cache = make_cache(torch, peqa, gen, [450] * 6, 2, 64, 16)
        table = cache.tensors[2]
        spare = table[3:].clone()
        table[3:] = -1
        goal = table if name != "spare" else torch.cat((spare, table[3:]))
        to = None if name == "none" else cache if name == "itself" else peqa.kv_cache(*cache.tensors[:2], goal)
        weights = torch.rand((6, 2, 452), generator=gen).cuda()
        kept = torch.empty((3, 2, 100), dtype=torch.int32, device="cuda")
        room = peqa.cache_evict_workspace_bytes(cache, 3, 450, 100)
        ws = torch.empty(room, dtype=torch.uint8, device="cuda")
        before = [cache.tensors[w][table[:3].long()].clone() for w in (0, 1)]
        peqa.cache_evict(cache, torch.tensor(lens, dtype=torch.int32, device="cuda"), 450, weights, weights, 100, 4, 30, kept, None, ws, room, to=to)
        at = goal[:3].long()
        rows = [cache.tensors[w][at].permute(0, 2, 1, 3, 4).flatten(2, 3)[s, :, :min(100, lens[s])] for w in (0, 1) for s in range(3)]
        results.append([kept, weights] + rows)
        if name == "spare":
            assert all(torch.equal(cache.tensors[w][table[:3].long()].view(torch.int16), before[w].view(torch.int16)) for w in (0, 1))
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)

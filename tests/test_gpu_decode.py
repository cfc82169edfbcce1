"""The paged-cache calls (peqa_rope_append, peqa_paged_attention) against plain implementations in 64 bits.

Tolerances.  Stored bf16 numbers: half a unit in the last of 8 places (at most 2^-8 of the number), and of the fp32 rotation before
it 2^-21 of the pair's size.  Stored 8-bit numbers: half a step, 2^-4 of the number or half of the least one, 2^-10.
Attention: with w the weights, v the values, a relative error of every weight of at most E moves the output by 2 E sum w |v|.
E adds the scores' fp32 rounding (under 2^-16 for the scores of these inputs), the exponential's (2^-20) and that of the weights:
2^-17 in two bf16 parts, 2^-12 as fp16; taken are 2^-14 and 2^-10 of sum w |v| in all, and bf16's 2^-8 of the output."""
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


def make_cache(torch, peqa, gen, lens, kv_heads, dim, page, fp8=False, layout="heads", spare=3, scales=True, poison=True):
    """Pools with pages in random places for sequences of the given capacities, NaN wherever no position is."""
    needed = [max(1, -(-n // page)) for n in lens]
    total = sum(needed) + spare
    shape = {"heads": (total, kv_heads, page, dim), "slots": (total, page, kv_heads, dim), "both": (total, 2, kv_heads, page, dim)}[layout]

    def pool(shape):
        x = torch.randn(shape, generator=gen)
        return ((x * 20).clamp(-448, 448).to(torch.float8_e4m3fn) if fp8 else x.to(torch.bfloat16)).cuda()
    if layout == "both":
        b = pool(shape)
        k, v = b[:, 0], b[:, 1]
    else:
        k, v = pool(shape), pool(shape)
        if layout == "slots":
            k, v = k.transpose(1, 2), v.transpose(1, 2)
    order = torch.randperm(total, generator=gen)[:sum(needed)]
    table = torch.full((len(lens), max(needed) + 1), 0x7FFFFFF0, dtype=torch.int32)
    at, used = 0, torch.zeros((total, page), dtype=torch.bool)
    for i, n in enumerate(needed):
        table[i, :n] = order[at:at + n].to(torch.int32)
        for j in range(lens[i]):
            used[order[at + j // page], j % page] = True
        at += n
    if poison:
        hole = (~used).cuda()[:, None, :, None].expand(total, kv_heads, page, dim)
        for x in (k, v):
            y = x.view(torch.uint8) if fp8 else x.view(torch.int16)
            y.masked_fill_(hole, 0x7F if fp8 else 0x7FC0)
    ks = vs = None
    if fp8 and scales:
        ks, vs = (0.02 + 0.05 * torch.rand(kv_heads, generator=gen)).cuda(), (0.02 + 0.05 * torch.rand(kv_heads, generator=gen)).cuda()
    table = table.cuda()[:, :max(needed)]                       # a row stride of its own
    return peqa.kv_cache(k, v, table, ks, vs)


def read(cache, which, seq, head, n):
    """Positions 0 .. n-1 of one head, in 64 bits on the host, and which of them are there."""
    import torch
    pool, table, scale = cache.tensors[which], cache.tensors[2].cpu(), cache.tensors[3 + which]
    page = cache.page_size
    rows, there = [], []
    for b in range(-(-n // page)):
        p = int(table[seq, b])
        ok = 0 <= p < cache.n_pages
        x = pool[p if ok else 0, head]
        rows.append(x.float().cpu().double())
        there += [ok] * page
    x = torch.cat(rows)[:n].numpy()
    if scale is not None:
        x = x * float(scale[head])
    return x, np.array(there[:n], bool)


def reference(cache, q, lens, max_len, scale, window=0, seq=None):
    rows, heads, dim = q.shape
    q = q.float().cpu().double().numpy()
    group = heads // cache.kv_heads
    out, lse, size = np.zeros(q.shape), np.full((rows, heads), -math.inf), np.zeros(q.shape)
    for r in range(rows):
        s = r if seq is None else seq[r]
        n = min(lens[r], max_len)
        if n <= 0 or not 0 <= s < cache.n_seqs:
            continue
        lo = max(0, n - window) if window else 0
        for h in range(cache.kv_heads):
            k, there = read(cache, 0, s, h, n)
            v, _ = read(cache, 1, s, h, n)
            take = there & (np.arange(n) >= lo)
            if not take.any():
                continue
            k, v = k[take], v[take]
            for i in range(h * group, (h + 1) * group):
                z = k @ q[r, i] * scale
                m = z.max()
                w = np.exp(z - m)
                lse[r, i] = m + math.log(w.sum())
                w /= w.sum()
                out[r, i] = w @ v
                size[r, i] = w @ np.abs(v)
    return out, lse, size


def check_attention(torch, peqa, cache, q, lens, max_len, window=0, seq=None, scale=None, fp8=False):
    rows, heads, dim = q.shape
    scale = dim ** -0.5 if scale is None else scale
    dev = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    # rows of an output with room between them, which stays
    wide = torch.full((rows, heads * dim + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide[:, :heads * dim].unflatten(1, (heads, dim))
    lse = torch.full((rows, heads), 7.0, device="cuda")
    room = peqa.paged_attention_workspace_bytes(cache, heads, rows, max_len, window)
    assert room > 0
    ws = torch.full((room,), 0xFF, dtype=torch.uint8, device="cuda")
    peqa.paged_attention(cache, q, dev(lens), max_len, scale, out, ws, room, lse=lse, seq=dev(seq), window=window)
    first = out.clone()
    want, want_lse, size = reference(cache, q, lens, max_len, scale, window, seq)
    got = out.float().cpu().double().numpy()
    assert np.isfinite(got).all()
    off = np.abs(got - want) - (2.0 ** -8 * np.abs(want) * 1.01 + 2.0 ** (-10 if fp8 else -14) * size + 1e-30)
    assert (off <= 0).all(), (off.max(), np.unravel_index(off.argmax(), off.shape))
    got_lse = lse.cpu().double().numpy()
    empty = np.isinf(want_lse)
    assert (got_lse[empty] == -math.inf).all()
    assert (np.abs(got_lse[~empty] - want_lse[~empty]) <= 2.0 ** -14 * (1 + np.abs(want_lse[~empty]))).all()
    assert (wide[:, heads * dim:] == 7.0).all()
    peqa.paged_attention(cache, q, dev(lens), max_len, scale, out, ws, room, seq=dev(seq), window=window)      # without lse: the same bits
    assert torch.equal(out, first)


LENS = [0, 1, 7, 8, 9, 31, 32, 33, 127, 128, 129, 300, 513]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim,page,layout", [
    (4, 4, 128, 16, "heads"), (8, 2, 128, 8, "slots"), (10, 2, 64, 32, "both"), (16, 2, 128, 64, "heads"), (18, 2, 64, 16, "slots"),
    (12, 1, 128, 1024, "heads"), (40, 2, 128, 16, "both"), (3, 3, 256, 16, "heads"), (34, 2, 256, 128, "slots"), (1, 1, 64, 8, "heads"),
    (33, 1, 128, 16, "heads"), (16, 1, 256, 8, "both"),
])
def test_attention(env, fp8, heads, kv_heads, dim, page, layout):
    torch, peqa = env
    print("attention", fp8, heads, kv_heads, dim, page, layout, flush=True)
    gen = torch.Generator().manual_seed(1000 + heads + dim + page)
    cache = make_cache(torch, peqa, gen, LENS, kv_heads, dim, page, fp8, layout)
    q = torch.randn((len(LENS), heads, dim), generator=gen).to(torch.bfloat16).cuda()
    check_attention(torch, peqa, cache, q, LENS, 513, fp8=fp8)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 100, 512, 513, 2 ** 31 - 1])
def test_window(env, fp8, window):
    torch, peqa = env
    print("window", fp8, window, flush=True)
    gen = torch.Generator().manual_seed(window % 1000)
    cache = make_cache(torch, peqa, gen, LENS, 2, 128, 16, fp8)
    q = torch.randn((len(LENS), 4, 128), generator=gen).to(torch.bfloat16).cuda()
    check_attention(torch, peqa, cache, q, LENS, 513, window=window, fp8=fp8)


@pytest.mark.parametrize("fp8,heads,kv_heads,dim,lens", [
    (False, 2, 1, 128, [20001]), (True, 2, 1, 128, [20001, 5]), (False, 24, 2, 64, [9000, 1, 0]), (True, 20, 1, 256, [7777, 4097]),
    (False, 16, 8, 256, [4100, 33]), (False, 1, 1, 128, [70000]),
])
def test_split_and_joined(env, fp8, heads, kv_heads, dim, lens):
    """Lengths that are cut into many chunks beside ones of a single chunk or none."""
    torch, peqa = env
    print("split", fp8, heads, kv_heads, dim, lens, flush=True)
    gen = torch.Generator().manual_seed(heads + dim)
    cache = make_cache(torch, peqa, gen, lens, kv_heads, dim, 32, fp8)
    q = torch.randn((len(lens), heads, dim), generator=gen).to(torch.bfloat16).cuda()
    check_attention(torch, peqa, cache, q, lens, max(lens), fp8=fp8)
    check_attention(torch, peqa, cache, q, lens, max(lens), window=5000, fp8=fp8)


@pytest.mark.parametrize("fp8,heads,kv_heads,dim,rows,most,window", [
    (False, 8, 8, 128, 20, 16384, 0), (True, 32, 4, 128, 40, 16384, 0), (False, 24, 2, 64, 50, 32768, 0), (True, 34, 2, 256, 60, 16384, 0),
    (False, 5, 5, 256, 30, 16384, 0), (False, 4, 4, 128, 1000, 2048, 0), (True, 4, 4, 64, 300, 4096, 1500), (False, 18, 1, 128, 200, 16384, 0),
    (True, 8, 4, 128, 100, 16384, 3000), (False, 3, 3, 64, 90, 16384, 4097),
])
def test_equal_shares(env, fp8, heads, kv_heads, dim, rows, most, window):
    """Bounds that make a launch of equal shares of all rows: few long rows among short and empty ones, in every order of lengths."""
    torch, peqa = env
    print("shares", fp8, heads, kv_heads, dim, rows, most, window, flush=True)
    gen = torch.Generator().manual_seed(rows + dim)
    lens = [int(n) for n in torch.randint(0, 200, (rows,), generator=gen)]
    for r, n in ((0, 0), (1, 1), (2, min(most, 4500)), (3, 64), (rows // 2, min(most, 9000)), (rows - 2, 2047), (rows - 1, 0)):
        lens[r] = n
    page = 64
    cache = make_cache(torch, peqa, gen, lens, kv_heads, dim, page, fp8)
    k, v, table, ks, vs = cache.tensors
    wide = torch.full((rows, most // page), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    cache = peqa.kv_cache(k, v, wide, ks, vs)
    q = torch.randn((rows, heads, dim), generator=gen).to(torch.bfloat16).cuda()
    check_attention(torch, peqa, cache, q, lens, most, window=window, fp8=fp8)
    check_attention(torch, peqa, cache, q, [min(n, 5) for n in lens], most, window=window, fp8=fp8)     # nothing but short rows


@pytest.mark.parametrize("fp8,heads,kv_heads,dim,rows,most,window", [
    (False, 16, 1, 256, 7, 130, 0), (False, 24, 2, 256, 9, 500, 0), (False, 18, 1, 256, 3, 9000, 0), (False, 16, 1, 256, 40, 16384, 0),
    (False, 12, 1, 256, 300, 250, 0), (False, 20, 1, 256, 520, 380, 100), (False, 33, 3, 256, 50, 8192, 3001), (True, 9, 1, 256, 12, 500, 0),
    (True, 17, 1, 256, 600, 200, 0), (False, 4, 4, 128, 520, 380, 0), (True, 2, 2, 64, 1030, 380, 0), (False, 3, 1, 256, 5, 400, 0),
])
def test_wide_heads_and_many_short_rows(env, fp8, heads, kv_heads, dim, rows, most, window):
    """Heads of 256 with more than eight to a key head, and items by the thousand whose rows one wave walks, in every form of a launch."""
    torch, peqa = env
    print("wide", fp8, heads, kv_heads, dim, rows, most, window, flush=True)
    gen = torch.Generator().manual_seed(rows + heads)
    lens = [int(n) for n in torch.randint(0, min(most, 300) + 1, (rows,), generator=gen)]
    lens[0], lens[1], lens[2], lens[rows - 1] = most, 0, 1, min(most, 4200)
    cache = make_cache(torch, peqa, gen, lens, kv_heads, dim, 32, fp8)
    q = torch.randn((rows, heads, dim), generator=gen).to(torch.bfloat16).cuda()
    check_attention(torch, peqa, cache, q, lens, most, window=window, fp8=fp8)


def test_rows_of_one_sequence_and_rows_of_none(env):
    """Several query rows of the same sequence (a prompt's tokens), sequences out of range, lengths past max_len and negative."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(5)
    cache = make_cache(torch, peqa, gen, [200, 64], 2, 128, 16)
    seq = [0, 0, 0, 1, 1, -1, 2, 0, 1]
    lens = [1, 2, 200, 64, 63, 10, 10, 5000, -5]
    q = torch.randn((len(seq), 8, 128), generator=gen).to(torch.bfloat16).cuda()
    check_attention(torch, peqa, cache, q, lens, 200, seq=seq)
    check_attention(torch, peqa, cache, q, lens, 61, seq=seq)        # cut for every row


def test_pages_that_are_not_there(env):
    """Holes in the table: their positions do not count; a row of holes only is empty."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(6)
    for fp8 in (False, True):
        cache = make_cache(torch, peqa, gen, [300, 300, 64], 2, 128, 16, fp8)
        table = cache.tensors[2]
        table[0, 1], table[0, 7], table[0, 18] = -1, cache.n_pages, 2 ** 31 - 1
        table[1, 3:9] = -2 ** 31
        table[2] = -1
        q = torch.randn((3, 4, 128), generator=gen).to(torch.bfloat16).cuda()
        check_attention(torch, peqa, cache, q, [300, 290, 64], 300, fp8=fp8)


def test_large_scores_and_equal_ones(env):
    """Scores far apart (one position takes all) and all equal; a scale of 0."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(7)
    cache = make_cache(torch, peqa, gen, [700], 1, 128, 16)
    q = (torch.randn((1, 8, 128), generator=gen) * 30).to(torch.bfloat16).cuda()
    check_attention(torch, peqa, cache, q, [700], 700, scale=0.0)
    # scores of hundreds: their fp32 rounding, 2^-24 of 128 products, is what moves the weights, under 2^-14 of them
    check_attention(torch, peqa, cache, q, [700], 700, scale=0.25)


@pytest.mark.parametrize("gap", [9.7, 12.1, 17.67])
@pytest.mark.parametrize("lens", [[100], [700, 3], [20001]])
def test_small_weights_of_8_bit_values(env, lens, gap):
    """Some positions `gap` above all others and with values of 0: the result is made of weights of e^-gap, each of which may be
    off by its own rounding only."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(12)
    cache = make_cache(torch, peqa, gen, lens, 1, 128, 32, True, scales=False)
    k, v, table, _, _ = cache.tensors
    k.zero_()
    v.copy_((torch.rand(v.shape, generator=gen) * 100 + 1).to(torch.float8_e4m3fn))
    for r, n in enumerate(lens):
        for j in range(n):
            if j % 1000 < 256 and j % 32 == 3:
                page, slot = int(table[r, j // 32]), j % 32
                k[page, 0, slot, 0] = 16.0
                v[page, 0, slot] = 0.0
    q = torch.zeros((len(lens), 4, 128))
    q[..., 0] = 1.0
    check_attention(torch, peqa, cache, q.to(torch.bfloat16).cuda(), lens, max(lens), scale=gap / 16, fp8=True)


def test_offsets_past_32_bits(env):
    """Pages behind 2^32 bytes and 2^31 elements of a pool."""
    torch, peqa = env
    pages, kv, page, dim = 131072 + 1500, 1, 128, 128
    k = torch.empty((pages, kv, page, dim), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    assert k.numel() > 2 ** 31
    gen = torch.Generator().manual_seed(8)
    used = [pages - 1, 3, pages - 700, 131072]
    for p in used:
        k[p] = torch.randn((kv, page, dim), generator=gen).to(torch.bfloat16).cuda()
        v[p] = torch.randn((kv, page, dim), generator=gen).to(torch.bfloat16).cuda()
    cache = peqa.kv_cache(k, v, torch.tensor([used], dtype=torch.int32, device="cuda"))
    q = torch.randn((1, 4, dim), generator=gen).to(torch.bfloat16).cuda()
    check_attention(torch, peqa, cache, q, [500], 512)
    new = torch.randn((2, 1, dim), generator=gen).to(torch.bfloat16).cuda()
    at = torch.tensor([5, 300], dtype=torch.int32, device="cuda")
    peqa.rope_append(cache, None, new, -new, at, None, None, None, seq=torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert torch.equal(k[used[0], 0, 5], new[0, 0]) and torch.equal(v[used[2], 0, 300 - 256], -new[1, 0])


def test_other_stream_and_graph(env):
    """Append and attention captured together and replayed with new inputs in place, against eager calls."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(9)
    lens = [900, 77, 1]
    cache = make_cache(torch, peqa, gen, [4096, 100, 100], 2, 128, 16, poison=False)
    ref = peqa.kv_cache(cache.tensors[0].clone(), cache.tensors[1].clone(), cache.tensors[2])
    qkv = torch.randn((3, 12, 128), generator=gen).to(torch.bfloat16).cuda()
    q, k, v = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
    pos = torch.tensor([n - 1 for n in lens], dtype=torch.int32, device="cuda")
    n = pos + 1
    cos, sin = torch.rand((4096, 64), device="cuda"), torch.rand((4096, 64), device="cuda")
    room = peqa.paged_attention_workspace_bytes(cache, 8, 3, 4096)
    ws = torch.zeros(room, dtype=torch.uint8, device="cuda")

    def step(c, rotated, out):
        peqa.rope_append(c, q, k, v, pos, cos, sin, rotated)
        peqa.paged_attention(c, rotated, n, 4096, 0.1, out, ws, room)

    rotated, out, rotated2, out2 = (torch.empty((3, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(4))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache, rotated, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cache, rotated, out)
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step(ref, rotated2, out2)
        torch.cuda.synchronize()
        assert torch.equal(got, out2) and torch.equal(rotated, rotated2)
        assert all(torch.equal(a, b) for a, b in zip(cache.tensors[:2], ref.tensors[:2]))
        qkv.copy_(torch.randn(qkv.shape, generator=gen).to(torch.bfloat16))
        pos += 1
        n += 1


# ---- appending ------------------------------------------------------------------------------------------------------

def rotate64(x, cos, sin, interleaved):
    """x [T, heads, dim], cos, sin [T, rot / 2], 64 bits."""
    x = x.copy()
    half = cos.shape[1]
    a, b = (np.arange(half) * 2, np.arange(half) * 2 + 1) if interleaved else (np.arange(half), np.arange(half) + half)
    c, s = cos[:, None], sin[:, None]
    u, w = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    x[..., a], x[..., b] = u, w
    return x


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim,rot,page,layout", [
    (4, 4, 128, 128, 16, "heads"), (8, 2, 64, 64, 8, "slots"), (5, 1, 256, 64, 64, "both"), (3, 3, 128, 16, 1024, "heads"),
    (1, 1, 64, 32, 16, "slots"), (6, 2, 256, 256, 32, "heads"), (2, 2, 128, 0, 16, "both"),
])
def test_append(env, fp8, interleaved, heads, kv_heads, dim, rot, page, layout):
    torch, peqa = env
    print("append", fp8, interleaved, heads, kv_heads, dim, rot, page, layout, flush=True)
    gen = torch.Generator().manual_seed(heads + dim + rot)
    cap = [100, 37, 64]
    cache = make_cache(torch, peqa, gen, cap, kv_heads, dim, page, fp8, layout, poison=False)
    before = [x.clone() for x in cache.tensors[:2]]
    seq, pos = [], []
    for s, n in enumerate(cap):
        for p in range(0, n, 1 + s):
            seq.append(s)
            pos.append(p)
    # tokens that are skipped, and their queries' rows zero: no position, no sequence, past the table, past the rotation's tables
    blocks = cache.n_blocks
    table = cache.tensors[2]
    seq += [0, -1, 3, 0, 0]
    pos += [-1, 0, 0, blocks * page, 10 ** 9]
    skipped = 5
    T = len(pos)
    x = torch.randn((T, (heads + 2 * kv_heads) * dim + 8), generator=gen).to(torch.bfloat16).cuda()
    q, k, v = (x[:, a * dim:b * dim].unflatten(1, (b - a, dim)) for a, b in ((0, heads), (heads, heads + kv_heads), (heads + kv_heads, heads + 2 * kv_heads)))
    n_pos = 128
    ang = np.random.default_rng(rot).uniform(-3, 3, (n_pos, max(rot // 2, 1)))
    cos, sin = (torch.tensor(f(ang), dtype=torch.float32).cuda() for f in (np.cos, np.sin))
    q_out = torch.full((T, heads, dim), 5.0, dtype=torch.bfloat16, device="cuda")
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    peqa.rope_append(cache, q, k, v, dev(pos), cos if rot else None, sin if rot else None, q_out, seq=dev(seq), interleaved=interleaved)
    torch.cuda.synchronize()

    good = slice(0, T - skipped)
    host = lambda a: a.float().cpu().double().numpy()  # noqa: E731
    rows = np.array(pos[good])
    c64, s64 = host(cos)[rows][:, :rot // 2], host(sin)[rows][:, :rot // 2]
    bound = lambda want, size: 2.0 ** -8 * np.abs(want) * 1.01 + 2.0 ** -21 * size  # noqa: E731
    size_of = lambda a: np.abs(a).max(-1, keepdims=True) * 2  # noqa: E731
    want_q = rotate64(host(q)[good], c64, s64, interleaved)
    assert (np.abs(host(q_out)[good] - want_q) <= bound(want_q, size_of(want_q))).all()
    assert (q_out[T - skipped:] == 0).all()
    touched = torch.zeros((cache.n_pages, page), dtype=torch.bool)
    wants = rotate64(host(k)[good], c64, s64, interleaved), host(v)[good]
    for which in range(2):
        pool, want, scale = cache.tensors[which], wants[which], cache.tensors[3 + which]
        got = np.stack([host(pool[int(table[s, p // page]), :, p % page]) for s, p in zip(seq[good], pos[good])])
        if fp8:
            want = want / host(scale)[:, None]
            past = np.abs(want) > 448
            assert (np.abs(got - want)[~past] <= (2.0 ** -4 * np.abs(want) + 2.0 ** -10)[~past] * 1.001 + 1e-6).all()
            assert (np.abs(got[past]) == 448).all() and (np.sign(got) * np.sign(want))[past].all()
        else:
            assert (np.abs(got - want) <= bound(want, size_of(want))).all()
            if which or not rot:
                assert (got == want).all()
        for s, p in zip(seq[good], pos[good]):
            touched[int(table[s, p // page]), p % page] = True
        stay = (~touched).cuda()[:, None, :, None].expand(pool.shape)
        kind = torch.uint8 if fp8 else torch.int16
        assert torch.equal(pool.view(kind)[stay], before[which].view(kind)[stay])
    # in place, and keys and values without queries: the same
    after = [t.clone() for t in cache.tensors[:2]]
    x2 = x.clone()
    q2 = x2[:, :heads * dim].unflatten(1, (heads, dim))
    peqa.rope_append(cache, q2, k, v, dev(pos), cos if rot else None, sin if rot else None, q2, seq=dev(seq), interleaved=interleaved)
    assert torch.equal(q2, q_out) and torch.equal(x2[:, heads * dim:], x[:, heads * dim:])
    peqa.rope_append(cache, None, k, v, dev(pos), cos if rot else None, sin if rot else None, None, seq=dev(seq), interleaved=interleaved)
    kind = torch.uint8 if fp8 else torch.int16
    assert all(torch.equal(a.view(kind), b.view(kind)) for a, b in zip(after, cache.tensors[:2]))


def test_append_special_numbers(env):
    """8-bit storage of what has no 8-bit number: too large ones and infinities become the largest, NaN stays; ties go to even."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(3)
    cache = make_cache(torch, peqa, gen, [16], 1, 64, 16, True, scales=False, poison=False)
    vals = [math.inf, -math.inf, math.nan, 448.0, 460.0, -1e30, 0.0, -0.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 17.0, 19.0, -17.0, 27.0, 1.0625]
    want = [448, -448, math.nan, 448, 448, -448, 0, 0, 2.0 ** -9, 0, 2.0 ** -8, 16, 20, -16, 28, 1.0]
    v = torch.tensor(vals * 4, dtype=torch.bfloat16, device="cuda").view(1, 1, 64)
    peqa.rope_append(cache, None, v, v, torch.tensor([9], dtype=torch.int32, device="cuda"), None, None, None)
    for which in range(2):
        got = cache.tensors[which][int(cache.tensors[2][0, 0]), 0, 9].float().cpu().numpy()
        np.testing.assert_array_equal(got, np.array(want * 4, np.float32))


def test_one_token_of_every_sequence(env):
    """seq left out: token t is sequence t's; a single token."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(4)
    cache = make_cache(torch, peqa, gen, [40, 40, 40], 2, 128, 16, poison=False)
    for T in (3, 1):
        k = torch.randn((T, 2, 128), generator=gen).to(torch.bfloat16).cuda()
        pos = torch.tensor([39, 0, 17][:T], dtype=torch.int32, device="cuda")
        peqa.rope_append(cache, None, k, -k, pos, None, None, None)
        for t in range(T):
            p = int(pos[t])
            page = int(cache.tensors[2][t, p // 16])
            assert torch.equal(cache.tensors[0][page, :, p % 16], k[t]) and torch.equal(cache.tensors[1][page, :, p % 16], -k[t])

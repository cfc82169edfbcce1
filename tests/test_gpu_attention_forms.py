"""Every form of peqa_paged_attention's launch, for every kernel that it can launch: whole items by one, four or eight waves, chunks, equal
shares, each with one column block and two, and items whose positions are walked in several pieces.  The form that a call takes is asked
for, so that a case cannot move to another one unnoticed.  Against 64 bits on the GPU, with the tolerance of tests/test_gpu_decode.py."""
import ctypes
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_2305_14152_amd import peqa
    peqa.lib()
    return torch, peqa


class Plan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("hb", "waves", "blocks", "per_wg", "splits", "chunk_units", "shares", "entries")] + \
               [("grid", ctypes.c_longlong)] + [(n, ctypes.c_size_t) for n in ("part_bytes", "ml_bytes", "parts_bytes")]


def plan_of(peqa, cache, rows, heads, most, window=0):
    f = peqa.lib()._ZN4peqa11attend_planEPK13peqa_kv_cacheiiii          # peqa::attend_plan
    f.argtypes, f.restype = [ctypes.POINTER(peqa.KVCache)] + [ctypes.c_int] * 4, Plan
    return f(ctypes.byref(cache), rows, heads, most, window)


def make_cache(torch, peqa, gen, lens, kv_heads, dim, page, fp8, most):
    """Pages in random places, NaN wherever no position is; tables as long as `most` asks for, what is past a sequence not there."""
    needed = [-(-n // page) for n in lens]
    total = sum(needed) + 2

    def pool():
        x = torch.randn((total, kv_heads, page, dim), device="cuda", generator=gen, dtype=torch.float32 if fp8 else torch.bfloat16)
        return (x * 20).clamp(-448, 448).to(torch.float8_e4m3fn) if fp8 else x
    k, v = pool(), pool()
    order = torch.randperm(total, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((len(lens), -(-most // page)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r, n in enumerate(needed):
        if n:
            table[r, :n] = order[at:at + n]
            at += n
            if lens[r] % page:
                for x in (k, v):
                    x.view(torch.uint8 if fp8 else torch.int16)[int(table[r, n - 1]), :, lens[r] % page:] = 0x7F if fp8 else 0x7FC0
    for x in (k, v):
        x.view(torch.uint8 if fp8 else torch.int16)[order[at:].long()] = 0x7F if fp8 else 0x7FC0
    scales = [0.02 + 0.05 * torch.rand(kv_heads, device="cuda", generator=gen) for _ in range(2)] if fp8 else [None, None]
    return peqa.kv_cache(k, v, table, *scales)


def check(torch, peqa, cache, q, lens, most, window=0):
    """The call against the formula in 64 bits, a row and a key head at a time."""
    rows, heads, dim = q.shape
    k_pool, v_pool, table, k_scale, v_scale = cache.tensors
    fp8, kv_heads, page = k_scale is not None, cache.kv_heads, cache.page_size
    scale = dim ** -0.5
    out, lse = torch.empty_like(q), torch.empty((rows, heads), device="cuda")
    room = peqa.paged_attention_workspace_bytes(cache, heads, rows, most, window)
    ws = torch.full((room,), 0xFF, dtype=torch.uint8, device="cuda")
    peqa.paged_attention(cache, q, torch.tensor(lens, dtype=torch.int32, device="cuda"), most, scale, out, ws, room, lse=lse, window=window)
    want, size = (torch.zeros(q.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    want_lse = torch.full((rows, heads), -math.inf, dtype=torch.float64, device="cuda")
    group = heads // kv_heads
    for r, n in enumerate(lens):
        lo = max(0, n - window) if window else 0
        if n == 0:
            continue
        pages = table[r, lo // page:-(-n // page)]
        there = pages >= 0
        take = there.repeat_interleave(page)
        at = torch.arange(lo // page * page, lo // page * page + take.numel(), device="cuda")
        take &= (at >= lo) & (at < n)
        if not bool(take.any()):
            continue
        index = pages.clamp_min(0).long()
        for h in range(kv_heads):
            k, v = (p.view(torch.uint8 if fp8 else p.dtype)[index, h].view(p.dtype).reshape(-1, dim)[take].double() for p in (k_pool, v_pool))
            if fp8:
                k, v = k * k_scale[h].double(), v * v_scale[h].double()
            mine = slice(h * group, h * group + group)
            z = (q[r, mine].double() @ k.T.contiguous()) * scale
            want_lse[r, mine] = torch.logsumexp(z, 1)
            w = torch.softmax(z, 1)
            want[r, mine], size[r, mine] = w @ v, w @ v.abs()
    off = (out.double() - want).abs() - (2.0 ** -8 * 1.01 * want.abs() + 2.0 ** (-10 if fp8 else -14) * size + 1e-30)
    assert bool((off <= 0).all()), (float(off.max()), int(off.argmax()))
    empty = want_lse.isinf()
    assert torch.equal(lse.isinf(), empty) and bool((lse[empty] < 0).all())
    assert bool(((lse.double() - want_lse).abs()[~empty] <= 2.0 ** -14 * (1 + want_lse.abs()[~empty])).all())
    again = torch.empty_like(q)
    peqa.paged_attention(cache, q, torch.tensor(lens, dtype=torch.int32, device="cuda"), most, scale, again, ws, room, window=window)
    assert torch.equal(again, out)


# rows, key heads, longest row, and what they are to make of it: waves, chunks, shares
FORMS = {
    "one wave": (140, 4, 200, 1, False, False),
    "one wave, longer": (520, 4, 380, 1, False, False),
    "four waves": (9, 2, 100, 4, False, False),
    "four waves, longer": (300, 4, 700, 4, False, False),
    "eight waves": (9, 2, 400, 8, False, False),
    "chunks": (3, 2, 9000, 4, True, False),
    "shares": (40, 4, 5000, 4, False, True),
}


HEADS = [(64, False, 5), (64, False, 11), (64, False, 17), (64, True, 6), (64, True, 16), (64, True, 19), (128, False, 8), (128, False, 16), (128, True, 3),
         (128, True, 9), (128, True, 32), (256, False, 7), (256, False, 9), (256, True, 8), (256, True, 12), (256, True, 18)]


def two_blocks(dim, fp8, group):
    return group > (16 if fp8 else 8) and not (dim == 256 and fp8)


@pytest.mark.parametrize("dim,fp8,group,form", [h + (f,) for f in FORMS for h in HEADS if f != "eight waves" or (h[0] < 256 and not two_blocks(*h))])
def test_every_kernel_in_every_form(env, dim, fp8, group, form):
    torch, peqa = env
    rows, kv_heads, most, waves, chunks, shares = FORMS[form]
    two = two_blocks(dim, fp8, group)
    print("form", form, dim, fp8, group, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(dim + group)
    draw = torch.Generator().manual_seed(rows + group)
    lens = [int(n) for n in torch.randint(0, min(most, 130), (rows,), generator=draw)]
    lens[0], lens[1], lens[2], lens[rows // 2], lens[rows - 1] = most, 1, most * 2 // 3 + 1, 0, min(most, 33)
    cache = make_cache(torch, peqa, gen, lens, kv_heads, dim, 16, fp8, most)
    heads = kv_heads * group
    p = plan_of(peqa, cache, rows, heads, most)
    assert (p.hb, p.waves) == (2 if two else 1, waves) and (p.splits > 1, p.shares > 0, p.entries > 0) == (chunks, shares, chunks or shares), form
    q = torch.randn((rows, heads, dim), device="cuda", generator=gen).to(torch.bfloat16)
    check(torch, peqa, cache, q, lens, most)
    check(torch, peqa, cache, q, lens, most, window=most // 2 + 3)


@pytest.mark.parametrize("dim,fp8,group", [(128, False, 1), (64, True, 2), (256, False, 3), (128, True, 17)])
@pytest.mark.parametrize("rows", [257, 300, 500])
def test_shares_of_more_rows_than_a_workgroup_has_threads(env, dim, fp8, group, rows):
    torch, peqa = env
    print("many rows", dim, fp8, group, rows, flush=True)
    gen, draw, most = torch.Generator(device="cuda").manual_seed(rows), torch.Generator().manual_seed(rows + group), 2500
    lens = [int(n) for n in torch.randint(0, 100, (rows,), generator=draw)]
    for r in (0, 3, 4, 255, 256, rows - 1):
        lens[r] = most - 7 * r % 100
    lens[1] = lens[rows - 2] = 0
    cache = make_cache(torch, peqa, gen, lens, 1, dim, 16, fp8, most)
    assert plan_of(peqa, cache, rows, group, most).shares > 0
    q = torch.randn((rows, group, dim), device="cuda", generator=gen).to(torch.bfloat16)
    check(torch, peqa, cache, q, lens, most)
    check(torch, peqa, cache, q, lens, most, window=2047)
    check(torch, peqa, cache, q, [0] * rows, most)
    check(torch, peqa, cache, q, [min(n, 65) for n in lens], most)


def test_shares_of_a_thousand_rows(env):
    torch, peqa = env
    gen, rows, most = torch.Generator(device="cuda").manual_seed(1), 1000, 1200
    lens = [int(n) for n in torch.randint(0, 300, (rows,), generator=torch.Generator().manual_seed(1))]
    lens[17], lens[999], lens[0] = most, most, 0
    cache = make_cache(torch, peqa, gen, lens, 1, 64, 32, False, most)
    assert plan_of(peqa, cache, rows, 4, most).shares > 0
    check(torch, peqa, cache, torch.randn((rows, 4, 64), device="cuda", generator=gen).to(torch.bfloat16), lens, most)


PIECE = 4096                                                     # positions whose pages are in LDS at a time


@pytest.mark.parametrize("dim,fp8,kv_heads,group,rows,most,page,window", [
    (128, False, 4, 2, 20, 33000, 64, 0), (128, False, 4, 9, 20, 33000, 16, 21001), (128, True, 4, 2, 40, 30000, 64, 0), (64, True, 4, 17, 40, 30000, 32, 0),
    (256, False, 4, 1, 30, 24000, 128, 0), (64, False, 4, 3, 40, 30000, 8, 0),
])
def test_shares_of_several_pieces(env, dim, fp8, kv_heads, group, rows, most, page, window):
    """Rows of more than twice what every share has, so that shares are longer than a piece, with pages that are not there."""
    torch, peqa = env
    print("pieces", dim, fp8, kv_heads, group, rows, most, page, window, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + dim)
    lens = [most - 701 * r for r in range(rows)] if rows * 701 < most else [most - (most // (rows + 9)) * r for r in range(rows)]
    lens[3], lens[5] = 0, 77
    cache = make_cache(torch, peqa, gen, lens, kv_heads, dim, page, fp8, most)
    heads = kv_heads * group
    p = plan_of(peqa, cache, rows, heads, most, window)
    counts = [min(n, window) if window else n for n in lens]
    assert p.shares > 0 and sum(counts) * kv_heads * p.blocks > 1.05 * PIECE * p.shares
    q = torch.randn((rows, heads, dim), device="cuda", generator=gen).to(torch.bfloat16)
    check(torch, peqa, cache, q, lens, most, window)
    # holes of a page and of many, anywhere
    table = cache.tensors[2]
    table.masked_fill_(torch.rand(table.shape, device="cuda", generator=gen) < 0.1, -1)
    table[0, 1000 // page:9000 // page] = -1
    table[2] = -1
    check(torch, peqa, cache, q, lens, most, window)


@pytest.mark.parametrize("dim,fp8,kv_heads,group,lens", [(128, False, 8, 2, [300001]), (256, True, 8, 3, [300001]), (64, False, 2, 1, [4100] * 600 + [9001]),
                                                         (128, True, 2, 20, [9000, 0, 4097, 8192] + [5] * 600)])
def test_chunks_and_items_of_several_pieces(env, dim, fp8, kv_heads, group, lens):
    torch, peqa = env
    print("long", dim, fp8, kv_heads, group, len(lens), lens[0], flush=True)
    gen = torch.Generator(device="cuda").manual_seed(dim)
    most = max(lens)
    cache = make_cache(torch, peqa, gen, lens, kv_heads, dim, 128, fp8, most)
    p = plan_of(peqa, cache, len(lens), kv_heads * group, most)
    assert p.shares == 0 and (p.chunk_units * 64 > PIECE or p.splits == 1 and most > PIECE) and (p.splits > 1) == (len(lens) == 1)
    q = torch.randn((len(lens), kv_heads * group, dim), device="cuda", generator=gen).to(torch.bfloat16)
    check(torch, peqa, cache, q, lens, most)
    cache.tensors[2][0, 3::7] = -1
    check(torch, peqa, cache, q, lens, most, window=most - 1000)

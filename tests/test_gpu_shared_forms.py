"""Every form of peqa_shared_attention's launch, for every kernel that it can launch: 16, 32 and 64 columns in all waves, 128 and 256 in waves of their own,
parts joined by a workgroup and by a wave of one; with odd numbers of rows, pages that are not there, rows that end among the shared positions, scores
that rise along the positions, infinite values, pools past 2^31 elements.  The form that a call takes is asked for, so that a case cannot move
to another one unnoticed.  Against 64 bits on the GPU, with the tolerances of tests/test_gpu_shared.py: 2^-8 of the output and 2^-14, against 8-bit
values 2^-10, of sum w |v|; of log-sum-exp 2^-14, and 2^-21 of itself."""
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
    _fields_ = [("wide", ctypes.c_bool)] + \
               [(n, ctypes.c_int) for n in ("hb", "columns", "tiles", "chunk", "chunks", "own_chunk", "own_splits", "own_blocks", "own_columns", "join_each")] + \
               [(n, ctypes.c_longlong) for n in ("prefix_wgs", "own_items")] + [(n, ctypes.c_size_t) for n in ("part_bytes", "ml_bytes")]


def plan_of(peqa, cache, rows, heads, most, shared):
    f = peqa.lib()._ZN4peqa11shared_planEPK13peqa_kv_cacheiiii          # peqa::shared_plan
    f.argtypes, f.restype = [ctypes.POINTER(peqa.KVCache)] + [ctypes.c_int] * 4, Plan
    plan = f(ctypes.byref(cache), rows, heads, most, shared)
    assert plan.part_bytes + plan.ml_bytes == peqa.shared_attention_workspace_bytes(cache, heads, rows, most, shared)
    return plan


def bits(torch, fp8):
    return (torch.uint8, 0x7F) if fp8 else (torch.int16, 0x7FC0)


def make_cache(torch, peqa, gen, shared, own, kv, dim, page, fp8, spare=2, rising=False):
    """Pages in random places; the last sequence's positions are the shared ones, the others have `own` behind them and nothing in front; NaN
    wherever no position is.  rising: keys that are the same in all elements and grow along the positions, to 4 / sqrt(dim)."""
    blocks = -(-(shared + max(own)) // page)
    spans = [(shared, shared + n) for n in own] + [(0, shared)]
    needed = sum(-(-b // page) - a // page if b > a else 0 for a, b in spans)
    total = needed + spare
    order = torch.randperm(total, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((len(spans), blocks), -1, dtype=torch.int32, device="cuda")
    kind, nan = bits(torch, fp8)

    def pool():
        x = torch.randn((total, kv, page, dim), device="cuda", generator=gen)
        return (x * 20).clamp(-448, 448).to(torch.float8_e4m3fn) if fp8 else x.to(torch.bfloat16)
    k, v = pool(), pool()
    hole = torch.ones((total, page), dtype=torch.bool, device="cuda")
    at = 0
    for s, (a, b) in enumerate(spans):
        if b <= a:
            continue
        n = -(-b // page) - a // page
        table[s, a // page:a // page + n] = order[at:at + n]
        p = torch.arange(a, b, device="cuda")
        where = order[at:at + n].long()[p // page - a // page]
        hole[where, p % page] = False
        if rising:
            x = (p / (shared + max(own)) * 4 * dim ** -0.5 * (20 if fp8 else 1))[:, None, None].expand(b - a, kv, dim)
            k.view(kind)[where, :, p % page] = x.to(k.dtype).view(kind)
        at += n
    for x in (k, v):
        x.view(kind).masked_fill_(hole[:, None, :, None], nan)
    scales = [0.02 + 0.05 * torch.rand(kv, device="cuda", generator=gen) for _ in range(2)] if fp8 else [None, None]
    return peqa.kv_cache(k, v, table, *scales)


def positions(torch, cache, seq, a, b, h):
    """Positions a .. b-1 whose pages are there, their keys and values of a head in 64 bits."""
    k_pool, v_pool, table, k_scale, v_scale = cache.tensors
    page, kind = cache.page_size, bits(torch, k_scale is not None)[0]
    p = torch.arange(a, b, device="cuda")
    pages = table[seq, p // page].long()
    there = (pages >= 0) & (pages < cache.n_pages)
    index, slot = pages[there], (p % page)[there]
    k, v = (x.view(kind)[index, h, slot].view(x.dtype).double() for x in (k_pool, v_pool))
    return (p[there], k * k_scale[h].double(), v * v_scale[h].double()) if k_scale is not None else (p[there], k, v)


def reference(torch, cache, q, lens, prefix, shared, scale):
    rows, heads, dim = q.shape
    group = heads // cache.kv_heads
    out, size = (torch.zeros(q.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full((rows, heads), -math.inf, dtype=torch.float64, device="cuda")
    for h in range(cache.kv_heads):
        mine = slice(h * group, h * group + group)
        first, first_k, first_v = positions(torch, cache, prefix, 0, shared, h)
        for r, n in enumerate(lens):
            seen = int((first < n).sum())
            k, v = first_k[:seen], first_v[:seen]
            if n > shared:
                k, v = (torch.cat(x) for x in zip((k, v), positions(torch, cache, r, shared, n, h)[1:]))
            if k.shape[0]:
                z = (q[r, mine].double() @ k.T.contiguous()) * scale
                w = torch.softmax(z, 1)
                lse[r, mine], out[r, mine], size[r, mine] = torch.logsumexp(z, 1), w @ v, w @ v.abs()
    return out, lse, size


def check(torch, peqa, cache, q, lens, most, shared, scale):
    rows, heads, _ = q.shape
    room = peqa.shared_attention_workspace_bytes(cache, heads, rows, most, shared)
    ws = torch.full((room,), 255, dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, float("nan")), torch.full((rows, heads), float("nan"), device="cuda")
    index = torch.tensor(lens, dtype=torch.int32, device="cuda")
    peqa.shared_attention(cache, q, index, most, rows, shared, scale, out, ws, room, lse=lse)
    want, want_lse, size = reference(torch, cache, q, [max(0, min(n, most)) for n in lens], rows, shared, scale)
    fine = want.isfinite()
    assert torch.equal(out.isfinite(), fine) and torch.equal(out.double()[~fine], want[~fine])
    off = (out.double() - want).abs() - 2.0 ** -8 * want.abs() - 2.0 ** (-10 if cache.dtype else -14) * size
    assert bool((off[fine] <= 0).all()), (float(off[fine].max()), int(off.nan_to_num(-1).argmax()))
    none = want_lse.isinf()
    assert torch.equal(lse.isinf(), none) and bool((lse[none] < 0).all())
    assert bool(((lse.double() - want_lse).abs()[~none] <= 2.0 ** -14 + 2.0 ** -21 * want_lse.abs()[~none]).all())
    again = torch.empty_like(q)
    peqa.shared_attention(cache, q, index, most, rows, shared, scale, again, ws, room)
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))


# rows, key heads, heads of one, shared positions, own ones; waves with columns of their own, blocks of columns, columns that a workgroup joins
FORMS = {
    "16 columns": (3, 2, 3, 700, 90, False, 1, 1),
    "32 columns": (7, 1, 4, 1111, 200, False, 2, 1),
    "64 columns": (15, 2, 4, 901, 130, False, 4, 1),
    "64 columns, waves join": (16, 17, 4, 211, 40, False, 4, 4),
    "128 columns": (13, 3, 8, 1501, 300, True, 1, 1),
    "128 columns, waves join": (71, 3, 5, 97, 41, True, 1, 4),
    "256 columns": (31, 16, 8, 4101, 70, True, 2, 4),
    "256 columns, several tiles": (57, 16, 8, 2051, 33, True, 2, 4),
}
WIDE = {   # what heads of 256 are given: 32 columns at most, none in waves of their own
    "16 columns": (1, 1), "32 columns": (2, 1), "64 columns": (2, 1), "64 columns, waves join": (2, 4), "128 columns": (2, 1), "128 columns, waves join": (2, 4),
}


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("form,dim,page", [(f, d, p) for f in FORMS for d, p in ((64, 8), (128, 16), (128, 64), (256, 32)) if d < 256 or f in WIDE])
def test_forms(env, form, dim, page, fp8):
    torch, peqa = env
    rows, kv, group, shared, most_own, wide, hb, each = FORMS[form]
    print("shared", form, dim, page, fp8, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + dim + page)
    pick = torch.Generator().manual_seed(rows)
    own = [most_own] + [int(n) for n in torch.randint(0, most_own + 1, (rows - 1,), generator=pick)]
    most, heads = shared + most_own, kv * group
    for rising in (False, True):
        cache = make_cache(torch, peqa, gen, shared, own, kv, dim, page, fp8, rising=rising)
        plan = plan_of(peqa, cache, rows, heads, most, shared)
        assert (plan.wide, plan.hb, plan.join_each) == ((wide, hb, each) if dim < 256 else (False, *WIDE[form]))
        q = torch.randn((rows, heads, dim), device="cuda", generator=gen).to(torch.bfloat16)
        if rising:
            q.fill_(1.0)
            q[1::2] = -0.5
        lens = [shared + n for n in own]
        check(torch, peqa, cache, q, lens, most, shared, 40 * dim ** -0.5 if rising else dim ** -0.5)
    # (the rising cache again) pages that are not there, rows that end among the shared positions or are empty
    table = cache.tensors[2]
    for b in {0, 2, 3, shared // page // 2, shared // page} & set(range(table.shape[1])):
        table[rows, b] = -1 if b % 2 else cache.n_pages
    table[0, shared // page] = 2 ** 31 - 1
    lens = [n if r % 3 else (0, shared // 2 + 1, -3, 1, shared - 1, shared)[r // 3 % 6] for r, n in enumerate(lens)]
    check(torch, peqa, cache, q, lens, most, shared, 7 * dim ** -0.5)
    table[rows, :] = -1
    check(torch, peqa, cache, q, lens, most, shared, 7 * dim ** -0.5)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("form", ["64 columns", "128 columns", "256 columns"])
def test_infinite_values(env, form, dim):
    """An infinite value makes its element infinite, of its sign, for the rows that see it, values of both signs make it NaN."""
    torch, peqa = env
    rows, kv, group, shared, most_own, *_ = FORMS[form]
    print("infinite", form, dim, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(dim)
    cache = make_cache(torch, peqa, gen, shared, [most_own] * rows, kv, dim, 32, False)
    v, table = cache.tensors[1], cache.tensors[2].cpu()
    place = lambda s, p: (int(table[s, p // 32]), kv - 1, p % 32)  # noqa: E731
    for p, d, value in ((5, 3, math.inf), (shared - 1, 4, -math.inf), (70, 9, math.inf), (shared // 2, 9, math.inf)):
        v[(*place(rows, p), d)] = value
    v[(*place(1, shared + 7), 11)] = -math.inf
    v[(*place(rows - 1, shared + most_own - 1), 12)] = math.inf
    q = torch.randn((rows, kv * group, dim), device="cuda", generator=gen).to(torch.bfloat16)
    # (scores of the order of one: no weight vanishes)
    check(torch, peqa, cache, q, [shared + most_own] * (rows - 1) + [shared + most_own - 1], shared + most_own, shared, 0.2 * dim ** -0.5)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("rows,kv,group,shared,hb", [(21, 2, 8, 1000, 1), (128, 2, 8, 8200, 2)])
def test_far_pages(env, rows, kv, group, shared, hb, fp8):
    """Pools past 2^31 elements, with waves that have columns of their own: whole pages of more positions than a stage."""
    torch, peqa = env
    print("far", rows, shared, fp8, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    page, dim, pages = 256, 128, 40000
    near = make_cache(torch, peqa, gen, shared, [30] * rows, kv, dim, page, fp8)
    kind = bits(torch, fp8)[0]
    scattered = 39999 - 7 * torch.randperm(near.n_pages, device="cuda", generator=gen)
    pools = [torch.zeros((pages, kv, page, dim), dtype=x.dtype, device="cuda") for x in near.tensors[:2]]
    for far, x in zip(pools, near.tensors[:2]):
        far.view(kind)[scattered] = x.view(kind)
    table = near.tensors[2]
    far = peqa.kv_cache(*pools, torch.where(table < 0, table, scattered[table.clamp_min(0).long()].to(torch.int32)), *near.tensors[3:])
    most = shared + 30
    plan = plan_of(peqa, far, rows, kv * group, most, shared)
    assert (plan.wide, plan.hb) == (True, hb)
    q = torch.randn((rows, kv * group, dim), device="cuda", generator=gen).to(torch.bfloat16)
    lens = torch.full((rows,), most, dtype=torch.int32, device="cuda")
    room = plan.part_bytes + plan.ml_bytes
    ws, got = torch.empty(room, dtype=torch.uint8, device="cuda"), []
    for cache in (near, far):
        out, lse = torch.empty_like(q), torch.empty((rows, kv * group), device="cuda")
        peqa.shared_attention(cache, q, lens, most, rows, shared, dim ** -0.5, out, ws, room, lse=lse)
        got.append((out, lse))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    check(torch, peqa, far, q, [most] * rows, most, shared, dim ** -0.5)

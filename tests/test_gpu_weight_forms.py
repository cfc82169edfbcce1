"""What positions are given (peqa_paged_attention_weights) in every form of the attention's launch: whole items by one, four and eight waves, chunks and
equal shares, and in every form of the second kernel, one, two and four heads in flight.  The form that a call takes is asked for.  Against 64 bits on the
GPU, with the tolerances of tests/test_gpu_evict.py: 2^-14 of what is added, 2^-17 of it and of what was there before; out and lse are those of
peqa_paged_attention, bit for bit."""
import pytest

from test_gpu_attention_forms import make_cache, plan_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_2305_14152_amd import peqa
    peqa.lib()
    return torch, peqa


def given(torch, cache, q, lens, window, seq, scale, room):
    """What positions are given, and how many of a sequence's there are."""
    rows, heads, dim = q.shape
    k_pool, _, table, k_scale, _ = cache.tensors
    group, page = heads // cache.kv_heads, cache.page_size
    kind = torch.uint8 if k_scale is not None else torch.int16
    want = torch.zeros((cache.n_seqs, cache.kv_heads, room), dtype=torch.float64, device="cuda")
    longest = [0] * cache.n_seqs
    for r, (s, n) in enumerate(zip(seq, lens)):
        if n <= 0 or not 0 <= s < cache.n_seqs:
            continue
        longest[s] = max(longest[s], n)
        p = torch.arange(max(0, n - window) if window else 0, n, device="cuda")
        pages = table[s, p // page].long()
        p, pages = p[(pages >= 0) & (pages < cache.n_pages)], pages[(pages >= 0) & (pages < cache.n_pages)]
        if not p.numel():
            continue
        for h in range(cache.kv_heads):
            k = k_pool.view(kind)[pages, h, p % page].view(k_pool.dtype).double()
            if k_scale is not None:
                k = k * k_scale[h].double()
            want[s, h, p] += torch.softmax((q[r, h * group:(h + 1) * group].double() @ k.T.contiguous()) * scale, 1).sum(0)
    return want, longest


def check(torch, peqa, gen, cache, q, lens, most, window=0, seq=None):
    rows, heads, dim = q.shape
    scale, room = dim ** -0.5, -(-most // 4) * 4 + 4
    index = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    (a, b), (la, lb) = (torch.empty_like(q) for _ in range(2)), (torch.empty((rows, heads), device="cuda") for _ in range(2))
    bytes_ = peqa.paged_attention_workspace_bytes(cache, heads, rows, most, window)
    peqa.paged_attention(cache, q, index(lens), most, scale, a, torch.empty(bytes_, dtype=torch.uint8, device="cuda"), bytes_, lse=la, seq=index(seq), window=window)
    bytes_ = peqa.paged_attention_weights_workspace_bytes(cache, heads, rows, most, window)
    ws = torch.full((bytes_,), 255, dtype=torch.uint8, device="cuda")
    old = torch.rand((cache.n_seqs, cache.kv_heads, room), device="cuda", generator=gen)
    new = torch.full_like(old, -7.0)
    peqa.paged_attention_weights(cache, q, index(lens), most, scale, b, old, new, ws, bytes_, lse=lb, seq=index(seq), window=window)
    assert torch.equal(a, b) and torch.equal(la, lb)
    want, longest = given(torch, cache, q, lens, window, seq or range(rows), scale, room)
    behind = torch.arange(room, device="cuda") >= torch.tensor(longest, device="cuda")[:, None, None]
    off = (new.double() - old.double() - want).abs() - 2.0 ** -14 * want - 2.0 ** -17 * (old.double() + want)
    assert bool((off.masked_fill(behind, -1.0) <= 0).all()), (float(off.masked_fill(behind, -1.0).max()), int(off.masked_fill(behind, -1.0).argmax()))
    assert bool((new.masked_fill(~behind, -7.0) == -7.0).all())
    same = old.clone()
    peqa.paged_attention_weights(cache, q, index(lens), most, scale, b, same, same, ws, bytes_, seq=index(seq), window=window)
    assert torch.equal(same, torch.where(behind, old, new))


# rows, key heads, longest row; waves, chunks, shares; workgroups of the second kernel more than 1024 (none: finished within the attention)
FORMS = {
    "one wave": (140, 4, 200, 1, False, False, None),
    "four waves": (300, 4, 700, 4, False, False, None),
    "eight waves": (9, 2, 400, 8, False, False, None),
    "chunks": (3, 2, 9000, 4, True, False, False),
    "chunks, many of the second": (1, 4, 300000, 4, True, False, True),
    "shares": (40, 4, 5000, 4, False, True, False),
    "shares, many of the second": (60, 4, 5000, 4, False, True, True),
}
HEADS = [(64, False, 1), (64, False, 20), (64, True, 8), (64, True, 17), (128, False, 4), (128, False, 12), (128, True, 3), (128, True, 11), (256, False, 2), (256, True, 9), (256, False, 16)]


def there(form, dim, fp8, group):
    """Whether there is such a kernel; of the largest calls, heads of 64 and 128 with up to eight to a key head."""
    if form == "eight waves":
        return dim < 256 and group <= (16 if fp8 else 8)
    return form != "chunks, many of the second" or (dim < 256 and group <= 8)


@pytest.mark.parametrize("form,dim,fp8,group", [(f, *h) for f in FORMS for h in HEADS if there(f, *h)])
def test_forms(env, form, dim, fp8, group):
    torch, peqa = env
    rows, kv, most, waves, chunks, shares, many = FORMS[form]
    print("weights", form, dim, fp8, group, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + dim)
    pick = torch.Generator().manual_seed(rows)
    lens = [most] + [int(n) for n in torch.randint(0, most + 1, (rows - 1,), generator=pick)]
    lens[-1] = lens[-1] if rows < 3 else 0
    cache = make_cache(torch, peqa, gen, lens, kv, dim, 32 if dim == 64 else 16, fp8, most)
    plan = plan_of(peqa, cache, rows, kv * group, most)
    within = plan.blocks == 1 and plan.splits == 1 and plan.shares == 0
    if plan.blocks == 1 and dim <= 128:
        assert (plan.waves, plan.splits > 1, plan.shares > 0) == (waves, chunks, shares) and within == (many is None)
    assert many is None or (-(-most // 1024) * rows * kv > 1024) == many
    q = torch.randn((rows, kv * group, dim), device="cuda", generator=gen).to(torch.bfloat16)
    check(torch, peqa, gen, cache, q, lens, most)
    # a bound below the longest row, and above all behind a window; pages that are not there; a length past the bound
    table, page = cache.tensors[2], cache.page_size
    table[0, [0, most // page // 2]] = -1
    if rows > 1:
        table[1, :] = cache.n_pages
    cut = most - 3
    check(torch, peqa, gen, cache, q, [min(n, cut) for n in lens], cut)
    check(torch, peqa, gen, cache, q, lens, most, window=most * 3 // 5)


@pytest.mark.parametrize("dim,fp8,group", [(128, False, 1), (64, True, 8), (128, False, 12)])
def test_rows_of_one_sequence_in_shares(env, dim, fp8, group):
    """Few sequences' rows in equal shares: sums over rows that several workgroups have, sequences that are none, one with no row."""
    torch, peqa = env
    gen = torch.Generator(device="cuda").manual_seed(dim)
    kv, most, rows = 4, 5000, 60
    cache = make_cache(torch, peqa, gen, [most, 3000, 700, 40], kv, dim, 16, fp8, most)
    seq = [(0, 1, 0, 5, 2, 0, -1)[r % 7] for r in range(rows)]
    lens = [max(0, (most, 3000, 700)[s] - r * 11) if 0 <= s < 3 else 100 for r, s in enumerate(seq)]
    assert plan_of(peqa, cache, rows, kv * group, most).shares > 0
    q = torch.randn((rows, kv * group, dim), device="cuda", generator=gen).to(torch.bfloat16)
    print("weights of rows of one sequence", dim, fp8, group, flush=True)
    check(torch, peqa, gen, cache, q, lens, most, seq=seq)
    check(torch, peqa, gen, cache, q, lens, most, window=2111, seq=seq)

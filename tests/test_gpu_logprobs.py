"""Log probabilities and their gradient (peqa_token_logprobs, peqa_token_logprobs_bwd) against 64 bits.

Tolerances.  lse, logp and entropy: sums of positive fp32 terms, whose rounding averages out (taken: 2^-18 of the sum), differences to
the maximum rounded to 2^-24 of the logits' size: 2^-17 (1 + |value|) + 2^-21 (largest |logit| that counts).  Gradients: 2^-17 of every
term's size, and bf16's rounding (2^-8) where the logits are bf16."""
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


def call(torch, peqa, x, targets, top):
    T, V = x.shape
    logp, H, lse = (torch.full((T,), 9.0, device="cuda") for _ in range(3))
    tl = torch.full((T, top), 9.0, device="cuda") if top else None
    ti = torch.full((T, top), -9, dtype=torch.int32, device="cuda") if top else None
    room = peqa.token_logprobs_workspace_bytes(T, V, top)
    assert room > 0
    ws = torch.full((room,), 0xFF, dtype=torch.uint8, device="cuda")
    peqa.token_logprobs(x, targets, logp, H, lse, tl, ti, ws, room)
    torch.cuda.synchronize()
    return logp, H, lse, tl, ti


def check(torch, peqa, x, targets, top):
    logp, H, lse, tl, ti = call(torch, peqa, x, targets, top)
    T, V = x.shape
    d = x.float().cpu().double().numpy()
    t = targets.cpu().numpy()
    for r in range(T):
        row = d[r]
        if (row == -math.inf).all():
            assert lse[r] == -math.inf and H[r] == 0 and (logp[r] == -math.inf if 0 <= t[r] < V else logp[r] == 0)
            if top:
                assert ti[r].tolist() == list(range(top)) and (tl[r] == -math.inf).all()
            continue
        m = row.max()
        e = np.exp(row - m)
        s = e.sum()
        w_lse = m + math.log(s)
        p = e / s
        w_H = math.log(s) - float((p * np.where(e > 0, row - m, 0)).sum())
        tol = lambda w: 2.0 ** -17 * (1 + abs(w)) + 2.0 ** -21 * abs(m)  # noqa: E731
        assert abs(float(lse[r]) - w_lse) <= tol(w_lse), (r, float(lse[r]), w_lse)
        assert abs(float(H[r]) - w_H) <= tol(w_H), (r, float(H[r]), w_H)
        w = row[t[r]] - w_lse if 0 <= t[r] < V else 0.0
        assert float(logp[r]) == w if not math.isfinite(w) else abs(float(logp[r]) - w) <= tol(w), (r, float(logp[r]), w)
        if top:
            ids = np.argsort(-row, kind="stable")[:top]
            assert ti[r].tolist() == ids.tolist(), r
            for got, j in zip(tl[r].tolist(), ids):
                w = row[j] - w_lse
                assert got == w if not math.isfinite(w) else abs(got - w) <= tol(w)
    # any of the outputs may be left out; without them the others are the same
    lse2 = torch.empty_like(lse)
    room = peqa.token_logprobs_workspace_bytes(T, V, 0)
    peqa.token_logprobs(x, None, None, None, lse2, None, None, torch.empty(room, dtype=torch.uint8, device="cuda"), room)
    assert (lse2 - lse).nan_to_num(0, 0, 0).abs().max() <= 2.0 ** -17 * (1 + lse.nan_to_num(0, 0, 0).abs().max())
    return logp, H, lse


def logits(torch, gen, T, V, dtype, pad=0, shift=0, std=3.0):
    """[T, V] in rows of V + pad, the first `shift` elements into its memory; what is no row's is NaN."""
    whole = torch.full((T * (V + pad) + shift + 8,), math.nan, dtype=dtype, device="cuda")
    x = whole[shift:shift + T * (V + pad)].view(T, V + pad)[:, :V]
    x.copy_((torch.randn((T, V), generator=gen) * std).to(dtype))
    return x, whole


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T,V,top,pad,shift", [
    (5, 1, 1, 0, 0), (3, 2, 2, 0, 1), (9, 7, 7, 0, 0), (4, 8, 5, 0, 0), (4, 9, 3, 0, 3), (7, 63, 32, 1, 0), (6, 1000, 32, 0, 0), (3, 1003, 20, 0, 5),
    (5, 8191, 32, 2, 1), (2, 8193, 1, 0, 0), (3, 32000, 20, 0, 0), (300, 513, 4, 0, 0), (1, 50257, 8, 0, 1), (4, 50257, 32, 0, 0),
    (1, 260001, 32, 3, 2), (2, 131072, 32, 0, 0), (260, 40000, 2, 0, 0), (1, 16385, 0, 0, 0), (1030, 5003, 3, 0, 0), (1025, 4200, 0, 0, 0),
])
def test_logprobs(env, f32, T, V, top, pad, shift):
    torch, peqa = env
    print("logprobs", f32, T, V, top, pad, shift, flush=True)
    gen = torch.Generator().manual_seed(T * 7 + V)
    x, _ = logits(torch, gen, T, V, torch.float32 if f32 else torch.bfloat16, pad, shift)
    targets = torch.randint(0, V, (T,), generator=gen, dtype=torch.int32)
    targets[0] = V - 1
    if T > 2:
        targets[1], targets[2] = -100, V
    check(torch, peqa, x, targets.cuda(), top)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T,V", [(12, 1000), (12, 32003), (12, 100001)])
def test_hard_rows(env, f32, T, V):
    """Masks of -inf and of the lowest value, nothing left, one word left, equal logits, sorted ones, large ones next to each other and in one
    column of the workgroup, signed zeros."""
    torch, peqa = env
    print("hard", f32, T, V, flush=True)
    dtype = torch.float32 if f32 else torch.bfloat16
    gen = torch.Generator().manual_seed(V)
    x, _ = logits(torch, gen, T, V, dtype)
    low = torch.finfo(dtype).min
    x[0] = -math.inf
    x[1] = -math.inf
    x[1, V - 3] = 2.0
    x[2] = low
    x[3, 5:] = low
    x[4] = 1.25
    x[5] = torch.linspace(-20, 20, V).to(dtype).cuda()
    x[6] = torch.linspace(20, -20, V).to(dtype).cuda()
    x[7, V // 2:V // 2 + 600] += 30
    j = torch.arange(V)
    x[8, ((j // 8) % 64 == 0).cuda()] += 40
    x[9] = torch.where(j % 2 == 0, 0.0, -0.0).to(dtype).cuda()
    x[10, ::3] = -math.inf
    x[11] = (j % 1000 == 999).to(dtype).cuda() * 300 - 100
    targets = torch.tensor([3, V - 3, 0, 1, 2, V - 1, 0, V // 2, 0, 1, 0, 999], dtype=torch.int32).cuda()
    check(torch, peqa, x, targets, 32)
    check(torch, peqa, x[8:9], targets[8:9], 32)
    check(torch, peqa, x[:2], targets[:2], 5)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T,V,top", [(40, 700, 32), (40, 1003, 20), (40, 4096, 32), (8, 50257, 32), (3, 200003, 31), (300, 1500, 32)])
def test_few_words_allowed(env, f32, T, V, top):
    """Fewer words than alternatives, the rest masked alike: the alternatives end with the first of the masked ones."""
    torch, peqa = env
    print("few", f32, T, V, top, flush=True)
    dtype = torch.float32 if f32 else torch.bfloat16
    gen = torch.Generator().manual_seed(V + top)
    x, _ = logits(torch, gen, T, V, dtype)
    for r in range(T):
        allowed = torch.randperm(V, generator=gen)[:r % (top + 3)]
        kept = x[r, allowed.cuda()].clone()
        x[r] = -math.inf if r % 2 == 0 else torch.finfo(dtype).min
        x[r, allowed.cuda()] = kept
    targets = torch.randint(0, V, (T,), generator=gen, dtype=torch.int32)
    check(torch, peqa, x, targets.cuda(), top)


def test_many_distinct_large_logits_in_few_columns(env):
    """More large logits than are gathered at once, all in the elements of few groups of threads."""
    torch, peqa = env
    V = 200000
    for T in (1, 300):
        x, _ = logits(torch, torch.Generator().manual_seed(1), T, V, torch.float32)
        j = torch.arange(V)
        few = ((j // 8) % 64 < 3)
        x[0, few.cuda()] = (1000 + 0.001 * torch.arange(int(few.sum()))).cuda()
        check(torch, peqa, x[:2] if T > 1 else x, torch.zeros(min(T, 2), dtype=torch.int32).cuda(), 32)
        if T > 1:
            out = call(torch, peqa, x, torch.zeros(T, dtype=torch.int32).cuda(), 32)
            want = torch.sort(x[0].cpu(), descending=True, stable=True)[1][:32]
            assert out[4][0].tolist() == want.tolist()


def test_nan_and_infinity(env):
    """A NaN or +inf makes a row's numbers NaN and no other row's; the alternatives stay words of the row."""
    torch, peqa = env
    for V in (500, 40000):
        x, _ = logits(torch, torch.Generator().manual_seed(2), 4, V, torch.bfloat16)
        good = call(torch, peqa, x.clone(), torch.zeros(4, dtype=torch.int32).cuda(), 8)
        x[1, 77], x[2, V - 1] = math.nan, math.inf
        x[3, :] = math.nan
        logp, H, lse, tl, ti = call(torch, peqa, x, torch.zeros(4, dtype=torch.int32).cuda(), 8)
        for r in (1, 2, 3):
            assert all(bool(a[r].isnan().all()) for a in (logp, H, lse, tl))
            assert ti[r].min() >= 0 and ti[r].max() < V and len(set(ti[r].tolist())) == 8
        assert all(torch.equal(a[0], b[0]) for a, b in zip((logp, H, lse, tl, ti), good))


def gradient64(x, t, g, h):
    out, size = np.zeros_like(x), np.zeros_like(x)
    for r in range(x.shape[0]):
        if (x[r] == -math.inf).all():
            continue
        live = 0 <= t[r] < x.shape[1]
        m = x[r].max()
        e = np.exp(x[r] - m)
        p = e / e.sum()
        lp = np.where(p > 0, x[r] - m - math.log(e.sum()), 0.0)
        H = -(p * lp).sum()
        gr = g[r] if live else 0.0
        out[r] = -gr * p - h[r] * p * (lp + H)
        size[r] = abs(gr) * p + abs(h[r]) * p * (np.abs(lp) + H)
        if live:
            out[r, t[r]] += gr
            size[r, t[r]] += abs(gr)
    return out, size


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T,V,pad,shift,d_pad,d_shift", [
    (4, 1, 0, 0, 0, 0), (5, 7, 0, 1, 0, 1), (5, 9, 0, 0, 3, 2), (6, 1000, 0, 0, 0, 0), (4, 4099, 1, 0, 1, 0), (3, 50257, 0, 0, 0, 0), (7, 32000, 8, 0, 0, 0),
    (3, 8193, 0, 3, 1, 2),
])
def test_gradient(env, f32, T, V, pad, shift, d_pad, d_shift):
    torch, peqa = env
    print("gradient", f32, T, V, pad, shift, flush=True)
    dtype = torch.float32 if f32 else torch.bfloat16
    gen = torch.Generator().manual_seed(V)
    x, _ = logits(torch, gen, T, V, dtype, pad, shift)
    if T > 3 and V > 5:
        x[1, ::2] = -math.inf
        x[2] = -math.inf
        x[3, 1:] = torch.finfo(dtype).min
    targets = torch.randint(0, V, (T,), generator=gen, dtype=torch.int32)
    targets[0] = -1
    g, h = torch.randn(T, generator=gen).cuda(), torch.randn(T, generator=gen).cuda()
    targets = targets.cuda()
    _, H, lse, _, _ = call(torch, peqa, x, targets, 0)
    host = lambda a: a.float().cpu().double().numpy()  # noqa: E731
    for use_g, use_h in ((True, True), (True, False), (False, True)):
        d, whole = logits(torch, gen, T, V, dtype, d_pad, d_shift)
        stay = whole.clone()
        peqa.token_logprobs_bwd(x, targets, lse, H if use_h else None, g if use_g else None, h if use_h else None, d)
        torch.cuda.synchronize()
        want, size = gradient64(host(x), targets.tolist(), host(g) * use_g, host(h) * use_h)
        off = np.abs(host(d) - want) - (2.0 ** -17 * size * 2 + (0 if f32 else 2.0 ** -8 * 1.01) * np.abs(want) + 1e-37)
        if not f32:
            off -= 2.0 ** -126                                   # subnormal results
        assert (off <= 0).all(), (use_g, use_h, off.max(), np.unravel_index(off.argmax(), off.shape))
        d.zero_()
        stay[d_shift:d_shift + T * (V + d_pad)].view(T, V + d_pad)[:, :V] = 0
        assert torch.equal(whole.isnan(), stay.isnan())          # nothing outside the rows was written
    # over the logits themselves
    both, _ = logits(torch, gen, T, V, dtype, d_pad, d_shift)
    peqa.token_logprobs_bwd(x, targets, lse, H, g, h, both)
    peqa.token_logprobs_bwd(x, targets, lse, H, g, h, x)
    assert torch.equal(both.contiguous(), x.contiguous())


def test_rows_without_a_gradient_are_zeros(env):
    """Ignored targets and factors of 0, whatever the row holds."""
    torch, peqa = env
    x = torch.full((3, 1000), math.nan, dtype=torch.bfloat16, device="cuda")
    targets = torch.tensor([-100, 5, 1000], dtype=torch.int32, device="cuda")
    d = torch.full_like(x, 3.0)
    peqa.token_logprobs_bwd(x, targets, torch.zeros(3, device="cuda"), torch.zeros(3, device="cuda"), torch.tensor([1.0, 0.0, 2.0], device="cuda"),
                            torch.zeros(3, device="cuda"), d)
    assert (d == 0).all()


def test_gradient_against_differences(env):
    """Central differences of the forward in 64 bits along random directions: the error of a difference of step 1e-4 is under 1e-6 of the
    sum of absolute gradients here."""
    torch, peqa = env
    rng = np.random.default_rng(0)
    T, V = 3, 500
    x = rng.normal(size=(T, V)) * 2
    x = x.astype(np.float32).astype(np.float64)
    t = [3, 499, 77]
    g, h = rng.normal(size=T), rng.normal(size=T)

    def loss(y):
        lse = np.log(np.exp(y).sum(1))
        p = np.exp(y - lse[:, None])
        return float((g * (y[range(T), t] - lse)).sum() + (h * -(p * (y - lse[:, None])).sum(1)).sum())

    xd = torch.tensor(x, dtype=torch.float32).cuda()
    targets = torch.tensor(t, dtype=torch.int32).cuda()
    _, H, lse, _, _ = call(torch, peqa, xd, targets, 0)
    d = torch.empty_like(xd)
    peqa.token_logprobs_bwd(xd, targets, lse, H, torch.tensor(g, dtype=torch.float32).cuda(), torch.tensor(h, dtype=torch.float32).cuda(), d)
    d = d.cpu().double().numpy()
    for _ in range(5):
        u = rng.normal(size=x.shape)
        step = 1e-4
        diff = (loss(x + step * u) - loss(x - step * u)) / (2 * step)
        assert abs(diff - (d * u).sum()) <= 1e-5 * np.abs(d * u).sum()


def test_graph_and_stream(env):
    """Forward and gradient captured, with the forward split over workgroups, against eager calls."""
    torch, peqa = env
    T, V, top = 4, 100000, 10
    gen = torch.Generator().manual_seed(11)
    x, _ = logits(torch, gen, T, V, torch.bfloat16)
    targets = torch.randint(0, V, (T,), generator=gen, dtype=torch.int32).cuda()
    g = torch.randn(T, generator=gen).cuda()
    room = peqa.token_logprobs_workspace_bytes(T, V, top)

    def buffers():
        return [torch.zeros(T, device="cuda") for _ in range(3)] + [torch.zeros((T, top), device="cuda"), torch.zeros((T, top), dtype=torch.int32, device="cuda"),
                torch.zeros(room, dtype=torch.uint8, device="cuda"), torch.zeros((T, V), dtype=torch.bfloat16, device="cuda")]

    def step(b):
        peqa.token_logprobs(x, targets, b[0], b[1], b[2], b[3], b[4], b[5], room)
        peqa.token_logprobs_bwd(x, targets, b[2], b[1], g, g, b[6])

    a, b = buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        step(b)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for i, (p, q) in enumerate(zip(a, b)) if i != 5)
        x.copy_((torch.randn((T, V), generator=gen) * 3).to(torch.bfloat16))

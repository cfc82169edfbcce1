"""Log probabilities and their gradient of logits far from zero, against 64 bits.

Tolerance of the gradient: what it is of logits near zero, for the same reasons: p_j = e^(x_j - lse) where x_j - lse and its exponential are
off by 2^-24 |x_j - lse| each and what is left of lse's own rounding is under 2^-17: 2 * 2^-17 of every term's size, and bf16's half unit,
2^-8 of the result, where the logits are bf16."""
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


def rows(torch, gen, T, V, dtype, pad=0, shift=0):
    """[T, V] in rows of V + pad, the first `shift` elements into its memory; what is no row's is NaN."""
    whole = torch.full((T * (V + pad) + shift + 8,), math.nan, dtype=dtype, device="cuda")
    x = whole[shift:shift + T * (V + pad)].view(T, V + pad)[:, :V]
    x.copy_((torch.randn((T, V), generator=gen) * 3).to(dtype))
    return x, whole


def forward(torch, peqa, x, targets, top=0):
    T, V = x.shape
    logp, H, lse = (torch.full((T,), 9.0, device="cuda") for _ in range(3))
    best, ids = (torch.full((T, top), 9.0, device="cuda"), torch.full((T, top), -9, dtype=torch.int32, device="cuda")) if top else (None, None)
    room = peqa.token_logprobs_workspace_bytes(T, V, top)
    peqa.token_logprobs(x, targets, logp, H, lse, best, ids, torch.full((room,), 0xFF, dtype=torch.uint8, device="cuda"), room)
    return logp, H, lse, best, ids


def host(t):
    return t.float().cpu().double().numpy()


def gradient64(x, t, g, h, lse=None):
    """The gradient, and the size of its terms; p_j from the row, or from what lse is said to be."""
    out, size = np.zeros_like(x), np.zeros_like(x)
    for r in range(x.shape[0]):
        m = x[r].max()
        if m == -math.inf:
            continue
        e = np.exp(x[r] - m)
        lp = x[r] - m - math.log(e.sum()) if lse is None else x[r] - lse[r]
        p = np.exp(lp)
        lp = np.where(p > 0, lp, 0.0)
        H = -(p * lp).sum()
        live = 0 <= t[r] < x.shape[1]
        gr = g[r] if live else 0.0
        out[r] = -gr * p - h[r] * p * (lp + H)
        size[r] = abs(gr) * p + abs(h[r]) * p * (np.abs(lp) + abs(H))
        if live:
            out[r, t[r]] += gr
            size[r, t[r]] += abs(gr)
    return out, size


def close(torch, d, want, size):
    off = np.abs(host(d) - want) - (2.0 ** -16 * size + 1e-37)
    if d.dtype == torch.bfloat16:
        off -= 2.0 ** -8 * 1.01 * np.abs(want) + 2.0 ** -126              # (and subnormal results)
    assert (off <= 0).all(), (off.max(), np.unravel_index(off.argmax(), off.shape))


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T,V,pad,shift,d_pad,d_shift", [(7, 9, 0, 1, 0, 1), (9, 1000, 0, 0, 0, 0), (8, 4099, 1, 0, 3, 2), (8, 32003, 0, 3, 5, 3), (10, 50257, 0, 0, 7, 0)])
def test_gradient_far_from_zero(env, f32, T, V, pad, shift, d_pad, d_shift):
    """Rows around 0, +-300, +-1000 and +-10000, rows of the lowest value only (p_j = 1 / V, though lse is the lowest value again), of one
    word more than that, and rows that a mask leaves a few words of."""
    torch, peqa = env
    print("far", f32, T, V, flush=True)
    dtype = torch.float32 if f32 else torch.bfloat16
    gen = torch.Generator().manual_seed(V)
    x, _ = rows(torch, gen, T, V, dtype, pad, shift)
    low = torch.finfo(dtype).min
    for r, far in enumerate((300, -1000, 10000, -10000)):
        x[r] = (x[r].float() + far).to(dtype)
    x[4] = low
    x[5] = low
    x[5, V // 2] = 1000.0
    x[6, 1::2] = -math.inf
    x[6, ::2] = low
    if T > 7:
        x[7] = (x[7].float() + 1000).to(dtype)
        x[7, 5:] = low
    targets = torch.randint(0, V, (T,), generator=gen, dtype=torch.int32)
    targets[1] = -1
    if T > 8:
        targets[8] = V
    targets = targets.cuda()
    g, h = torch.randn(T, generator=gen).cuda(), torch.randn(T, generator=gen).cuda()
    _, H, lse, _, _ = forward(torch, peqa, x, targets)
    for use_g, use_h in ((True, True), (True, False), (False, True)):
        d, whole = rows(torch, gen, T, V, dtype, d_pad, d_shift)
        outside = whole.clone()
        peqa.token_logprobs_bwd(x, targets, lse, H if use_h else None, g if use_g else None, h if use_h else None, d)
        torch.cuda.synchronize()
        close(torch, d, *gradient64(host(x), targets.tolist(), host(g) * use_g, host(h) * use_h))
        outside[d_shift:d_shift + T * (V + d_pad)].view(T, V + d_pad)[:, :V] = 0
        d.zero_()
        assert torch.equal(whole.isnan(), outside.isnan())
    # over the logits themselves
    both, _ = rows(torch, gen, T, V, dtype, d_pad, d_shift)
    peqa.token_logprobs_bwd(x, targets, lse, H, g, h, both)
    peqa.token_logprobs_bwd(x, targets, lse, H, g, h, x)
    assert torch.equal(both.contiguous(), x.contiguous())


@pytest.mark.parametrize("far", [0.0, 1000.0, -10000.0])
def test_an_lse_over_more_words_is_taken_as_it_is(env, far):
    """Two halves of the words with the lse of both: the halves' gradients are the whole row's, as exactly as lse is known in fp32."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(5)
    T, V = 4, 3000
    x = (torch.randn((T, V), generator=gen) * 3 + far).cuda()
    targets = torch.tensor([3, 1499, 1500, 2999], dtype=torch.int32, device="cuda")
    g = torch.randn(T, generator=gen).cuda()
    lse = forward(torch, peqa, x, targets)[2]
    zero = np.zeros(T)
    for part in range(2):
        t = targets - part * 1500
        y, d = x[:, part * 1500:part * 1500 + 1500], torch.empty((T, 1500), device="cuda")
        peqa.token_logprobs_bwd(y, t, lse, None, g, None, d)
        close(torch, d, *gradient64(host(y), t.tolist(), host(g), zero, host(lse)))


# ---- the forward ------------------------------------------------------------------------------------------------------
# logp, the alternatives' and the entropy do not depend on where a row lies: (x - m) - log s, with m the row's largest, x - m rounded to
# 2^-24 of itself, and sums of positive terms (taken: 2^-18).  2^-17 (1 + |value|) bounds each, whatever m is; lse alone has m's rounding.

def check_forward(torch, peqa, x, targets, top):
    T, V = x.shape
    logp, H, lse, best, ids = forward(torch, peqa, x, targets, top)
    near = lambda got, want: got == want if not math.isfinite(want) else abs(got - want) <= 2.0 ** -17 * (1 + abs(want))  # noqa: E731
    d, t = host(x), targets.tolist()
    for r in range(T):
        m = d[r].max()
        e = np.exp(d[r] - m)
        log_s = math.log(e.sum())
        p = e / e.sum()
        assert abs(float(lse[r]) - (m + log_s)) <= 2.0 ** -17 * (1 + log_s) + 2.0 ** -24 * abs(m + log_s), r
        assert near(float(H[r]), log_s - float((p * np.where(e > 0, d[r] - m, 0.0)).sum())), (r, float(H[r]))
        assert near(float(logp[r]), d[r, t[r]] - m - log_s if 0 <= t[r] < V else 0.0), (r, float(logp[r]))
        if top:
            order = np.argsort(-d[r], kind="stable")[:top]
            assert ids[r].tolist() == order.tolist(), r
            assert all(near(got, d[r, j] - m - log_s) for got, j in zip(best[r].tolist(), order)), r


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T,V,top", [(9, 7, 7), (9, 1000, 32), (9, 32003, 5), (9, 50257, 0), (300, 1500, 20), (9, 200003, 32)])
def test_forward_far_from_zero(env, f32, T, V, top):
    """Rows around +-1000 and +-10000, of the lowest value only (log probabilities -log V, entropy log V), of one word more, of half of them."""
    torch, peqa = env
    print("forward far", f32, T, V, top, flush=True)
    dtype = torch.float32 if f32 else torch.bfloat16
    gen = torch.Generator().manual_seed(V + T)
    x, _ = rows(torch, gen, T, V, dtype)
    low = torch.finfo(dtype).min
    for r, far in enumerate((1000, -1000, 10000, -10000)):
        x[r] = (x[r].float() + far).to(dtype)
    x[4] = low
    x[5] = low
    x[5, V // 2] = 3.0
    x[6, ::2] = low
    x[6, 1::2] = -math.inf
    x[7, 3:] = low
    targets = torch.randint(0, V, (T,), generator=gen, dtype=torch.int32)
    targets[1], targets[6] = -100, 2
    check_forward(torch, peqa, x, targets.cuda(), top)


@pytest.mark.parametrize("f32", [False, True])
def test_more_large_logits_in_a_slice_than_are_gathered(env, f32):
    """A row that is cut into slices, each with more than 1024 logits no smaller than its bound: large ones in eight of every 64 vectors of
    eight, so that with 32 alternatives the bound is among the small ones.  They are then found one by one within a slice."""
    torch, peqa = env
    V, top = 200000, 32
    slices = (V + 14) // 8 // 2048
    round256 = lambda n: (n + 255) // 256 * 256  # noqa: E731
    assert slices > 8 and peqa.token_logprobs_workspace_bytes(1, V, top) == round256(slices * 16) + round256(slices * top * 8)
    x, _ = rows(torch, torch.Generator().manual_seed(3), 1, V, torch.float32 if f32 else torch.bfloat16)
    large = (torch.arange(V) // 8) % 64 < 8
    assert int(large.sum()) // slices > 1500
    order = torch.randperm(int(large.sum()), generator=torch.Generator().manual_seed(4))
    x[0, large.cuda()] = (1000 + 0.001 * order).to(x.dtype).cuda()
    check_forward(torch, peqa, x, torch.tensor([9], dtype=torch.int32).cuda(), top)
    x[0, large.cuda()] = (1000 + 0.001 * torch.arange(len(order))).to(x.dtype).cuda()          # the last slice has the answer
    check_forward(torch, peqa, x, torch.tensor([V - 1], dtype=torch.int32).cuda(), top)

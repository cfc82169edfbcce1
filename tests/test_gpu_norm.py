"""Norms of queries and keys with the rotation (peqa_norm_rope_append, peqa_norm_rope, peqa_norm_rope_bwd) against plain implementations
in 64 bits.

Tolerances.  A head's sum of squares adds at most 16 + 4 positive numbers after one another, and a head's sum for dx as many products:
under 2^-18 of the size of what is added, and the steps around them (square root, products, rotation) add less; a stored bf16 number is off
by 2^-8 of itself, an 8-bit one by 2^-4 of itself or half of the least one, 2^-10.  A weight's gradient adds up to 64 numbers in a thread
(as many as these sizes leave to one), then 64, 32 and 32: 2^-16 of the sum of sizes, their own errors included."""
import numpy as np
import pytest

from test_gpu_decode import make_cache

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_2305_14152_amd import peqa
    peqa.lib()
    return torch, peqa


def tables(torch, n, rot, gen):
    """Cosines and sines of any angles, not of a circle's (longer contexts scale them)."""
    if not rot:
        return None, None
    angle = 6.3 * torch.rand((n, rot // 2), generator=gen)
    return (1.1 * angle.cos()).cuda(), (1.1 * angle.sin()).cuda()


def pairs(rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def host(t):
    return None if t is None else t.float().cpu().double().numpy()


def turned(x, cos, sin, pos, interleaved, back=False):
    """x [T, heads, dim] rotated, and the size of what was added for every element."""
    if cos is None:
        return x.copy(), np.abs(x)
    a, b = pairs(2 * cos.shape[1], interleaved)
    c, s = host(cos)[pos][:, None], host(sin)[pos][:, None] * (-1 if back else 1)
    y, size = x.copy(), np.abs(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    size[..., a] = np.abs(x[..., a] * c) + np.abs(x[..., b] * s)
    size[..., b] = np.abs(x[..., a] * s) + np.abs(x[..., b] * c)
    return y, size


def forward(x, w, cos, sin, pos, interleaved, eps=EPS):
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return turned(x * r * (1.0 if w is None else w), cos, sin, pos, interleaved)


def backward(x, w, cos, sin, pos, interleaved, dy, there, eps=EPS):
    """dx, dw and the sizes of what is added up for them; rows that are not `there` have none."""
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    g, g_size = turned(dy, cos, sin, pos, interleaved, back=True)
    z, live = x * r, there[:, None, None]
    dw, dw_size = (g * z * live).sum((0, 1)), (g_size * np.abs(z) * live).sum((0, 1))
    w = 1.0 if w is None else w
    u, u_size = g * w, g_size * np.abs(w)
    dx = r * (u - z * (u * z).mean(-1, keepdims=True)) * live
    return dx, r * (u_size + np.abs(z) * (u_size * np.abs(z)).mean(-1, keepdims=True)) * live, dw, dw_size


def near(got, want, size, step=2.0 ** -8):
    off = np.abs(got - want) - (step * np.abs(want) + 2.0 ** -17 * size + 1e-30)
    assert np.isfinite(got).all() and off.max() <= 0, (off.max(), np.unravel_index(off.argmax(), off.shape))


def inputs(torch, gen, T, heads, kv, dim, scale=1.0):
    """Members of a stacked linear's output."""
    both = (scale * torch.randn((T, (heads + 2 * kv) * dim), generator=gen)).to(torch.bfloat16).cuda()
    q, k, v = both.split([heads * dim, kv * dim, kv * dim], 1)
    return q.unflatten(1, (heads, dim)), k.unflatten(1, (kv, dim)), v.unflatten(1, (kv, dim))


CASES = [(1, 1, 1, 64, 64, False, True), (1, 32, 8, 128, 128, False, True), (2, 5, 5, 128, 64, True, True), (17, 8, 2, 256, 256, False, False),
         (333, 3, 1, 64, 16, False, True), (100, 12, 4, 256, 48, True, True), (64, 4, 4, 128, 0, False, True), (1000, 40, 8, 128, 128, False, True),
         (3000, 7, 1, 64, 64, True, False)]


@pytest.mark.parametrize("T,heads,kv,dim,rot,interleaved,weighted", CASES)
def test_training(env, T, heads, kv, dim, rot, interleaved, weighted):
    torch, peqa = env
    gen = torch.Generator().manual_seed(T * 1000 + heads)
    n = 77
    cos, sin = tables(torch, n, rot, gen)
    q, k, _ = inputs(torch, gen, T, heads, kv, dim)
    pos = torch.randint(0, n, (T,), generator=gen, dtype=torch.int32)
    if T > 2:
        pos[1] = -1
        pos[T - 1] = n if rot else -2 ** 31
    there = (pos >= 0).numpy() & ((pos < n).numpy() | (rot == 0))
    at = np.where(there, pos.numpy(), 0)
    pos = pos.cuda()
    wq, wk = ((1 + 0.3 * torch.randn(dim, generator=gen)).cuda() if weighted else None for _ in range(2))
    outs = [torch.full((T, h * dim + 8), float("nan"), dtype=torch.bfloat16, device="cuda")[:, :h * dim].unflatten(1, (h, dim)) for h in (heads, kv) * 2]
    peqa.norm_rope(q, k, pos, cos, sin, wq, wk, EPS, outs[0], outs[1], interleaved=interleaved)
    dq_out, dk_out, _ = inputs(torch, gen, T, heads, kv, dim)
    room = peqa.norm_rope_bwd_workspace_bytes(T, heads, kv, dim)
    ws = torch.full((room,), 255, dtype=torch.uint8, device="cuda")
    dws = [torch.full((dim,), float("nan"), device="cuda") for _ in range(2)]
    args = (q, k, pos, cos, sin, wq, wk, EPS, dq_out, dk_out)
    peqa.norm_rope_bwd(*args, outs[2], outs[3], *dws, ws, room, interleaved=interleaved)
    for x, w, y, dy, dx, dw in ((q, wq, outs[0], dq_out, outs[2], dws[0]), (k, wk, outs[1], dk_out, outs[3], dws[1])):
        X, W = host(x), host(w)
        want, size = forward(X, W, cos, sin, at, interleaved)
        near(host(y), want * there[:, None, None], size)
        want, size, grad, grad_size = backward(X, W, cos, sin, at, interleaved, host(dy), there)
        near(host(dx), want, size)
        off = np.abs(host(dw) - grad) - 2.0 ** -16 * grad_size
        assert off.max() <= 0, off.max()
    # the same bits without the weights' gradients, with one of them, and in the gradients' own place
    for which in ((None, None), (torch.empty_like(dws[0]), None), (None, torch.empty_like(dws[1]))):
        g, h = dq_out.clone(), dk_out.clone()
        peqa.norm_rope_bwd(*args[:8], g, h, g, h, *which, ws if any(w is not None for w in which) else None, room if any(w is not None for w in which) else 0,
                           interleaved=interleaved)
        assert torch.equal(g, outs[2]) and torch.equal(h, outs[3])
        for w, d in zip(which, dws):
            assert w is None or torch.equal(w, d)
    y, z = q.clone(), k.clone()
    peqa.norm_rope(y, z, pos, cos, sin, wq, wk, EPS, y, z, interleaved=interleaved)
    assert torch.equal(y, outs[0]) and torch.equal(z, outs[1])


def test_formulas_against_differences():
    """The 64-bit gradients that the kernels are held to, against central differences of the 64-bit forward."""
    rng = np.random.default_rng(0)
    import torch
    gen = torch.Generator().manual_seed(0)
    angle = 6.3 * torch.rand((5, 8), generator=gen)
    cos, sin = 1.1 * angle.cos(), 1.1 * angle.sin()
    for interleaved in (False, True):
        x, w, dy, pos = rng.normal(size=(3, 2, 24)), 1 + 0.3 * rng.normal(size=24), rng.normal(size=(3, 2, 24)), np.array([4, 0, 2])
        dx, _, dw, _ = backward(x, w, cos, sin, pos, interleaved, dy, np.ones(3, bool))
        f = lambda x, w: (forward(x, w, cos, sin, pos, interleaved)[0] * dy).sum()  # noqa: E731
        for _ in range(5):
            ex, ew = rng.normal(size=x.shape), rng.normal(size=w.shape)
            h = 1e-5
            assert abs((f(x + h * ex, w) - f(x - h * ex, w)) / (2 * h) - (dx * ex).sum()) <= 1e-7
            assert abs((f(x, w + h * ew) - f(x, w - h * ew)) / (2 * h) - (dw * ew).sum()) <= 1e-7


@pytest.mark.parametrize("scale", [0.0, 1e-30, 1e-4, 1e4, 1e15])
def test_sizes_of_heads(env, scale):
    """Heads of zeros, under eps and far above it."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(5)
    T, heads, kv, dim = 9, 4, 2, 128
    cos, sin = tables(torch, 16, 128, gen)
    q, k, _ = inputs(torch, gen, T, heads, kv, dim, scale)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
    y, z, dq, dk = (torch.empty((T, h, dim), dtype=torch.bfloat16, device="cuda") for h in (heads, kv) * 2)
    peqa.norm_rope(q, k, pos, cos, sin, w, w, EPS, y, z)
    dy, dz, _ = inputs(torch, gen, T, heads, kv, dim)
    peqa.norm_rope_bwd(q, k, pos, cos, sin, w, w, EPS, dy, dz, dq, dk, None, None, None, 0)
    at = np.arange(T)
    for x, out, d, dx in ((q, y, dy, dq), (k, z, dz, dk)):
        want, size = forward(host(x), host(w), cos, sin, at, False)
        near(host(out), want, size)
        want, size, _, _ = backward(host(x), host(w), cos, sin, at, False, host(d), np.ones(T, bool))
        near(host(dx), want, size)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,heads,kv,dim,rot,interleaved,page,layout", [
    (1, 1, 1, 64, 64, False, 8, "heads"), (16, 32, 8, 128, 128, False, 16, "slots"), (3, 6, 2, 256, 64, True, 32, "both"),
    (200, 8, 8, 128, 128, True, 16, "heads"), (77, 12, 1, 64, 16, False, 64, "heads"), (50, 4, 4, 256, 0, False, 8, "slots")])
def test_append(env, T, heads, kv, dim, rot, interleaved, page, layout, fp8):
    """Rotated by one number, stored at another; what is not a token's place stays as it was."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(T + dim)
    seqs, room, n = 3, 150, 900
    cache = make_cache(torch, peqa, gen, [room] * seqs, kv, dim, page, fp8=fp8, layout=layout)
    cos, sin = tables(torch, n, rot, gen)
    q, k, v = inputs(torch, gen, T, heads, kv, dim)
    places = torch.randperm(seqs * room, generator=gen)[:T]
    seq, place = (places // room).to(torch.int32), (places % room).to(torch.int32)
    pos = torch.randint(0, n, (T,), generator=gen, dtype=torch.int32)
    gone = np.zeros(T, bool)
    if T > 10:                                                # tokens that are skipped, each for a reason of its own
        place[1], seq[2], seq[3], pos[4], place[5] = -1, -1, seqs, -1, 2 ** 31 - 1
        gone[[1, 2, 3, 4, 5]] = True
        if rot:
            pos[6] = n
            gone[6] = True
        cache.tensors[2][int(seq[7]), int(place[7]) // page] = cache.n_pages
        gone |= ((seq == seq[7]) & (place // page == place[7] // page)).numpy()
    wq, wk = ((1 + 0.3 * torch.randn(dim, generator=gen)).cuda() for _ in range(2))
    out = torch.full((T, heads, dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    bits = torch.uint8 if fp8 else torch.int16
    before = [p.view(bits).clone() for p in cache.tensors[:2]]
    peqa.norm_rope_append(cache, q, k, v, pos.cuda(), cos, sin, wq, wk, EPS, out, place=place.cuda(), seq=seq.cuda(), interleaved=interleaved)
    at = np.where(gone, 0, pos.numpy())
    want, size = forward(host(q), host(wq), cos, sin, at, interleaved)
    near(host(out), want * ~gone[:, None, None], size)
    want, size = forward(host(k), host(wk), cos, sin, at, interleaved)
    table = cache.tensors[2].cpu().numpy()
    touched = torch.zeros(before[0].shape, dtype=torch.bool)
    for name, (pool, scale, x, sizes) in enumerate(((cache.tensors[0], cache.tensors[3], want, size), (cache.tensors[1], cache.tensors[4], host(v), np.abs(host(v))))):
        data = pool.float().cpu().double().numpy()
        for t in range(T):
            if gone[t]:
                continue
            p, s = table[seq[t], place[t] // page], int(place[t]) % page
            touched[p, :, s] = True
            got, should, part = data[p, :, s], x[t], sizes[t]
            if fp8:
                by = host(scale)[:, None]
                should, part = np.clip(should / by, -448, 448), part / by
                assert (np.abs(got - should) <= np.maximum(2.0 ** -4 * np.abs(should), 2.0 ** -10) + 2.0 ** -17 * part).all()
            else:
                near(got, should, part)
    for pool, old in zip(cache.tensors[:2], before):
        assert torch.equal(pool.view(bits).cpu()[~touched], old.cpu()[~touched])
    # places of their own or none: the same as long as they are the positions; without queries
    if rot == 0 or room <= n:
        where = torch.where(torch.from_numpy(gone), -1, place).cuda()
        a, b = torch.empty_like(out), torch.empty_like(out)
        peqa.norm_rope_append(cache, q, k, v, where, cos, sin, wq, wk, EPS, a, seq=seq.cuda(), interleaved=interleaved)
        kept = [p.view(bits).clone() for p in cache.tensors[:2]]
        peqa.norm_rope_append(cache, q, k, v, where, cos, sin, wq, wk, EPS, b, place=where, seq=seq.cuda(), interleaved=interleaved)
        assert torch.equal(a, b) and all(torch.equal(p.view(bits), o) for p, o in zip(cache.tensors[:2], kept))
        peqa.norm_rope_append(cache, None, k, v, where, cos, sin, None, wk, EPS, None, seq=seq.cuda(), interleaved=interleaved)
        assert all(torch.equal(p.view(bits), o) for p, o in zip(cache.tensors[:2], kept))


def test_stream_and_graph(env):
    """A captured forward and backward, replayed over changing inputs on a stream of their own, against eager calls."""
    torch, peqa = env
    gen = torch.Generator().manual_seed(8)
    T, heads, kv, dim = 700, 8, 2, 128
    cos, sin = tables(torch, 1000, 128, gen)
    q, k, _ = inputs(torch, gen, T, heads, kv, dim)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    w = (1 + 0.3 * torch.randn(dim, generator=gen)).cuda()
    room = peqa.norm_rope_bwd_workspace_bytes(T, heads, kv, dim)

    def step(out, ws):
        y, z, dq, dk, dw, dv = out
        peqa.norm_rope(q, k, pos, cos, sin, w, w, EPS, y, z)
        peqa.norm_rope_bwd(q, k, pos, cos, sin, w, w, EPS, y, z, dq, dk, dw, dv, ws, room)

    def fresh():
        return [torch.empty((T, h, dim), dtype=torch.bfloat16, device="cuda") for h in (heads, kv) * 2] + [torch.empty(dim, device="cuda") for _ in range(2)]
    stream, graph, got = torch.cuda.Stream(), torch.cuda.CUDAGraph(), fresh()
    ws = torch.empty(room, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step(got, ws)
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step(got, ws)
    for i in range(4):
        q.copy_(torch.randn(q.shape, generator=gen).to(torch.bfloat16))
        pos.copy_(torch.randint(0, 1000, (T,), generator=gen, dtype=torch.int32))
        want = fresh()
        step(want, torch.empty(room, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i

"""Cases of the operators that decoders with normalised heads, shared prompts and bounded caches need beside the PEQA linears, through
the calls of paper_2305_14152_amd.peqa (`own` true) or in elementary torch operations in 32 bits (`own` false).

A case is a dict of plain values; its "kind" is one of

  append   peqa.norm_rope_append: queries and keys of new tokens normalised per head and rotated by their positions, keys and values
           stored in a paged cache at places of their own
  train    peqa.norm_rope and peqa.norm_rope_bwd: the same without a cache, and the gradients of its inputs and of the norms' weights
  shared   peqa.shared_attention: one query token per row; the first positions of all rows are one sequence's
  weights  peqa.paged_attention_weights: attention over the cache that also adds up what every position was given
  evict    peqa.cache_evict: the positions with the least of it leave the cache
"""
import math

import torch

own = False

FP8_MAX = 448.0
THETA = 10000.0
EPS = 1e-6


def listed():
    return [
        # one decoding step of sixteen sequences that were cut before, so that a token's place is not its position: latency
        {"name": "append_step_gqa", "kind": "append", "rows": 16, "seqs": 16, "heads": 32, "kv_heads": 8, "dim": 128, "rot": 128,
         "interleaved": False, "page": 64, "fp8": False, "most": 1024, "behind": 500},
        # three prompts of uneven length at once, half of every head rotated in neighbouring pairs, 8-bit cache
        {"name": "append_prompts_fp8", "kind": "append", "rows": 5003, "seqs": 3, "heads": 40, "kv_heads": 8, "dim": 128, "rot": 64,
         "interleaved": True, "page": 16, "fp8": True, "most": 2048, "behind": 0},
        # a short odd training batch of a small decoder with wide heads and frozen norms: launches and latency
        {"name": "train_short", "kind": "train", "rows": 129, "heads": 8, "kv_heads": 2, "dim": 256, "rot": 256, "interleaved": False,
         "trained": False},
        # the benchmark's training step: 2048 tokens of a 7B layer, norms trained too
        {"name": "train_7b", "kind": "train", "rows": 2048, "heads": 32, "kv_heads": 32, "dim": 128, "rot": 128, "interleaved": False,
         "trained": True},
        # three answers to one short question: latency
        {"name": "shared_few_7b", "kind": "shared", "rows": 3, "heads": 32, "kv_heads": 32, "dim": 128, "page": 16, "fp8": False,
         "shared": 555, "most": 77},
        # sixteen samples behind a prompt as long as the training context
        {"name": "shared_batch_7b", "kind": "shared", "rows": 16, "heads": 32, "kv_heads": 32, "dim": 128, "page": 64, "fp8": False,
         "shared": 2048, "most": 512},
        # a full serving batch behind a long system prompt, eight heads to a key head: the prefix is a matrix product
        {"name": "shared_many_gqa", "kind": "shared", "rows": 64, "heads": 64, "kv_heads": 8, "dim": 128, "page": 32, "fp8": False,
         "shared": 8192, "most": 1024},
        # questions about one long document on an 8-bit cache
        {"name": "shared_document_fp8", "kind": "shared", "rows": 32, "heads": 64, "kv_heads": 8, "dim": 128, "page": 128, "fp8": True,
         "shared": 65537, "most": 333},
        # the smallest accumulating attention: one short sequence
        {"name": "weights_one_7b", "kind": "weights", "rows": 1, "heads": 32, "kv_heads": 32, "dim": 128, "page": 16, "fp8": False,
         "most": 333, "uneven": False, "window": 0},
        # a serving batch of uneven lengths with eight heads to a key head
        {"name": "weights_batch_gqa", "kind": "weights", "rows": 32, "heads": 64, "kv_heads": 8, "dim": 128, "page": 32, "fp8": False,
         "most": 8192, "uneven": True, "window": 0},
        # one sequence cut by a third where it lies, an odd number of positions
        {"name": "evict_one_gqa", "kind": "evict", "rows": 1, "kv_heads": 8, "dim": 128, "page": 16, "fp8": False, "most": 1501,
         "keep": 1001, "sinks": 4, "recent": 200, "uneven": False, "inplace": True},
        # sixteen 7B sequences of uneven lengths cut to half of the training context
        {"name": "evict_batch_7b", "kind": "evict", "rows": 16, "kv_heads": 32, "dim": 128, "page": 64, "fp8": False, "most": 2048,
         "keep": 1024, "sinks": 4, "recent": 256, "uneven": True, "inplace": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, no more work than the largest listed one of its kind."""
    kind = rng.choice(["append", "train", "shared", "shared", "weights", "weights", "evict", "evict"])
    bytes_, flops = (max(work(c)[k] for c in listed() if c["kind"] == kind) for k in ("bytes", "flops"))
    while True:
        kv = rng.choice([1, 2, 4, 5, 8, 8, 16, 32, 40, 64])
        group = rng.choice([1, 1, 1, 2, 4, 8, 8, 12, 16])
        if kv * group > 128:
            continue
        c = {"kind": kind, "heads": kv * group, "kv_heads": kv, "dim": rng.choice([64, 128, 128, 128, 256])}
        if kind in ("append", "train"):
            c["rot"] = rng.choice([c["dim"], c["dim"], c["dim"] // 2, c["dim"] // 4])
            c["interleaved"] = rng.random() < 0.4
        if kind != "train":
            c["page"] = rng.choice([8, 16, 16, 32, 64, 128, 256])
            c["fp8"] = rng.random() < 0.4
        if kind == "append":
            c["rows"] = _log_int(rng, 1, 6000)
            c["seqs"] = c["rows"] if c["rows"] <= 64 else rng.randint(1, 8)
            c["most"] = max(_log_int(rng, 64, 4096), -(-c["rows"] // c["seqs"]) + 100)
            c["behind"] = rng.choice([0, 0, _log_int(rng, 1, 5000)])
            room = c["seqs"] * c["most"]
        elif kind == "train":
            c["rows"] = _log_int(rng, 1, 8192)
            c["trained"] = rng.random() < 0.6
            room = 0
        elif kind == "shared":
            c["rows"] = _log_int(rng, 1, 128)
            c["shared"] = _log_int(rng, 1, 131072)
            c["most"] = _log_int(rng, 1, 4096)
            room = c["shared"] + c["rows"] * c["most"]
        else:
            c["rows"] = _log_int(rng, 1, 128)
            c["most"] = _log_int(rng, 1, 65536)
            c["uneven"] = c["rows"] > 1 and rng.random() < 0.7
            room = c["rows"] * c["most"]
            if kind == "weights":
                c["window"] = rng.choice([0, 0, 0, _log_int(rng, 16, 8192)])
            else:
                del c["heads"]
                c["keep"] = max(1, int(c["most"] * rng.uniform(0.2, 0.98)))
                c["sinks"] = min(c["keep"] // 4, rng.choice([0, 1, 4, 16]))
                c["recent"] = int(c["keep"] * rng.uniform(0.0, 0.5))
                c["inplace"] = rng.random() < 0.6
        w = work(c)
        if room * kv * c["dim"] <= 1 << 28 and w["bytes"] <= bytes_ and w["flops"] <= max(flops, 1.0):
            return c


def _lengths(c):
    """Lengths of the rows' sequences: uneven ones spread from a few tokens to the longest, the second row of several empty."""
    if not c.get("uneven", True):
        return [c["most"]] * c["rows"]
    n = [max(1, round(c["most"] * (0.02 + 0.98 * (0.618034 * i % 1.0)))) for i in range(c["rows"])]
    n[0] = c["most"]
    if c["rows"] > 2:
        n[1] = 0
    return n


def _shared_lengths(c):
    """The rows' own positions behind the shared ones; a row without any sees nothing at all."""
    n = _lengths(c)
    return [c["shared"] + m if m else 0 for m in n], n


def work(c):
    """Bytes and flops of one pass: inputs read once, outputs written once."""
    element = 1 if c.get("fp8") else 2
    if c["kind"] in ("append", "train"):
        q, kv = c["rows"] * c["heads"] * c["dim"], c["rows"] * c["kv_heads"] * c["dim"]
        tables = 4.0 * c["rows"] * c["rot"] + 12.0 * c["rows"]
        if c["kind"] == "append":
            return {"bytes": 4.0 * (q + kv) + 2.0 * kv * element + tables, "flops": 5.0 * (q + kv)}
        # forward: both read and written; backward: inputs and gradients read, gradients written
        return {"bytes": 10.0 * (q + kv) + 2 * tables, "flops": 20.0 * (q + kv)}
    row = c["kv_heads"] * c["dim"] * element * 2
    if c["kind"] == "shared":
        lens, mine = _shared_lengths(c)
        queries = c["rows"] * c["heads"] * c["dim"]
        positions = sum(mine) + c["shared"]
        return {"bytes": float(row) * positions + 4.0 * queries + 4.0 * c["rows"] * c["heads"] + 4.0 * (positions // c["page"] + 2 * c["rows"]),
                "flops": 4.0 * sum(lens) * c["heads"] * c["dim"]}
    if c["kind"] == "weights":
        tokens = sum(min(n, c["window"]) if c["window"] else n for n in _lengths(c))
        return {"bytes": float(row) * tokens + 4.0 * c["rows"] * c["heads"] * c["dim"] + 4.0 * c["rows"] * c["heads"] + 8.0 * tokens * c["kv_heads"]
                + 4.0 * (tokens // c["page"] + 2 * c["rows"]),
                "flops": 4.0 * tokens * c["heads"] * c["dim"] + 2.0 * tokens * c["heads"]}
    lens = _lengths(c)
    # in place, what is in front of the first one to leave stays where it is: little more than the sinks
    moved = sum(max(0, c["keep"] - c["sinks"]) if n > c["keep"] else 0 for n in lens) if c["inplace"] else sum(min(n, c["keep"]) for n in lens)
    return {"bytes": 2.0 * row * moved + 4.0 * c["kv_heads"] * (sum(lens) + c["rows"] * (c["most"] + c["keep"])), "flops": 2.0 * c["kv_heads"] * sum(lens)}


# ---- inputs -------------------------------------------------------------------------------------------------------

def _pool(c, pages, gen):
    x = torch.randn((pages, c["kv_heads"], c["page"], c["dim"]), device="cuda", generator=gen, dtype=torch.float32 if c["fp8"] else torch.bfloat16)
    return (16.0 * x).clamp_(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn) if c["fp8"] else x


def _cache(c, needed, gen):
    """Pools of pages and the table of a cache whose sequences have `needed` pages each, at places without order."""
    blocks, total = max(max(needed), 1), sum(needed)
    order = torch.randperm(total + 3, device="cuda", generator=gen)[:total].to(torch.int32)
    table = torch.zeros((len(needed), blocks), dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(needed):
        table[i, :n] = order[at:at + n]
        at += n
    s = {"k_pool": _pool(c, total + 3, gen), "v_pool": _pool(c, total + 3, gen), "table": table, "k_scale": None, "v_scale": None}
    if c["fp8"]:
        s["k_scale"] = 0.05 + 0.02 * torch.rand(c["kv_heads"], device="cuda", generator=gen)
        s["v_scale"] = 0.05 + 0.02 * torch.rand(c["kv_heads"], device="cuda", generator=gen)
    return s


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _tables(c, positions):
    angle = torch.outer(torch.arange(positions, device="cuda", dtype=torch.float64),
                        THETA ** (-torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64) / c["rot"]))
    return {"cos": angle.cos().float(), "sin": angle.sin().float()}


def _places(c):
    """(sequence, place) of the new tokens of an append: one per sequence at uneven places, or pieces of prompts."""
    if c["rows"] == c["seqs"]:
        return list(range(c["rows"])), [(c["most"] - 1 - 37 * i) % c["most"] for i in range(c["rows"])]
    each = -(-c["rows"] // c["seqs"])
    seq = [i // each for i in range(c["rows"])]
    return seq, [i % each + 7 * s for i, s in enumerate(seq)]


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": c}
    normal = lambda *shape, dtype=torch.bfloat16: torch.randn(shape, device="cuda", generator=gen, dtype=dtype)  # noqa: E731
    if c["kind"] in ("append", "train"):
        # queries, keys and values as the linears before leave them: side by side in one row per token
        both = normal(c["rows"], (c["heads"] + 2 * c["kv_heads"]) * c["dim"]) * 1.5
        q, kv = c["heads"] * c["dim"], c["kv_heads"] * c["dim"]
        s["q"] = both[:, :q].unflatten(1, (c["heads"], c["dim"]))
        s["k"] = both[:, q:q + kv].unflatten(1, (c["kv_heads"], c["dim"]))
        s["v"] = both[:, q + kv:].unflatten(1, (c["kv_heads"], c["dim"]))
        s["q_weight"] = 1.0 + 0.2 * normal(c["dim"], dtype=torch.float32)
        s["k_weight"] = 1.0 + 0.2 * normal(c["dim"], dtype=torch.float32)
        s["q_out"] = torch.empty((c["rows"], c["heads"], c["dim"]), device="cuda", dtype=torch.bfloat16)
    if c["kind"] == "append":
        seq, place = _places(c)
        s |= _cache(c, [-(-c["most"] // c["page"])] * c["seqs"], gen)
        s["seq"], s["place"] = _int32(seq), _int32(place)
        s["pos"] = s["place"] + c["behind"] if c["behind"] else s["place"]
        s |= _tables(c, c["most"] + c["behind"])
    elif c["kind"] == "train":
        s["pos"] = _int32([i % 2048 for i in range(c["rows"])])
        s |= _tables(c, min(c["rows"], 2048))
        s["k_out"] = torch.empty((c["rows"], c["kv_heads"], c["dim"]), device="cuda", dtype=torch.bfloat16)
        s["d_q_out"], s["d_k_out"] = normal(c["rows"], c["heads"], c["dim"]), normal(c["rows"], c["kv_heads"], c["dim"])
        # the gradients go where the linears' backward takes them: side by side
        d = torch.zeros_like(both)
        s["dq"], s["dk"] = d[:, :q].unflatten(1, (c["heads"], c["dim"])), d[:, q:q + kv].unflatten(1, (c["kv_heads"], c["dim"]))
        s["d_q_weight"] = torch.empty(c["dim"], device="cuda") if c["trained"] else None
        s["d_k_weight"] = torch.empty(c["dim"], device="cuda") if c["trained"] else None
    elif c["kind"] == "shared":
        lens, mine = _shared_lengths(c)
        # the last row of the table is the prefix's; the others' own pages begin with the one that the shared positions end in
        first = c["shared"] // c["page"]
        needed = [-(-n // c["page"]) - first if n else 0 for n in lens] + [-(-c["shared"] // c["page"])]
        s |= _cache(c, needed, gen)
        table = torch.zeros((c["rows"] + 1, -(-max(max(lens), c["shared"]) // c["page"])), dtype=torch.int32, device="cuda")
        width = min(s["table"].shape[1], table.shape[1] - first)
        table[:-1, first:first + width] = s["table"][:-1, :width]
        table[-1, :needed[-1]] = s["table"][-1, :needed[-1]]
        s["table"] = table
        s["lens"], s["most"] = _int32(lens), max(lens)
    elif c["kind"] == "weights":
        lens = _lengths(c)
        s |= _cache(c, [-(-n // c["page"]) for n in lens], gen)
        s["lens"], s["most"] = _int32(lens), max(lens)
        s["before"] = torch.rand((c["rows"], c["kv_heads"], -(-c["most"] // 4) * 4), device="cuda", generator=gen)
        s["after"] = torch.zeros_like(s["before"])
    else:
        lens = _lengths(c)
        s |= _cache(c, [-(-n // c["page"]) for n in lens], gen)
        s["lens"], s["most"] = _int32(lens), max(lens)
        # few positions with much, many with little, some that were never looked at
        room = (c["rows"], c["kv_heads"], -(-c["most"] // 4) * 4)
        w = torch.exp(2.5 * normal(*room, dtype=torch.float32))
        s["before"] = w.masked_fill_(torch.rand(room, device="cuda", generator=gen) < 0.15, 0.0)
        s["after"] = torch.zeros(room, device="cuda")
        s["kept"] = torch.empty((c["rows"], c["kv_heads"], c["keep"]), dtype=torch.int32, device="cuda")
        s["new_lens"] = torch.empty(c["rows"], dtype=torch.int32, device="cuda")
        for name in ("k", "v"):
            s["to_" + name] = s[name + "_pool"]
        s["to_table"] = s["table"]
        if not c["inplace"]:
            to = _cache(c, [-(-min(n, c["keep"]) // c["page"]) for n in lens], gen)
            s |= {"to_k": to["k_pool"], "to_v": to["v_pool"], "to_table": to["table"]}
    if c["kind"] in ("shared", "weights"):
        s["q"] = normal(c["rows"], c["heads"], c["dim"])
        s["scale"] = c["dim"] ** -0.5
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((c["rows"], c["heads"]), device="cuda")
    if own:
        from paper_2305_14152_amd import peqa
        if c["kind"] != "train":
            s["cache"] = peqa.kv_cache(s["k_pool"], s["v_pool"], s["table"], s["k_scale"], s["v_scale"])
        room = 0
        if c["kind"] == "train":
            room = peqa.norm_rope_bwd_workspace_bytes(c["rows"], c["heads"], c["kv_heads"], c["dim"])
        elif c["kind"] == "shared":
            room = peqa.shared_attention_workspace_bytes(s["cache"], c["heads"], c["rows"], s["most"], c["shared"])
        elif c["kind"] == "weights":
            room = peqa.paged_attention_weights_workspace_bytes(s["cache"], c["heads"], c["rows"], s["most"], c["window"])
        elif c["kind"] == "evict":
            room = peqa.cache_evict_workspace_bytes(s["cache"], c["rows"], s["most"], c["keep"])
            s["to"] = None if c["inplace"] else peqa.kv_cache(s["to_k"], s["to_v"], s["to_table"], s["k_scale"], s["v_scale"])
        s["room"] = room
        s["ws"] = torch.zeros(max(room, 16), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------

def _run_own(s):
    from paper_2305_14152_amd import peqa
    c = s["case"]
    if c["kind"] == "append":
        peqa.norm_rope_append(s["cache"], s["q"], s["k"], s["v"], s["pos"], s["cos"], s["sin"], s["q_weight"], s["k_weight"], EPS, s["q_out"],
                              place=s["place"] if c["behind"] else None, seq=s["seq"], interleaved=c["interleaved"])
    elif c["kind"] == "train":
        peqa.norm_rope(s["q"], s["k"], s["pos"], s["cos"], s["sin"], s["q_weight"], s["k_weight"], EPS, s["q_out"], s["k_out"],
                       interleaved=c["interleaved"])
        peqa.norm_rope_bwd(s["q"], s["k"], s["pos"], s["cos"], s["sin"], s["q_weight"], s["k_weight"], EPS, s["d_q_out"], s["d_k_out"], s["dq"], s["dk"],
                           s["d_q_weight"], s["d_k_weight"], s["ws"], s["room"], interleaved=c["interleaved"])
    elif c["kind"] == "shared":
        peqa.shared_attention(s["cache"], s["q"], s["lens"], s["most"], c["rows"], c["shared"], s["scale"], s["out"], s["ws"], s["room"], lse=s["lse"])
    elif c["kind"] == "weights":
        peqa.paged_attention_weights(s["cache"], s["q"], s["lens"], s["most"], s["scale"], s["out"], s["before"], s["after"], s["ws"], s["room"],
                                     lse=s["lse"], window=c["window"])
    else:
        peqa.cache_evict(s["cache"], s["lens"], s["most"], s["before"], s["after"], c["keep"], c["sinks"], c["recent"], s["kept"], s["new_lens"],
                         s["ws"], s["room"], to=s["to"])
    return _outputs(s)


def _outputs(s):
    kind = s["case"]["kind"]
    if kind == "append":
        return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}
    if kind == "evict":
        return {"k": s["to_k"], "v": s["to_v"], "weights": s["after"], "kept": s["kept"], "lens": s["new_lens"]}
    names = {"train": ("q_out", "k_out", "dq", "dk", "d_q_weight", "d_k_weight"), "shared": ("out", "lse"), "weights": ("out", "lse", "after")}
    return {n: s[n] for n in names[kind]}


def _rotate(x, cos, sin, interleaved):
    """x [rows, heads, dim] in 32 bits, cos and sin [rows, 1, rot / 2]."""
    half = cos.shape[-1]
    r, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :half], r[..., half:])
    u, w = a * cos - b * sin, a * sin + b * cos
    r = torch.stack((u, w), -1).flatten(-2) if interleaved else torch.cat((u, w), -1)
    return torch.cat((r, rest), -1)


def _normed(x):
    """x in 32 bits, and one over its root mean square."""
    x = x.float()
    return x, torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)


def _store(pool, x, page, slot, scale):
    """x [rows, kv_heads, dim] in 32 bits into the pool at (page, head, slot)."""
    if scale is not None:
        x = (x / scale[:, None]).clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        pool = pool.view(torch.uint8)
    pool[page, :, slot] = x.to(pool.dtype)


def _forward(s, name):
    x, r = _normed(s[name])
    cos, sin = s["cos"][s["pos"].long()][:, None], s["sin"][s["pos"].long()][:, None]
    return _rotate(x * r * s[name + "_weight"], cos, sin, s["case"]["interleaved"])


def _append(s):
    c = s["case"]
    place = s["place"].long()
    page, slot = s["table"][s["seq"].long(), place // c["page"]].long(), place % c["page"]
    s["q_out"].copy_(_forward(s, "q"))
    _store(s["k_pool"], _forward(s, "k"), page, slot, s["k_scale"])
    _store(s["v_pool"], s["v"].float(), page, slot, s["v_scale"])


def _backward(s, name):
    x, r = _normed(s[name])
    cos, sin = s["cos"][s["pos"].long()][:, None], s["sin"][s["pos"].long()][:, None]
    g = _rotate(s["d_%s_out" % name].float(), cos, -sin, s["case"]["interleaved"])       # turned back
    y = x * r
    if s["case"]["trained"]:
        s["d_%s_weight" % name].copy_((g * y).sum((0, 1)))
    g = g * s[name + "_weight"]
    s["d" + name].copy_(r * (g - y * (g * y).mean(-1, keepdim=True)))


def _train(s):
    s["q_out"].copy_(_forward(s, "q"))
    s["k_out"].copy_(_forward(s, "k"))
    _backward(s, "q")
    _backward(s, "k")


def _gather(pool, scale, table):
    """The pages of every row, [rows, kv_heads, positions, dim] in 32 bits."""
    x = (pool if scale is None else pool.view(torch.uint8))[table.long()].view(pool.dtype).float()
    if scale is not None:
        x = x * scale[:, None, None]
    return x.transpose(1, 2).flatten(2, 3)


def _softmax(scores):
    """(weights before division, their sums, log-sum-exp) over the last axis; rows of -inf only have sums of 0."""
    top = scores.amax(-1, keepdim=True).clamp_min(-3.0e38)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    return p, total, torch.where(total > 0, top + total.log(), -math.inf)


def _shared(s):
    c = s["case"]
    rows, kv, dim, n = c["rows"], c["kv_heads"], c["dim"], c["shared"]
    first = n // c["page"]
    blocks = -(-n // c["page"])
    k, v = (_gather(s[p + "_pool"], s[p + "_scale"], s["table"][-1:, :blocks])[0, :, :n] for p in ("k", "v"))
    mk, mv = (_gather(s[p + "_pool"], s[p + "_scale"], s["table"][:-1, first:]) for p in ("k", "v"))
    q, lens = s["q"].float().view(rows, kv, c["heads"] // kv, dim), s["lens"].long()[:, None]
    near = first * c["page"] + torch.arange(mk.shape[2], device="cuda")
    over = (torch.matmul(q.transpose(0, 1).flatten(1, 2), k.transpose(1, 2)) * s["scale"]).view(kv, rows, -1, n).transpose(0, 1)
    over = over.masked_fill(~(torch.arange(n, device="cuda") < lens)[:, None, None], -math.inf)
    mine = (torch.matmul(q, mk.transpose(2, 3)) * s["scale"]).masked_fill(~((near >= n) & (near < lens))[:, None, None], -math.inf)
    p, total, lse = _softmax(torch.cat((over, mine), -1))
    out = torch.matmul(p[..., :n].transpose(0, 1).flatten(1, 2), v).view(kv, rows, -1, dim).transpose(0, 1) + torch.matmul(p[..., n:], mv)
    s["out"].copy_((out / total.clamp_min(1e-30)).reshape(rows, c["heads"], dim))
    s["lse"].copy_(lse.reshape(rows, c["heads"]))


def _weights(s):
    c = s["case"]
    rows, kv, dim = c["rows"], c["kv_heads"], c["dim"]
    k, v = _gather(s["k_pool"], s["k_scale"], s["table"]), _gather(s["v_pool"], s["v_scale"], s["table"])
    q = s["q"].float().view(rows, kv, c["heads"] // kv, dim)
    at, lens = torch.arange(k.shape[2], device="cuda"), s["lens"].long()[:, None]
    seen = at < lens
    if c["window"]:
        seen &= at >= lens - c["window"]
    p, total, lse = _softmax((torch.matmul(q, k.transpose(2, 3)) * s["scale"]).masked_fill(~seen[:, None, None], -math.inf))
    p = p / total.clamp_min(1e-30)
    s["out"].copy_(torch.matmul(p, v).view(rows, c["heads"], dim))
    s["lse"].copy_(lse.reshape(rows, c["heads"]))
    n = c["most"]
    s["after"][..., :n] = torch.where((at < lens)[:, None, :n], s["before"][..., :n] + p.sum(2)[..., :n], s["after"][..., :n])


def _evict(s):
    c = s["case"]
    rows, kv, page = c["rows"], c["kv_heads"], c["page"]
    w, lens = s["before"], s["lens"].long()[:, None, None]
    at = torch.arange(w.shape[2], device="cuda").expand_as(w)
    held = (at < c["sinks"]) | (at >= lens - c["recent"])
    key = torch.where(at < lens, torch.where(held, math.inf, w), -math.inf)
    kept = torch.sort(key, dim=2, descending=True, stable=True)[1][..., :c["keep"]].sort(2)[0]
    there = kept < lens
    s["after"].zero_()
    s["after"][..., :c["keep"]] = torch.where(there, w.gather(2, kept), 0.0)
    s["kept"].copy_(torch.where(there, kept, -1))
    s["new_lens"].copy_(lens[:, 0, 0].clamp_max(c["keep"]))
    row, head, j = there.nonzero(as_tuple=True)
    old = kept[row, head, j]
    source, goal = s["table"][row, old // page].long(), s["to_table"][row, j // page].long()
    bits = torch.uint8 if c["fp8"] else torch.int16
    for_k = s["k_pool"].view(bits)[source, head, old % page]
    for_v = s["v_pool"].view(bits)[source, head, old % page]
    s["to_k"].view(bits)[goal, head, j % page] = for_k
    s["to_v"].view(bits)[goal, head, j % page] = for_v


def run(state):
    if own:
        return _run_own(state)
    {"append": _append, "train": _train, "shared": _shared, "weights": _weights, "evict": _evict}[state["case"]["kind"]](state)
    return _outputs(state)


# ---- in 64 bits ---------------------------------------------------------------------------------------------------

def exact(case, seed):
    """What run() returns for these inputs, from the definitions in 64 bits."""
    global own
    mode, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = mode
    c = case

    def head_norm(x, weight):
        return x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["dim"] + EPS) * weight

    def turned(x):
        angle = torch.complex(s["cos"].double(), s["sin"].double())[s["pos"].tolist()][:, None]
        half = c["rot"] // 2
        pairs = [(2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half) for i in range(half)]
        a, b = [p[0] for p in pairs], [p[1] for p in pairs]
        z = torch.complex(x[..., a], x[..., b]) * angle
        y = x.clone()
        y[..., a], y[..., b] = z.real, z.imag
        return y

    def head(name, table, h, lo, hi):
        """Positions lo .. hi-1 of key head h of the sequence with this row of the table."""
        pool, scale = s[name + "_pool"], s[name + "_scale"]
        b0 = lo // c["page"]
        pages = table[b0:-(-hi // c["page"])].long()
        x = pool.view(torch.uint8 if c["fp8"] else pool.dtype)[pages, h].view(pool.dtype).reshape(-1, c["dim"])[lo - b0 * c["page"]:hi - b0 * c["page"]]
        return x.float().double() * (1.0 if scale is None else scale[h].double())

    if c["kind"] == "train":
        out = {}
        for n in ("q", "k"):
            x, weight = s[n].double().requires_grad_(), s[n + "_weight"].double().requires_grad_()
            y = turned(head_norm(x, weight))
            dx, dw = torch.autograd.grad(y, (x, weight), s["d_%s_out" % n].double())
            out |= {n + "_out": y.detach(), "d" + n: dx, "d_%s_weight" % n: dw if c["trained"] else None}
        return out
    if c["kind"] == "append":
        got = {"k": turned(head_norm(s["k"].double(), s["k_weight"].double())), "v": s["v"].double()}
        out = {"q": turned(head_norm(s["q"].double(), s["q_weight"].double()))}
        table, place = s["table"].tolist(), s["place"].tolist()
        page = torch.tensor([table[n][p // c["page"]] for n, p in zip(s["seq"].tolist(), place)], device="cuda")
        slot = torch.tensor([p % c["page"] for p in place], device="cuda")
        for n in ("k", "v"):
            pool, x = s[n + "_pool"].float().double(), got[n]
            if c["fp8"]:
                x = (x / s[n + "_scale"].double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
            pool.permute(0, 2, 1, 3)[page, slot] = x
            out[n] = pool
        return out
    lens = s["lens"].tolist()
    if c["kind"] == "evict":
        pools = {n: s["to_" + n].float().double() for n in ("k", "v")}
        after = torch.zeros_like(s["before"], dtype=torch.float64)
        kept = torch.full_like(s["kept"], -1)
        for r, n in enumerate(lens):
            if n == 0:
                continue
            for h in range(c["kv_heads"]):
                w = s["before"][r, h, :n].double()
                if n > c["keep"]:
                    lo, hi = c["sinks"], n - c["recent"]
                    first = torch.argsort(w[lo:hi], descending=True, stable=True)[:c["keep"] - c["sinks"] - c["recent"]] + lo
                    take = torch.cat((torch.arange(lo, device="cuda"), first.sort()[0], torch.arange(hi, n, device="cuda")))
                else:
                    take = torch.arange(n, device="cuda")
                m = take.numel()
                kept[r, h, :m], after[r, h, :m] = take.to(torch.int32), w[take]
                goal, at = s["to_table"][r].long(), torch.arange(m, device="cuda")
                for name in ("k", "v"):
                    source = s[name + "_pool"].view(torch.uint8 if c["fp8"] else torch.bfloat16)
                    x = source[s["table"][r].long()[take // c["page"]], h, take % c["page"]].view(s[name + "_pool"].dtype)
                    pools[name][goal[at // c["page"]], h, at % c["page"]] = x.float().double()
        return {**pools, "weights": after, "kept": kept, "lens": torch.tensor([min(n, c["keep"]) for n in lens], dtype=torch.int32)}
    group = c["heads"] // c["kv_heads"]
    out = torch.zeros((c["rows"], c["heads"], c["dim"]), device="cuda", dtype=torch.float64)
    lse = torch.full((c["rows"], c["heads"]), -math.inf, device="cuda", dtype=torch.float64)
    after = s["after"].double() if c["kind"] == "weights" else None
    for h in range(c["kv_heads"]):
        members = slice(h * group, (h + 1) * group)
        if c["kind"] == "shared":
            k, v = (head(n, s["table"][-1], h, 0, c["shared"]) for n in ("k", "v"))
            far = (s["q"][:, members].double() @ k.T) * float(s["scale"])
        for r, n in enumerate(lens):
            lo = c["shared"] if c["kind"] == "shared" else max(0, n - c["window"]) if c["window"] else 0
            if n <= lo:
                continue
            mk, mv = (head(name, s["table"][r], h, lo, n) for name in ("k", "v"))
            z = (s["q"][r, members].double() @ mk.T) * float(s["scale"])
            if c["kind"] == "shared":
                z = torch.cat((far[r], z), 1)
            p = torch.softmax(z, 1)
            lse[r, members] = torch.logsumexp(z, 1)
            if c["kind"] == "shared":
                out[r, members] = p[:, :c["shared"]] @ v + p[:, c["shared"]:] @ mv
            else:
                out[r, members] = p @ mv
                after[r, h, :n] = s["before"][r, h, :n].double()
                after[r, h, lo:n] += p.sum(0)
    return {"out": out, "lse": lse} if c["kind"] == "shared" else {"out": out, "lse": lse, "after": after}

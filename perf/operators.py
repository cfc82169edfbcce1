"""Cases of the decoding and scoring operators beside the PEQA linears: what a program that serves or scores with a
quantized decoder does between its linears and after the last of them, through the calls of paper_2305_14152_amd.peqa
(`own` true) or in elementary torch operations in 32 bits (`own` false).

A case is a dict of plain values; its "kind" is one of

  append     peqa.rope_append: queries and keys of new tokens rotated by their positions, keys and values stored in a
             paged cache (bf16, or 8-bit floats with a scale per head)
  attend     peqa.paged_attention: one query token per row over its sequence's pages
  logprobs   peqa.token_logprobs: log probabilities of given tokens, entropy, log-sum-exp and the top alternatives
  logprobs_bwd  peqa.token_logprobs_bwd: the gradient of log probabilities and entropies with respect to the logits
"""
import math

import torch

own = False

FP8_MAX = 448.0
THETA = 10000.0
LOGIT_STD = 2.5


def listed():
    return [
        # one decoding step of sixteen 7B sequences: a few hundred kilobytes, launches and latency
        {"name": "append_step_7b", "kind": "append", "rows": 16, "seqs": 16, "heads": 32, "kv_heads": 32, "dim": 128, "rot": 128,
         "interleaved": False, "page": 64, "fp8": False, "most": 1024},
        # three prompts of uneven length at once, heads of 256 with a quarter of them rotated in neighbouring pairs, shared keys, 8-bit cache
        {"name": "append_prompts_fp8", "kind": "append", "rows": 5555, "seqs": 3, "heads": 32, "kv_heads": 8, "dim": 256, "rot": 64,
         "interleaved": True, "page": 16, "fp8": True, "most": 2048},
        # the smallest attention: one short 7B sequence
        {"name": "attend_one_7b", "kind": "attend", "rows": 1, "heads": 32, "kv_heads": 32, "dim": 128, "page": 16, "fp8": False,
         "most": 333, "uneven": False, "window": 0},
        # sixteen 7B sequences of uneven lengths up to the training context
        {"name": "attend_batch_7b", "kind": "attend", "rows": 16, "heads": 32, "kv_heads": 32, "dim": 128, "page": 64, "fp8": False,
         "most": 2048, "uneven": True, "window": 0},
        # seven 13B sequences behind a sliding window that starts inside a page
        {"name": "attend_window_13b", "kind": "attend", "rows": 7, "heads": 40, "kv_heads": 40, "dim": 128, "page": 16, "fp8": False,
         "most": 4999, "uneven": True, "window": 1000},
        # one very long document, eight heads to a key: the length has to be split
        {"name": "attend_long_gqa", "kind": "attend", "rows": 1, "heads": 64, "kv_heads": 8, "dim": 128, "page": 128, "fp8": False,
         "most": 131072, "uneven": False, "window": 0},
        # a full serving batch on an 8-bit cache
        {"name": "attend_many_gqa_fp8", "kind": "attend", "rows": 64, "heads": 64, "kv_heads": 8, "dim": 128, "page": 32, "fp8": True,
         "most": 8192, "uneven": True, "window": 0},
        # the end of a decoding step: sixteen rows of the 32000-word head, twenty alternatives each
        {"name": "logprobs_step_7b", "kind": "logprobs", "rows": 16, "vocab": 32000, "stride": 32000, "f32": False, "top": 20, "masked": 0.0, "ignored": 0.0},
        # perplexity of a text of the training context
        {"name": "logprobs_text_7b", "kind": "logprobs", "rows": 2048, "vocab": 32000, "stride": 32000, "f32": False, "top": 0, "masked": 0.0, "ignored": 0.1},
        # an odd vocabulary in padded rows, most words forbidden by a grammar, five alternatives
        {"name": "logprobs_odd_f32", "kind": "logprobs", "rows": 333, "vocab": 100003, "stride": 100008, "f32": True, "top": 5, "masked": 0.9, "ignored": 0.0},
        # a short batch whose loss has an entropy term, 32-bit logits of an odd width
        {"name": "logprobs_bwd_odd_f32", "kind": "logprobs_bwd", "rows": 100, "vocab": 50001, "stride": 50004, "f32": True, "entropy": True, "ignored": 0.0},
        # the loss gradient of one training sequence, a tenth of the tokens not trained on
        {"name": "logprobs_bwd_train_7b", "kind": "logprobs_bwd", "rows": 2048, "vocab": 32000, "stride": 32000, "f32": False, "entropy": False, "ignored": 0.1},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, no more work than the largest listed one of its kind."""
    kind = rng.choice(["append", "attend", "attend", "attend", "logprobs", "logprobs", "logprobs_bwd"])
    limit = max(work(c)["bytes"] for c in listed() if c["kind"] == kind)
    while True:
        if kind in ("append", "attend"):
            kv = rng.choice([1, 2, 4, 5, 8, 8, 16, 32, 40, 64])
            group = rng.choice([1, 1, 1, 2, 4, 8, 8, 12, 16])
            c = {"kind": kind, "heads": kv * group, "kv_heads": kv, "dim": rng.choice([64, 128, 128, 128, 256]),
                 "page": rng.choice([8, 16, 16, 32, 64, 128, 256]), "fp8": rng.random() < 0.4}
            if c["heads"] > 128:
                continue
            if kind == "append":
                c["rows"] = _log_int(rng, 1, 6000)
                c["seqs"] = c["rows"] if c["rows"] <= 64 else rng.randint(1, 8)
                c["rot"] = rng.choice([c["dim"], c["dim"], c["dim"] // 2, c["dim"] // 4])
                c["interleaved"] = rng.random() < 0.4
                c["most"] = max(_log_int(rng, 64, 4096), -(-c["rows"] // c["seqs"]) + 1)
                if c["seqs"] * c["most"] * kv * c["dim"] > 1 << 27:
                    continue
            else:
                c["rows"] = _log_int(rng, 1, 128)
                c["most"] = _log_int(rng, 1, 131072)
                c["uneven"] = c["rows"] > 1 and rng.random() < 0.7
                c["window"] = rng.choice([0, 0, 0, _log_int(rng, 16, 8192)])
                if c["rows"] * c["most"] * kv * c["dim"] > 1 << 29:      # what the pages of all sequences may hold
                    continue
        else:
            vocab = _log_int(rng, 1000, 260000)
            f32 = rng.random() < 0.4
            unit = 4 if f32 else 8
            c = {"kind": kind, "rows": _log_int(rng, 1, 4096), "vocab": vocab, "stride": -(-vocab // unit) * unit, "f32": f32,
                 "ignored": rng.choice([0.0, 0.1, 0.5])}
            if kind == "logprobs":
                c["top"] = rng.choice([0, 0, 1, 2, 5, 20, 32])
                c["masked"] = rng.choice([0.0, 0.0, 0.9, 0.999])
            else:
                c["entropy"] = rng.random() < 0.5
        if work(c)["bytes"] <= limit and 3072 not in c.values():
            return c


def _lengths(c):
    """Lengths of the rows' sequences: uneven ones spread from a few tokens to the longest, the second row of several empty."""
    if not c["uneven"]:
        return [c["most"]] * c["rows"]
    n = [max(1, round(c["most"] * (0.02 + 0.98 * (0.618034 * i % 1.0)))) for i in range(c["rows"])]
    n[0] = c["most"]
    if c["rows"] > 2:
        n[1] = 0
    return n


def _places(c):
    """(sequence, position) of the new tokens of an append: one per sequence at uneven positions, or pieces of prompts."""
    if c["rows"] == c["seqs"]:
        return list(range(c["rows"])), [(c["most"] - 1 - 37 * i) % c["most"] for i in range(c["rows"])]
    seq, pos = [], []
    left = c["rows"]
    for s in range(c["seqs"]):
        last = s == c["seqs"] - 1
        n = left if last else min(c["most"], left // (c["seqs"] - s) + 11 * s)
        n = max(n, left - (c["seqs"] - 1 - s) * c["most"])
        seq += [s] * min(n, left)
        pos += list(range(min(n, left)))
        left -= min(n, left)
    return seq, pos


def work(c):
    """Bytes and flops of one pass: inputs read once, outputs written once."""
    if c["kind"] == "append":
        q, kv = c["rows"] * c["heads"] * c["dim"], c["rows"] * c["kv_heads"] * c["dim"]
        tables = 4.0 * c["rows"] * c["rot"]
        return {"bytes": 4.0 * q + 4.0 * kv + kv * (2 if c["fp8"] else 4) + tables + 8.0 * c["rows"],
                "flops": 3.0 * c["rot"] * c["rows"] * (c["heads"] + c["kv_heads"])}
    if c["kind"] == "attend":
        tokens = sum(min(n, c["window"]) if c["window"] else n for n in _lengths(c))
        element = 1 if c["fp8"] else 2
        return {"bytes": 2.0 * tokens * c["kv_heads"] * c["dim"] * element + 4.0 * c["rows"] * c["heads"] * c["dim"] + 4.0 * c["rows"] * c["heads"]
                + 4.0 * (tokens // c["page"] + 2 * c["rows"]),
                "flops": 4.0 * tokens * c["heads"] * c["dim"]}
    element = 4 if c["f32"] else 2
    if c["kind"] == "logprobs":
        return {"bytes": float(c["rows"]) * (c["vocab"] * element + 16 + 8 * c["top"]), "flops": 5.0 * c["rows"] * c["vocab"]}
    return {"bytes": float(c["rows"]) * (2 * c["vocab"] * element + 20), "flops": 6.0 * c["rows"] * c["vocab"]}


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


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": c}
    bf16 = torch.bfloat16
    if c["kind"] == "append":
        seq, pos = _places(c)
        s |= _cache(c, [-(-c["most"] // c["page"])] * c["seqs"], gen)
        # queries, keys and values as the linears before leave them: side by side in one row per token
        both = torch.randn((c["rows"], (c["heads"] + 2 * c["kv_heads"]) * c["dim"]), device="cuda", generator=gen, dtype=bf16)
        q, kv = c["heads"] * c["dim"], c["kv_heads"] * c["dim"]
        s["q"] = both[:, :q].unflatten(1, (c["heads"], c["dim"]))
        s["k"] = both[:, q:q + kv].unflatten(1, (c["kv_heads"], c["dim"]))
        s["v"] = both[:, q + kv:].unflatten(1, (c["kv_heads"], c["dim"]))
        s["seq"], s["pos"] = _int32(seq), _int32(pos)
        angle = torch.outer(torch.arange(c["most"], device="cuda", dtype=torch.float64),
                            THETA ** (-torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64) / c["rot"]))
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["q_out"] = torch.empty((c["rows"], c["heads"], c["dim"]), device="cuda", dtype=bf16)
    elif c["kind"] == "attend":
        lens = _lengths(c)
        s |= _cache(c, [-(-n // c["page"]) for n in lens], gen)
        s["q"] = torch.randn((c["rows"], c["heads"], c["dim"]), device="cuda", generator=gen, dtype=bf16)
        s["lens"], s["most"], s["scale"] = _int32(lens), max(lens), c["dim"] ** -0.5
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((c["rows"], c["heads"]), device="cuda")
    else:
        x = torch.randn((c["rows"], c["stride"]), device="cuda", generator=gen) * LOGIT_STD
        if c.get("masked"):
            x.masked_fill_(torch.rand(x.shape, device="cuda", generator=gen) < c["masked"], -math.inf)
            x[:, 0] = 0.0                                       # (a word that is always allowed)
        s["logits"] = (x if c["f32"] else x.to(bf16))[:, :c["vocab"]]
        targets = torch.randint(0, c["vocab"], (c["rows"],), device="cuda", generator=gen, dtype=torch.int32)
        if c["ignored"]:
            targets[torch.rand(c["rows"], device="cuda", generator=gen) < c["ignored"]] = -100
        s["targets"] = targets
        if c["kind"] == "logprobs":
            s |= {n: torch.empty(c["rows"], device="cuda") for n in ("logp", "entropy", "lse")}
            s["top_logp"] = torch.empty((c["rows"], c["top"]), device="cuda") if c["top"] else None
            s["top_ids"] = torch.empty((c["rows"], c["top"]), device="cuda", dtype=torch.int32) if c["top"] else None
        else:
            # what the forward left behind, and the gradients that come from the loss
            y = s["logits"].float()
            s["lse"] = torch.logsumexp(y, 1)
            p = torch.exp(y - s["lse"][:, None])
            s["entropy"] = s["lse"] - (p * y).sum(1) if c["entropy"] else None
            s["d_logp"] = -(0.5 + torch.rand(c["rows"], device="cuda", generator=gen)) / c["rows"]
            s["d_entropy"] = 0.1 * torch.randn(c["rows"], device="cuda", generator=gen) / c["rows"] if c["entropy"] else None
            s["d_logits"] = torch.empty((c["rows"], c["stride"]), device="cuda", dtype=s["logits"].dtype)[:, :c["vocab"]]
    if own:
        from paper_2305_14152_amd import peqa
        if c["kind"] in ("append", "attend"):
            s["cache"] = peqa.kv_cache(s["k_pool"], s["v_pool"], s["table"], s["k_scale"], s["v_scale"])
        s["room"] = 0
        if c["kind"] == "attend":
            s["room"] = peqa.paged_attention_workspace_bytes(s["cache"], c["heads"], c["rows"], s["most"], c["window"])
        if c["kind"] == "logprobs":
            s["room"] = peqa.token_logprobs_workspace_bytes(c["rows"], c["vocab"], c["top"])
        s["ws"] = torch.zeros(max(s["room"], 16), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------

def _run_own(s):
    from paper_2305_14152_amd import peqa
    c = s["case"]
    if c["kind"] == "append":
        peqa.rope_append(s["cache"], s["q"], s["k"], s["v"], s["pos"], s["cos"], s["sin"], s["q_out"], seq=s["seq"], interleaved=c["interleaved"])
        return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}
    if c["kind"] == "attend":
        peqa.paged_attention(s["cache"], s["q"], s["lens"], s["most"], s["scale"], s["out"], s["ws"], s["room"], lse=s["lse"], window=c["window"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["kind"] == "logprobs":
        peqa.token_logprobs(s["logits"], s["targets"], s["logp"], s["entropy"], s["lse"], s["top_logp"], s["top_ids"], s["ws"], s["room"])
        return {n: s[n] for n in ("logp", "entropy", "lse", "top_logp", "top_ids")}
    peqa.token_logprobs_bwd(s["logits"], s["targets"], s["lse"], s["entropy"], s["d_logp"], s["d_entropy"], s["d_logits"])
    return {"d_logits": s["d_logits"]}


def _rotate(x, cos, sin, interleaved):
    """x [rows, heads, dim] in 32 bits, cos and sin [rows, 1, rot / 2]."""
    half = cos.shape[-1]
    r, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :half], r[..., half:])
    u, w = a * cos - b * sin, a * sin + b * cos
    r = torch.stack((u, w), -1).flatten(-2) if interleaved else torch.cat((u, w), -1)
    return torch.cat((r, rest), -1)


def _store(pool, x, page, slot, scale):
    """x [rows, kv_heads, dim] in 32 bits into the pool at (page, head, slot)."""
    if scale is not None:
        x = (x / scale[:, None]).clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        pool = pool.view(torch.uint8)
    pool[page, :, slot] = x.to(pool.dtype)


def _append(s):
    c = s["case"]
    pos = s["pos"].long()
    page, slot = s["table"][s["seq"].long(), pos // c["page"]].long(), pos % c["page"]
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]
    _store(s["k_pool"], _rotate(s["k"].float(), cos, sin, c["interleaved"]), page, slot, s["k_scale"])
    _store(s["v_pool"], s["v"].float(), page, slot, s["v_scale"])
    return {"q": _rotate(s["q"].float(), cos, sin, c["interleaved"]).to(torch.bfloat16), "k": s["k_pool"], "v": s["v_pool"]}


def _gather(pool, scale, table):
    """The pages of every row, [rows, kv_heads, positions, dim] in 32 bits."""
    x = (pool if scale is None else pool.view(torch.uint8))[table.long()].view(pool.dtype).float()
    if scale is not None:
        x = x * scale[:, None, None]
    return x.transpose(1, 2).flatten(2, 3)


def _attend(s):
    c = s["case"]
    rows, kv, dim = c["rows"], c["kv_heads"], c["dim"]
    k, v = _gather(s["k_pool"], s["k_scale"], s["table"]), _gather(s["v_pool"], s["v_scale"], s["table"])
    q = s["q"].float().view(rows, kv, c["heads"] // kv, dim)
    at, lens = torch.arange(k.shape[2], device="cuda"), s["lens"].long()[:, None]
    seen = at < lens
    if c["window"]:
        seen &= at >= lens - c["window"]
    scores = (torch.matmul(q, k.transpose(2, 3)) * s["scale"]).masked_fill(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_min(-3.0e38)     # (finite for rows without a position)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / total.clamp_min(1e-30)
    lse = torch.where(total > 0, top + total.log(), -math.inf)
    return {"out": out.view(rows, c["heads"], dim).to(torch.bfloat16), "lse": lse.view(rows, c["heads"])}


def _logprobs(s):
    c = s["case"]
    x = s["logits"].float()
    top = x.amax(1, keepdim=True)
    y = x - top
    e = torch.exp(y)
    total = e.sum(1)
    log = total.log()
    lse = top[:, 0] + log
    entropy = log - torch.where(e > 0, e * y, 0.0).sum(1) / total
    t = s["targets"].long()
    logp = torch.where(t >= 0, x.gather(1, t.clamp_min(0)[:, None])[:, 0] - lse, 0.0)
    out = {"logp": logp, "entropy": entropy, "lse": lse, "top_logp": None, "top_ids": None}
    if c["top"]:
        best, ids = torch.sort(x, dim=1, descending=True, stable=True)
        out["top_logp"], out["top_ids"] = best[:, :c["top"]] - lse[:, None], ids[:, :c["top"]].to(torch.int32)
    return out


def _logprobs_bwd(s):
    logp = s["logits"].float() - s["lse"][:, None]
    p = torch.exp(logp)
    t = s["targets"].long()
    g = torch.where(t >= 0, s["d_logp"], 0.0)[:, None]
    d = -g * p
    d.scatter_add_(1, t.clamp_min(0)[:, None], g)
    if s["d_entropy"] is not None:
        d = d - s["d_entropy"][:, None] * p * (logp + s["entropy"][:, None])
    return {"d_logits": d.to(s["logits"].dtype)}


def run(state):
    if own:
        return _run_own(state)
    return {"append": _append, "attend": _attend, "logprobs": _logprobs, "logprobs_bwd": _logprobs_bwd}[state["case"]["kind"]](state)


# ---- in 64 bits ---------------------------------------------------------------------------------------------------

def _exact_append(c, s):
    got = {}
    where = s["pos"].tolist()
    turn = torch.complex(s["cos"].double(), s["sin"].double())[where]           # [rows, rot / 2]
    for name in ("q", "k"):
        x = s[name].double().clone()
        for i in range(c["rot"] // 2):
            a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + c["rot"] // 2)
            z = torch.complex(x[..., a], x[..., b]) * turn[:, i, None]
            x[..., a], x[..., b] = z.real, z.imag
        got[name] = x
    got["v"] = s["v"].double()
    table = s["table"].tolist()
    page = [table[n][p // c["page"]] for n, p in zip(s["seq"].tolist(), where)]
    slot = [p % c["page"] for p in where]
    out = {"q": got["q"]}
    for name in ("k", "v"):
        pool = s[name + "_pool"].double()
        x = got[name]
        if c["fp8"]:
            x = (x / s[name + "_scale"].double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
        pool.permute(0, 2, 1, 3)[torch.tensor(page, device="cuda"), torch.tensor(slot, device="cuda")] = x
        out[name] = pool
    return out


def _exact_attend(c, s):
    rows, kv, heads = c["rows"], c["kv_heads"], c["heads"]
    out = torch.zeros((rows, heads, c["dim"]), device="cuda", dtype=torch.float64)
    lse = torch.full((rows, heads), -math.inf, device="cuda", dtype=torch.float64)
    for r, n in enumerate(s["lens"].tolist()):
        lo = max(0, n - c["window"]) if c["window"] else 0
        if n <= lo:
            continue
        pages = s["table"][r, :-(-n // c["page"])].long()
        for h in range(kv):
            k, v = (s[m].view(torch.uint8 if c["fp8"] else s[m].dtype)[pages, h].view(s[m].dtype).reshape(-1, c["dim"])[lo:n].float().double()
                    for m in ("k_pool", "v_pool"))
            if c["fp8"]:
                k, v = k * s["k_scale"][h].double(), v * s["v_scale"][h].double()
            members = slice(h * (heads // kv), (h + 1) * (heads // kv))
            z = (s["q"][r, members].double() @ k.T) * float(s["scale"])
            lse[r, members] = torch.logsumexp(z, 1)
            out[r, members] = torch.softmax(z, 1) @ v
    return {"out": out, "lse": lse}


def _exact_logprobs(c, s):
    x = s["logits"].double()
    log = torch.log_softmax(x, 1)
    p = log.exp()
    t = s["targets"].long()
    rows = torch.arange(c["rows"], device="cuda")
    out = {"logp": torch.where(t >= 0, log[rows, t.clamp_min(0)], 0.0), "entropy": -torch.special.xlogy(p, p).sum(1),
           "lse": torch.logsumexp(x, 1), "top_logp": None, "top_ids": None}
    if c["top"]:
        ids = torch.argsort(x, dim=1, descending=True, stable=True)[:, :c["top"]]
        out["top_logp"], out["top_ids"] = log.gather(1, ids), ids.to(torch.int32)
    return out


def _exact_logprobs_bwd(c, s):
    x = s["logits"].double()
    lse = s["lse"].double()[:, None]
    p = (x - lse).exp()
    t = s["targets"].long()
    hot = torch.zeros_like(p)
    live = t >= 0
    hot[live.nonzero()[:, 0], t[live]] = 1.0
    d = s["d_logp"].double()[:, None] * (hot - p) * live[:, None]
    if c["entropy"]:
        d = d - s["d_entropy"].double()[:, None] * p * (x - lse + s["entropy"].double()[:, None])
    return {"d_logits": d}


def exact(case, seed):
    """What run() returns for these inputs, from the definitions in 64 bits."""
    global own
    mode, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = mode
    return {"append": _exact_append, "attend": _exact_attend, "logprobs": _exact_logprobs, "logprobs_bwd": _exact_logprobs_bwd}[case["kind"]](case, s)

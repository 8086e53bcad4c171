"""The attention half of a decoder layer, as it is measured: rotary positions with the quantised cache's write, the
cache read back, attention over prompts, and attention of single tokens over the cache.

A case is one call that an inference engine makes for one layer, on inputs drawn from a seed: bf16 queries, keys and
values, a paged cache of e4m3 codes with one fp32 scale per token and head, page tables in the order an allocator
leaves them (shuffled), stale bytes in pages and slots that hold no token.

Kinds of case:

* ``rope``    rotate queries and keys, write keys and values into the cache (``moe_rope_cache``).
* ``read``    sequences' keys and values back from the cache as packed bf16 (``moe_cache_read``).
* ``prompt``  causal attention over packed prompts (``moe_attn_prefill``).
* ``step``    attention of one token per sequence over the cache, behind a prefix that all share or none
              (``moe_attn_decode``).

With ``own`` false the operators run in elementary torch operations in 32 bits, rounded once; ``exact`` states them in
64 bits, sequence by sequence.
"""
import math
import random

import torch

own = False

E4M3_MAX = 448.0
STALE = -1          # page table entries behind a sequence's last page
TABLE_ROWS = 32768  # positions that the rotary table covers


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # A decode step's batch: 16 new tokens, whole heads rotated. Latency.
        {"name": "rope_step_16", "kind": "rope", "tokens": 16, "q_heads": 32, "kv_heads": 8, "dim": 128, "rot": 128,
         "interleaved": False, "page": 64, "keep_k": False},
        # A prompt's chunk from one packed projection, half of each head rotated; rotated keys kept for the attention.
        {"name": "rope_prompt_8192", "kind": "rope", "tokens": 8192, "q_heads": 32, "kv_heads": 8, "dim": 128, "rot": 64,
         "interleaved": True, "page": 64, "keep_k": True},
        # A few short sequences read back, small heads.
        {"name": "read_short_301", "kind": "read", "batch": 3, "longest": 301, "kv_heads": 8, "dim": 64, "page": 16},
        # Long contexts read back for the next chunk of their prompts.
        {"name": "read_long_32768", "kind": "read", "batch": 4, "longest": 32768, "kv_heads": 8, "dim": 128, "page": 64},
        # The shortest prompt: latency; one head per group, small heads.
        {"name": "prompt_17", "kind": "prompt", "batch": 1, "longest": 17, "past": 0, "q_heads": 16, "kv_heads": 16,
         "dim": 64},
        # A prefill batch of packed prompts of different lengths.
        {"name": "prompt_packed_2048", "kind": "prompt", "batch": 8, "longest": 2048, "past": 0, "q_heads": 32,
         "kv_heads": 8, "dim": 128},
        # The last, odd chunk of a long prompt behind 8192 tokens already read.
        {"name": "prompt_chunk_509", "kind": "prompt", "batch": 1, "longest": 509, "past": 8192, "q_heads": 32,
         "kv_heads": 8, "dim": 128},
        # One long prompt at once.
        {"name": "prompt_long_16384", "kind": "prompt", "batch": 1, "longest": 16384, "past": 0, "q_heads": 32,
         "kv_heads": 8, "dim": 128},
        # Single-user decode, short context: latency.
        {"name": "step_1_255", "kind": "step", "batch": 1, "longest": 255, "prefix": 0, "q_heads": 32, "kv_heads": 8,
         "dim": 128, "page": 64},
        # Single-user decode, long context: few rows, one long axis.
        {"name": "step_1_65536", "kind": "step", "batch": 1, "longest": 65536, "prefix": 0, "q_heads": 32, "kv_heads": 8,
         "dim": 128, "page": 64},
        # A batched decode step over contexts of all lengths.
        {"name": "step_64_ragged_8192", "kind": "step", "batch": 64, "longest": 8192, "prefix": 0, "q_heads": 64,
         "kv_heads": 8, "dim": 128, "page": 64},
        # Users behind one long system prompt, each with a short conversation of its own.
        {"name": "step_48_prefix_8191", "kind": "step", "batch": 48, "longest": 512, "prefix": 8191, "q_heads": 32,
         "kv_heads": 8, "dim": 128, "page": 64},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


HEADS = ((32, 8, 128), (64, 8, 128), (16, 16, 64), (28, 4, 128), (24, 8, 64), (16, 1, 128), (40, 8, 128), (8, 8, 128))


def draw(rng):
    kind = rng.choice(("rope", "read", "prompt", "step"))
    hq, hkv, dim = rng.choice(HEADS)
    page = rng.choice((16, 32, 64, 128))
    if kind == "rope":
        return {"kind": kind, "tokens": min(_log(rng, 1, 8192), 8192 * 32 * 128 // (hq * dim)), "q_heads": hq,
                "kv_heads": hkv, "dim": dim, "rot": rng.choice((dim, dim // 2, dim // 4)),
                "interleaved": rng.random() < 0.5, "page": page, "keep_k": rng.random() < 0.5}
    if kind == "read":
        batch = _log(rng, 1, 32)
        most = 4 * 32768 // batch * 8 * 128 // (max(hkv, 8) * dim)
        return {"kind": kind, "batch": batch, "longest": _log(rng, 16, min(most, 65535)), "kv_heads": hkv, "dim": dim,
                "page": page}
    if kind == "prompt":
        batch = _log(rng, 1, 12)
        past = rng.choice((0, 0, _log(rng, 16, 8192)))
        most = min(8192, 12000 * 32 // max(hq, 32)) // batch  # the square of the packed tokens is what costs
        return {"kind": kind, "batch": batch, "longest": _log(rng, 16, max(16, most // (2 if past else 1))),
                "past": past // batch, "q_heads": hq, "kv_heads": hkv, "dim": dim}
    batch = _log(rng, 1, 64)
    prefix = rng.choice((0, 0, _log(rng, 16, 8192)))
    most = 8192 if batch > 8 else 65536 // batch
    return {"kind": kind, "batch": batch, "longest": _log(rng, 16, most if not prefix else max(32, most // 8)),
            "prefix": prefix, "q_heads": hq, "kv_heads": hkv, "dim": dim, "page": page}


def _lengths(case):
    """The sequences' lengths: one of the longest, the others spread below it, now and then an idle one of none."""
    n, longest = case["batch"], case["longest"]
    r = random.Random(1009 * n + longest)
    return [longest if i == n // 2 else int(longest * r.random() ** 1.5) for i in range(n)]


def work(case):
    kind, d, hkv = case["kind"], case["dim"], case["kv_heads"]
    if kind == "rope":
        t, hq = case["tokens"], case["q_heads"]
        moved = 2 * (2 * hq + 2 * hkv + (hkv if case["keep_k"] else 0)) * d + 2 * hkv * (d + 4) + 4 * case["rot"]
        return {"bytes": t * moved, "flops": t * 3 * (hq + hkv) * case["rot"]}
    lens = _lengths(case)
    total = sum(lens)
    if kind == "read":
        return {"bytes": 2 * total * hkv * (d + 4 + 2 * d), "flops": 2 * total * hkv * d}
    hq = case["q_heads"]
    if kind == "prompt":
        pairs = sum(n * case["past"] + n * (n + 1) // 2 for n in lens)
        keys = total + case["batch"] * case["past"]
        return {"bytes": 4 * d * (total * hq + keys * hkv), "flops": 4 * d * hq * pairs}
    b, p = case["batch"], case["prefix"]
    return {"bytes": 2 * (total + p) * hkv * (d + 4) + 4 * b * hq * d, "flops": 4 * d * hq * (total + b * p)}


# ----------------------------------------------------------------------------------------------- inputs
def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _keys(g, *shape):
    """Keys as projections give them: a few channels are many times the others'."""
    d = shape[-1]
    loud = 1.0 + 5.0 * (torch.rand(d, generator=g, device="cuda") < 0.04)
    return _normal(g, *shape) * loud


def _quantised(x):
    """e4m3 codes (as bytes) and one fp32 scale per last-axis row of fp32 `x`."""
    amax = x.abs().amax(-1)
    s = amax / torch.full_like(amax, E4M3_MAX)
    q = torch.where(s[..., None] > 0, x / s[..., None], x).clamp(-E4M3_MAX, E4M3_MAX)
    return q.to(torch.float8_e4m3fn).view(torch.uint8), s


def _pool(g, pages, hkv, page, d):
    """A cache's pages as a server has them: whatever was there before."""
    def codes():
        return torch.randint(0, 256, (pages, hkv, page, d), generator=g, device="cuda", dtype=torch.uint8)

    def scales():
        return _normal(g, pages, hkv, page).exp()
    return {"k": codes(), "v": codes(), "k_scale": scales(), "v_scale": scales()}


def _fill(g, pool, table, longest):
    """Keys and values of the tokens that the page table's rows hold (whole pages; the rest of the last is stale)."""
    page, d = pool["k"].shape[2:]
    hkv = pool["k"].shape[1]
    for row, n in zip(table, longest):
        full = row[:-(-n // page)].long()
        if not n:
            continue
        for name, make in (("k", _keys), ("v", _normal)):
            codes, s = _quantised(make(g, len(full), hkv, page, d))
            tail = n - (len(full) - 1) * page
            last = full[-1]
            keep_c, keep_s = pool[name][last, :, tail:].clone(), pool[name + "_scale"][last, :, tail:].clone()
            pool[name][full], pool[name + "_scale"][full] = codes, s
            pool[name][last, :, tail:], pool[name + "_scale"][last, :, tail:] = keep_c, keep_s


def _table(g, lens, page, spare=3):
    """Page tables of sequences of these lengths, pages in shuffled order; and how many pages there are."""
    need = [-(-n // page) for n in lens]
    order = torch.randperm(sum(need) + spare, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(max(need), 1)), STALE, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return table, sum(need) + spare


def _offsets(lens):
    return torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, d, hkv = case["kind"], case["dim"], case["kv_heads"]
    state = {"kind": kind, "case": dict(case)}
    if kind == "rope":
        t, hq, page = case["tokens"], case["q_heads"], case["page"]
        # queries, keys and values are one projection's output: rows of all heads
        row = torch.cat([_normal(g, t, hq, d), _keys(g, t, hkv, d), _normal(g, t, hkv, d)], 1).bfloat16()
        state.update(q=row[:, :hq], k=row[:, hq:hq + hkv], v=row[:, hq + hkv:])
        f = 10000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"]) / 4.0
        angle = torch.arange(TABLE_ROWS, device="cuda", dtype=torch.float64)[:, None] * f
        state["table"] = torch.cat([angle.cos(), angle.sin()], 1).float()  # one row per position: cosines, sines
        start = torch.randint(0, TABLE_ROWS - t + 1, (1,), generator=g, device="cuda")
        state["positions"] = (start + torch.arange(t, device="cuda")).to(torch.int32)
        pages = -(-t // page) + 3
        state["pool"] = _pool(g, pages, hkv, page, d)
        order = torch.randperm(pages, generator=g, device="cuda")
        at = torch.arange(t, device="cuda")
        state["slots"] = (order[at // page] * page + at % page).to(torch.int32)
        return state
    lens = _lengths(case)
    if kind == "prompt":
        hq, past = case["q_heads"], case["past"]
        n = sum(lens)
        keys = [x + past for x in lens]
        if past:
            state.update(q=_normal(g, n, hq, d).bfloat16(), k=_keys(g, sum(keys), hkv, d).bfloat16(),
                         v=_normal(g, sum(keys), hkv, d).bfloat16())
        else:
            row = torch.cat([_normal(g, n, hq, d), _keys(g, n, hkv, d), _normal(g, n, hkv, d)], 1).bfloat16()
            state.update(q=row[:, :hq], k=row[:, hq:hq + hkv], v=row[:, hq + hkv:])
        state.update(cu_q=_offsets(lens), cu_k=_offsets(keys), longest=max(keys))
        return state
    page = case["page"]
    rows = lens + ([case["prefix"]] if kind == "step" else [])
    table, pages = _table(g, rows, page)
    state["pool"] = _pool(g, pages, hkv, page, d)
    _fill(g, state["pool"], table, rows)
    widest = max(1, max(-(-n // page) for n in lens))
    state["pages"] = table[:len(lens), :widest].contiguous()
    state["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    state["longest"] = max(lens)
    if kind == "read":
        state.update(cu=_offsets(lens), total=sum(lens))
        return state
    state["q"] = _normal(g, len(lens), case["q_heads"], d).bfloat16()
    if case["prefix"]:
        state["prefix_pages"] = table[-1, :-(-case["prefix"] // page)].contiguous()
    return state


# ------------------------------------------------------------------------------------------ plain forms
def _rotated(x, cos, sin, interleaved):
    x = x.float()
    r = 2 * cos.shape[-1]
    cos, sin = cos[:, None], sin[:, None]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_rope(s):
    c = s["case"]
    row = s["table"][s["positions"].long()]
    cos, sin = row[:, :c["rot"] // 2], row[:, c["rot"] // 2:]
    q = _rotated(s["q"], cos, sin, c["interleaved"])
    k = _rotated(s["k"], cos, sin, c["interleaved"])
    pool, slot = s["pool"], s["slots"].long()
    page, at = slot // c["page"], slot % c["page"]
    pool["k"][page, :, at], pool["k_scale"][page, :, at] = _quantised(k)
    pool["v"][page, :, at], pool["v_scale"][page, :, at] = _quantised(s["v"].float())
    return {"q": q.bfloat16(), **({"k": k.bfloat16()} if c["keep_k"] else {}), "cache": _values_of(pool)}


def _values_of(pool):
    return {n: t.view(torch.float8_e4m3fn) if t.dtype == torch.uint8 else t for n, t in pool.items()}


def _gathered(pool, name, pages):
    """fp32 rows [N, heads, tokens, dim] of page table rows [N, P], every slot of every page."""
    at = pages.clamp(min=0).long()
    x = pool[name][at].view(torch.float8_e4m3fn).float() * pool[name + "_scale"][at][..., None]
    return x.transpose(1, 2).flatten(2, 3)


def _plain_read(s):
    lens = s["lens"].long()
    cu = s["cu"].long()
    row = torch.repeat_interleave(torch.arange(len(lens), device=lens.device), lens, output_size=s["total"])
    at = torch.arange(s["total"], device=lens.device) - cu[row]
    size = s["case"]["page"]
    page, at = s["pages"][row, at // size].long(), at % size
    pool = s["pool"]
    return {n: (pool[n][page, :, at].view(torch.float8_e4m3fn).float() * pool[n + "_scale"][page, :, at][..., None]).bfloat16()
            for n in ("k", "v")}


def _plain_prompt(s):
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    (tq, hq, d), (tk, hkv) = q.shape, k.shape[:2]
    cu_q, cu_k = s["cu_q"].long(), s["cu_k"].long()
    at_q, at_k = torch.arange(tq, device=q.device), torch.arange(tk, device=q.device)
    of_q, of_k = torch.bucketize(at_q, cu_q[1:], right=True), torch.bucketize(at_k, cu_k[1:], right=True)
    last = at_q - cu_q[of_q + 1] + cu_k[of_q + 1]  # the last key that a query sees: sequences end together
    hidden = (of_q[:, None] != of_k[None]) | (at_k[None] > last[:, None])
    grouped = q.view(tq, hkv, hq // hkv, d).permute(1, 2, 0, 3).reshape(hkv, -1, d)
    p = torch.matmul(grouped, k.permute(1, 2, 0).contiguous()).view(hkv, -1, tq, tk)
    p.mul_(1.0 / math.sqrt(d)).masked_fill_(hidden, -math.inf)
    p.sub_(p.amax(-1, keepdim=True)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(hkv, -1, tk), v.transpose(0, 1).contiguous()).view(hkv, -1, tq, d) / total
    return o.permute(2, 0, 1, 3).reshape(tq, hq, d).bfloat16()


def _plain_step(s):
    c = s["case"]
    b, hkv, d = c["batch"], c["kv_heads"], c["dim"]
    scale = 1.0 / math.sqrt(d)
    q = s["q"].float().view(b, hkv, -1, d)
    k, v = _gathered(s["pool"], "k", s["pages"]), _gathered(s["pool"], "v", s["pages"])
    there = (torch.arange(k.shape[2], device=q.device) < s["lens"][:, None])[:, None]
    v = torch.where(there[..., None], v, 0.0)
    scores = (torch.matmul(q, k.transpose(2, 3).contiguous()) * scale).masked_fill(~there[:, :, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    if c["prefix"]:
        # the shared rows' products once for all sequences: every sequence's queries are rows of one matrix
        pk, pv = (_gathered(s["pool"], n, s["prefix_pages"][None])[0, :, :c["prefix"]] for n in ("k", "v"))
        rows = q.transpose(0, 1).reshape(hkv, -1, d)
        shared = (torch.matmul(rows, pk.transpose(1, 2).contiguous()) * scale).view(hkv, b, -1, c["prefix"]).transpose(0, 1)
        top = torch.maximum(top, shared.amax(-1, keepdim=True))
    top = torch.where(top == -math.inf, 0.0, top)
    p = (scores - top).exp()
    total, o = p.sum(-1, keepdim=True), torch.matmul(p, v)
    if c["prefix"]:
        p = (shared - top).exp()
        total = total + p.sum(-1, keepdim=True)
        o = o + torch.matmul(p.transpose(0, 1).reshape(hkv, -1, c["prefix"]), pv).view(hkv, b, -1, d).transpose(0, 1)
    return torch.where(total > 0, o / total, 0.0).reshape(b, -1, d).bfloat16()


# -------------------------------------------------------------------------------- the framework's calls
def _own_buffers(s):
    """What a program that serves allocates once: the cache's handle, outputs, workspaces."""
    import paper_2606_10493_amd as moe
    c, kind = s["case"], s["kind"]
    dims = moe.MoeAttnDims(c.get("q_heads", c["kv_heads"]), c["kv_heads"], c["dim"])
    b = {"moe": moe, "dims": dims}
    if "pool" in s:
        p = s["pool"]
        b["cache"] = moe.KVCache(p["k"], p["v"], p["k_scale"], p["v_scale"])
    if kind == "read":
        shape = (s["total"], c["kv_heads"], c["dim"])
        b.update(k=torch.empty(shape, dtype=torch.bfloat16, device="cuda"),
                 v=torch.empty(shape, dtype=torch.bfloat16, device="cuda"))
        return b
    b["out"] = torch.empty(s["q"].shape, dtype=torch.bfloat16, device="cuda")
    if kind == "rope":
        b["layout"] = moe.MOE_ROPE_INTERLEAVED if c["interleaved"] else moe.MOE_ROPE_HALF
        b["k"] = torch.empty(s["k"].shape, dtype=torch.bfloat16, device="cuda") if c["keep_k"] else None
        return b
    need = (moe.moe_attn_prefill_workspace(dims, c["batch"], s["q"].shape[0], s["longest"]) if kind == "prompt" else
            moe.moe_attn_decode_workspace(dims, c["batch"], s["longest"], c["prefix"]))
    b["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    return b


def _own(s):
    b = s.get("own")
    if b is None:
        b = s["own"] = _own_buffers(s)
    moe, dims, kind = b["moe"], b["dims"], s["kind"]
    if kind == "rope":
        moe.moe_rope_cache(dims, s["q"], s["k"], s["v"], s["positions"], s["table"], b["layout"], s["slots"], b["cache"],
                           b["out"], b["k"])
        return {"q": b["out"], **({"k": b["k"]} if b["k"] is not None else {}), "cache": _values_of(s["pool"])}
    if kind == "read":
        moe.moe_cache_read(dims, b["cache"], s["pages"], s["cu"], b["k"], b["v"])
        return {"k": b["k"], "v": b["v"]}
    scale = 1.0 / math.sqrt(dims.head_dim)
    if kind == "prompt":
        moe.moe_attn_prefill(dims, s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], s["longest"], scale, b["out"], b["ws"])
    else:
        moe.moe_attn_decode(dims, s["q"], b["cache"], s["pages"], s["lens"], s["longest"], scale, b["out"], b["ws"],
                            prefix_pages=s.get("prefix_pages"), prefix_len=s["case"]["prefix"])
    return b["out"]


def run(state):
    if own:
        return _own(state)
    return {"rope": _plain_rope, "read": _plain_read, "prompt": _plain_prompt, "step": _plain_step}[state["kind"]](state)


# -------------------------------------------------------------------------------------------- in 64 bits
def _e4m3_steps():
    """All non-negative e4m3 values, from the format: 3 bits of mantissa, exponents from -6, subnormals below, 448."""
    return torch.tensor([m * 2.0 ** -9 for m in range(8)]
                        + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1],
                        dtype=torch.float64, device="cuda")


def _exact_quantised(x):
    """The nearest e4m3 values (ties to the even code) of x over max|x| / 448, and that scale, in 64 bits."""
    s = x.abs().amax(-1) / E4M3_MAX
    y = x / torch.where(s > 0, s, 1.0)[..., None]
    steps = _e4m3_steps()
    mid = (steps[1:] + steps[:-1]) / 2
    up, down = torch.bucketize(y.abs(), mid, right=True), torch.bucketize(y.abs(), mid)
    return torch.copysign(steps[torch.where(up % 2 == 0, up, down)], y), s


def _exact_rows(pool, name, row, n):
    """[heads, n, dim] of one page table row, in 64 bits."""
    page = pool[name].shape[2]
    at = row[:-(-n // page)].long()
    x = pool[name][at].view(torch.float8_e4m3fn).double() * pool[name + "_scale"][at].double()[..., None]
    return torch.cat(list(x), 1)[:, :n]


def _exact_attention(q, k, v, hidden=None):
    """q [heads, rows, dim] over k, v [heads, keys, dim]."""
    d = q.shape[-1]
    w = torch.matmul(q, k.mT.contiguous()) / d ** 0.5
    if hidden is not None:
        w = w.masked_fill(hidden, -math.inf)
    return torch.matmul(torch.softmax(w, -1), v)


def exact(case, seed):
    s = prepare(case, seed)
    kind, d, hkv = case["kind"], case["dim"], case["kv_heads"]
    if kind == "rope":
        half = case["rot"] // 2
        turn = s["table"][s["positions"].long()].double()
        turn = torch.complex(turn[:, :half], turn[:, half:])[:, None]

        def turned(x):
            x = x.double().clone()
            lo, hi = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else (slice(0, half), slice(half, 2 * half))
            z = torch.complex(x[..., lo].contiguous(), x[..., hi].contiguous()) * turn
            x[..., lo], x[..., hi] = z.real, z.imag
            return x
        k = turned(s["k"])
        out = {"q": turned(s["q"]), **({"k": k} if case["keep_k"] else {}), "cache": {}}
        pool = s["pool"]
        for name, x in (("k", k), ("v", s["v"].double())):
            held = pool[name].view(torch.float8_e4m3fn).double()
            scales = pool[name + "_scale"].double()
            slot = s["slots"].long()
            page, at = slot // case["page"], slot % case["page"]
            held[page, :, at], scales[page, :, at] = _exact_quantised(x)
            out["cache"][name], out["cache"][name + "_scale"] = held, scales
        return out
    lens = _lengths(case)
    pool = s.get("pool")
    if kind == "read":
        return {n: torch.cat([_exact_rows(pool, n, s["pages"][i], x).transpose(0, 1) if x else
                              torch.empty(0, hkv, d, dtype=torch.float64, device="cuda") for i, x in enumerate(lens)])
                for n in ("k", "v")}
    hq = case["q_heads"]
    g = hq // hkv
    if kind == "step":
        p = case["prefix"]
        front = {n: _exact_rows(pool, n, s["prefix_pages"], p) for n in ("k", "v")} if p else None
        out = torch.zeros(len(lens), hq, d, dtype=torch.float64, device="cuda")
        for i, n in enumerate(lens):
            parts = [[front[x]] if p else [] for x in ("k", "v")]
            if n:
                for part, x in zip(parts, ("k", "v")):
                    part.append(_exact_rows(pool, x, s["pages"][i], n))
            if n or p:
                k, v = (torch.cat(x, 1) for x in parts)
                out[i] = _exact_attention(s["q"][i].double().view(hkv, g, d), k, v).reshape(hq, d)
        return out
    out = torch.zeros(sum(lens), hq, d, dtype=torch.float64, device="cuda")
    past, at_q, at_k = case["past"], 0, 0
    for n in lens:
        for h in range(hkv):
            k, v = (s[x][at_k:at_k + n + past, h].double()[None] for x in ("k", "v"))
            for lo in range(0, n, 2048):
                rows = slice(at_q + lo, at_q + min(n, lo + 2048))
                i = torch.arange(lo, min(n, lo + 2048), device="cuda")
                hidden = torch.arange(n + past, device="cuda")[None] > past + i[:, None]
                q = s["q"][rows, h * g:(h + 1) * g].double().transpose(0, 1)
                out[rows, h * g:(h + 1) * g] = _exact_attention(q, k, v, hidden).transpose(0, 1)
        at_q, at_k = at_q + n, at_k + n + past
    return out

"""Timed cases of the paged cache: page tables, cache writes and attention of new tokens over it.

A case names an operator:

  append   pages and slots for the new tokens of a batch of sequences, from their lengths (`rf2_paged_append`)
  release  pages of finished sequences go back on the list of free ones (`rf2_paged_release`)
  store    rows of K and V go to their slots in the cache (`rf2_paged_store`)
  attn     the new tokens attend to the cache, their own rows included (`rf2_paged_attn`)

`run` computes a pass with plain torch operations, or, where `own` is true, makes the calls of a program that uses the
framework.  The lengths of a case's sequences follow from the case (`lens` is their seed), values and the order of the
pages from the seed of `prepare`.

The cache: with P tokens to a page, channel c of K of head h at slot s = page * P + r is element
    k_cache[page, h, r // 32, c // 8, r % 32, c % 8]
and of V, whose keys stand in groups of 16 in the order 0-3, 8-11, 4-7, 12-15,
    v_cache[page, h, r // 32, r % 32 // 16 * 2 + r % 8 // 4, c, r % 16 // 8 * 4 + r % 4].
"""
import math
import random

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}

DEFAULTS = dict(op="attn", seqs=1, heads=32, kv=8, d=128, page=64, dtype="bf16", causal=True, lse=False, fused_qkv=False,
                new_lo=1, new_hi=1, single=0.0, ctx_lo=0, ctx_hi=0, pad=0, evict=0.0, done=0.0, short=False, lens=1)


def _case(name, **over):
    return dict(DEFAULTS, name=name, **over)


def listed():
    return [
        # Tables of one step of a small batch, a token each: nothing but latency.
        _case("append_step", op="append", seqs=24, ctx_lo=100, ctx_hi=4000),
        # Tables of a large batch that takes in prompts of very different lengths.
        _case("append_prompts", op="append", seqs=256, page=32, new_lo=4, new_hi=2000, ctx_lo=20, ctx_hi=8000, pad=37, lens=2),
        # A few of a batch's sequences are finished.
        _case("release_few", op="release", seqs=32, ctx_lo=100, ctx_hi=4000, done=0.1, lens=3),
        # Half of a large batch is finished, with pages evicted from its tables before.
        _case("release_batch", op="release", seqs=512, page=32, ctx_lo=200, ctx_hi=16000, done=0.5, evict=0.2, lens=4),
        # K and V of one step's tokens, slices of a joint projection.
        _case("store_step", op="store", seqs=48, ctx_lo=100, ctx_hi=2000, fused_qkv=True, lens=5),
        # K and V of three new frames of a 480p video model, 30 x 52 tokens each, behind frames that are cached.
        _case("store_frames", op="store", heads=40, kv=40, new_lo=4680, new_hi=4680, ctx_lo=4690, ctx_hi=4690, fused_qkv=True),
        # The smallest attention: one token of one sequence over a short cache.
        _case("attn_one", heads=24, kv=24, d=64, page=32, ctx_lo=200, ctx_hi=200),
        # A step of a batch, a token each, four query heads to a K/V head.
        _case("attn_steps", seqs=64, ctx_lo=300, ctx_hi=9000, lens=6),
        # A step of few sequences with very long caches.
        _case("attn_steps_long", seqs=4, heads=40, kv=8, page=128, dtype="fp16", ctx_lo=20000, ctx_hi=110000, lse=True, lens=7),
        # Three new frames of a 480p video model attend to the 21 frames cached and to each other, all in both directions.
        _case("attn_frames", heads=40, kv=40, causal=False, new_lo=4680, new_hi=4680, ctx_lo=28080, ctx_hi=28080, fused_qkv=True),
        # Ragged chunks of prompts, each token over what stands before it.
        _case("attn_prompts", seqs=5, page=32, new_lo=300, new_hi=2600, ctx_lo=50, ctx_hi=6000, fused_qkv=True, lens=8),
        # One step that mixes single tokens with a chunk of a prompt, rows of padding behind them, a third of the older
        # pages evicted.
        _case("attn_mixed", seqs=16, heads=16, kv=4, d=64, page=128, dtype="fp16", new_lo=700, new_hi=700, single=0.9,
              ctx_lo=500, ctx_hi=6000, pad=5, evict=0.33, lse=True, lens=9),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    c = dict(DEFAULTS)
    c["op"] = rng.choices(["append", "release", "store", "attn"], [2, 1, 2, 5])[0]
    c["kv"] = rng.choice([1, 2, 4, 5, 8, 10, 24])
    c["heads"] = c["kv"] * rng.choice([1, 1, 2, 3, 4, 5, 8])
    c["d"] = rng.choice([128, 128, 64])
    c["page"] = rng.choice([32, 64, 64, 128, 256])
    c["dtype"] = rng.choice(["bf16", "bf16", "fp16"])
    c["causal"] = rng.random() < 0.7
    c["lse"] = rng.random() < 0.4
    c["fused_qkv"] = rng.random() < 0.5
    c["lens"] = rng.randrange(1 << 20)
    c["pad"] = rng.choice([0, 0, rng.randint(1, 300)])
    kind = rng.choice(["steps", "steps", "chunk", "prompts", "mixed"])
    c["seqs"] = 1 if kind == "chunk" else _log_uniform(rng, 1, 400 if c["op"] in ("append", "release") else 100)
    c["ctx_hi"] = _log_uniform(rng, 16, 60000 if c["seqs"] <= 8 else 9000)
    c["ctx_lo"] = rng.choice([0, c["ctx_hi"] // 8, c["ctx_hi"]])
    if kind != "steps":
        c["new_hi"] = _log_uniform(rng, 2, 4000 if kind == "chunk" else 1500)
        c["new_lo"] = rng.choice([c["new_hi"], max(1, c["new_hi"] // 20)])
    if kind == "mixed":
        c["single"] = 0.8
    if c["op"] in ("attn", "release"):
        c["evict"] = rng.choice([0.0, 0.0, 0.4])
    c["done"] = rng.choice([0.05, 0.3, 1.0]) if c["op"] == "release" else 0.0
    c["short"] = c["op"] == "append" and rng.random() < 0.15
    # no more than the largest listed cases cost: elements of the padded logits, of the padded cache and of the tables
    while _too_large(c):
        if c["seqs"] > 1:
            c["seqs"] = c["seqs"] // 2
        else:
            c["ctx_hi"], c["ctx_lo"] = c["ctx_hi"] // 2, c["ctx_lo"] // 2
            c["new_hi"], c["new_lo"] = max(1, c["new_hi"] // 2), max(1, c["new_lo"] // 2)
    return c


def _too_large(c):
    new, ctx = _lengths(c)
    longest = max(n + x for n, x in zip(new, ctx))
    tokens = sum(new) + sum(ctx)
    logits = c["seqs"] * max(new) * c["heads"] * longest if c["op"] == "attn" else 0
    return logits > 3e9 or c["seqs"] * longest * c["kv"] * c["d"] > 6e8 or tokens > 1.2e6


# ---- lengths, pages and inputs ------------------------------------------------------------------------------

def _lengths(c):
    """New and cached tokens of each sequence, as lists."""
    rng = random.Random(c["lens"])
    new, ctx = [], []
    for _ in range(c["seqs"]):
        one = rng.random() < c["single"]
        new.append(1 if one else _log_uniform(rng, c["new_lo"], c["new_hi"]))
        ctx.append(max(c["ctx_lo"], _log_uniform(rng, max(1, c["ctx_lo"]), c["ctx_hi"]) if c["ctx_hi"] else 0))
    if c["single"] and c["seqs"] > 1:
        new[rng.randrange(c["seqs"])] = c["new_hi"]        # a chunk there is
    return new, ctx


def _pages(c, tokens):
    return -(-tokens // c["page"])


def _evicted(c, ctx):
    """Pages evicted of each sequence: a run of whole cached pages behind the first one."""
    return [int(c["evict"] * max(0, x // c["page"] - 1)) for x in ctx]


def _row(c):
    """Row length of the block table."""
    new, ctx = _lengths(c)
    return max(_pages(c, n + x) for n, x in zip(new, ctx)) + 2


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    new, ctx = _lengths(c)
    cached = [n + x for n, x in zip(new, ctx)] if c["op"] in ("store", "attn") else ctx
    held = [_pages(c, x) for x in cached]
    need = sum(_pages(c, n + x) - _pages(c, x) for n, x in zip(new, ctx))
    n_pages = sum(held) + need + 7
    row = _row(c)
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    s = dict(case=c, new=new, ctx=ctx, n_pages=n_pages)

    # block table: sequence after sequence takes pages of the random order, what is left is the free list
    first = torch.tensor([sum(held[:i]) for i in range(c["seqs"])], device=DEV)[:, None]
    col, have = torch.arange(row, device=DEV)[None], _ints(held)[:, None]
    table = torch.where(col < have, order[(first + col).clamp(max=n_pages - 1)], -1)
    gone = _ints(_evicted(c, ctx))[:, None]
    table = torch.where((col >= 1) & (col < 1 + gone), -1, table)
    s["block_table"] = table.to(torch.int32).contiguous()
    s["free_pages"] = torch.cat([order[sum(held):], torch.full((sum(held),), -1, dtype=torch.int32, device=DEV)])
    left = n_pages - sum(held)
    s["n_free"] = _ints([max(0, need - 1) if c["short"] and need else left])
    s["seq_len"] = _ints(cached)
    s["new_len"] = _ints(new)
    total = s["total"] = sum(new)
    rows = s["rows"] = total + c["pad"]
    s["cu_new"] = _ints([sum(new[:i]) for i in range(c["seqs"] + 1)])
    if c["op"] == "release":
        rng = random.Random(c["lens"] + 1)
        done = [rng.random() < c["done"] for _ in range(c["seqs"])]
        s["done"] = torch.tensor(done, device=DEV)
    if c["op"] in ("append", "release"):
        s["seq_len_out"], s["n_free_out"] = torch.empty_like(s["seq_len"]), torch.empty_like(s["n_free"])
        s["cu_out"], s["slots_out"] = torch.empty_like(s["cu_new"]), _ints([0] * rows)
        s["status"] = _ints([0])
    else:
        t = TYPES[c["dtype"]]
        tiles = (n_pages, c["kv"], c["page"] // 32)
        s["k_cache"] = torch.randn(*tiles, c["d"] // 8, 32, 8, generator=gen, device=DEV, dtype=torch.float32).to(t)
        s["v_cache"] = torch.randn(*tiles, 4, c["d"], 8, generator=gen, device=DEV, dtype=torch.float32).to(t)
        # q, k and v of a layer: three tensors, or the parts of one projection's output
        parts = [c["heads"], c["kv"], c["kv"]]
        qkv = torch.randn(rows, sum(parts), c["d"], generator=gen, device=DEV).to(t)
        q, k, v = qkv.split(parts, 1)
        if not c["fused_qkv"]:
            q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        s["q"], s["k"], s["v"] = q, k, v
        if c["op"] == "store":
            at = torch.arange(total, device=DEV)
            seq = (at[:, None] >= s["cu_new"][None, 1:]).sum(1)
            pos = _ints(ctx)[seq] + at - s["cu_new"][seq]
            page = table[seq, pos // c["page"]]
            slots = page * c["page"] + pos % c["page"]
            s["slots"] = torch.cat([slots, torch.full((c["pad"],), -1, device=DEV)]).to(torch.int32)
        else:
            s["o"] = torch.zeros(rows, c["heads"], c["d"], dtype=t, device=DEV)
            s["lse"] = torch.zeros(rows, c["heads"], device=DEV) if c["lse"] else None
    if own:
        from paper_2512_24086_amd import rf2
        s["plan"] = rf2.PagedPlan(heads=c["heads"], kv_heads=c["kv"], head_dim=c["d"], page=c["page"], n_pages=n_pages,
                                  max_seqs=c["seqs"], max_pages=row, max_tokens=max(1, rows), dtype=TYPES[c["dtype"]],
                                  causal=c["causal"])
        s["workspace"] = s["plan"].alloc_workspace(DEV) if c["op"] == "attn" else None
    return s


# ---- the operators as plain torch operations ----------------------------------------------------------------

def _plain_append(s):
    c = s["case"]
    P, row, rows = c["page"], s["block_table"].shape[1], s["rows"]
    old, new, n_free, free = s["seq_len"], s["new_len"], s["n_free"], s["free_pages"]
    cu = torch.cat([torch.zeros_like(n_free), new.cumsum(0)])
    have, want = (old + P - 1) // P, (old + new + P - 1) // P
    base = torch.cat([torch.zeros_like(n_free), (want - have).cumsum(0)])
    bad = ((new < 0) | (old < 0) | (old > row * P)).any() | (n_free < 0) | (n_free > s["n_pages"])
    status = bad.int() + 2 * (want > row).any() + 4 * (cu[-1:] > rows) + 8 * (base[-1:] > n_free)
    fine = status == 0
    # table: columns `have` to `want` of a row are pages from the top of the free list
    col = torch.arange(row, device=DEV)[None]
    take = n_free - 1 - (base[:-1, None] + col - have[:, None])
    fresh = (col >= have[:, None]) & (col < want[:, None]) & fine
    table = torch.where(fresh, free[take.clamp(0, free.numel() - 1)], s["block_table"])
    s["block_table"].copy_(table)
    # slots: sequence of a token by comparison with the sums
    at = torch.arange(rows, device=DEV)
    seq = (at[:, None] >= cu[None, 1:]).sum(1).clamp(max=c["seqs"] - 1)
    pos = (old[seq] + at - cu[seq]).clamp(min=0, max=row * P - 1)
    slots = torch.where((at < cu[-1]) & fine, table[seq, pos // P] * P + pos % P, -1)
    return {"block_table": s["block_table"], "seq_len": torch.where(fine, old + new, old).int(), "cu_new": (cu * fine).int(),
            "n_free": torch.where(fine, n_free - base[-1:], n_free).int(), "slots": slots.int(), "status": status.int()}


def _plain_release(s):
    c = s["case"]
    P, row = c["page"], s["block_table"].shape[1]
    old, n_free, free = s["seq_len"], s["n_free"], s["free_pages"]
    col = torch.arange(row, device=DEV)[None]
    back = (s["done"][:, None] & (col < ((old + P - 1) // P)[:, None]) & (s["block_table"] >= 0)).flatten()
    rank = back.cumsum(0)
    status = (rank[-1:] + n_free > s["n_pages"]).int()
    fine = status == 0
    # the place of every page that goes back; the others write their own value to where they are (behind the list: a spare place)
    to = torch.where(back & fine, n_free + rank - 1, free.numel())
    wide = torch.cat([free, free[:1]])
    wide[to] = s["block_table"].flatten()
    s["free_pages"].copy_(wide[:-1])
    return {"free_pages": s["free_pages"], "seq_len": torch.where(s["done"] & fine, 0, old).int(),
            "n_free": (n_free + rank[-1:] * fine).int(), "status": status}


def _plain_store(s):
    c = s["case"]
    P, n = c["page"], s["total"]
    slot = s["slots"][:n].long()
    page, r = slot // P, slot % P
    k, v = s["k"][:n], s["v"][:n]
    s["k_cache"][page, :, r // 32, :, r % 32] = k.reshape(n, c["kv"], c["d"] // 8, 8)
    s["v_cache"][page, :, r // 32, r % 32 // 16 * 2 + r % 8 // 4, :, r % 16 // 8 * 4 + r % 4] = v
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attn(s):
    c = s["case"]
    P, B, d, kv, G = c["page"], c["seqs"], c["d"], c["kv"], c["heads"] // c["kv"]
    M, L = max(s["new"]), max(n + x for n, x in zip(s["new"], s["ctx"]))
    # K and V of every sequence, padded to the longest: [B, kv, L, d]
    pos = torch.arange(L, device=DEV)
    page, r = s["block_table"][:, pos // P].long(), pos % P
    there = (page >= 0) & (pos < s["seq_len"][:, None])
    page = page.clamp(min=0)
    k = s["k_cache"][page, :, r // 32, :, r % 32].float().view(B, L, kv, d).transpose(1, 2)
    v = s["v_cache"][page, :, r // 32, r % 32 // 16 * 2 + r % 8 // 4, :, r % 16 // 8 * 4 + r % 4].float().transpose(1, 2)
    v = torch.where(there[:, None, :, None], v, 0.0)
    # the new tokens, padded to the most: [B, kv, M * G, d]
    t = torch.arange(M, device=DEV)
    live = t < s["new_len"][:, None]
    at = (s["cu_new"][:-1, None] + t)[live]
    q = torch.zeros(B, M, c["heads"], d, device=DEV)
    q[live] = s["q"][at].float()
    q = q.view(B, M, kv, G, d).transpose(1, 2).reshape(B, kv, M * G, d)
    x = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    x = x.view(B, kv, M, G, L)
    sees = there[:, None].expand(B, M, L)
    if c["causal"]:
        sees = sees & (pos < (s["seq_len"] - s["new_len"] + 1)[:, None, None] + t[:, None])
    x.masked_fill_(~sees[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, kv, M * G, L), v).view(B, kv, M, G, d) / torch.where(total == 0, 1.0, total)
    s["o"][at] = o.transpose(1, 2).reshape(B, M, c["heads"], d)[live].to(s["o"].dtype)
    if s["lse"] is None:
        return {"o": s["o"]}
    lse = (top + total.log()).transpose(1, 2).reshape(B, M, c["heads"])
    s["lse"][at] = lse[live]
    return {"o": s["o"], "lse": s["lse"]}


# ---- one pass -----------------------------------------------------------------------------------------------

def run(state):
    s = state
    op = s["case"]["op"]
    if not own:
        return {"append": _plain_append, "release": _plain_release, "store": _plain_store, "attn": _plain_attn}[op](s)
    plan = s["plan"]
    if op == "append":
        plan.rf2_paged_append(s["seq_len"], s["new_len"], s["free_pages"], s["n_free"], s["block_table"], s["seq_len_out"],
                              s["n_free_out"], s["cu_out"], s["slots_out"], s["status"])
        return {"block_table": s["block_table"], "seq_len": s["seq_len_out"], "cu_new": s["cu_out"], "n_free": s["n_free_out"],
                "slots": s["slots_out"], "status": s["status"]}
    if op == "release":
        plan.rf2_paged_release(s["done"], s["seq_len"], s["block_table"], s["free_pages"], s["n_free"], s["seq_len_out"],
                               s["n_free_out"], s["status"])
        return {"free_pages": s["free_pages"], "seq_len": s["seq_len_out"], "n_free": s["n_free_out"], "status": s["status"]}
    if op == "store":
        plan.rf2_paged_store(s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    plan.rf2_paged_attn(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["seq_len"], s["cu_new"], s["workspace"], s["o"],
                        s["lse"])
    return {"o": s["o"]} if s["lse"] is None else {"o": s["o"], "lse": s["lse"]}


# ---- what a pass cannot do without --------------------------------------------------------------------------

def work(case):
    c = case
    new, ctx = _lengths(c)
    total, row_bytes = sum(new), 2 * c["kv"] * c["d"] * 2
    if c["op"] == "append":
        need = 0 if c["short"] else sum(_pages(c, n + x) - _pages(c, x) for n, x in zip(new, ctx))
        return {"bytes": 4.0 * (4 * c["seqs"] + total + c["pad"] + 2 * need + c["seqs"] + 4), "flops": 0}
    if c["op"] == "release":
        rng = random.Random(c["lens"] + 1)
        pages = sum(_pages(c, x) for x in ctx if rng.random() < c["done"])
        return {"bytes": 4.0 * (2 * c["seqs"] + 2 * pages + 3) + c["seqs"], "flops": 0}
    if c["op"] == "store":
        return {"bytes": total * (2.0 * row_bytes + 4), "flops": 0}
    gone = [e * c["page"] for e in _evicted(c, ctx)]
    keys = sum(n + x - e for n, x, e in zip(new, ctx, gone))
    pairs = sum(n * (x - e) + (n * (n + 1) // 2 if c["causal"] else n * n) for n, x, e in zip(new, ctx, gone))
    out = total * c["heads"] * (c["d"] * 4 + (4 if c["lse"] else 0))
    entries = 4 * sum(_pages(c, n + x) for n, x in zip(new, ctx))
    return {"bytes": float(keys * row_bytes + out + entries), "flops": 4.0 * pairs * c["heads"] * c["d"]}


# ---- the definition, in 64 bits -----------------------------------------------------------------------------

def exact(case, seed):
    c = case
    if c["op"] in ("append", "release"):
        return None                     # whole numbers
    s = prepare(dict(c), seed)
    P, d, G = c["page"], c["d"], c["heads"] // c["kv"]
    r = torch.arange(P, device=DEV)
    # keys of a page in order, from the tiles: [32, ...] of K, and the storage order of V
    order = [(key // 16 * 2 + key % 8 // 4, key % 16 // 8 * 4 + key % 4) for key in range(32)]
    if c["op"] == "store":
        k, v = s["k_cache"].double(), s["v_cache"].double()
        slots = s["slots"].tolist()
        for group in range(32):         # the tokens of one place in a tile at a time
            at = [n for n, slot in enumerate(slots) if slot >= 0 and slot % 32 == group]
            if not at:
                continue
            page = torch.tensor([slots[n] // P for n in at], device=DEV)
            tile = torch.tensor([slots[n] % P // 32 for n in at], device=DEV)
            rows_k, rows_v = (s[x][torch.tensor(at, device=DEV)].double() for x in ("k", "v"))
            k[page, :, tile, :, group] = torch.stack(rows_k.split(8, 2), 2)
            g, e = order[group]
            v[page, :, tile, g, :, e] = rows_v
        return {"k_cache": k, "v_cache": v}
    o = torch.zeros(s["rows"], c["heads"], d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["rows"], c["heads"], dtype=torch.float64, device=DEV)
    g_of, e_of = (torch.tensor([x[i] for x in order], device=DEV) for i in (0, 1))
    start = 0
    for i, (n, x) in enumerate(zip(s["new"], s["ctx"])):
        length = n + x
        pages = s["block_table"][i, :_pages(c, length)].long()
        key = torch.arange(pages.numel() * P, device=DEV)
        kept = ((pages >= 0).repeat_interleave(P) & (key < length)).nonzero()[:, 0]
        mine = pages[kept // P]
        inside = r[kept % P]
        limit = torch.arange(x + 1, length + 1, device=DEV) if c["causal"] else torch.full((n,), length, device=DEV)
        seen = kept[None] < limit[:, None]
        for h in range(c["kv"]):
            k = s["k_cache"][mine, h, inside // 32, :, inside % 32].double().flatten(1)
            v = s["v_cache"][mine, h, inside // 32, g_of[inside % 32], :, e_of[inside % 32]].double()
            for g in range(G):
                q = s["q"][start:start + n, h * G + g].double()
                logits = (q @ k.t().contiguous() / math.sqrt(d)).masked_fill(~seen, -math.inf)
                sums = torch.logsumexp(logits, 1)
                p = torch.where(seen, torch.exp(logits - sums[:, None].clamp(min=-1e300)), 0.0)
                o[start:start + n, h * G + g] = p @ v
                lse[start:start + n, h * G + g] = sums
        start += n
    return {"o": o, "lse": lse} if c["lse"] else {"o": o}

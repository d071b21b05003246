"""Plain forms of the paged cache's operators, for its tests (no test cases here): tables by loops over tokens, attention in
64 bits from rows of K and V that stand beside the cache."""
import math

import numpy as np
import torch

BAD_LENGTH, SEQ_FULL, TOKENS_FULL, POOL_FULL = 1, 2, 4, 8


def ceil_div(a, b):
    return -(-a // b)


def append(seq_len, new_len, free_pages, n_free, table, n_tokens, page, n_pages):
    """(table, seq_len, n_free, cu_new, slots, status) as lists and arrays; the table given is not changed."""
    table, row = table.copy(), table.shape[1]
    status = 0
    if any(n < 0 for n in new_len) or any(not 0 <= x <= row * page for x in seq_len) or not 0 <= n_free <= n_pages:
        status |= BAD_LENGTH
    good = [(x, n) for x, n in zip(seq_len, new_len) if n >= 0 and 0 <= x <= row * page]
    if any(x + n > row * page for x, n in good):
        status |= SEQ_FULL
    if sum(n for _, n in good) > n_tokens:
        status |= TOKENS_FULL
    if sum(ceil_div(x + n, page) - ceil_div(x, page) for x, n in good) > n_free:
        status |= POOL_FULL
    slots = [-1] * n_tokens
    if status:
        return table, list(seq_len), n_free, [0] * (len(seq_len) + 1), slots, status
    cu, top = [0], n_free
    for s, (x, n) in enumerate(zip(seq_len, new_len)):
        for i in range(ceil_div(x, page), ceil_div(x + n, page)):
            top -= 1
            table[s, i] = free_pages[top]
        for t in range(n):
            p = table[s, (x + t) // page]
            if 0 <= p < n_pages:
                slots[cu[-1] + t] = int(p) * page + (x + t) % page
        cu.append(cu[-1] + n)
    return table, [x + n for x, n in zip(seq_len, new_len)], top, cu, slots, 0


def release(done, seq_len, table, free_pages, n_free, page, n_pages):
    """(free_pages, seq_len, n_free, status)."""
    row = table.shape[1]
    if any(not 0 <= x <= row * page for x in seq_len) or not 0 <= n_free <= n_pages:
        return list(free_pages), list(seq_len), n_free, BAD_LENGTH
    back = [int(p) for s, x in enumerate(seq_len) if done[s] for p in table[s, :ceil_div(x, page)] if 0 <= p < n_pages]
    if n_free + len(back) > n_pages:
        return list(free_pages), list(seq_len), n_free, POOL_FULL
    out = list(free_pages)
    out[n_free:n_free + len(back)] = back
    return out, [0 if d else x for d, x in zip(done, seq_len)], n_free + len(back), 0


def put(cache_k, cache_v, slots, k, v, page):
    """Rows of K and V ([n, kv, d]) to their slots, element by element of the header's formulas."""
    for n, slot in enumerate(slots):
        if slot < 0:
            continue
        P, r = slot // page, slot % page
        cache_k[P, :, r // 32, :, r % 32] = k[n].reshape(k.shape[1], -1, 8)
        cache_v[P, :, r // 32, r % 32 // 16 * 2 + r % 8 // 4, :, r % 16 // 8 * 4 + r % 4] = v[n]


def put_many(cache_k, cache_v, slots, k, v, page):
    """The same for a tensor of valid slots at once."""
    P, r = slots // page, slots % page
    cache_k[P, :, r // 32, :, r % 32] = k.reshape(*k.shape[:2], -1, 8)
    cache_v[P, :, r // 32, r % 32 // 16 * 2 + r % 8 // 4, :, r % 16 // 8 * 4 + r % 4] = v


def attention(q, k, v, kept, n_new, causal, scale, eps_half):
    """One sequence: q [n, heads, d], k and v [len, kv, d], kept [len] (False: in a hole).  Returns o, lse and how far a kernel
    may be off that rounds probabilities and results to a type of half step `eps_half` and sums in fp32.

    A probability is off by eps_half of itself when it is rounded, so o by eps_half * sum p |v|, and by eps_half * |o| when o
    is rounded.  A logit, a sum of d products in fp32, is off by at most d 2^-24 sum |q k| scale (plus 2^-20 for the
    exponent's own arithmetic: logits below 8 in size, two roundings, and an exponential good to 2^-22), a probability by as
    much of itself, numerator and denominator alike: twice that.  The sums of up to 2^17 terms in fp32 add 2^-16: blocks of
    at most 2^12 units a lane, each sum rounded by 2^-24 of a partial sum no larger than the whole."""
    n, heads, d = q.shape
    length, kv = k.shape[0], k.shape[1]
    G = heads // kv
    q, k, v = q.double(), k.double(), v.double()
    o = torch.zeros(n, heads, d, dtype=torch.float64, device=q.device)
    lse = torch.full((n, heads), -math.inf, dtype=torch.float64, device=q.device)
    tol, lse_tol = torch.zeros_like(o), torch.zeros_like(lse)
    limit = torch.arange(n, device=q.device) + (length - n_new + 1) if causal else torch.full((n,), length, device=q.device)
    sees = kept[None] & (torch.arange(length, device=q.device)[None] < limit[:, None])
    any_key = sees.any(1)
    for h in range(heads):
        kh, vh = k[:, h // G], v[:, h // G]
        vh = torch.where(kept[:, None], vh, 0.0)
        x = (q[:, h] @ kh.t().contiguous()) * scale
        x = torch.where(sees, x, -math.inf)
        top = torch.where(any_key, x.amax(1), 0.0) if length else torch.zeros(n, dtype=torch.float64, device=q.device)
        p = torch.exp(x - top[:, None])
        total = torch.where(any_key, p.sum(1), 1.0)
        p = p / total[:, None]
        o[:, h] = p @ vh
        lse[:, h] = torch.where(any_key, top + total.log(), -math.inf)
        sizes = torch.where(kept[:, None], kh, 0.0).abs()
        off = d * 2.0 ** -24 * (torch.where(sees, (q[:, h].abs() @ sizes.t().contiguous()) * scale, 0.0).amax(1) if length
                                else torch.zeros(n, dtype=torch.float64, device=q.device)) + 2.0 ** -20
        spread = p @ vh.abs()
        tol[:, h] = eps_half * (o[:, h].abs() + spread) * (1 + 2.0 ** -6) + (2 * off[:, None] + 2.0 ** -16) * spread + 1e-30
        lse_tol[:, h] = off + 2.0 ** -16 + 2.0 ** -23 * lse[:, h].abs().clamp(max=1e30)
    return o, lse, tol, lse_tol


class Batch:
    """A batch of sequences with its cache.  Pages stand in a random order; what no token has stays as `fill` (NaN)."""

    def __init__(self, *, new, ctx, heads, kv, d, page, dtype=torch.bfloat16, seed=0, device="cuda", holes=(), extra_pages=3,
                 extra_row=1, fill=float("nan"), q_scale=1.0, pad=0, fused=False):
        gen = torch.Generator(device="cpu")
        gen.manual_seed(seed)
        self.new, self.ctx, self.heads, self.kv, self.d, self.page, self.dtype = list(new), list(ctx), heads, kv, d, page, dtype
        self.len = [n + x for n, x in zip(new, ctx)]
        held = [ceil_div(x, page) for x in self.len]
        self.n_pages = sum(held) + extra_pages
        self.row = max(held + [1]) + extra_row
        order = torch.randperm(self.n_pages, generator=gen).tolist()
        table = np.full((len(new), self.row), -1, dtype=np.int32)
        at = 0
        for s, n in enumerate(held):
            table[s, :n] = order[at:at + n]
            at += n
        shape = (self.n_pages, kv, page // 32)
        k_cache = torch.full((*shape, d // 8, 32, 8), fill, dtype=dtype)
        v_cache = torch.full((*shape, 4, d, 8), fill, dtype=dtype)
        self.k = [torch.randn(x, kv, d, generator=gen).to(dtype) for x in self.len]
        self.v = [torch.randn(x, kv, d, generator=gen).to(dtype) for x in self.len]
        for s, x in enumerate(self.len):
            pos = torch.arange(x)
            slots = torch.from_numpy(table[s])[pos // page].long() * page + pos % page
            if x:
                put_many(k_cache, v_cache, slots, self.k[s], self.v[s], page)
        self.kept = [torch.ones(x, dtype=torch.bool) for x in self.len]
        for s, p, mark in holes:             # column p of row s is no page
            table[s, p] = mark
            self.kept[s][p * page:(p + 1) * page] = False
        total = sum(new)
        rows = total + pad
        qkv = torch.randn(rows, heads + (2 * kv if fused else 0), d, generator=gen) * q_scale
        self.qkv = qkv.to(dtype).to(device)
        self.q = self.qkv[:, :heads]
        self.total, self.rows = total, rows
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.cu = torch.from_numpy(cu).to(device)
        self.table = torch.from_numpy(table).to(device)
        self.seq_len = torch.tensor(self.len, dtype=torch.int32, device=device)
        self.k_cache, self.v_cache = k_cache.to(device), v_cache.to(device)
        self.device = device

    def plan(self, causal=True, scale=None, **over):
        from paper_2512_24086_amd import rf2
        args = dict(heads=self.heads, kv_heads=self.kv, head_dim=self.d, page=self.page, n_pages=self.n_pages,
                    max_seqs=len(self.new), max_pages=self.row, max_tokens=max(1, self.rows), dtype=self.dtype, causal=causal, scale=scale)
        args.update(over)
        return rf2.PagedPlan(**args)

    def run(self, plan, with_lse=True, stream=None):
        o = torch.full((self.rows, self.heads, self.d), 7.0, dtype=self.dtype, device=self.device)
        lse = torch.full((self.rows, self.heads), 7.0, device=self.device) if with_lse else None
        plan.rf2_paged_attn(self.q, self.k_cache, self.v_cache, self.table, self.seq_len, self.cu, plan.alloc_workspace(self.device), o,
                            lse, stream)
        return o, lse

    def check(self, o, lse, causal=True, scale=None):
        """Every row against the definition; rows of padding are as they were.  Returns the largest share of the tolerance used."""
        scale = scale if scale is not None else 1.0 / math.sqrt(self.d)
        half = torch.finfo(self.dtype).eps / 2
        worst, at = 0.0, 0
        for s, n in enumerate(self.new):
            dev = [x.to(self.device) for x in (self.k[s], self.v[s], self.kept[s])]
            want, want_lse, tol, lse_tol = attention(self.q[at:at + n], *dev, n, causal, scale, half)
            got = o[at:at + n].double()
            if n:
                share = ((got - want).abs() / tol).max().item()
                assert share <= 1.0, (s, share)
                worst = max(worst, share)
                if lse is not None:
                    got_lse = lse[at:at + n].double()
                    none = torch.isinf(want_lse)
                    assert torch.equal(none, torch.isinf(got_lse)) and (got_lse[none] < 0).all(), s
                    assert ((got_lse - want_lse).abs()[~none] <= lse_tol[~none]).all(), (s, (got_lse - want_lse)[~none].abs().max())
            at += n
        assert (o[at:] == 7.0).all() and (lse is None or (lse[at:] == 7.0).all()), "rows of padding were written"
        return worst

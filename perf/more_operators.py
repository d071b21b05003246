"""Timed cases of what is done to Q and K before attention: norms of each head's rows and rotation by positions of several axes.

A case names an operator:

  rope      Q and K rotated by their tokens' positions (`rf2_rope_apply`, a plan without a norm)
  norm      rows of each head normalised, weighted and rotated in one pass (`rf2_rope_apply`)
  backward  gradients of Q, K and the weights of the norm (`rf2_rope_backward`)
  permute   window permutation and block means of a layer, Q and K normalised and rotated on the way (`rf2_permute_rope`)
  store     new tokens of a paged cache: Q normalised and rotated, K too and into the cache, V into the cache (`rf2_paged_store_rope`)

`run` computes a pass with plain torch operations, or, where `own` is true, makes the calls of a program that uses the
framework.

A row x of d channels of one head of token n, with weights w: y = x w / sqrt(mean(x^2) + eps).  Pair i of its d / 2 pairs (channels 2i and
2i + 1, or i and i + d/2) turns by the angle pos[n, a] f: the first dim_0 / 2 pairs belong to axis 0, the next dim_1 / 2 to axis 1, ...; the
j-th pair of axis a has f = theta^(-2j / dim_a).  Pairs behind the last axis stay.
"""
import math
import random

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32}
EPS = 1e-6

# Tokens: T x H x W of a grid (axes 3, 2: time, height, width or height, width), or T of packed sequences (axes 1), `text` behind them.
DEFAULTS = dict(op="norm", batch=1, T=1, H=1, W=1, text=0, heads=8, kv=8, d=128, layout="bnhd", joint=False, dtype="bf16",
                weights="bf16", halves=False, axes=3, dim0=44, dim1=42, dim2=42, theta=10000.0, first=0, runs=1, own_pos=False, block=128,
                block_k=0, sink=0, page=64, pad=0, lens=1)


def _case(name, **over):
    return dict(DEFAULTS, name=name, **over)


def listed():
    text = dict(axes=1, dim0=128, dim1=0, dim2=0, halves=True, theta=1e6)
    return [
        # The smallest call: one token of a text model, rotation alone.
        _case("rope_token", op="rope", heads=8, kv=2, d=64, axes=1, dim0=64, dim1=0, dim2=0, halves=True, first=900),
        # Q and K of a 480p video layer, normalised by the model's own code before.
        _case("rope_video480p", op="rope", T=21, H=30, W=52, heads=40, kv=40, layout="bhnd"),
        # One step of a batch: a token each, slices of a joint projection, positions far into their sequences.
        _case("norm_step", T=48, runs=48, heads=32, kv=8, joint=True, first=100000, **text),
        # A layer of a small image model.
        _case("norm_image", H=64, W=64, heads=10, kv=10, joint=True, axes=2, dim0=64, dim1=64),
        # Prompts packed one behind the other, an odd number of tokens, four query heads to a K/V head.
        _case("norm_prompts", T=8191, runs=7, heads=32, kv=8, dtype="fp16", weights="f32", joint=True, lens=2, **text),
        # The headline layer: 720p video, 40 heads.
        _case("norm_video720p", T=21, H=45, W=80, heads=40, kv=40, layout="bhnd"),
        # Training on short clips: two of them, odd sizes.
        _case("backward_clips", op="backward", batch=2, T=5, H=17, W=13, heads=16, kv=4, d=64, dtype="fp16", weights="f32",
              axes=3, dim0=16, dim1=24, dim2=24, own_pos=True),
        # Training of a 480p video layer.
        _case("backward_video480p", op="backward", T=21, H=30, W=52, heads=40, kv=40),
        # The layer's first call: an image with text behind it, norms of the text's own.
        _case("permute_image", op="permute", H=64, W=64, text=205, heads=12, kv=12, layout="bnhd", dim0=16, dim1=56, dim2=56),
        # The same of the headline layer.
        _case("permute_video720p", op="permute", T=21, H=45, W=80, heads=40, kv=40, layout="bhnd", sink=1),
        # Serving: a step's tokens into the cache, with rows of padding behind them.
        _case("store_step", op="store", T=48, runs=48, heads=32, kv=8, joint=True, first=100000, pad=16, **text),
        # Serving: three new frames of a 480p video model.
        _case("store_frames", op="store", T=3, H=30, W=52, heads=40, kv=40, joint=True, first=18),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _tokens(c):
    return c["T"] * c["H"] * c["W"] + c["text"]


def draw(rng):
    c = dict(DEFAULTS)
    c["op"] = rng.choices(["rope", "norm", "backward", "permute", "store"], [2, 3, 3, 2, 2])[0]
    permute, store = c["op"] == "permute", c["op"] == "store"
    c["d"] = rng.choice([128, 128, 64])
    c["kv"] = rng.choice([1, 2, 3, 5, 8, 10, 12, 40])
    c["heads"] = c["kv"] * (1 if permute or c["kv"] == 40 else rng.choice([1, 1, 2, 3, 4, 8]))
    c["dtype"] = "bf16" if permute else rng.choice(["bf16", "bf16", "fp16"])
    c["weights"] = rng.choice([c["dtype"], c["dtype"], "f32"])
    c["layout"] = "bnhd" if store else rng.choice(["bnhd", "bhnd"])
    c["joint"] = c["layout"] == "bnhd" and not permute and rng.random() < 0.6
    c["batch"] = 1 if store else rng.choice([1, 1, 2, 3])
    c["halves"] = rng.random() < 0.4
    c["theta"] = rng.choice([100.0, 10000.0, 500000.0, 1e6])
    c["axes"] = rng.choice([2, 3]) if permute else rng.choice([1, 2, 3, 3])
    # even parts of the channels to each axis, all of them or a few fewer
    whole = c["d"] - rng.choice([0, 0, 0, 8, c["d"] // 2])
    cuts = sorted(rng.sample(range(1, whole // 2), c["axes"] - 1))
    parts = [2 * (b - a) for a, b in zip([0] + cuts, cuts + [whole // 2])] + [0, 0]
    c["dim0"], c["dim1"], c["dim2"] = parts[:3]
    if c["axes"] == 1:
        c["T"] = _log_uniform(rng, 1, 20000)
        if store and rng.random() < 0.5:
            c["T"] = min(c["T"], 64)        # a step, a token each
            c["runs"] = c["T"]
        else:
            c["runs"] = rng.choice([1, 1 if store else c["T"], max(1, c["T"] // 700)])
        c["first"] = rng.choice([0, _log_uniform(rng, 1, 1000000)])
    else:
        c["T"] = 1 if c["axes"] == 2 else _log_uniform(rng, 1, 24)
        c["H"], c["W"] = _log_uniform(rng, 2, 80), _log_uniform(rng, 2, 80)
        c["first"] = rng.choice([0, rng.randint(1, 400)])
        c["text"] = 0 if store else rng.choice([0, 0, rng.randint(1, 300)])
    c["own_pos"] = c["batch"] > 1 and not permute and rng.random() < 0.5
    if permute:
        c["block"], c["block_k"] = rng.choice([(64, 0), (128, 0), (128, 64), (64, 128), (256, 128)])
        c["sink"] = 1 if c["T"] > 2 and rng.random() < 0.5 else 0
    if store:
        c["page"] = rng.choice([32, 64, 128, 256])
        c["pad"] = rng.choice([0, 0, rng.randint(1, 100)])
    c["lens"] = rng.randrange(1 << 20)
    most = 2048 * min(c["block"], c["block_k"] or c["block"]) if permute else 1 << 20          # (of a layer)
    while c["batch"] * _tokens(c) * (c["heads"] + 2 * c["kv"]) * c["d"] > 6e8 or _tokens(c) > most:
        side = max("THW", key=lambda x: c[x])
        c[side] = (c[side] + 1) // 2
        c["runs"] = min(c["runs"], c["T"])
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------

def _axes(c):
    return [c["dim0"], c["dim1"], c["dim2"]][:c["axes"]]


def _positions(c):
    """[batch, tokens, axes] int32, or [tokens, axes] where the batch shares them."""
    n = c["T"] * c["H"] * c["W"]
    at = torch.arange(n, device=DEV)
    if c["axes"] == 1:
        # sequences one behind the other, each from its own place on
        rng = random.Random(c["lens"])
        starts = sorted([0] + rng.sample(range(1, n), c["runs"] - 1))
        begins = torch.tensor([rng.randint(c["first"] // 2, c["first"]) - s for s in starts], device=DEV)
        run_of = torch.bucketize(at, torch.tensor(starts, device=DEV), right=True) - 1
        pos = (at + begins[run_of])[:, None]
    else:
        t, h, w = at // (c["H"] * c["W"]) + c["first"], at // c["W"] % c["H"] - c["H"] // 2, at % c["W"] - c["W"] // 2
        pos = torch.stack([t, h, w][3 - c["axes"]:], 1)
        # text behind the grid: on the diagonal
        more = torch.arange(c["text"], device=DEV) + max(c["T"] + c["first"], c["H"], c["W"])
        pos = torch.cat([pos, more[:, None].expand(-1, c["axes"])])
    if c["own_pos"]:
        pos = torch.stack([pos + 3 * b for b in range(c["batch"])])
    return pos.to(torch.int32).contiguous()


def _order(c):
    """Tokens in window order: windows of the frames behind the sink's, window by window, then the sink's frames, then the text."""
    shapes = {256: (4, 8, 8), 128: (2, 8, 8), 64: (4, 4, 4)} if c["T"] > 1 else {256: (1, 16, 16), 128: (1, 8, 16), 64: (1, 8, 8)}
    wt, wh, ww = shapes[c["block"]]
    n = c["T"] * c["H"] * c["W"]
    at = torch.arange(n, device=DEV)
    t, h, w = at // (c["H"] * c["W"]), at // c["W"] % c["H"], at % c["W"]
    sink = t < c["sink"]
    slab = torch.where(sink, t + c["T"], (t - c["sink"]) // wt)
    window = (slab * c["H"] + h // wh) * c["W"] + w // ww
    return torch.cat([torch.argsort(window * n + at), torch.arange(n, n + c["text"], device=DEV)])


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    t, wt = TYPES[c["dtype"]], TYPES[c["weights"]]
    B, N, d = c["batch"], _tokens(c) + c["pad"], c["d"]
    parts = [c["heads"], c["kv"], c["kv"]]

    def rows(heads):
        # channels of different size, as projections have them
        size = torch.rand(heads, 1, d, generator=gen, device=DEV) * 2 + 0.3
        x = (torch.randn(B, heads, N, d, generator=gen, device=DEV) * size).to(t)
        return x if c["layout"] == "bhnd" else x.transpose(1, 2).contiguous()

    def weight():
        return (1 + 0.3 * torch.randn(d, generator=gen, device=DEV)).to(wt)

    s = dict(case=c)
    if c["joint"]:
        s["q"], s["k"], s["v"] = rows(sum(parts)).split(parts, 2)
    else:
        s["q"], s["k"] = rows(c["heads"]), rows(c["kv"])
        if c["op"] in ("permute", "store"):
            s["v"] = rows(c["kv"])
    s["pos"] = _positions(c)
    if c["pad"]:
        s["pos"] = torch.cat([s["pos"], torch.zeros(c["pad"], c["axes"], dtype=torch.int32, device=DEV)])
    # each pair's axis, and its frequency
    axis = sum([[a] * (dim // 2) for a, dim in enumerate(_axes(c))], [])
    freq = sum([[c["theta"] ** (-2.0 * j / dim) for j in range(dim // 2)] for dim in _axes(c)], [])
    more = d // 2 - len(axis)
    s["axis"] = torch.tensor(axis + [0] * more, device=DEV)
    s["freq"] = torch.tensor(freq + [0.0] * more, dtype=torch.float64, device=DEV)
    names = [] if c["op"] == "rope" else ["wq", "wk", "wq_text", "wk_text"] if c["text"] and c["op"] == "permute" else ["wq", "wk"]
    for name in ("wq", "wk", "wq_text", "wk_text"):
        s[name] = weight() if name in names else None
    if c["op"] in ("rope", "norm"):
        s["q_out"], s["k_out"] = (torch.empty(x.shape, dtype=t, device=DEV) for x in (s["q"], s["k"]))
    elif c["op"] == "backward":
        s["dq_out"], s["dk_out"] = rows(c["heads"]), rows(c["kv"])
        s["dq"], s["dk"] = (torch.empty(x.shape, dtype=t, device=DEV) for x in (s["q"], s["k"]))
        s["dwq"], s["dwk"] = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    elif c["op"] == "permute":
        s["order"] = _order(c)
        b = s["block_k"] = c["block_k"] or c["block"]
        tq, tk = -(-N // c["block"]), -(-N // b)
        s["qp"] = torch.empty(B, c["heads"], tq * c["block"], d, dtype=t, device=DEV)
        s["kp"] = torch.empty(B, c["heads"], tk, b // 64, d // 8, 64, 8, dtype=t, device=DEV)
        s["vp"] = torch.empty(B, c["heads"], tk, b // 64, 8, d, 8, dtype=t, device=DEV)
        s["qbar"], s["kbar"] = torch.empty(B, c["heads"], tq, d, device=DEV), torch.empty(B, c["heads"], tk, d, device=DEV)
    else:
        # slots of the tokens: a run in pages of any order, or a page of its own for each sequence
        P, n = c["page"], _tokens(c)
        alone = c["runs"] == n
        n_pages = n + 3 if alone else -(-(n + P) // P) + 3
        order = torch.randperm(n_pages, generator=gen, device=DEV)
        at = torch.arange(n, device=DEV) + P // 3
        slots = order[at - P // 3] * P + at * 7 % P if alone else order[at // P] * P + at % P
        s["slots"] = torch.cat([slots, torch.full((c["pad"],), -1, device=DEV)]).to(torch.int32)
        s["cu_new"] = torch.tensor([0, n], dtype=torch.int32, device=DEV)
        tiles = (n_pages, c["kv"], P // 32)
        s["k_cache"] = torch.randn(*tiles, d // 8, 32, 8, generator=gen, device=DEV).to(t)
        s["v_cache"] = torch.randn(*tiles, 4, d, 8, generator=gen, device=DEV).to(t)
        s["q"], s["k"], s["v"] = s["q"][0], s["k"][0], s["v"][0]
        s["q_out"] = torch.zeros(N, c["heads"], d, dtype=t, device=DEV)
    if own:
        from paper_2512_24086_amd import rf2
        s["rope"] = rf2.RopePlan(heads=c["heads"], kv_heads=c["kv"], head_dim=d, axis_dims=_axes(c), theta=c["theta"],
                                 pairing=rf2.RF2_ROPE_HALVES if c["halves"] else rf2.RF2_ROPE_PAIRS,
                                 norm=rf2.RF2_NORM_NONE if c["op"] == "rope" else rf2.RF2_NORM_RMS, eps=EPS, dtype=t, weight_dtype=wt,
                                 layout=rf2.RF2_LAYOUT_BHND if c["layout"] == "bhnd" else rf2.RF2_LAYOUT_BNHD)
        if c["op"] == "backward":
            s["workspace"] = s["rope"].alloc_workspace(DEV)
        elif c["op"] == "permute":
            s["plan"] = rf2.Plan(batch=B, heads=c["heads"], head_dim=d, T=c["T"], H=c["H"], W=c["W"], block=c["block"], sparsity=0.8,
                                 sink_frames=c["sink"], text_tokens=c["text"], block_k=c["block_k"],
                                 qkv_layout=rf2.RF2_LAYOUT_BHND if c["layout"] == "bhnd" else rf2.RF2_LAYOUT_BNHD)
        elif c["op"] == "store":
            s["plan"] = rf2.PagedPlan(heads=c["heads"], kv_heads=c["kv"], head_dim=d, page=c["page"], n_pages=n_pages, max_seqs=1,
                                      max_pages=n_pages, max_tokens=N, dtype=t)
    return s


# ---- the operators as plain torch operations --------------------------------------------------------------------

def _angles(s):
    """Cosine and sine of each token's pairs, [batch or 1, 1, tokens, d/2] or [batch or 1, tokens, 1, d/2] as the rows lie."""
    phi = s["pos"].double()[..., s["axis"]] * s["freq"]
    phi = phi if phi.dim() == 3 else phi[None]
    phi = phi.unsqueeze(1 if s["case"]["layout"] == "bhnd" else 2)
    return phi.cos().float(), phi.sin().float()


def _turn(s, x, cos, sin):
    if s["case"]["halves"]:
        u, v = x.chunk(2, -1)
        return torch.cat([u * cos - v * sin, v * cos + u * sin], -1)
    u, v = x[..., 0::2], x[..., 1::2]
    return torch.stack([u * cos - v * sin, v * cos + u * sin], -1).flatten(-2)


def _forward(s, x, w, cos, sin):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
    return _turn(s, x, cos, sin)


def _plain_apply(s):
    cos, sin = _angles(s)
    return {"q": _forward(s, s["q"], s["wq"], cos, sin).to(s["q"].dtype), "k": _forward(s, s["k"], s["wk"], cos, sin).to(s["k"].dtype)}


def _gradient(s, x, w, dz, cos, sin):
    g = _turn(s, dz.float(), cos, -sin)
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    x = x * r
    dw = (g * x).sum((0, 1, 2), dtype=torch.float64).float()
    g = g * w.float()
    return (r * (g - x * (g * x).mean(-1, keepdim=True))).to(dz.dtype), dw


def _plain_backward(s):
    cos, sin = _angles(s)
    dq, dwq = _gradient(s, s["q"], s["wq"], s["dq_out"], cos, sin)
    dk, dwk = _gradient(s, s["k"], s["wk"], s["dk_out"], cos, sin)
    return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


def _blocks(s, x, b):
    """Rows [batch, heads, tokens, d] in window order, cut into blocks of b, zeros behind the last: [batch, heads, blocks, b, d]."""
    x = x[:, :, s["order"]]
    n = x.shape[2]
    return torch.nn.functional.pad(x, (0, 0, 0, -n % b)).unflatten(2, (-1, b))


def _means(x, n):
    b = x.shape[3]
    count = (n - torch.arange(x.shape[2], device=DEV) * b).clamp(max=b)
    return x.sum(3) / count[:, None]


def _plain_permute(s):
    c = s["case"]
    b, d, n, video = s["block_k"], c["d"], _tokens(c), c["T"] * c["H"] * c["W"]
    cos, sin = _angles(s)
    heads_first = (lambda x: x) if c["layout"] == "bhnd" else (lambda x: x.transpose(1, 2))
    text = (torch.arange(n, device=DEV) >= video)[:, None]

    def weights(w, of_text):
        w = w.float()
        if of_text is not None:
            w = torch.where(text, of_text.float(), w)
            w = w[None] if c["layout"] == "bhnd" else w[:, None]
        return w

    q = _blocks(s, heads_first(_forward(s, s["q"], weights(s["wq"], s["wq_text"]), cos, sin)), c["block"])
    k = _blocks(s, heads_first(_forward(s, s["k"], weights(s["wk"], s["wk_text"]), cos, sin)), b)
    v = _blocks(s, heads_first(s["v"]), b)
    qbar, kbar = _means(q, n), _means(k, n)
    # K: row r of a block is (half, part, 32 rows); tiles [part][d/8][half, 32][8]
    kp = k.unflatten(3, (2, b // 64, 32)).unflatten(6, (d // 8, 8)).permute(0, 1, 2, 4, 6, 3, 5, 7).to(s["k"].dtype)
    # V: keys of a group of 16 in the order 0-3, 8-11, 4-7, 12-15, then (half, part, 4 chunks, 8 keys); tiles [part][half, 4][d][8]
    v = v.unflatten(3, (b // 16, 2, 2, 4)).transpose(4, 5).flatten(3, 6).unflatten(3, (2, b // 64, 4, 8))
    vp = v.permute(0, 1, 2, 4, 3, 5, 7, 6)
    return {"qp": q.flatten(2, 3).to(s["q"].dtype).contiguous(), "kp": kp.contiguous().view(s["kp"].shape),
            "vp": vp.contiguous().view(s["vp"].shape), "qbar": qbar, "kbar": kbar}


def _plain_store(s):
    c = s["case"]
    P, n, d = c["page"], _tokens(c), c["d"]
    cos, sin = (x[0, :n] for x in _angles(s))
    s["q_out"][:n] = _forward(s, s["q"][:n], s["wq"], cos, sin).to(s["q"].dtype)
    k = _forward(s, s["k"][:n], s["wk"], cos, sin).to(s["k"].dtype)
    slot = s["slots"][:n].long()
    page, r = slot // P, slot % P
    s["k_cache"][page, :, r // 32, :, r % 32] = k.reshape(n, c["kv"], d // 8, 8)
    s["v_cache"][page, :, r // 32, r % 32 // 16 * 2 + r % 8 // 4, :, r % 16 // 8 * 4 + r % 4] = s["v"][:n]
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


# ---- one pass ---------------------------------------------------------------------------------------------------

def run(state):
    s = state
    op = s["case"]["op"]
    if not own:
        return {"rope": _plain_apply, "norm": _plain_apply, "backward": _plain_backward, "permute": _plain_permute,
                "store": _plain_store}[op](s)
    rope = s["rope"]
    if op in ("rope", "norm"):
        rope.rf2_rope_apply(s["q"], s["k"], s["pos"], s["q_out"], s["k_out"], s["wq"], s["wk"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "backward":
        rope.rf2_rope_backward(s["q"], s["k"], s["pos"], s["dq_out"], s["dk_out"], s["dq"], s["dk"], s["wq"], s["wk"], s["dwq"], s["dwk"],
                               s["workspace"])
        return {"dq": s["dq"], "dk": s["dk"], "dwq": s["dwq"], "dwk": s["dwk"]}
    if op == "permute":
        s["plan"].rf2_permute_rope(rope, s["q"], s["k"], s["v"], s["pos"], s["qp"], s["kp"], s["vp"], s["qbar"], s["kbar"], s["wq"], s["wk"],
                                   s["wq_text"], s["wk_text"])
        return {"qp": s["qp"], "kp": s["kp"], "vp": s["vp"], "qbar": s["qbar"], "kbar": s["kbar"]}
    s["plan"].rf2_paged_store_rope(rope, s["q"], s["k"], s["v"], s["pos"], s["slots"], s["k_cache"], s["v_cache"], s["q_out"], s["wq"], s["wk"],
                                   s["cu_new"])
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    c = case
    n, h = c["batch"] * _tokens(c), c["heads"] + c["kv"]
    rows = 2.0 * n * h * c["d"]                       # bytes of Q and K
    pos = 4.0 * _tokens(c) * c["axes"] * (c["batch"] if c["own_pos"] else 1)
    turn, norm = 3.0 * n * h * c["d"], 4.0 * n * h * c["d"]
    if c["op"] == "rope":
        return {"bytes": 2 * rows + pos, "flops": turn}
    if c["op"] == "norm":
        return {"bytes": 2 * rows + pos, "flops": turn + norm}
    if c["op"] == "backward":
        return {"bytes": 3 * rows + pos + 16 * c["d"], "flops": turn + 3 * norm}
    v = 2.0 * n * c["kv"] * c["d"]
    if c["op"] == "store":
        return {"bytes": 2 * (rows + v) + pos + 4.0 * n, "flops": turn + norm}
    b, bk = c["block"], c["block_k"] or c["block"]
    tq, tk = -(-_tokens(c) // b), -(-_tokens(c) // bk)
    out = c["batch"] * c["heads"] * c["d"] * (2.0 * (tq * b + 2 * tk * bk) + 4.0 * (tq + tk))
    return {"bytes": rows + v + out + pos, "flops": turn + norm + n * h * c["d"]}


# ---- the definition, in 64 bits -----------------------------------------------------------------------------------

def _unit(s, b):
    """e^(i phi) of the tokens of one element of the batch, [tokens, d/2]."""
    pos = s["pos"] if s["pos"].dim() == 2 else s["pos"][b]
    phi = torch.empty(pos.shape[0], s["freq"].numel(), dtype=torch.float64, device=DEV)
    for i, (a, f) in enumerate(zip(s["axis"].tolist(), s["freq"].tolist())):
        phi[:, i] = pos[:, a].double() * f
    return torch.polar(torch.ones_like(phi), phi)


def _as_complex(x, halves):
    half = x.shape[-1] // 2
    return torch.complex(x[:, :half], x[:, half:]) if halves else torch.view_as_complex(x.reshape(-1, half, 2))


def _as_real(z, halves):
    return torch.cat([z.real, z.imag], 1) if halves else torch.view_as_real(z).flatten(1)


def _exact_rows(x, w, unit, halves):
    """Rows of one head, [tokens, d], in 64 bits; w: [d] or [tokens, d]."""
    x = x.double()
    if w is not None:
        x = x / (x.pow(2).sum(1, keepdim=True) / x.shape[1] + EPS).sqrt() * w.double()
    return _as_real(_as_complex(x, halves) * unit, halves)


def _exact_order(c):
    """The window order, window by window."""
    depth = {64: 4, 128: 2, 256: 4}[c["block"]]
    wt, wh, ww = (depth,) + ((4, 4) if c["block"] == 64 else (8, 8))
    if c["T"] == 1:
        wt, wh, ww = 1, {64: 8, 128: 8, 256: 16}[c["block"]], {64: 8, 128: 16, 256: 16}[c["block"]]
    order = []
    for begin, end, step in ((c["sink"], c["T"], wt), (0, c["sink"], 1)):
        for t0 in range(begin, end, step):
            for h0 in range(0, c["H"], wh):
                for w0 in range(0, c["W"], ww):
                    order += [(t * c["H"] + h) * c["W"] + w for t in range(t0, min(t0 + step, end))
                              for h in range(h0, min(h0 + wh, c["H"])) for w in range(w0, min(w0 + ww, c["W"]))]
    n = len(order)
    return torch.tensor(order + list(range(n, n + c["text"])), device=DEV)


def exact(case, seed):
    c = case
    s = prepare(dict(c), seed)
    B, d, halves = c["batch"], c["d"], c["halves"]
    first = c["layout"] == "bhnd"

    def of(x, b, h):
        return x[b, h] if first else x[b, :, h]

    if c["op"] in ("rope", "norm", "backward"):
        out = {}
        for name, heads in (("q", c["heads"]), ("k", c["kv"])):
            x, w = s[name], s["w" + name]
            z = torch.empty(x.shape, dtype=torch.float64, device=DEV)
            dw = torch.zeros(d, dtype=torch.float64, device=DEV)
            for b in range(B):
                unit = _unit(s, b)
                for h in range(heads):
                    if c["op"] != "backward":
                        of(z, b, h).copy_(_exact_rows(of(x, b, h), w, unit, halves))
                        continue
                    # dz / dx by the chain rule, with the norm n = sqrt(mean(x^2) + eps): d(x/n) = dx / n - x (x . dx) / (d n^3)
                    row = of(x, b, h).double()
                    back = _as_real(_as_complex(of(s[f"d{name}_out"], b, h).double(), halves) * unit.conj(), halves)
                    n = (row.pow(2).sum(1, keepdim=True) / d + EPS).sqrt()
                    dw += (back * row / n).sum(0)
                    back = back * w.double()
                    of(z, b, h).copy_(back / n - row * (row * back).sum(1, keepdim=True) / (d * n ** 3))
            out["d" + name if c["op"] == "backward" else name] = z
            if c["op"] == "backward":
                out["dw" + name] = dw
        return {k: out[k] for k in (("dq", "dk", "dwq", "dwk") if c["op"] == "backward" else ("q", "k"))}

    if c["op"] == "store":
        n, P = _tokens(c), c["page"]
        unit = _unit(s, 0)[:n]
        q = torch.zeros(s["q_out"].shape, dtype=torch.float64, device=DEV)
        for h in range(c["heads"]):
            q[:n, h] = _exact_rows(s["q"][:n, h], s["wq"], unit, halves)
        k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
        slots = s["slots"].tolist()
        for key in range(32):           # the tokens of one place in a tile at a time
            at = [i for i, slot in enumerate(slots) if slot >= 0 and slot % 32 == key]
            if not at:
                continue
            page = torch.tensor([slots[i] // P for i in at], device=DEV)
            tile = torch.tensor([slots[i] % P // 32 for i in at], device=DEV)
            at = torch.tensor(at, device=DEV)
            place = [0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15].index(key % 16) + key // 16 * 16
            for h in range(c["kv"]):
                k_cache[page, h, tile, :, key] = _exact_rows(s["k"][at, h], s["wk"], unit[at], halves).view(-1, d // 8, 8)
                v_cache[page, h, tile, place // 8, :, place % 8] = s["v"][at, h].double()
        return {"q": q, "k_cache": k_cache, "v_cache": v_cache}

    order, video = _exact_order(c), c["T"] * c["H"] * c["W"]
    n, b_k = _tokens(c), c["block_k"] or c["block"]
    out = {x: torch.zeros(s[x].shape, dtype=torch.float64, device=DEV) for x in ("qp", "kp", "vp", "qbar", "kbar")}
    r = torch.arange(n, device=DEV)
    blk, row, half = r // b_k, r % b_k, b_k // 2
    place = torch.tensor([0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15], device=DEV)[row % 16] + row // 16 * 16
    for b in range(B):
        unit = _unit(s, b)
        for h in range(c["heads"]):
            z = {}
            for x in ("q", "k"):
                w, wt = s["w" + x], s[f"w{x}_text"]
                if wt is not None:
                    w = torch.cat([w.double()[None].expand(video, d), wt.double()[None].expand(n - video, d)])
                z[x] = _exact_rows(of(s[x], b, h), w, unit, halves)[order]
            out["qp"][b, h, :n] = z["q"]
            out["kp"][b, h, blk, row % half // 32, :, row // half * 32 + row % 32] = z["k"].view(n, d // 8, 8)
            out["vp"][b, h, blk, place % half // 32, place // half * 4 + place % 32 // 8, :, place % 8] = of(s["v"], b, h).double()[order]
            for x, size in (("q", c["block"]), ("k", b_k)):
                padded = torch.cat([z[x], z[x].new_zeros(-n % size, d)]).view(-1, size, d).sum(1)
                padded[:-1] /= size
                padded[-1] /= n - (padded.shape[0] - 1) * size
                out[x + "bar"][b, h] = padded
    return out

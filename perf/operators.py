"""The operators for packed requests and their plain forms: attention, block norms and adapted projections.

A program that serves many requests on one backbone puts their rows behind one another: views of different sizes, tokens of
different streams.  Three operators work on such rows, with an engine or without one:

  attention       softmax(score) V for every sequence of a packed batch, its keys beside it or in a longer cache; scores may be
                  capped (c tanh(s / c)), lowered by distance (in a line, or on a grid of patches) and masked (causal, with a
                  prefix that everybody sees)
  block_norm      what stands between two blocks: norm of the branch, gate of the request, LayerScale, residual sum, norm of
                  the sum and its modulation by the request
  adapter_linear  one projection for all rows, beside it the low-rank adapter of each row's request

`run` computes them with elementary torch operations in 32 bits, or, with `own`, makes the framework's calls.  Widths and
heads are those of the ViT-S, ViT-B, ViT-L and ViT-g backbones of `vpe_inputs` and `bench.py`, or generic.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _attention(name, q, k, heads, kv_heads, head_dim, dtype="bf16", cache=0, causal=False, prefix="", cap=0.0, bias="", grid=0):
    """q, k: rows of every sequence.  cache: rows that each sequence's keys may take (0: keys are packed too).  prefix: per
    sequence, how many first keys everybody sees.  bias: "line" or "grid" (grid: patches in a row of it)."""
    c = dict(kind="attention", q=q, k=k, heads=heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, cache=cache, causal=causal,
             prefix=prefix, cap=cap, bias=bias, grid=grid)
    return dict(c, name=name) if name else c


def _norm(name, rows, width, requests, dtype="bf16", post="layer", pre="layer", alpha=1.0):
    """post, pre: "layer", "rms" or "none" for the norm of the branch and of the sum.  requests 0: no gates and modulation."""
    c = dict(kind="norm", rows=rows, width=width, requests=requests, dtype=dtype, post=post, pre=pre, alpha=alpha)
    return dict(c, name=name) if name else c


def _adapters(name, rows, k, n, rank, adapters, dtype="bf16", mixed=False, bias=True):
    """mixed: every row has an adapter of its own choice (tokens of many streams); else rows of a request lie together."""
    c = dict(kind="adapters", rows=rows, k=k, n=n, rank=rank, adapters=adapters, dtype=dtype, mixed=mixed, bias=bias)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one learned query reads one 476 x 630 view of a ViT-S: the smallest call of a head that pools by attention
        _attention("pool_one_view", "1", "1531", 6, 6, 64),
        # single tokens of 24 streams against their caches, 16384 rows reserved for each
        _attention("tokens_cached", ",".join(["1"] * 24), "9,16384,257,12001,1374,8192,16000,4097,63,64,65,5480,"
                   "3333,15999,10240,700,12288,1,2048,14000,6001,900,16383,11111", 32, 8, 128, cache=16384),
        # five views of different sizes through a ViT-B in one pass, scores lowered by the distance on the patch grid
        _attention("views_packed", "1369,768,247,1530,441", "1369,768,247,1530,441", 12, 12, 64, bias="grid", grid=37),
        # two long texts behind their images: rows see the image and what is before them, scores capped
        _attention("reader_long", "8192,7001", "8192,7001", 16, 4, 128, causal=True, prefix="1374,257", cap=30.0),
        # one view of a ViT-S in fp32, capped and with distances in a line: for a user who checks numbers
        _attention("view_f32", "1531", "1531", 6, 6, 64, dtype="f32", cap=50.0, bias="line"),
        # between two blocks for a single token
        _norm("norm_one_row", 1, 1536, 1),
        # between two blocks of a ViT-g, eight 518 x 518 views with gates and modulation of their own
        _norm("norm_views", 10992, 1536, 8),
        # an odd width, fp32, RMS norms, a weighted residual, no requests
        _norm("norm_odd_f32", 2741, 777, 0, dtype="f32", post="rms", pre="rms", alpha=0.81),
        # QKV of a ViT-g for one token
        _adapters("adapter_one_row", 1, 1536, 4608, 16, 4),
        # tokens of 48 streams with 32 adapters between them
        _adapters("adapters_mixed", 48, 4096, 4096, 16, 32, mixed=True),
        # QKV of a ViT-g, eight 518 x 518 views, an adapter for each
        _adapters("adapters_views", 10992, 1536, 4608, 32, 8),
        # the first MLP product of a ViT-S in fp32, two views
        _adapters("adapters_f32", 3062, 384, 1536, 8, 2, dtype="f32"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))

    most = {c["kind"]: work(c) for c in listed() if c["name"] in ("reader_long", "norm_views", "adapters_views")}
    most_bytes = work(listed()[1])["bytes"]
    while True:
        kind = rng.choice(("attention", "attention", "norm", "adapters"))
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        if kind == "norm":
            case = _norm(None, log(1, 16384), rng.choice((384, 768, 1024, 1536, log(64, 4096))), rng.choice((0, 1, 3, 8)), dtype,
                         rng.choice(("layer", "rms", "none")), rng.choice(("layer", "rms", "none")), rng.choice((1.0, 0.81)))
        elif kind == "adapters":
            case = _adapters(None, log(1, 12000), 64 * log(4, 64), rng.choice((64 * log(4, 72), log(200, 4608))), 8 * log(1, 8),
                             log(1, 32), dtype, rng.random() < 0.4, rng.random() < 0.7)
        else:
            head_dim = rng.choice((64, 64, 128))
            kv_heads = rng.choice((1, 2, 4, 6, 8, 12))
            heads = kv_heads * rng.choice((1, 1, 2, 4))
            form = rng.choice(("tokens", "views", "reader"))
            n = log(1, 32) if form == "tokens" else rng.randint(1, 8)
            ks = [log(1, 16384) if form == "tokens" else log(40, 4096 if form == "views" else 8192) for _ in range(n)]
            qs = [min(k, rng.choice((1, 1, 1, 2, 5))) for k in ks] if form == "tokens" else ks
            causal = form != "views"
            case = _attention(None, ",".join(map(str, qs)), ",".join(map(str, ks)), heads, kv_heads, head_dim, dtype,
                              cache=max(ks) + rng.randint(0, 300) if form == "tokens" else 0, causal=causal,
                              prefix=",".join(str(rng.randint(0, k)) for k in ks) if form == "reader" else "",
                              cap=rng.choice((0.0, 0.0, 20.0, 50.0)),
                              bias=rng.choice(("", "", "line")) if causal else rng.choice(("", "line", "grid")), grid=rng.randint(5, 60))
        w = work(case)
        if w["flops"] * (16.0 if dtype == "f32" else 1.0) <= most[kind]["flops"] * (4.0 if kind == "norm" else 1.0) and w["bytes"] <= most_bytes:
            return case


# ------------------------------------------------------------------ the work of a pass
def _lengths(text):
    return [int(n) for n in text.split(",") if n]


def _visible(nq, nk, causal, prefix):
    """Pairs of a query and a key it sees: row i stands at nk - nq + i and sees the keys up to there, and the prefix."""
    if not causal:
        return float(nq) * nk
    return float(sum(min(nk, max(0, nk - nq + i + 1, prefix)) for i in range(nq)))


def work(case):
    if case["kind"] == "attention":
        qs, ks = _lengths(case["q"]), _lengths(case["k"])
        prefix = _lengths(case["prefix"]) or [0] * len(qs)
        esz = 2.0 if case["dtype"] == "bf16" else 4.0
        pairs = sum(_visible(a, b, case["causal"], p) for a, b, p in zip(qs, ks, prefix))
        rows = esz * case["head_dim"] * (2.0 * case["heads"] * sum(qs) + 2.0 * case["kv_heads"] * sum(ks)) + 4.0 * case["heads"] * sum(qs)
        if case["bias"] == "grid":
            rows += 8.0 * sum(ks)
        return {"bytes": rows, "flops": 4.0 * case["head_dim"] * case["heads"] * pairs}
    esz = 2.0 if case["dtype"] == "bf16" else 4.0
    if case["kind"] == "norm":
        cells = float(case["rows"]) * case["width"]
        return {"bytes": cells * (8.0 + 2.0 * esz) + 4.0 * case["width"] * (5.0 + 3.0 * case["requests"]), "flops": 20.0 * cells}
    rows, k, n, r, a = (float(case[x]) for x in ("rows", "k", "n", "rank", "adapters"))
    used = min(rows, a)
    return {"bytes": esz * (rows * (k + n) + k * n + used * r * (k + n)) + 4.0 * n, "flops": 2.0 * rows * (k * n + r * (k + n))}


# ------------------------------------------------------------------ what a program has in hand before the call
def _gen(seed):
    return torch.Generator("cuda").manual_seed(77_000 + seed)


def _normal(gen, shape, std=1.0, dtype=torch.float32):
    return (std * torch.randn(shape, generator=gen, device="cuda")).to(dtype)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _prepare_attention(case, gen):
    qs, ks, T = _lengths(case["q"]), _lengths(case["k"]), DTYPE[case["dtype"]]
    H, KH, D, cache = case["heads"], case["kv_heads"], case["head_dim"], case["cache"]
    q_at = _offsets(qs)
    k_at = [i * cache for i in range(len(ks) + 1)] if cache else _offsets(ks)
    st = dict(case=case, qs=qs, ks=ks, q_at=q_at, k_at=k_at, prefix=_lengths(case["prefix"]))
    if not cache and not case["bias"] == "grid" and H == KH and qs == ks:
        qkv = _normal(gen, (q_at[-1], 3, H, D), 1.6, T)            # one product has written all three: rows of 3 H D
        st["q"], st["k"], st["v"] = qkv[:, 0], qkv[:, 1], qkv[:, 2]
    else:
        st["q"] = _normal(gen, (q_at[-1], H, D), 1.6, T)
        st["k"], st["v"] = (_normal(gen, (k_at[-1], KH, D), 1.6, T) for _ in range(2))
    st["out"] = torch.empty((q_at[-1], H, D), dtype=T, device="cuda")
    st["lse"] = torch.empty((q_at[-1], H), device="cuda")
    st["slopes"] = st["coords"] = None
    if case["bias"]:
        st["slopes"] = torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda") / H) * (1.0 + 0.1 * torch.rand(H, generator=gen, device="cuda"))
    if case["bias"] == "grid":
        cell = torch.cat([torch.arange(n, device="cuda") for n in ks])
        st["coords"] = torch.stack([(cell // case["grid"]).float(), (cell % case["grid"]).float()], 1).contiguous()
    if own:
        import paper_2508_11584_amd as vpe
        st["q_offsets"], st["k_offsets"] = _int32(q_at), _int32(k_at)
        st["k_lengths"] = _int32(ks) if cache else None
        st["prefix_rows"] = _int32(st["prefix"]) if st["prefix"] else None
        need = vpe.attention_workspace_bytes(st["q"], st["k"], sequences=len(qs), max_q=max(qs), max_k=max(ks))
        st["workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    return st


def _prepare_norm(case, gen):
    R, W, N, T = case["rows"], case["width"], case["requests"], DTYPE[case["dtype"]]
    st = dict(case=case, x=_normal(gen, (R, W), 2.0), branch=_normal(gen, (R, W), 1.0, T))
    st["x"] += 3.0 * torch.randn((R, 1), generator=gen, device="cuda")              # rows away from zero, as a residual stream is
    for which in ("post", "pre"):
        st[which + "_gain"] = None if case[which] == "none" else 1.0 + _normal(gen, (W,), 0.1)
        st[which + "_bias"] = _normal(gen, (W,), 0.1) if case[which] == "layer" else None
    st["layer_scale"] = 0.1 + _normal(gen, (W,), 0.02)
    for which in ("gate", "scale", "shift"):
        st[which] = _normal(gen, (N, W), 0.3) + (1.0 if which == "gate" else 0.0) if N else None
    st["request"] = (torch.arange(R, device="cuda") * N // R).int() if N else None
    st["out"] = torch.empty_like(st["x"])
    st["normed"] = torch.empty((R, W), dtype=T, device="cuda")
    return st


def _prepare_adapters(case, gen):
    R, K, N, r, A, T = (case[x] for x in ("rows", "k", "n", "rank", "adapters", "dtype"))
    T = DTYPE[T]
    st = dict(case=case, x=_normal(gen, (R, K), 1.0, T), weight=_normal(gen, (N, K), 1.0 / math.sqrt(K), T))
    st["bias"] = _normal(gen, (N,), 0.1) if case["bias"] else None
    st["a"] = _normal(gen, (A, r, K), 1.0 / math.sqrt(K), T)
    st["b"] = _normal(gen, (A, N, r), 0.5 / math.sqrt(r), T)
    st["scale"] = 0.5 + torch.rand(A, generator=gen, device="cuda")
    if case["mixed"]:
        st["adapter"] = torch.randint(-1, A, (R,), generator=gen, device="cuda").int()       # -1: the shared projection alone
    else:
        st["adapter"] = (torch.arange(R, device="cuda") * A // R).int()
    st["out"] = torch.empty((R, N), dtype=T, device="cuda")
    if own:
        import paper_2508_11584_amd as vpe
        st["workspace"] = torch.empty(max(vpe.adapter_linear_workspace_bytes(st["x"], st["weight"], st["a"]), 1), dtype=torch.uint8, device="cuda")
    return st


_PREPARE = {"attention": _prepare_attention, "norm": _prepare_norm, "adapters": _prepare_adapters}


def prepare(case, seed):
    return _PREPARE[case["kind"]](case, _gen(seed))


# ------------------------------------------------------------------ a pass in elementary operations
def _plain_attention(st):
    case = st["case"]
    H, KH, D = case["heads"], case["kv_heads"], case["head_dim"]
    G, cap = H // KH, case["cap"]
    out, lse = torch.empty_like(st["out"]), torch.empty_like(st["lse"])
    for s, (nq, nk) in enumerate(zip(st["qs"], st["ks"])):
        q0, k0 = st["q_at"][s], st["k_at"][s]
        q = st["q"][q0:q0 + nq].float().permute(1, 0, 2).reshape(KH, G * nq, D)
        k = st["k"][k0:k0 + nk].float().permute(1, 2, 0).contiguous()
        v = st["v"][k0:k0 + nk].float().permute(1, 0, 2).contiguous()
        score = (torch.matmul(q, k) * D ** -0.5).view(H, nq, nk)
        if cap:
            score = cap * torch.tanh(score / cap)
        at = torch.arange(nq, device="cuda").view(nq, 1) + (nk - nq)
        key = torch.arange(nk, device="cuda")
        if case["bias"] == "line":
            score = score - st["slopes"].view(H, 1, 1) * (at - key).abs().float()
        elif case["bias"] == "grid":
            d = st["coords"][q0:q0 + nq].view(nq, 1, 2) - st["coords"][k0:k0 + nk]
            score = score - st["slopes"].view(H, 1, 1) * (d * d).sum(2).sqrt()
        if case["causal"]:
            seen = (key <= at) | (key < (st["prefix"][s] if st["prefix"] else 0))
            score = score.masked_fill(~seen, -math.inf)
        top = score.amax(2, keepdim=True)
        e = torch.exp(score - top)
        total = e.sum(2, keepdim=True)
        o = torch.matmul(e.view(KH, G * nq, nk), v).view(H, nq, D) / total
        out[q0:q0 + nq] = o.permute(1, 0, 2).to(out.dtype)
        lse[q0:q0 + nq] = (top + torch.log(total)).view(H, nq).t()
    return out, lse


def _plain_normalised(x, kind, gain, bias):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * gain
    return y if bias is None else y + bias


def _plain_norm(st):
    case = st["case"]
    y = _plain_normalised(st["branch"].float(), case["post"], st["post_gain"], st["post_bias"]) * st["layer_scale"]
    row = st["request"].long() if case["requests"] else None
    if row is not None:
        y = y * st["gate"][row]
    x = case["alpha"] * st["x"] + y
    h = _plain_normalised(x, case["pre"], st["pre_gain"], st["pre_bias"])
    if row is not None:
        h = h * (1.0 + st["scale"][row]) + st["shift"][row]
    return x, h.to(st["normed"].dtype)


def _plain_adapters(st):
    x = st["x"].float()
    y = torch.matmul(x, st["weight"].float().t())
    if st["bias"] is not None:
        y += st["bias"]
    for a in range(st["case"]["adapters"]):
        mine = (st["adapter"] == a).float().view(-1, 1) * st["scale"][a]
        y += torch.matmul(torch.matmul(x, st["a"][a].float().t()) * mine, st["b"][a].float().t())
    return y.to(st["out"].dtype)


# ------------------------------------------------------------------ a pass as a user's program makes it
def _own_attention(st):
    import paper_2508_11584_amd as vpe
    case = st["case"]
    vpe.attention(st["q"], st["k"], st["v"], st["out"], q_offsets=st["q_offsets"], k_offsets=st["k_offsets"], k_lengths=st["k_lengths"],
                  max_q=max(st["qs"]), max_k=max(st["ks"]), causal=case["causal"], prefix=st["prefix_rows"], cap=case["cap"],
                  slopes=st["slopes"], q_coords=st["coords"], k_coords=st["coords"], lse=st["lse"], workspace=st["workspace"],
                  stream=torch.cuda.current_stream())
    return st["out"], st["lse"]


def _own_norm(st):
    import paper_2508_11584_amd as vpe
    case = st["case"]
    kind = {"none": vpe.VPE_NORM_NONE, "layer": vpe.VPE_NORM_LAYER, "rms": vpe.VPE_NORM_RMS}
    vpe.block_norm(st["x"], st["out"], branch=st["branch"], normed=st["normed"], post=kind[case["post"]], post_gain=st["post_gain"],
                   post_bias=st["post_bias"], pre=kind[case["pre"]], pre_gain=st["pre_gain"], pre_bias=st["pre_bias"],
                   layer_scale=st["layer_scale"], residual_scale=case["alpha"], gate=st["gate"], scale=st["scale"], shift=st["shift"],
                   request=st["request"], eps=EPS, stream=torch.cuda.current_stream())
    return st["out"], st["normed"]


def _own_adapters(st):
    import paper_2508_11584_amd as vpe
    vpe.adapter_linear(st["x"], st["weight"], st["out"], bias=st["bias"], a=st["a"], b=st["b"], adapter=st["adapter"], scale=st["scale"],
                       workspace=st["workspace"], stream=torch.cuda.current_stream())
    return st["out"]


_PLAIN = {"attention": _plain_attention, "norm": _plain_norm, "adapters": _plain_adapters}
_OWN = {"attention": _own_attention, "norm": _own_norm, "adapters": _own_adapters}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state)


# ------------------------------------------------------------------ the same from the definitions, in 64 bits
def _exact_attention(st):
    case = st["case"]
    H, G, D = case["heads"], case["heads"] // case["kv_heads"], case["head_dim"]
    out = torch.empty(st["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
    for s in range(len(st["qs"])):
        rows = slice(st["q_at"][s], st["q_at"][s] + st["qs"][s])
        keys = slice(st["k_at"][s], st["k_at"][s] + st["ks"][s])
        nq, nk = st["qs"][s], st["ks"][s]
        i, j = torch.meshgrid(torch.arange(nq, device="cuda"), torch.arange(nk, device="cuda"), indexing="ij")
        behind = j - (i + nk - nq)                                    # how far the key is behind the row's own place
        hidden = behind > 0
        if not case["causal"]:
            hidden = torch.zeros_like(hidden)
        elif st["prefix"]:
            hidden = hidden & (j >= st["prefix"][s])
        far = None
        if case["bias"] == "line":
            far = behind.double().abs()
        elif case["bias"] == "grid":
            a, b = st["coords"][rows].double(), st["coords"][keys].double()
            far = torch.hypot(a[:, None, 0] - b[None, :, 0], a[:, None, 1] - b[None, :, 1])
        for h in range(H):
            x = torch.mm(st["q"][rows, h].double(), st["k"][keys, h // G].double().t().contiguous()) / math.sqrt(D)
            if case["cap"] > 0.0:
                x = torch.tanh(x.div(case["cap"])).mul(case["cap"])
            if far is not None:
                x = x - far * st["slopes"][h].double()
            x[hidden] = -math.inf
            z = torch.logsumexp(x, 1)
            out[rows, h] = torch.mm(torch.exp(x - z.unsqueeze(1)), st["v"][keys, h // G].double())
            lse[rows, h] = z
    return out, lse


def _exact_norm(st):
    case = st["case"]

    def wide(t):
        return None if t is None else t.double()

    def normal(x, kind, gain, bias):
        if kind == "none":
            return x
        if kind == "layer":
            var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
            y = (x - mean) / torch.sqrt(var + EPS)
        else:
            y = x / torch.sqrt(x.square().sum(1, keepdim=True) / x.shape[1] + EPS)
        y = y * wide(gain)
        return y if bias is None else y + wide(bias)

    add = normal(wide(st["branch"]), case["post"], st["post_gain"], st["post_bias"]) * wide(st["layer_scale"])
    which = st["request"].long() if case["requests"] else None
    if which is not None:
        add = add * wide(st["gate"]).index_select(0, which)
    x = wide(st["x"]) * case["alpha"] + add
    h = normal(x, case["pre"], st["pre_gain"], st["pre_bias"])
    if which is not None:
        h = h + h * wide(st["scale"]).index_select(0, which) + wide(st["shift"]).index_select(0, which)
    return x, h


def _exact_adapters(st):
    x = st["x"].double()
    y = torch.mm(x, st["weight"].double().t().contiguous())
    if st["bias"] is not None:
        y = y + st["bias"].double()
    for a in range(st["case"]["adapters"]):
        rows = torch.nonzero(st["adapter"] == a).flatten()
        if len(rows):
            low = torch.mm(x[rows], st["a"][a].double().t().contiguous())
            y[rows] += st["scale"][a].double() * torch.mm(low, st["b"][a].double().t().contiguous())
    return y


_EXACT = {"attention": _exact_attention, "norm": _exact_norm, "adapters": _exact_adapters}


def exact(case, seed):
    return _EXACT[case["kind"]](prepare(case, seed))

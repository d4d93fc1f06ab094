"""What the speed of a worker's step is measured on: the operators that run a batch the scheduler
picked, whose members belong to different applications of one model and have different lengths.

Kinds of case (the field "kind"):
  adapt   low-rank adapters of many applications added to a shared projection's output: every
          row of the batch has its own adapter, or none
  cache   keys and values quantised into a paged cache as they are written, and read back
  attend  attention of the batch's new tokens over that cache: single tokens, prompt chunks
          (each token sees those up to itself) and trees of drafted tokens (a 64-bit mask a token)

Widths, ranks, heads and pages are generic; batches (64, 128) and the number of applications (32) are
those of the repository's configurations.  Lengths are ragged: the requests of a batch have contexts
drawn between two bounds, fixed by the case.  Inputs are made on the GPU.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
TOP = {"int8": 127.0, "fp8": 448.0}
CODES = {"int8": torch.int8, "fp8": torch.float8_e4m3fn}
TINY = 2.0 ** -100          # a vector whose largest magnitude is below this is stored as zeros


def _adapt(name, rows, adapters, d_in, d_out, rank, dtype="bf16", ragged=False, prompts=0, none=0.0,
           base=True, pad=0, salt=1):
    """prompts > 0: the rows are that many requests' tokens, one adapter a request; 0: every row is
    a request of its own.  ragged: adapters' ranks between 0 and rank.  none: share of requests
    without an adapter.  pad: extra elements between rows."""
    c = dict(kind="adapt", rows=rows, adapters=adapters, d_in=d_in, d_out=d_out, rank=rank,
             dtype=dtype, ragged=ragged, prompts=prompts, none=none, base=base, pad=pad, salt=salt)
    return dict(c, name=name) if name else c


def _cached(name, kind, requests, rows, lo, hi, heads, group, dim, page, fmt, dtype="bf16",
            ragged=False, tree=False, salt=1):
    """requests with lo..hi tokens cached before and `rows` new ones (ragged: 0..rows)."""
    c = dict(kind=kind, requests=requests, rows=rows, lo=lo, hi=hi, heads=heads, group=group, dim=dim,
             page=page, format=fmt, dtype=dtype, ragged=ragged, tree=tree, salt=salt)
    return dict(c, name=name) if name else c


def listed():
    return [
        # four requests of different applications decode a token on a small model
        _adapt("adapt-few", 4, 8, 1024, 1024, 8),
        # a full batch decodes: 64 requests spread over 32 applications
        _adapt("adapt-batch", 64, 32, 4096, 4096, 16),
        # odd widths, padded rows, adapters of different ranks, requests without one
        _adapt("adapt-odd", 37, 21, 1000, 1501, 12, dtype="f16", ragged=True, none=0.2, pad=3),
        # prompts of 16 requests go through a wide projection
        _adapt("adapt-prompts", 8192, 32, 4096, 4096, 64, prompts=16, none=0.1),
        # 64 requests write one token each, and read it back
        _cached("cache-step", "cache", 64, 1, 16, 4096, 8, 1, 128, 16, "int8"),
        # odd heads and dimensions, ragged rows, 32-bit activations
        _cached("cache-odd", "cache", 21, 37, 0, 300, 5, 1, 80, 32, "fp8", dtype="f32", ragged=True),
        # prompts of 16 requests, 16384 tokens in all, fill their pages
        _cached("cache-prompts", "cache", 16, 1024, 0, 512, 8, 1, 128, 64, "fp8"),
        # one request decodes a token over a short context: the latency of the call
        _cached("attend-one", "attend", 1, 1, 200, 300, 4, 4, 64, 16, "int8", dtype="f16"),
        # a full batch of 64 decodes over ragged contexts
        _cached("attend-batch", "attend", 64, 1, 64, 8192, 8, 4, 128, 16, "int8"),
        # four requests decode over a hundred thousand tokens each
        _cached("attend-long", "attend", 4, 1, 65536, 131072, 8, 8, 128, 64, "fp8"),
        # 16 requests check trees of up to 24 drafted tokens
        _cached("attend-tree", "attend", 16, 24, 0, 12000, 8, 4, 128, 32, "fp8", ragged=True,
                tree=True),
        # chunks of four prompts after a shared context: bound by the products
        _cached("attend-chunk", "attend", 4, 2048, 1024, 4096, 8, 4, 128, 64, "int8", ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["adapt", "adapt", "cache", "cache", "attend", "attend", "attend"])
    salt = rng.randrange(1 << 20)
    if kind == "adapt":
        prompts = rng.choice([0, 0, _log(rng, 1, 32)])
        width = lambda: rng.choice([8, 8, 1]) * _log(rng, 64, 360)  # noqa: E731
        rows = _log(rng, 64, 8192) if prompts else _log(rng, 1, 128)
        return _adapt(None, rows, _log(rng, 1, 64), width(), width(),
                      rng.choice([8, 16, 32, 64, _log(rng, 1, 64)]), dtype=rng.choice(["bf16", "f16"]),
                      ragged=rng.random() < 0.3, prompts=min(prompts, rows), none=rng.choice([0.0, 0.0, 0.15]),
                      base=rng.random() < 0.8, pad=rng.choice([0, 0, 0, 8, 3]), salt=salt)
    page = rng.choice([16, 32, 64, 128, 256])
    dim = rng.choice([64, 128, 128, 80, 96, 192, 256, _log(rng, 16, 256)])
    heads, group = _log(rng, 1, 16), rng.choice([1, 2, 4, 8, 7])
    fmt, dtype = rng.choice(["int8", "fp8"]), rng.choice(["bf16", "bf16", "f16"])
    if kind == "cache":
        rows = rng.choice([1, _log(rng, 2, 1024)])
        requests = max(1, min(_log(rng, 1, 128), 16384 // rows))
        return _cached(None, kind, requests, rows, 0, _log(rng, 16, 2048), heads, 1, dim, page, fmt,
                       dtype=rng.choice([dtype, "f32"]), ragged=rng.random() < 0.5, salt=salt)
    form = rng.choice(["step", "step", "tree", "chunk"])
    rows = 1 if form == "step" else _log(rng, 2, 64) if form == "tree" else _log(rng, 2, 1024)
    hi = _log(rng, 32, 131072 if form == "step" else 16384 if form == "tree" else 4096)
    requests = _log(rng, 1, 64)
    while requests > 1 and requests * (hi + rows) * heads * dim > (1 << 28):
        requests = requests * 2 // 3
    while heads > 1 and (requests * (hi + rows) * heads * dim > (1 << 28) or
                         requests * rows * (hi + rows) * heads * group * dim > (1 << 37)):
        heads = heads * 2 // 3
    while requests > 1 and requests * rows * (hi + rows) * heads * group * dim > (1 << 37):
        requests = requests * 2 // 3
    return _cached(None, kind, requests, rows, rng.choice([0, hi // 4, hi]), hi, heads, group, dim, page, fmt,
                   dtype=dtype, ragged=rng.random() < 0.5, tree=form == "tree", salt=salt)


# -- what a case fixes --------------------------------------------------------------
def _adapter_rows(c):
    """Each row's adapter, or -1, and each adapter's rank."""
    r = random.Random(c["salt"] * 7919 + c["rows"])
    pick = lambda: -1 if r.random() < c["none"] else r.randrange(c["adapters"])  # noqa: E731
    ranks = [r.randint(0, c["rank"]) if c["ragged"] else c["rank"] for _ in range(c["adapters"])]
    if not c["prompts"]:
        return [pick() for _ in range(c["rows"])], ranks
    cuts = sorted(r.randrange(c["rows"] + 1) for _ in range(c["prompts"] - 1))
    ids = []
    for a, b in zip([0] + cuts, cuts + [c["rows"]]):
        ids += [pick()] * (b - a)
    return ids, ranks


def _lengths(c):
    """Each request's context and number of new rows."""
    r = random.Random(c["salt"] * 7919 + c["requests"])
    ctx = [r.randint(c["lo"], c["hi"]) for _ in range(c["requests"])]
    rows = [r.randint(0, c["rows"]) if c["ragged"] else c["rows"] for _ in range(c["requests"])]
    if not sum(rows):
        rows[-1] = c["rows"]
    return ctx, rows


def _dim_pad(c):
    return -(-c["dim"] // 64) * 64


def work(case):
    c = case
    if c["kind"] == "adapt":
        ids, ranks = _adapter_rows(c)
        width = c["d_in"] + c["d_out"]
        n = c["rows"] * (c["d_in"] + c["d_out"] * (2 if c["base"] else 1)) + width * sum(ranks[a] for a in set(ids) if a >= 0)
        return {"bytes": 2 * n + 4 * c["rows"], "flops": 2 * width * sum(ranks[a] for a in ids if a >= 0)}
    size = {"bf16": 2, "f16": 2, "f32": 4}[c["dtype"]]
    ctx, rows = _lengths(c)
    T = sum(rows)
    if c["kind"] == "cache":
        # written: activations in, codes and scales out; read back: the reverse
        v = 2 * T * c["heads"]
        return {"bytes": 2 * v * (c["dim"] * (size + 1) + 4), "flops": 4 * v * c["dim"]}
    hq = c["heads"] * c["group"]
    tokens = sum(a + m for a, m in zip(ctx, rows) if m)
    pairs = sum(m * a + (m * (m + 1)) // 2 for a, m in zip(ctx, rows))
    return {"bytes": tokens * c["heads"] * 2 * (c["dim"] + 4) + T * hq * (2 * size * c["dim"] + 4),
            "flops": 4 * pairs * hq * c["dim"]}


# -- inputs --------------------------------------------------------------------------
def _stride(rows, width, pad, g, dtype):
    """A [rows][width] matrix of normals whose rows are width + pad apart."""
    return torch.randn(rows, width + pad, generator=g, device=DEV).to(dtype)[:, :width]


def _quantise(x, fmt):
    """Codes (as 32-bit values) and scales of vectors along the last axis."""
    amax = x.abs().amax(-1, keepdim=True)
    bad, low = ~torch.isfinite(amax), amax < TINY
    inv = TOP[fmt] / torch.where(bad | low, 1.0, amax)
    code = torch.where(bad | low, 0.0, x * inv)
    code = code.round() if fmt == "int8" else code.to(torch.float8_e4m3fn).float()
    scale = torch.where(bad, math.nan, torch.where(low, 0.0, amax / TOP[fmt]))
    return code, scale[..., 0]


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = DTYPES[c["dtype"]]
    if c["kind"] == "adapt":
        ids, ranks = _adapter_rows(c)
        n, R = c["adapters"], c["rank"]
        s = dict(case=c, adapter=torch.tensor(ids, dtype=torch.int32, device=DEV),
                 x=_stride(c["rows"], c["d_in"], c["pad"], g, dt),
                 down=(torch.randn(n, R, c["d_in"], generator=g, device=DEV) / math.sqrt(c["d_in"])).to(dt),
                 up=(torch.randn(n, c["d_out"], R, generator=g, device=DEV) / math.sqrt(R)).to(dt),
                 scale=torch.rand(n, generator=g, device=DEV) + 0.5,
                 rank=torch.tensor(ranks, dtype=torch.int32, device=DEV) if c["ragged"] else None,
                 base=_stride(c["rows"], c["d_out"], c["pad"], g, dt) if c["base"] else None)
        return s
    ctx, rows = _lengths(c)
    P, H, D, Dp = c["page"], c["heads"], c["dim"], _dim_pad(c)
    pages = [-(-(a + m) // P) for a, m in zip(ctx, rows)]
    total = sum(pages) + 3
    ids = torch.randperm(total, generator=g, device=DEV).to(torch.int32).cpu()
    table = torch.full((c["requests"], max(max(pages), 1)), -1, dtype=torch.int32)
    at = 0
    for r, k in enumerate(pages):
        table[r, :k] = ids[at:at + k]
        at += k
    off = [0]
    for m in rows:
        off.append(off[-1] + m)
    T = off[-1]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    s = dict(case=c, table=table.to(DEV), length=ints([a + m for a, m in zip(ctx, rows)]), row_off=ints(off),
             n_rows=T, max_rows=max(rows), max_length=max(a + m for a, m in zip(ctx, rows)))
    code = CODES[c["format"]]
    if c["kind"] == "cache":
        # keys and values as a fused projection leaves them: side by side in one row
        kv = torch.randn(T, 2 * H * D, generator=g, device=DEV) * torch.exp(torch.randn(T, 1, generator=g, device=DEV))
        kv = kv.to(dt)
        s["k"], s["v"] = kv[:, :H * D].unflatten(1, (H, D)), kv[:, H * D:].unflatten(1, (H, D))
        for n in ("kv_k", "kv_v"):
            s[n] = torch.zeros(total, H, P, Dp, dtype=torch.uint8, device=DEV).view(code)
            s[n + "_scale"] = torch.zeros(total, H, P, device=DEV)
        return s
    for n in ("kv_k", "kv_v"):
        x = torch.randn(total, H, P, D, generator=g, device=DEV)
        q, s[n + "_scale"] = _quantise(x, c["format"])
        s[n] = torch.zeros(total, H, P, Dp, dtype=torch.uint8, device=DEV).view(code)
        s[n][..., :D] = q.to(code)
    s["q"] = (2.0 * torch.randn(T, H * c["group"], D, generator=g, device=DEV)).to(dt)
    s["tree"] = None
    if c["tree"]:
        # drafted token i hangs under a random earlier one, or under the context
        r = random.Random(seed)
        masks = []
        for m in rows:
            mine = []
            for i in range(m):
                up = r.randrange(-1, i)
                mine.append((mine[up] if up >= 0 else 0) | (1 << i))
            masks += [v - (1 << 64) if v >= 1 << 63 else v for v in mine]
        s["tree"] = torch.tensor(masks, dtype=torch.int64, device=DEV)
    return s


# -- the plain forms -------------------------------------------------------------------
def _plain_adapt(s):
    c = s["case"]
    n, R = c["adapters"], c["rank"]
    h = (s["x"].float() @ s["down"].float().flatten(0, 1).T).unflatten(1, (n, R))
    mine = s["adapter"][:, None] == torch.arange(n, device=DEV)
    keep = mine[:, :, None]
    if s["rank"] is not None:
        keep = keep & (torch.arange(R, device=DEV) < s["rank"][:, None])
    h = torch.where(keep, h * s["scale"][:, None], 0.0).flatten(1)
    y = h @ s["up"].float().transpose(1, 2).flatten(0, 1)
    if s["base"] is not None:
        y = s["base"].float() + y
    return y.to(s["x"].dtype)


def _places(s):
    """Each row's page and slot."""
    row = torch.arange(s["n_rows"], device=DEV)
    req = torch.searchsorted(s["row_off"][1:].contiguous(), row.to(torch.int32), right=True)
    pos = (s["length"][req] - s["row_off"][req + 1] + row).long()
    P = s["case"]["page"]
    return s["table"][req, pos // P].long()[:, None], torch.arange(s["case"]["heads"], device=DEV)[None], (pos % P)[:, None]


def _plain_store(s, x, name, at):
    D, fmt = s["case"]["dim"], s["case"]["format"]
    code, scale = _quantise(x.float(), fmt)
    code = torch.nn.functional.pad(code, (0, s[name].shape[-1] - D)).to(CODES[fmt])
    s[name].view(torch.uint8)[at] = code.view(torch.uint8)
    s[name + "_scale"][at] = scale


def _plain_load(s, name, at):
    code = s[name].view(torch.uint8)[at].view(CODES[s["case"]["format"]])
    return (code.float() * s[name + "_scale"][at][..., None])[..., :s["case"]["dim"]]


def _plain_cache(s):
    at = _places(s)
    _plain_store(s, s["k"], "kv_k", at)
    _plain_store(s, s["v"], "kv_v", at)
    dt = s["k"].dtype
    return {"k": _plain_load(s, "kv_k", at).to(dt), "v": _plain_load(s, "kv_v", at).to(dt),
            "k_scale": s["kv_k_scale"], "v_scale": s["kv_v_scale"]}


def _plain_whole(s, name, L):
    """[requests][heads][L][D]: the cached vectors of every request, zeros past its length."""
    page = s["table"].clamp(min=0).long()
    x = s[name].view(torch.uint8)[page].view(CODES[s["case"]["format"]])[..., :s["case"]["dim"]].float()
    x = x * s[name + "_scale"][page][..., None]
    x = x.transpose(1, 2).flatten(2, 3)[:, :, :L]
    live = torch.arange(L, device=DEV) < s["length"][:, None]
    return torch.where(live[:, None, :, None], x, 0.0)


def _plain_attend(s):
    c = s["case"]
    H, G, D, M, L = c["heads"], c["group"], c["dim"], s["max_rows"], s["max_length"]
    k, v = _plain_whole(s, "kv_k", L), _plain_whole(s, "kv_v", L)
    n = s["row_off"][1:] - s["row_off"][:-1]
    i = torch.arange(M, device=DEV)
    there = i < n[:, None]                                    # [requests][M]
    row = torch.where(there, s["row_off"][:-1, None] + i, 0).long()
    q = s["q"].float()[row].unflatten(2, (H, G)).permute(0, 2, 1, 3, 4).reshape(-1, H, M * G, D)
    score = (q @ k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(D))
    t = torch.arange(L, device=DEV)
    context = (s["length"] - n)[:, None, None]
    if s["tree"] is None:
        sees = t <= context + i[:, None]
    else:
        j = t - context                                       # the drafted token's number
        bit = (s["tree"][row][:, :, None] >> j.clamp(0, 63)) & 1
        sees = (j < 0) | ((bit == 1) & (j < n[:, None, None]))
    sees = sees.repeat_interleave(G, 1)[:, None]
    score = score.masked_fill(~sees, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    o = torch.where(total > 0, (p @ v) / total, 0.0)
    lse = top + torch.log(total)
    o = o.unflatten(2, (M, G)).transpose(1, 2)[there].flatten(1, 2)
    lse = lse[..., 0].unflatten(2, (M, G)).transpose(1, 2)[there].flatten(1)
    return {"out": o.to(s["q"].dtype), "lse": lse}


# -- the framework's calls ----------------------------------------------------------------
_worker = None              # a serving program keeps one


def _own(s):
    global _worker
    from paper_2209_00159_amd import worker as W
    c = s["case"]
    if _worker is None:
        _worker = W.Worker()
    if c["kind"] == "adapt":
        if "adapters" not in s:
            s["adapters"] = W.Adapters(_worker, s["down"], s["up"], scale=s["scale"], rank=s["rank"])
        return s["adapters"].apply(s["x"], s["adapter"], base=s["base"])
    if "cache" not in s:
        s["cache"] = W.Cache(_worker, s["kv_k"], s["kv_v"], s["kv_k_scale"], s["kv_v_scale"], head_dim=c["dim"])
        s["batch"] = W.Batch(s["row_off"], s["length"], s["table"], n_rows=s["n_rows"], max_rows=s["max_rows"],
                             max_length=s["max_length"])
    if c["kind"] == "cache":
        s["cache"].write(s["batch"], s["k"], s["v"])
        k, v = s["cache"].read(s["batch"], dtype=s["k"].dtype)
        return {"k": k, "v": v, "k_scale": s["kv_k_scale"], "v_scale": s["kv_v_scale"]}
    out, lse = s["cache"].attend(s["batch"], s["q"], tree=s["tree"], lse=True)
    return {"out": out, "lse": lse}


def run(state):
    if own:
        return _own(state)
    return {"adapt": _plain_adapt, "cache": _plain_cache, "attend": _plain_attend}[state["case"]["kind"]](state)


# -- the definitions in 64 bits ---------------------------------------------------------------
def _exact_adapt(s):
    y = torch.zeros(s["x"].shape[0], s["up"].shape[1], dtype=torch.float64, device=DEV)
    if s["base"] is not None:
        y += s["base"].double()
    for a in sorted(set(s["adapter"].tolist()) - {-1}):
        rows = torch.nonzero(s["adapter"] == a)[:, 0]
        R = s["down"].shape[1] if s["rank"] is None else int(s["rank"][a])
        h = s["x"][rows].double() @ s["down"][a, :R].double().T
        y[rows] += float(s["scale"][a]) * (h @ s["up"][a, :, :R].double().T)
    return y


def _exact_vectors(x, fmt):
    """Vectors as the cache holds them, in 64 bits: the nearest multiples (or e4m3 multiples) of
    their scale."""
    x = x.double()
    amax = x.abs().amax(-1, keepdim=True)
    scale = torch.where(amax < TINY, 0.0, amax / TOP[fmt])
    u = torch.where(scale > 0, x / torch.where(scale > 0, scale, 1.0), 0.0)
    if fmt == "int8":
        u = torch.round(u)
    else:
        # e4m3: 3 fraction bits down to 2^-6, then multiples of 2^-9
        step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3.0)
        u = torch.round(u / step) * step
    return u * scale, scale[..., 0]


def _exact_cache(s):
    c = s["case"]
    out = {}
    off, length, table = (s[n].tolist() for n in ("row_off", "length", "table"))
    at = [(table[r][(length[r] - off[r + 1] + t) // c["page"]], (length[r] - off[r + 1] + t) % c["page"])
          for r in range(c["requests"]) for t in range(off[r], off[r + 1])]
    page, slot = (torch.tensor(v, device=DEV) for v in zip(*at))
    for n in ("k", "v"):
        out[n], scale = _exact_vectors(s[n], c["format"])
        pool = torch.zeros(s["kv_" + n + "_scale"].shape, dtype=torch.float64, device=DEV)
        pool.transpose(1, 2)[page, slot] = scale
        out[n + "_scale"] = pool
    return out


def _exact_attend(s):
    c = s["case"]
    G, H, P = c["group"], c["heads"], c["page"]
    off, length, table = (s[n].tolist() for n in ("row_off", "length", "table"))
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for r in range(c["requests"]):
        a, b, L = off[r], off[r + 1], length[r]
        if a == b or not L:
            continue
        pages = torch.tensor(table[r][:-(-L // P)], device=DEV)
        sees = torch.zeros(b - a, L, dtype=torch.bool, device=DEV)
        sees[:, :L - (b - a)] = True
        if s["tree"] is None:
            sees[:, L - (b - a):] = torch.ones(b - a, b - a, dtype=torch.bool, device=DEV).tril()
        else:
            for j in range(b - a):
                sees[:, L - (b - a) + j] = ((s["tree"][a:b] >> j) & 1) == 1
        some = sees.any(-1)
        for h in range(H):
            k, v = (s[n][pages, h].reshape(-1, s[n].shape[-1])[:L, :c["dim"]].float().double() *
                    s[n + "_scale"][pages, h].reshape(-1)[:L, None].double() for n in ("kv_k", "kv_v"))
            for i in range(h * G, (h + 1) * G):
                z = (s["q"][a:b, i].double() @ k.T) / math.sqrt(c["dim"])
                z[~sees] = -math.inf
                lse[a:b, i] = torch.logsumexp(z, -1)
                w = torch.exp(z - torch.where(some, lse[a:b, i], 0.0)[:, None])
                out[a:b, i] = w @ v
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    return {"adapt": _exact_adapt, "cache": _exact_cache, "attend": _exact_attend}[case["kind"]](s)

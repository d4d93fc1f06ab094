"""The worker's operators (adapters, the 8-bit paged cache, attention over it) against plain forms in
64 bits, at the sizes, masks and values where they can go wrong, and their refusals."""
import math

import pytest
import torch

import worker_plain as P
from paper_2209_00159_amd import orloj as O
from paper_2209_00159_amd import worker as W

pytestmark = pytest.mark.gpu

FORMATS = [torch.int8, torch.float8_e4m3fn]


def say(*a):
    print(*a, flush=True)


@pytest.fixture(scope="module")
def worker():
    return W.Worker()


# -- adapters ---------------------------------------------------------------------
def adapt_inputs(seed, rows, n, d_in, d_out, rank, dtype, pad=0, ragged=False, none=0.2, ids=None):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    ids = torch.randint(0, max(n, 1), (rows,), generator=g) if ids is None else ids
    ids = torch.where(torch.rand(rows, generator=g) < none, -1, ids).to(torch.int32)
    if n == 0:
        ids[:] = -1
    return dict(x=r(rows, d_in + pad).to(dtype)[:, :d_in], adapter=ids,
                down=(r(n, rank, d_in) / math.sqrt(d_in)).to(dtype), up=r(n, d_out, rank).to(dtype),
                scale=torch.rand(n, generator=g) * 2 - 0.5,
                rank=torch.randint(0, rank + 1, (n,), generator=g, dtype=torch.int32) if ragged else None,
                base=r(rows, d_out + pad).to(dtype)[:, :d_out])


def on(worker, d):
    """Copies on the device that keep their strides."""
    out = {}
    for k, v in d.items():
        if isinstance(v, torch.Tensor) and v.dim() == 2 and not v.is_contiguous():
            whole = torch.empty(v.shape[0], v.stride(0), dtype=v.dtype, device=worker.device)
            whole[:, :v.shape[1]] = v.to(worker.device)
            out[k] = whole[:, :v.shape[1]]
        else:
            out[k] = v.to(worker.device) if isinstance(v, torch.Tensor) else v
    return out


def check_adapt(worker, d, use_base=True, use_scale=True):
    dev = on(worker, d)
    ad = W.Adapters(worker, dev["down"], dev["up"], scale=dev["scale"] if use_scale else None, rank=dev["rank"])
    got = ad.apply(dev["x"], dev["adapter"], base=dev["base"] if use_base else None)
    worker.sync()
    want, mag = P.adapt(d["x"], d["adapter"], d["down"], d["up"], d["scale"] if use_scale else None, d["rank"],
                        d["base"] if use_base else None)
    dtype = d["x"].dtype
    # one rounding of the result, sums in 32 bits, h with 16 significant bits or more; 2^-24: the
    # smallest 16-bit floats
    depth = d["x"].shape[1] + d["down"].shape[1] + 8
    bound = P.UNIT[dtype] * want.abs() + mag * (2.0 ** -15 + depth * 2.0 ** -24) * (1 + P.UNIT[dtype]) + 2.0 ** -24
    err = (got.cpu().double() - want).abs()
    assert bool((err <= bound).all()), float((err / bound).max())
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,n,d_in,d_out,rank,pad,ragged", [
    (1, 1, 1, 1, 1, 0, False),
    (1, 4, 64, 64, 8, 0, False),
    (3, 2, 7, 5, 3, 1, True),
    (16, 3, 128, 256, 16, 0, False),
    (17, 5, 136, 72, 8, 0, True),
    (37, 21, 333, 517, 12, 3, True),
    (64, 32, 1024, 1000, 16, 0, False),
    (65, 7, 520, 264, 64, 8, True),
    (128, 4, 256, 128, 128, 0, True),
    (130, 3, 2048, 96, 33, 0, False),
    (700, 6, 512, 640, 24, 0, True),
    (1025, 4, 7, 5, 3, 0, True),
    (1030, 5, 333, 517, 12, 3, True),
    (1100, 6, 512, 640, 24, 0, True),
    (1100, 3, 1032, 96, 33, 8, False),
    (1200, 4, 256, 136, 128, 0, True),
])
def test_adapters(worker, dtype, rows, n, d_in, d_out, rank, pad, ragged):
    say("adapt", dtype, rows, n, d_in, d_out, rank, pad, ragged)
    d = adapt_inputs(rows + d_in, rows, n, d_in, d_out, rank, dtype, pad, ragged)
    check_adapt(worker, d)
    check_adapt(worker, d, use_base=False, use_scale=False)


@pytest.mark.parametrize("rows", [150, 1150])
@pytest.mark.parametrize("ids", ["one", "none", "pairs", "blocks"])
def test_adapters_of_adjacent_rows(worker, ids, rows):
    say("adapt ids", ids, rows)
    i = torch.arange(rows)
    pick = dict(one=i * 0 + 2, none=i * 0 - 1, pairs=i // 2 % 5, blocks=i // 40 % 5)[ids]
    d = adapt_inputs(5, rows, 5, 256, 384, 16, torch.bfloat16, none=0.0, ids=pick)
    got = check_adapt(worker, d)
    if ids == "none":
        assert torch.equal(got.cpu(), d["base"])


def test_adapters_without_work(worker):
    say("adapt without work")
    d = adapt_inputs(1, 0, 3, 64, 32, 8, torch.float16)
    dev = on(worker, d)
    assert W.Adapters(worker, dev["down"], dev["up"]).apply(dev["x"], dev["adapter"]).shape == (0, 32)
    check_adapt(worker, adapt_inputs(2, 9, 0, 64, 32, 8, torch.float16))


def test_adapters_in_place_and_range(worker):
    say("adapt in place")
    d = adapt_inputs(3, 40, 5, 256, 264, 16, torch.float16)
    dev = on(worker, d)
    ad = W.Adapters(worker, dev["down"], dev["up"], scale=dev["scale"])
    want = ad.apply(dev["x"], dev["adapter"], base=dev["base"])
    out = dev["base"].clone()
    assert torch.equal(ad.apply(dev["x"], dev["adapter"], base=out, out=out), want)
    # h beyond what 16 bits hold (|h| about 2^24), y within it
    big = dict(d, x=d["x"] * 2000, down=d["down"] * 500, up=(d["up"] * 2.0 ** -13).to(torch.float16), scale=d["scale"] * 2.0 ** -7)
    big["x"], big["down"] = big["x"].to(torch.float16), (d["down"].float() * 8000).to(torch.float16)
    check_adapt(worker, big)
    # a row's infinity or NaN stays in its row
    x = d["x"].clone()
    x[3, 5], x[20, 0] = math.inf, math.nan
    got = ad.apply(x.to(worker.device), dev["adapter"], base=dev["base"])
    rest = [t for t in range(40) if t not in (3, 20)]
    assert torch.equal(got[rest], want[rest])
    for t in (3, 20):
        assert bool(torch.isfinite(got[t]).all()) == (int(d["adapter"][t]) < 0)
    worker.sync()


# -- the cache ----------------------------------------------------------------------
REQUESTS = [[(0, 1)], [(3, 5), (0, 0), (17, 1), (31, 40), (0, 16)], [(15, 1)] * 20 + [(100, 60)]]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,heads,page,requests", [
    (1, 1, 16, 0), (64, 2, 16, 1), (80, 5, 32, 1), (128, 8, 16, 2), (131, 3, 64, 1), (192, 1, 128, 1), (256, 2, 256, 2)])
def test_cache(worker, fmt, dtype, dim, heads, page, requests):
    say("cache", fmt, dtype, dim, heads, page, requests)
    p = P.Paged(REQUESTS[requests], page, heads, dim, fmt, seed=dim)
    before = {n: t.clone() for n, t in p.pool.items()}
    cache, batch = p.cache(W, worker), p.batch(W, worker)
    # a strided view: keys and values side by side
    kv = torch.randn(p.T, heads, 2, dim, generator=p.g) * torch.exp(torch.randn(p.T, heads, 1, 1, generator=p.g))
    kv[0, 0, 0] = 0.0
    if p.T > 3:
        kv[1, -1, 0] = 2.0 ** -120
        kv[2, 0, 1, dim // 2] = math.inf
        kv[3, 0, 0, 0] = math.nan
        kv[3, 0, 1, 0] = -0.0
    kv = kv.to(dtype)
    dev = kv.to(worker.device)
    cache.write(batch, dev[:, :, 0], dev[:, :, 1])
    got = dict(zip(("k", "v"), cache.read(batch, dtype=torch.float32)))
    low = dict(zip(("k", "v"), cache.read(batch, dtype=dtype)))
    worker.sync()
    for j, n in enumerate(("k", "v")):
        x = kv[:, :, j].double()
        amax = x.abs().amax(-1)
        scale = amax / P.TOP[fmt]
        scale[amax < 2.0 ** -100] = 0.0
        bad = ~torch.isfinite(amax)
        pool, ps = getattr(cache, n).view(torch.uint8).cpu(), getattr(cache, n + "_scale").cpu()
        used = torch.zeros(ps.shape, dtype=torch.bool)
        for r in range(len(p.length)):
            for row in range(p.off[r], p.off[r + 1]):
                page_, slot = p.at(r, p.context[r] + row - p.off[r])
                used[page_, :, slot] = True
                s = ps[page_, :, slot].double()
                code = pool[page_, :, slot].view(fmt).double()
                assert torch.equal(torch.isnan(s), bad[row])
                fine = ~bad[row]
                # one rounding of the scale; codes to the nearest of their grid (2^-18: how near a
                # tie x (top / amax) in 32 bits, with three roundings and codes to 448, can fall)
                assert bool(((s - scale[row]).abs()[fine] <= 2.0 ** -23 * scale[row][fine]).all())
                assert bool((code[..., dim:] == 0).all()) and bool((code[bad[row]] == 0).all())
                unit = torch.where(scale[row] > 0, x[row].T / torch.where(scale[row] > 0, scale[row], 1.0), 0.0).T
                unit = torch.where(fine[:, None], unit, 0.0)
                step = torch.ones_like(unit) if fmt == torch.int8 else \
                    torch.exp2(torch.floor(torch.log2(unit.abs().clamp(min=2.0 ** -6))) - 3.0)
                off = (code[..., :dim] - unit).abs()
                assert bool((off <= 0.5 * step + unit.abs() * 2.0 ** -21).all())
                # reading back: the product, rounded once
                want = (code[..., :dim].float() * s.float()[:, None])
                assert torch.equal(torch.nan_to_num(got[n][row].cpu(), nan=7.0), torch.nan_to_num(want, nan=7.0))
                assert torch.equal(torch.nan_to_num(low[n][row].cpu().float(), nan=7.0),
                                   torch.nan_to_num(want.to(dtype).float(), nan=7.0))
        # nothing else was written
        assert torch.equal(pool[~used], before[n][~used])
        assert torch.equal(torch.nan_to_num(ps[~used], nan=7.0), torch.nan_to_num(before[n + "_scale"][~used], nan=7.0))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_cache_codes_are_those_of_32_bit_arithmetic(worker, fmt, dtype):
    """scale = amax (1 / top), code = x ((1 / amax) top) to the nearest, each step rounded to 32
    bits: the same codes, ties and all."""
    say("cache codes", fmt, dtype)
    p = P.Paged([(0, 700)], 64, 4, 128, fmt, seed=3)
    cache, batch = p.cache(W, worker), p.batch(W, worker)
    x = torch.randn(700, 4, 128, generator=p.g).to(dtype)
    x[::3] = (x[::3] * 8).round() / 8                 # many ties
    cache.write(batch, x.to(worker.device), x.to(worker.device))
    worker.sync()
    f = x.float()
    amax = f.abs().amax(-1)
    top = torch.tensor(P.TOP[fmt])
    inv = (torch.tensor(1.0) / amax) * top
    y = f * inv[..., None]
    want = y.round().to(torch.int8) if fmt == torch.int8 else y.to(torch.float8_e4m3fn)
    for pool, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        for t in range(700):
            page, slot = p.at(0, t)
            assert torch.equal(pool[page, :, slot].cpu().view(torch.uint8), want[t].view(torch.uint8)), t
            assert torch.equal(scale[page, :, slot].cpu(), amax[t] * (torch.tensor(1.0) / top))


def test_cache_of_many_requests(worker):
    """A row's request is found among many, empty ones between them."""
    say("cache of many requests")
    g = torch.Generator().manual_seed(9)
    req = [(int(c), int(m)) for c, m in zip(torch.randint(0, 40, (1500,), generator=g),
                                            torch.randint(0, 3, (1500,), generator=g))]
    p = P.Paged(req, 16, 1, 64, torch.int8)
    cache, batch = p.cache(W, worker), p.batch(W, worker)
    x = torch.randn(p.T, 1, 64, generator=g, device="cpu").to(worker.device)
    cache.write(batch, x, -x)
    k, v = cache.read(batch, dtype=torch.float32)
    worker.sync()
    assert torch.equal(k, -v)
    assert float((k - x).abs().max()) <= 0.51 * float(x.abs().max()) / 127
    whole = W.Batch(torch.tensor([0] + p.length).cumsum(0).to(torch.int32).to(worker.device),
                    batch._keep[1], batch._keep[2])
    at = torch.tensor([sum(p.length[:r]) + p.context[r] + i for r in range(1500) for i in range(p.rows[r])])
    assert torch.equal(cache.read(whole, dtype=torch.float32)[0].cpu()[at], k.cpu())
    worker.sync()


def test_pages_past_32_bits(worker):
    """Pages more than 2^32 bytes into the cache hold what near ones do."""
    say("pages past 32 bits")
    far = W.Cache.empty(worker, 8300, 8, 256, 256, torch.int8)      # 512 KiB a page
    near = W.Cache.empty(worker, 4, 8, 256, 256, torch.int8)
    i = lambda v: torch.tensor(v, dtype=torch.int32, device=worker.device)  # noqa: E731
    assert far.k.numel() > 2 ** 32
    g = torch.Generator().manual_seed(1)
    k, v, q = (torch.randn(300, h, 256, generator=g).to(torch.bfloat16).to(worker.device) for h in (8, 8, 16))
    got = []
    for cache, pages in ((far, [8299, 8230]), (near, [1, 3])):
        batch = W.Batch(i([0, 300]), i([300]), i([pages]))
        cache.write(batch, k, v)
        one = W.Batch(i([0, 1]), i([300]), i([pages]))
        got.append([*cache.read(batch, dtype=torch.float32), cache.attend(batch, q), cache.attend(one, q[:1])])
    worker.sync()
    for a, b in zip(*got):
        assert torch.equal(a, b)


# -- attention -----------------------------------------------------------------------
def check_attend(worker, p, q, scale=None, tree=None, layout=None):
    dev = q.to(worker.device)
    if layout is not None:
        dev = layout(dev)
    t = None if tree is None else tree.to(worker.device)
    out, lse = p.cache(W, worker).attend(p.batch(W, worker), dev, scale=scale, tree=t, lse=True)
    worker.sync()
    s = q.shape[2] ** -0.5 if scale is None else scale
    want, want_lse, bound, lse_bound = P.attend(p, q, s, tree)
    unit = P.UNIT[q.dtype]
    err = (out.cpu().double() - want).abs()
    bound = bound * (1 + unit) + want.abs() * unit + 2.0 ** -24
    assert bool((err <= bound).all()), float((err / bound).max())
    gone = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse.cpu()), gone)
    off = (lse.cpu().double() - want_lse).abs()[~gone]
    assert bool((off <= lse_bound[~gone]).all()), float((off / lse_bound[~gone]).max())
    assert bool((out.cpu()[gone] == 0).all())
    return out, lse


def queries(p, group, dtype, size=2.0):
    return (size * torch.randn(p.T, p.heads * group, p.dim, generator=p.g)).to(dtype)


STEPS = [(0, 1), (1, 1), (14, 1), (15, 1), (16, 1), (30, 1), (31, 1), (32, 1), (62, 1), (63, 1), (64, 1), (127, 1),
         (128, 1), (200, 0), (255, 1), (256, 1), (700, 1)]
CHUNKS = [(0, 1), (0, 2), (0, 17), (5, 0), (3, 16), (15, 31), (40, 33), (100, 70), (1, 130), (257, 5)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,heads,group,page", [
    (64, 2, 1, 16), (128, 2, 4, 16), (128, 1, 7, 64), (80, 3, 2, 32), (1, 1, 1, 16), (192, 1, 16, 128), (256, 2, 8, 256),
    (200, 1, 33, 16)])
@pytest.mark.parametrize("form", ["steps", "chunks"])
def test_attend(worker, fmt, dtype, dim, heads, group, page, form):
    say("attend", fmt, dtype, dim, heads, group, page, form)
    p = P.Paged(STEPS if form == "steps" else CHUNKS, page, heads, dim, fmt, seed=dim + group).fill()
    check_attend(worker, p, queries(p, group, dtype))


def random_tree(p, seed, empty=0.0):
    g = torch.Generator().manual_seed(seed)
    masks = []
    for m in p.rows:
        mine = []
        for i in range(m):
            up = int(torch.randint(-1, i, (1,), generator=g)) if i else -1
            v = (mine[up] if up >= 0 else 0) | 1 << i
            mine.append(v)
        mine = [0 if float(torch.rand(1, generator=g)) < empty else v for v in mine]
        masks += [v - (1 << 64) if v >> 63 else v for v in mine]
    return torch.tensor(masks, dtype=torch.int64)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim,heads,group,page", [(64, 2, 4, 16), (128, 1, 3, 32), (96, 2, 8, 64)])
def test_attend_trees(worker, fmt, dim, heads, group, page):
    say("tree", fmt, dim, heads, group, page)
    req = [(0, 1), (0, 24), (7, 64), (0, 64), (33, 16), (500, 9), (64, 0), (15, 17), (1000, 48)]
    p = P.Paged(req, page, heads, dim, fmt, seed=group).fill()
    tree = random_tree(p, 3, empty=0.3)
    q = queries(p, group, torch.bfloat16)
    out, lse = check_attend(worker, p, q, tree=tree)
    assert bool(torch.isinf(lse).any())            # rows that see nothing
    # bits past a request's rows are ignored
    more = tree.clone()
    for r, m in enumerate(p.rows):
        if m < 64:
            more[p.off[r]:p.off[r + 1]] |= torch.tensor(-1 << m, dtype=torch.int64)
    again = p.cache(W, worker).attend(p.batch(W, worker), q.to(worker.device), tree=more.to(worker.device))
    assert torch.equal(again, out)
    # a chain is what no tree means
    chain = torch.cat([torch.tensor([(1 << i + 1) - 1 if i < 63 else -1 for i in range(m)], dtype=torch.int64)
                       for m in p.rows])
    check_attend(worker, p, q, tree=chain)


@pytest.mark.parametrize("fmt", FORMATS)
def test_attend_what_a_row_does_not_see(worker, fmt):
    """A drafted token with NaN keys and values touches the rows that see it, and no other."""
    say("attend unseen", fmt)
    p = P.Paged([(20, 6), (0, 6), (300, 6)], 16, 2, 64, fmt, seed=4).fill()
    tree = random_tree(p, 8)
    q = queries(p, 4, torch.float16)
    cache, batch = p.cache(W, worker), p.batch(W, worker)
    dev, t = q.to(worker.device), tree.to(worker.device)
    want = cache.attend(batch, dev, tree=t)
    for which in (cache.k_scale, cache.v_scale):
        for r in range(3):
            page, slot = p.at(r, p.context[r] + 2)
            which[page, :, slot] = math.nan
        got = cache.attend(batch, dev, tree=t)
        worker.sync()
        for r in range(3):
            for row in range(p.off[r], p.off[r + 1]):
                if int(tree[row]) >> 2 & 1:
                    assert bool(torch.isnan(got[row]).all())
                else:
                    assert torch.equal(got[row], want[row])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("k_size,v_size,q_size", [(1e-6, 1e8, 3e6), (1e4, 1e-9, 1e-4), (1e-20, 1e25, 1e20), (30.0, 1.0, 5.0),
                                                  (0.0, 1.0, 1.0)])
def test_attend_sizes(worker, fmt, k_size, v_size, q_size):
    """Large and small keys, values and queries; scores that leave one token all the weight."""
    say("attend sizes", fmt, k_size, v_size, q_size)
    p = P.Paged([(0, 3), (100, 1), (333, 2)], 16, 2, 128, fmt, seed=6).fill(k_size, v_size)
    check_attend(worker, p, queries(p, 2, torch.bfloat16, q_size))


def test_attend_lengths_that_are_split(worker):
    say("attend split")
    p = P.Paged([(5000, 1), (20, 1), (9999, 1), (0, 1), (16384, 1)], 64, 1, 64, torch.int8, seed=2).fill()
    check_attend(worker, p, queries(p, 8, torch.float16))
    p = P.Paged([(3000, 8), (4100, 20)], 16, 1, 128, torch.float8_e4m3fn, seed=2).fill()
    check_attend(worker, p, queries(p, 4, torch.bfloat16))


def test_attend_layouts(worker):
    """Queries inside a fused projection's rows, heads outermost, unaligned; an output inside another."""
    say("attend layouts")
    p = P.Paged([(50, 3), (7, 20)], 16, 2, 64, torch.int8, seed=1).fill()
    q = queries(p, 2, torch.bfloat16)
    want, _ = check_attend(worker, p, q)

    def fused(d):
        whole = torch.zeros(d.shape[0], 3 * d.shape[1], d.shape[2], dtype=d.dtype, device=d.device)
        whole[:, :d.shape[1]] = d
        return whole[:, :d.shape[1]]

    def heads_first(d):
        return d.transpose(0, 1).contiguous().transpose(0, 1)

    def unaligned(d):
        whole = torch.zeros(d.shape[0], d.shape[1], d.shape[2] + 3, dtype=d.dtype, device=d.device)
        whole[..., 1:-2] = d
        return whole[..., 1:-2]

    for layout in (fused, heads_first, unaligned):
        got, _ = check_attend(worker, p, q, layout=layout)
        assert torch.equal(got, want)
    for layout in (fused, heads_first, unaligned):
        out = layout(torch.zeros_like(want))
        got = p.cache(W, worker).attend(p.batch(W, worker), q.to(worker.device), out=out)
        assert got is out and torch.equal(out, want)
    worker.sync()


def test_attend_scale_and_no_sums(worker):
    say("attend scale")
    p = P.Paged([(40, 2), (0, 5)], 16, 1, 64, torch.int8, seed=1).fill()
    q = queries(p, 4, torch.bfloat16)
    for scale in (1.0, -0.25, 0.0):
        out, _ = check_attend(worker, p, q, scale=scale)
        assert torch.equal(p.cache(W, worker).attend(p.batch(W, worker), q.to(worker.device), scale=scale), out)


# -- streams, graphs, repeated calls ---------------------------------------------------------
def step(cache, batch, ad, x, ids, q, k, v, tree):
    cache.write(batch, k, v)
    kv = cache.read(batch, dtype=torch.float32)
    return (ad.apply(x, ids), *cache.attend(batch, q, tree=tree, lse=True), *kv)


def step_inputs(worker, seed, requests):
    p = P.Paged(requests, 16, 2, 64, torch.int8, seed=seed).fill()
    d = adapt_inputs(seed, p.T, 6, 128, 256, 16, torch.bfloat16)
    dev = on(worker, d)
    r = lambda *s: torch.randn(*s, generator=p.g).to(torch.bfloat16).to(worker.device)  # noqa: E731
    return dict(cache=p.cache(W, worker), batch=p.batch(W, worker), ad=W.Adapters(worker, dev["down"], dev["up"]),
                x=dev["x"], ids=dev["adapter"], q=r(p.T, 8, 64), k=r(p.T, 2, 64), v=r(p.T, 2, 64),
                tree=random_tree(p, seed).to(worker.device))


def test_the_same_bits_every_time(worker):
    say("same bits")
    a = step_inputs(worker, 1, [(2000, 5), (37, 12), (0, 64), (9000, 1)])
    b = step_inputs(worker, 2, [(10, 5), (3, 1)])
    want = [t.clone() for t in step(**a)]
    for _ in range(3):
        step(**b)
        for x, y in zip(step(**a), want):
            assert torch.equal(x, y)
    worker.sync()


def test_another_stream(worker):
    say("another stream")
    a = step_inputs(worker, 3, [(2000, 5), (37, 12)])
    want = [t.clone() for t in step(**a)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    home = torch.cuda.current_stream()
    try:
        worker.ctx.set_stream(side)
        with torch.cuda.stream(side):
            got = step(**a)
        worker.sync()
    finally:
        worker.ctx.set_stream(home)
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    for x, y in zip(step(**a), want):
        assert torch.equal(x, y)
    worker.sync()


def test_captured_step():
    """A captured step replays with other inputs, lengths and pages, also after larger calls."""
    say("captured step")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        worker = W.Worker(O.Context(stream=stream))
        reqs = ([(1500, 5), (37, 12), (0, 3)], [(10, 5), (700, 12), (1490, 3)], [(63, 5), (0, 12), (1, 3)])
        sets = [step_inputs(worker, 10 + i, r) for i, r in enumerate(reqs)]
        a = sets[0]
        a["batch"]._rows.max_length = 1600
        pages = torch.full((3, 128), -1, dtype=torch.int32, device=worker.device)
        a["batch"]._keep += (pages,)
        pages[:, :a["batch"]._keep[2].shape[1]] = a["batch"]._keep[2]
        a["batch"]._rows.d_pages, a["batch"]._rows.max_pages = pages.data_ptr(), 128
        n = 1 + max(s["cache"].k.shape[0] for s in sets)
        big = W.Cache.empty(worker, n, 2, 64)
        a["cache"], first = big, a["cache"]
        step(**a)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            outs = step(**a)
        for rnd in range(2):
            for i, s in enumerate(sets):
                src = first if i == 0 else s["cache"]
                for name in ("k", "v", "k_scale", "v_scale"):
                    d, t = getattr(big, name), getattr(src, name)
                    d.view(torch.uint8)[:t.shape[0]] = t.view(torch.uint8)
                if i:
                    a["batch"]._keep[0].copy_(s["batch"]._keep[0])
                    a["batch"]._keep[1].copy_(s["batch"]._keep[1])
                    t = s["batch"]._keep[2]
                    pages.fill_(-1)
                    pages[:, :t.shape[1]] = t
                    for name in ("x", "ids", "q", "k", "v", "tree"):
                        a[name].copy_(s[name])
                elif rnd:
                    continue
                for o in outs:
                    o.fill_(-3.0)
                g.replay()
                torch.cuda.synchronize()
                want = step(**dict(s, cache=big, batch=a["batch"], ad=a["ad"]))
                torch.cuda.synchronize()
                for x, y in zip(outs, want):
                    assert torch.equal(x, y)
                # larger calls in between: the captured one keeps its scratch
                step(**step_inputs(worker, 50 + i, [(4000 << i, 60 >> i), (0, 64)]))
        worker.sync()
        del g


def test_scratch_cannot_grow_under_capture():
    say("capture without scratch")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        worker = W.Worker(O.Context(stream=stream))
        d = on(worker, adapt_inputs(1, 8, 2, 64, 64, 8, torch.bfloat16))
        ad = W.Adapters(worker, d["down"], d["up"])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            y = torch.zeros(8, 64, dtype=torch.bfloat16, device=worker.device)
            with pytest.raises(O.OrlojError) as ei:
                ad.apply(d["x"], d["adapter"], out=y)
            assert ei.value.code == O.ORLOJ_E_INVALID and "capture" in str(ei.value)
        g.replay()
        ad.apply(d["x"], d["adapter"])
        worker.sync()


# -- refusals ----------------------------------------------------------------------------
def data_error(worker, text):
    with pytest.raises(O.OrlojError) as ei:
        worker.sync()
    assert ei.value.code == O.ORLOJ_E_DATA and text in str(ei.value), str(ei.value)
    worker.sync()                                     # reported once


def test_data_errors(worker):
    """What is wrong in device data is reported, is not acted on, and leaves the other rows alone."""
    say("data errors")
    d = on(worker, adapt_inputs(1, 8, 4, 64, 64, 8, torch.bfloat16, none=0.0))
    ad = W.Adapters(worker, d["down"], d["up"])
    want = ad.apply(d["x"], d["adapter"])
    for wrong in (4, -2, 1 << 30):
        ids = d["adapter"].clone()
        ids[3] = wrong
        got = ad.apply(d["x"], ids)
        data_error(worker, "adapter-id")
        assert torch.equal(got[[0, 1, 2, 4, 5, 6, 7]], want[[0, 1, 2, 4, 5, 6, 7]])
    for wrong in (9, -1):
        ranks = torch.full((4,), 8, dtype=torch.int32, device=worker.device)
        ranks[int(d["adapter"][5])] = wrong
        W.Adapters(worker, d["down"], d["up"], rank=ranks).apply(d["x"], d["adapter"])
        data_error(worker, "rank")

    p = P.Paged([(40, 2), (7, 3), (100, 1)], 16, 2, 64, torch.int8, seed=1).fill()
    q = queries(p, 2, torch.bfloat16).to(worker.device)
    cache, b = p.cache(W, worker), p.batch(W, worker)
    want = cache.attend(b, q)
    off, length, pages = b._keep
    kept = [0, 1, 5]                                  # the rows of requests 0 and 2

    def run(text, **with_):
        t = dict(row_off=off, length=length, pages=pages, n_rows=6, max_rows=3, max_length=101)
        bad = W.Batch(**dict(t, **with_))
        got = cache.attend(bad, q)
        data_error(worker, text)
        assert torch.equal(got[kept], want[kept])
        kb, _ = cache.read(bad, dtype=torch.float32)
        data_error(worker, text)
        state = [t.view(torch.uint8).clone() for t in (cache.k, cache.v)]
        k = torch.ones(6, 2, 64, device=worker.device)
        cache.write(bad, k, k)
        data_error(worker, text)
        for t, s in zip((cache.k, cache.v), state):
            t.view(torch.uint8).copy_(s)
        scales = p.cache(W, worker)
        cache.k_scale.copy_(scales.k_scale)
        cache.v_scale.copy_(scales.v_scale)

    def changed(t, i, v):
        t = t.clone()
        t[i] = v
        return t

    run("length", length=changed(length, 1, 2))
    run("length", length=changed(length, 1, 102))
    run("length", length=changed(length, 1, -5))
    run("page", pages=changed(pages, (1, 0), p.n_pages))
    run("page", pages=changed(pages, (1, 0), -1))
    # offsets: a wrong one concerns the requests beside it
    kept = [0, 1]
    run("row-offsets", row_off=changed(off, 2, 1))
    run("row-offsets", row_off=changed(off, 3, 7))
    kept = [0, 1, 5]
    run("row-offsets", max_rows=2)


def test_refusals(worker):
    say("refusals")
    dev = worker.device
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device=dev)  # noqa: E731

    def refused(code, f):
        with pytest.raises(O.OrlojError) as ei:
            f()
        assert ei.value.code == code, str(ei.value)

    i32 = dict(dtype=torch.int32)
    ad = W.Adapters(worker, z(2, 8, 64), z(2, 32, 8))
    for bad in (lambda: W.Adapters(worker, z(2, 8, 64), z(2, 32, 4)),
                lambda: W.Adapters(worker, z(2, 8, 64), z(3, 32, 8)),
                lambda: W.Adapters(worker, z(2, 64, 8).transpose(1, 2), z(2, 32, 8)),
                lambda: W.Adapters(worker, z(2, 8, 64).cpu(), z(2, 32, 8)),
                lambda: W.Adapters(worker, z(2, 8, 64), z(2, 32, 8), scale=z(3, dtype=torch.float32)),
                lambda: ad.apply(z(4, 63), z(4, **i32)), lambda: ad.apply(z(4, 64), z(5, **i32)),
                lambda: ad.apply(z(64, 4).T, z(4, **i32)),
                lambda: ad.apply(z(4, 64), z(4, **i32), base=z(3, 32)),
                lambda: ad.apply(z(4, 64), z(4, **i32), out=z(5, 32))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: W.Adapters(worker, z(2, 8, 64, dtype=torch.float32), z(2, 32, 8, dtype=torch.float32)),
                lambda: ad.apply(z(4, 64, dtype=torch.float16), z(4, **i32)),
                lambda: ad.apply(z(4, 64), z(4, dtype=torch.int64))):
        with pytest.raises(TypeError):
            bad()
    refused(O.ORLOJ_E_UNSUPPORTED, lambda: W.Adapters(worker, z(1, 129, 8), z(1, 8, 129)).apply(z(1, 8), z(1, **i32)))
    y = z(4, 64)
    refused(O.ORLOJ_E_INVALID, lambda: ad.apply(z(4, 64), z(4, **i32), base=y[:2].view(4, 32), out=y[:, :32]))

    def cache_of(page=16, dim=64, heads=2, dtype=torch.int8):
        pad = W.dim_pad(dim)
        return W.Cache(worker, z(4, heads, page, pad, dtype=dtype), z(4, heads, page, pad, dtype=dtype),
                       z(4, heads, page, dtype=torch.float32), z(4, heads, page, dtype=torch.float32), dim)

    def batch_of(rows=2, length=4, **kw):
        return W.Batch(torch.tensor([0, rows], **i32).to(dev), torch.tensor([length], **i32).to(dev), z(1, 4, **i32), **kw)

    c, b = cache_of(), batch_of()
    assert (b.n_rows, b.max_rows, b.max_length) == (2, 2, 4)
    refused(O.ORLOJ_E_INVALID, lambda: cache_of(page=24).write(b, z(2, 2, 64), z(2, 2, 64)))
    refused(O.ORLOJ_E_INVALID, lambda: cache_of(page=512).read(b))
    refused(O.ORLOJ_E_UNSUPPORTED, lambda: cache_of(dim=257).attend(b, z(2, 2, 257)))
    refused(O.ORLOJ_E_INVALID, lambda: c.attend(b, z(2, 3, 64)))                      # 3 heads over 2
    refused(O.ORLOJ_E_INVALID, lambda: c.attend(b, z(2, 2, 64), scale=math.inf))
    refused(O.ORLOJ_E_UNSUPPORTED, lambda: c.attend(batch_of(65, 65), z(65, 2, 64), tree=z(65, dtype=torch.int64)))
    refused(O.ORLOJ_E_INVALID, lambda: c.attend(batch_of(n_rows=2, max_rows=-1, max_length=4), z(2, 2, 64)))
    refused(O.ORLOJ_E_UNSUPPORTED, lambda: c.read(batch_of(n_rows=2, max_rows=2, max_length=(1 << 30) + 1)))
    refused(O.ORLOJ_E_INVALID, lambda: c.attend(batch_of(n_rows=2, max_rows=1, max_length=4), z(2, 2, 64)))
    for bad in (lambda: W.Cache(worker, c.k, c.v, c.k_scale, c.v_scale, 65),
                lambda: W.Cache(worker, c.k, c.v, c.k_scale[:2], c.v_scale, 64),
                lambda: c.write(b, z(2, 2, 63), z(2, 2, 64)), lambda: c.write(b, z(3, 2, 64), z(2, 2, 64)),
                lambda: c.attend(b, z(2, 4, 32)), lambda: c.attend(b, z(2, 2, 64), tree=z(3, dtype=torch.int64)),
                lambda: c.attend(b, z(2, 64, 2).transpose(1, 2)),
                lambda: W.Batch(z(3, **i32), z(1, **i32), z(1, 4, **i32))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: c.attend(b, z(2, 2, 64, dtype=torch.float32)), lambda: c.read(b, dtype=torch.int8),
                lambda: c.write(b, z(2, 2, 64), z(2, 2, 64, dtype=torch.float16)),
                lambda: c.attend(b, z(2, 2, 64), tree=z(2, **i32)),
                lambda: W.Cache.empty(worker, 2, 2, 64, dtype=torch.uint8),
                lambda: W.Batch(z(2, dtype=torch.int64), z(1, **i32), z(1, 4, **i32))):
        with pytest.raises(TypeError):
            bad()
    worker.sync()


def test_nothing_to_do(worker):
    say("nothing to do")
    i32 = dict(dtype=torch.int32, device=worker.device)
    c = W.Cache.empty(worker, 0, 2, 64)
    none = W.Batch(torch.zeros(1, **i32), torch.zeros(0, **i32), torch.zeros(0, 3, **i32))
    z = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device=worker.device)
    c.write(none, z, z)
    assert c.read(none)[0].shape == (0, 2, 64) and c.attend(none, z).shape == (0, 2, 64)
    rest = W.Batch(torch.zeros(3, **i32), torch.zeros(2, **i32), torch.zeros(2, 0, **i32))
    c.write(rest, z, z)
    assert c.attend(rest, z).shape == (0, 2, 64)
    worker.sync()

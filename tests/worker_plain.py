"""Plain 64-bit forms of the worker's operators (CPU), and the inputs their tests share."""
import math

import torch

TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def adapt(x, adapter, down, up, scale=None, rank=None, base=None):
    """(y, bound): base + s B (A x) in 64 bits and, per element, the sum of the magnitudes of
    all products behind it."""
    x = x.double()
    y = torch.zeros(x.shape[0], up.shape[1], dtype=torch.float64)
    mag = torch.zeros_like(y)
    if base is not None:
        y += base.double()
    for t, a in enumerate(adapter.tolist()):
        R = down.shape[1] if rank is None else int(rank[a]) if a >= 0 else 0
        if a < 0 or R == 0:
            continue
        s = 1.0 if scale is None else float(scale[a])
        A, B = down[a, :R].double(), up[a, :, :R].double()
        y[t] += s * (B @ (A @ x[t]))
        mag[t] = abs(s) * (B.abs() @ (A.abs() @ x[t].abs()))
    return y, mag


def e4m3(u):
    """The nearest e4m3 numbers, ties to even, in 64 bits."""
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(u / step) * step


class Paged:
    """Requests on shuffled pages: contexts and rows as lists; every slot that holds no token, and
    every page of no request, holds garbage."""

    def __init__(self, requests, page, heads, dim, dtype, seed=0, spare=3):
        self.page, self.heads, self.dim, self.dtype = page, heads, dim, dtype
        self.context, self.rows = [c for c, _ in requests], [m for _, m in requests]
        self.length = [c + m for c, m in requests]
        self.off = [0]
        for m in self.rows:
            self.off.append(self.off[-1] + m)
        self.T = self.off[-1]
        self.pad = (dim + 63) // 64 * 64
        g = torch.Generator().manual_seed(seed)
        self.g = g
        need = [-(-n // page) for n in self.length]
        self.n_pages = sum(need) + spare
        ids = torch.randperm(self.n_pages, generator=g).tolist()
        self.max_pages = max(need + [1]) + 1
        self.table = torch.full((len(requests), self.max_pages), 0x7fffffff, dtype=torch.int32)
        for r, k in enumerate(need):
            self.table[r, :k] = torch.tensor(ids[:k], dtype=torch.int32)
            del ids[:k]
        # garbage: any code (NaN codes among them), NaN and infinite scales
        shape = (self.n_pages, heads, page)
        self.pool = {}
        for n in ("k", "v"):
            self.pool[n] = torch.randint(0, 256, shape + (self.pad,), dtype=torch.uint8, generator=g)
            s = torch.full(shape, math.nan)
            s[::2] = math.inf
            self.pool[n + "_scale"] = s

    def fill(self, k_size=1.0, v_size=1.0):
        """Random codes and scales for every token, in the pools and as 64-bit vectors."""
        self.dense = []
        for r, n in enumerate(self.length):
            entry = {}
            for name, size in (("k", k_size), ("v", v_size)):
                x = torch.randn(n, self.heads, self.dim, generator=self.g)
                scale = torch.exp(torch.randn(n, self.heads, generator=self.g)) * size / 64.0
                if self.dtype == torch.int8:
                    code = (x * 40).round().clamp(-127, 127).to(torch.int8)
                else:
                    code = (x * 40).to(torch.float8_e4m3fn)
                entry[name] = code.double() * scale.double()[..., None]
                raw = torch.zeros(n, self.heads, self.pad, dtype=torch.uint8)
                raw[..., :self.dim] = code.view(torch.uint8)
                for t in range(0, n, self.page):
                    p, m = int(self.table[r, t // self.page]), min(self.page, n - t)
                    self.pool[name][p, :, :m] = raw[t:t + m].transpose(0, 1)
                    self.pool[name + "_scale"][p, :, :m] = scale[t:t + m].T
            self.dense.append(entry)
        return self

    def at(self, r, t):
        return int(self.table[r, t // self.page]), t % self.page

    def cache(self, W, worker):
        d = {n: (p if n.endswith("scale") else p.view(self.dtype)).to(worker.device) for n, p in self.pool.items()}
        return W.Cache(worker, d["k"], d["v"], d["k_scale"], d["v_scale"], head_dim=self.dim)

    def batch(self, W, worker, **bounds):
        d = worker.device
        i = lambda v: torch.tensor(v, dtype=torch.int32, device=d)  # noqa: E731
        b = dict(n_rows=self.T, max_rows=max(self.rows + [0]), max_length=max(self.length + [0]))
        return W.Batch(i(self.off), i(self.length), self.table.to(d), **dict(b, **bounds))


def attend(paged, q, scale, tree=None):
    """(out, lse, bound, lse_bound) in 64 bits.  The bounds are those of the arithmetic the operator
    promises: a query with 11 significant bits of its row's largest element (exact for the elements
    within 2^-14 of it), scores summed in 32 bits, weights with 11 significant bits."""
    T, Hq, D = q.shape
    group = Hq // paged.heads
    out = torch.zeros(T, Hq, D, dtype=torch.float64)
    bound = torch.zeros_like(out)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    lse_bound = torch.zeros_like(lse)
    qd = q.double()
    for r, n in enumerate(paged.length):
        a, b = paged.off[r], paged.off[r + 1]
        ctx = n - (b - a)
        for row in range(a, b):
            i = row - a
            if tree is None:
                sees = torch.arange(n) <= ctx + i
            else:
                m = int(tree[row]) & ((1 << 64) - 1)
                sees = torch.tensor([t < ctx or bool(m >> (t - ctx) & 1) for t in range(n)], dtype=torch.bool)
            if not bool(sees.any()):
                continue
            k = paged.dense[r]["k"][sees].repeat_interleave(group, 1)      # [n][Hq][D]
            v = paged.dense[r]["v"][sees].repeat_interleave(group, 1)
            s = scale * torch.einsum("hd,nhd->hn", qd[row], k)
            size = abs(scale) * torch.einsum("hd,nhd->hn", qd[row].abs(), k.abs())
            coarse = abs(scale) * torch.einsum("h,nhd->hn", qd[row].abs().amax(-1), k.abs())
            ds = (size * ((D + 8) * 2.0 ** -24) + coarse * 2.0 ** -25 + s.abs() * 2.0 ** -22).amax(-1)
            lse[row] = torch.logsumexp(s, -1)
            p = torch.exp(s - lse[row][:, None])
            out[row] = torch.einsum("hn,nhd->hd", p, v)
            mag = torch.einsum("hn,nhd->hd", p, v.abs())
            N = s.shape[1]
            rel = 2.0 ** -10 + 2 * ds + (N + 64) * 2.0 ** -24
            # weights far below the largest: absolute rounding of 2^-24 of it
            floor = (p.amax(-1) * 2.0 ** -24)[:, None] * v.abs().amax(0) * N
            bound[row] = mag * rel[:, None] + floor
            lse_bound[row] = ds + (N + 64) * 2.0 ** -24 + 2.0 ** -22 * (1 + s.abs().amax(-1))
    return out, lse, bound, lse_bound


UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}

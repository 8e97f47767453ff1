"""Plain 64-bit reference of the paged cache's operators, window by window, on the CPU, and the inputs of their tests."""
import math

import torch

F8 = torch.float8_e4m3fn
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "fp8": (torch.bfloat16, F8), "f32": (torch.float32, torch.float32)}


class Cache:
    """Pools, page table and lengths of a test, on the CPU; `dev` uploads what a call takes."""

    def __init__(self, seed, type="bf16", B=2, K=3, n_q=4, n_kv=2, D=64, page=16, lens=(5, 70), rows=None, extra_pages=2, order="pshd", layers=0):
        g = self.g = torch.Generator().manual_seed(seed)
        self.type, self.B, self.K, self.n_q, self.n_kv, self.D, self.page = type, B, K, n_q, n_kv, D, page
        self.dtype, self.kv_dtype = TYPES[type]
        self.lens = list(lens)
        assert len(self.lens) == B
        self.rows = rows
        need = [-(-(n + K + 1) // page) for n in self.lens]
        self.width = max(need)
        self.n_pages = sum(need) + extra_pages
        perm = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.table = torch.full((B, self.width), -1, dtype=torch.int32)
        at = 0
        for b in range(B):
            self.table[b, : need[b]] = perm[at : at + need[b]]
            at += need[b]
        # memory order of pages, slots and heads, as the pool's strides say
        shape = {"p": self.n_pages, "s": page, "h": n_kv}
        lead = (layers,) if layers else ()
        self.scales = (0.03, 0.02) if type == "fp8" else (1.0, 1.0)
        self.pools = []
        for scale in self.scales:
            x = torch.randn(*lead, *[shape[o] for o in order[:3]], D, generator=g) / scale
            x = self.store(x)
            back = [order.index(o) for o in "psh"]
            x = x.permute(*range(len(lead)), *[len(lead) + i for i in back], len(lead) + 3)
            self.pools.append(x)
        self.strides = dict(zip(("page_stride", "slot_stride", "head_stride"), self.pools[0].stride()[len(lead) :]))

    def store(self, x):
        return x.clamp(-448, 448).to(F8) if self.kv_dtype == F8 else x.to(self.kv_dtype)

    def dev_pools(self):
        out = []
        for p in self.pools:
            flat = torch.empty(p.numel(), dtype=torch.uint8 if p.dtype == F8 else p.dtype)
            q = flat.as_strided(p.shape, p.stride())
            q.copy_(p.view(torch.uint8) if p.dtype == F8 else p)
            d = flat.cuda().as_strided(p.shape, p.stride())
            out.append(d)
        return out

    def host(self, d):
        """A device pool's values as the CPU pools have them."""
        x = d.cpu()
        return x.view(F8) if self.kv_dtype == F8 else x

    def create(self, aj, **more):
        return aj.aj_cache_create(self.B, self.K, self.n_q, self.n_kv, self.D, self.page, self.n_pages, self.width,
                                  aj.AJ_F32 if self.type == "f32" else aj.AJ_BF16, aj.AJ_KV_FP8_E4M3 if self.type == "fp8" else aj.AJ_KV_SAME,
                                  **{**self.strides, **more})

    def n_rows(self, b):
        return self.K + 1 if self.rows is None else max(0, min(self.K + 1, self.rows[b]))

    def i32(self, x):
        return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")

    def slot(self, b, t):
        """(page, slot) of a token, or None if it is nowhere."""
        e = t // self.page
        if e >= self.width:
            return None
        p = int(self.table[b, e])
        return (p, t % self.page) if 0 <= p < self.n_pages else None


def random_tree(g, K, back=3):
    """Parents of K nodes, each under one of the `back` before it (or the root)."""
    return [max(-1, j - 1 - int(torch.randint(0, back, (1,), generator=g))) for j in range(K)]


def tree_rows(parent):
    """(depth per row, list of ancestor-or-self sets per row) of one tree, walked node by node."""
    depth, sets = [0], [{0}]
    for j, p in enumerate(parent):
        p = max(-1, min(p, j - 1))
        depth.append(depth[p + 1] + 1)
        sets.append(sets[p + 1] | {j + 1})
    return depth, sets


def masks(sets):
    words = (len(sets) + 31) // 32
    m = torch.zeros(len(sets), words, dtype=torch.int64)
    for r, s in enumerate(sets):
        for j in s:
            m[r, j // 32] |= 1 << (j % 32)
    return torch.where(m >= 2**31, m - 2**32, m).to(torch.int32)


def sees(c, b, r, t, window, sinks, depth=None, sets=None):
    """Whether row r of window b sees token t."""
    L = max(0, c.lens[b])
    d = lambda j: j if depth is None else max(0, min(depth[b][j], j))  # noqa: E731
    if t >= L:
        j = t - L
        if j > r or (sets is not None and j not in sets[b][r]):
            return False
    if c.slot(b, t) is None:
        return False
    pos = t if t < L else L + d(t - L)
    return not window or L + d(r) - pos < window or pos < sinks


def attend(c, q, scale, window=0, sinks=0, depth=None, sets=None):
    """out, lse, and how far off each may be, in 64 bits; rows that are not there are NaN.

    Weights of bf16 calls are rounded to bf16 (half a step, 2^-8 of each), and outputs are.  Scores are fp32 sums of D products: off by at most
    (D + 2) 2^-24 sum |q k| scale; a weight is off by twice the largest of these (its own and the sum's) and by the sum's own n + 8 roundings."""
    R, G = c.K + 1, c.n_q // c.n_kv
    out = torch.full((c.B, R, c.n_q, c.D), math.nan, dtype=torch.float64)
    tol = torch.zeros_like(out)
    lse = torch.full((c.B, R, c.n_q), math.nan, dtype=torch.float64)
    lse_tol = torch.zeros_like(lse)
    half = 2.0**-8 if c.type != "f32" else 2.0**-24
    for b in range(c.B):
        L = max(0, c.lens[b])
        T = min(L + c.n_rows(b), c.width * c.page)
        vis = torch.zeros(c.n_rows(b), T, dtype=torch.bool)
        for r in range(c.n_rows(b)):
            for t in range(T):
                vis[r, t] = sees(c, b, r, t, window, sinks, depth, sets)
        where = [c.slot(b, t) or (0, 0) for t in range(T)]
        pg, sl = torch.tensor([w[0] for w in where], dtype=torch.long), torch.tensor([w[1] for w in where], dtype=torch.long)
        wide = lambda p: (p.view(torch.uint8)[pg, sl].view(F8) if p.dtype == F8 else p[pg, sl]).double()  # noqa: E731
        k, v = wide(c.pools[0]) * c.scales[0], wide(c.pools[1]) * c.scales[1]
        for r in range(c.n_rows(b)):
            at = vis[r].nonzero().flatten()
            if not len(at):
                out[b, r], lse[b, r] = 0.0, -math.inf
                continue
            kk, vv = k[at].repeat_interleave(G, 1), v[at].repeat_interleave(G, 1)      # [n, n_q, D]
            x = q[b, r].double()
            s = (kk * x).sum(2) * scale
            err = (c.D + 2) * 2.0**-24 * ((kk * x).abs().sum(2) * scale).amax(0)        # [n_q]
            p = torch.softmax(s, 0)
            out[b, r] = (p[..., None] * vv).sum(0)
            size = (p[..., None] * vv.abs()).sum(0)
            weight = (half if c.type != "f32" else 0.0) + 2 * err[:, None] + (len(at) + 8) * 2.0**-24
            tol[b, r] = 1.01 * weight * size + half * (out[b, r].abs() + weight * size) + 1e-30
            lse[b, r] = torch.logsumexp(s, 0)
            lse_tol[b, r] = err + (len(at) + 8) * 2.0**-24 + 2.0**-22 * lse[b, r].abs()
    return out, lse, tol, lse_tol


def rotated(x, pos, inv_freq, rot, interleaved):
    """x [n, heads, D] in 64 bits turned by pos [n]."""
    y = x.clone()
    a = pos[:, None, None].double() * inv_freq.double()
    i = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
    j = i + 1 if interleaved else i + rot // 2
    y[..., i] = x[..., i] * a.cos() - x[..., j] * a.sin()
    y[..., j] = x[..., j] * a.cos() + x[..., i] * a.sin()
    return y


def normed(x, w, eps):
    x = x.double()
    return x if w is None else x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()

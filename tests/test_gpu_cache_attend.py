"""aj_cache_attend against the 64-bit reference: single tokens, chains and trees, windows and sinks, every storage type, ragged lengths and rows,
page sizes, memory orders, and slots that hold no visible token filled with NaN."""
import math

import pytest
import torch

import cache_ref as ref

pytestmark = pytest.mark.gpu


def poison(c):
    """NaN in every slot that no token of a window has."""
    used = torch.zeros(c.n_pages, c.page, dtype=torch.bool)
    for b in range(c.B):
        for t in range(max(0, c.lens[b]) + c.n_rows(b)):
            if (s := c.slot(b, t)):
                used[s] = True
    for p in c.pools:
        if p.dtype == ref.F8:
            p.view(torch.uint8)[~used] = 0x7F
        else:
            p[~used] = math.nan


def run(c, q, scale, window=0, sinks=0, depth=None, sets=None, lse=True, q_stride=0, stream=None):
    import paper_2504_20039_amd as aj
    R = c.K + 1
    pools = c.dev_pools()
    h = c.create(aj, window=window, sinks=sinks, q_stride=q_stride)
    dq = q.flatten(2).cuda()
    if q_stride:
        wide = torch.full((c.B, R, q_stride), math.nan, dtype=c.dtype, device="cuda")
        wide[..., : dq.shape[2]] = dq
        dq = wide
    out = torch.full((c.B, R, c.n_q * c.D), 9.0, dtype=c.dtype, device="cuda")
    out_lse = torch.full((c.B, R, c.n_q), 9.0, device="cuda") if lse else None
    mask = None if sets is None else torch.stack([ref.masks(s) for s in sets]).cuda()
    args = (h, dq, *pools, c.table.cuda(), c.i32(c.lens), scale, out)
    kw = dict(lse=out_lse, n_rows=c.i32(c.rows), depth=c.i32(depth), mask=mask, k_scale=c.scales[0], v_scale=c.scales[1])
    aj.aj_cache_attend(*args, **kw)
    torch.cuda.synchronize()
    first = out.clone()
    aj.aj_cache_attend(*args, **kw)      # the same bits again
    torch.cuda.synchronize()
    bits = torch.int32 if c.type == "f32" else torch.int16
    assert torch.equal(first.view(bits), out.view(bits))
    aj.aj_cache_destroy(h)
    return out.cpu().view(c.B, R, c.n_q, c.D).double(), None if out_lse is None else out_lse.cpu().double()


def check(c, q, got, got_lse, **kw):
    want, lse, tol, lse_tol = ref.attend(c, q, **kw)
    for b in range(c.B):
        n = c.n_rows(b)
        assert (got[b, n:] == 9.0).all()
        err = (got[b, :n] - want[b, :n]).abs()
        assert (err <= tol[b, :n]).all(), (b, err.max().item(), (err / tol[b, :n]).max().item())
        if got_lse is not None:
            assert (got_lse[b, n:] == 9.0).all()
            none = lse[b, :n] == -math.inf
            assert torch.equal(got_lse[b, :n] == -math.inf, none)
            e = torch.where(none, 0.0, got_lse[b, :n] - lse[b, :n]).abs()
            assert (e <= lse_tol[b, :n]).all(), (b, e.max().item())


def queries(c, size=2.0):
    return (torch.randn(c.B, c.K + 1, c.n_q, c.D, generator=c.g) * size).to(c.dtype)


CASES = [
    # one new token: lengths around the tiles' borders, none and one cached token, head layouts
    dict(type="bf16", K=0, B=9, lens=(0, 1, 31, 62, 63, 64, 126, 127, 128), n_q=8, n_kv=1, D=128),
    dict(type="bf16", K=0, B=3, lens=(5000, 17, 0), n_q=7, n_kv=1, D=128, page=64),
    dict(type="bf16", K=0, B=2, lens=(255, 700), n_q=6, n_kv=6, D=64, page=1),
    dict(type="bf16", K=0, B=1, lens=(3000,), n_q=40, n_kv=1, D=128, page=256),
    dict(type="bf16", K=0, B=2, lens=(300, 65), n_q=4, n_kv=2, D=256, page=32, order="phsd"),
    dict(type="fp8", K=0, B=4, lens=(0, 1300, 64, 191), n_q=8, n_kv=2, D=128, page=16),
    dict(type="fp8", K=0, B=2, lens=(500, 3), n_q=4, n_kv=4, D=64, page=2),
    dict(type="fp8", K=0, B=2, lens=(200, 129), n_q=2, n_kv=1, D=256),
    dict(type="f32", K=0, B=4, lens=(0, 900, 63, 64), n_q=4, n_kv=2, D=128),
    dict(type="f32", K=0, B=2, lens=(70, 200), n_q=3, n_kv=3, D=256, page=8),
    # chains
    dict(type="bf16", K=3, B=3, lens=(0, 61, 130), n_q=8, n_kv=1, D=128, page=4),
    dict(type="bf16", K=16, B=2, lens=(1000, 5), n_q=8, n_kv=2, D=128, rows=(17, 6)),
    dict(type="bf16", K=33, B=3, lens=(40, 0, 222), n_q=14, n_kv=2, D=64, rows=(0, 34, -1)),
    dict(type="bf16", K=64, B=2, lens=(200, 63), n_q=16, n_kv=2, D=128),
    dict(type="bf16", K=300, B=1, lens=(10,), n_q=2, n_kv=1, D=128, page=8),
    dict(type="bf16", K=20, B=2, lens=(100, 90), n_q=4, n_kv=1, D=256),
    dict(type="fp8", K=40, B=2, lens=(100, 257), n_q=8, n_kv=2, D=128),
    dict(type="fp8", K=9, B=2, lens=(33, 300), n_q=12, n_kv=1, D=256, page=8),
    dict(type="f32", K=40, B=2, lens=(100, 0), n_q=8, n_kv=2, D=64),
    dict(type="f32", K=70, B=1, lens=(77,), n_q=2, n_kv=1, D=128, order="hpsd"),
    dict(type="f32", K=34, B=2, lens=(5, 40), n_q=2, n_kv=2, D=256),
    # items in two, a few and many pieces, equal ones and ragged ones
    dict(type="bf16", K=37, B=5, lens=(1000, 600, 129, 0, 2100), n_q=4, n_kv=1, D=128),
    dict(type="bf16", K=37, B=6, lens=(520,) * 6, n_q=8, n_kv=2, D=128, page=64),
    dict(type="bf16", K=31, B=1, lens=(2500,), n_q=8, n_kv=2, D=64),
    dict(type="bf16", K=40, B=2, lens=(900, 2000), n_q=4, n_kv=1, D=256),
    dict(type="bf16", K=7, B=3, lens=(2500, 40, 700), n_q=4, n_kv=1, D=256, page=1),
    dict(type="fp8", K=33, B=3, lens=(1500, 256, 700), n_q=16, n_kv=2, D=128),
    dict(type="fp8", K=0, B=3, lens=(900, 20, 1700), n_q=16, n_kv=2, D=256, page=2),
    dict(type="f32", K=33, B=2, lens=(600, 1200), n_q=2, n_kv=1, D=64),
    dict(type="f32", K=33, B=1, lens=(700,), n_q=2, n_kv=1, D=256),
    dict(type="f32", K=0, B=2, lens=(1500, 33), n_q=8, n_kv=1, D=256, page=4),
    dict(type="f32", K=2, B=2, lens=(1500, 333), n_q=8, n_kv=1, D=128, rows=(3, 0)),
    # odd head sizes
    dict(type="bf16", K=5, B=2, lens=(64, 300), n_q=6, n_kv=2, D=80),
    dict(type="bf16", K=0, B=2, lens=(64, 300), n_q=5, n_kv=1, D=16),
    dict(type="bf16", K=30, B=1, lens=(90,), n_q=6, n_kv=2, D=208),
    dict(type="fp8", K=2, B=2, lens=(63, 200), n_q=6, n_kv=2, D=96),
    dict(type="fp8", K=0, B=1, lens=(140,), n_q=4, n_kv=2, D=48, order="phsd"),
    dict(type="f32", K=6, B=2, lens=(70, 64), n_q=4, n_kv=2, D=112),
    dict(type="f32", K=0, B=1, lens=(190,), n_q=4, n_kv=4, D=32, page=2),
    # windows and sinks
    dict(type="bf16", K=0, B=4, lens=(1000, 30, 64, 129), n_q=8, n_kv=2, D=128, window=64, sinks=4),
    dict(type="bf16", K=0, B=2, lens=(700, 300), n_q=4, n_kv=1, D=128, window=1, sinks=0),
    dict(type="bf16", K=12, B=2, lens=(500, 0), n_q=8, n_kv=2, D=128, window=7, sinks=1, page=1),
    dict(type="bf16", K=70, B=2, lens=(300, 20), n_q=4, n_kv=1, D=64, window=50, sinks=130, rows=(71, 40)),
    dict(type="fp8", K=3, B=3, lens=(640, 70, 5), n_q=8, n_kv=1, D=128, window=200, sinks=64, page=64),
    dict(type="f32", K=20, B=2, lens=(400, 64), n_q=4, n_kv=2, D=64, window=33, sinks=3),
    dict(type="bf16", K=40, B=2, lens=(100, 0), n_q=4, n_kv=1, D=64, window=2**31 - 1, sinks=2**31 - 1),
    dict(type="bf16", K=400, B=2, lens=(100, 0), n_q=2, n_kv=1, D=64, window=2**31 - 1, tree=5),
    # trees
    dict(type="bf16", K=15, B=3, lens=(100, 0, 63), n_q=8, n_kv=2, D=128, tree=3),
    dict(type="bf16", K=100, B=2, lens=(64, 31), n_q=8, n_kv=1, D=128, tree=20),
    dict(type="bf16", K=60, B=2, lens=(200, 9), n_q=4, n_kv=1, D=64, tree=2, window=6, sinks=2),
    dict(type="fp8", K=32, B=2, lens=(333, 17), n_q=16, n_kv=2, D=128, tree=3, rows=(33, 10)),
    dict(type="f32", K=36, B=2, lens=(20, 100), n_q=2, n_kv=1, D=128, tree=2, window=40, sinks=0),
]


@pytest.mark.parametrize("p", CASES, ids=lambda p: "-".join(f"{k}{v}" for k, v in p.items()).replace(" ", "")[:90])
def test_attend(p):
    p = dict(p)
    window, sinks, tree = (p.pop(k, 0) for k in ("window", "sinks", "tree"))
    c = ref.Cache(21, **p)
    poison(c)
    q = queries(c)
    depth = sets = None
    if tree:
        rows = [ref.tree_rows(ref.random_tree(c.g, c.K, tree)) for _ in range(c.B)]
        depth, sets = [r[0] for r in rows], [r[1] for r in rows]
    kw = dict(scale=c.D**-0.5, window=window, sinks=sinks, depth=depth, sets=sets)
    check(c, q, *run(c, q, **kw), **kw)


@pytest.mark.parametrize("type", ["bf16", "fp8", "f32"])
def test_masks_that_leave_rows_empty(type):
    """Without cached tokens, mask rows may be empty; bits behind a row count for nothing; depths are clamped; no lse."""
    c = ref.Cache(4, type=type, K=9, B=3, lens=(0, 0, 80), n_q=4, n_kv=1, D=64)
    poison(c)
    q = queries(c)
    sets = [[set() if r % 2 else {r, 9} for r in range(10)], [set() for _ in range(10)], [set() if r == 3 else {0, r} for r in range(10)]]
    depth = [[r + 50 for r in range(10)], [-r for r in range(10)], [r // 2 for r in range(10)]]
    kw = dict(scale=0.3, window=5, sinks=0, depth=depth, sets=sets)
    got, lse = run(c, q, **kw)
    check(c, q, got, lse, **kw)
    assert (got[1] == 0).all() and (got[0, 1] == 0).all()
    got2, none = run(c, q, lse=False, **kw)
    assert none is None and torch.equal(got, got2)


@pytest.mark.parametrize("type", ["bf16", "fp8", "f32"])
def test_pages_that_are_nowhere(type):
    """Bad page numbers anywhere, a window whose tokens all are, lengths behind the table, negative lengths."""
    c = ref.Cache(9, type=type, K=4, B=6, page=8, lens=(200, 30, 100, 64, 3, 0), n_q=8, n_kv=2, D=128)
    c.table[0, [0, 7, 9, 24]] = torch.tensor([-1, c.n_pages, 2**31 - 1, -2**31], dtype=torch.int32)
    c.table[1, :] = -1
    c.lens[2] = c.width * c.page - 2          # rows 2 and on are behind the table
    c.table[2] = torch.where(c.table[2] < 0, c.table[3, 0], c.table[2])
    c.lens[3] = c.width * c.page + 1000       # all rows are
    c.table[3] = torch.where(c.table[3] < 0, c.table[3, 0], c.table[3])
    c.lens[4] = -7
    poison(c)
    q = queries(c)
    for window, sinks in ((0, 0), (90, 2), (3, 0)):
        kw = dict(scale=0.1, window=window, sinks=sinks)
        got, lse = run(c, q, **kw)
        check(c, q, got, lse, **kw)
        assert (got[1] == 0).all() and (lse[1] == -math.inf).all()


def test_pages_outside_the_window_may_be_gone():
    """Tokens between the sinks and the window lie on pages that were given back: NaN there, or no page at all."""
    c = ref.Cache(13, K=5, B=2, page=16, lens=(600, 300), n_q=8, n_kv=2, D=128)
    for b, L in ((0, 600), (1, 300)):
        for e in range(1, (L - 99) // 16):
            if e % 2:
                for p in c.pools:
                    p[int(c.table[b, e])] = math.nan
            else:
                c.table[b, e] = -1
        for p in c.pools:     # and inside the pages at the borders
            p[int(c.table[b, 0]), 3:] = math.nan
            e, s = divmod(L - 99, 16)
            p[int(c.table[b, e]), :s] = math.nan
    q = queries(c)
    kw = dict(scale=0.1, window=100, sinks=3)
    got, lse = run(c, q, **kw)
    assert torch.isfinite(got).all()
    for p in c.pools:         # (the reference multiplies by zero)
        p[torch.isnan(p)] = 0.0
    check(c, q, got, lse, **kw)


@pytest.mark.parametrize("type", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("K", [5, 40])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_nan_and_infinity_in_tokens_that_a_row_does_not_see(type, K, D):
    """A draft row whose state overflowed: rows that do not see it are as if it were not there, rows that do are NaN or infinite."""
    c = ref.Cache(17, type=type, K=K, B=2, lens=(60, 100), n_q=8, n_kv=2, D=D)
    q = queries(c)
    kw = dict(scale=0.1)
    want, want_lse, tol, lse_tol = ref.attend(c, q, **kw)      # without them
    sk, sv = c.slot(0, 60 + 3), c.slot(1, 100 + 2)
    if type == "fp8":
        c.pools[0].view(torch.uint8)[sk] = 0x7F
        c.pools[1].view(torch.uint8)[sv] = 0x7F
    else:
        c.pools[0][sk] = math.nan
        c.pools[1][sv][:, ::2] = math.nan
        c.pools[1][sv][:, 1] = math.inf
    got, lse = run(c, q, **kw)
    near = (got - want).abs() <= tol
    near_lse = (lse - want_lse).abs() <= lse_tol
    for b, r in ((0, 3), (1, 2)):
        assert near[b, :r].all() and near_lse[b, :r].all()
    assert torch.isnan(got[0, 3:]).all()
    if type == "fp8":
        assert torch.isnan(got[1, 2:]).all()
    else:
        assert torch.isnan(got[1, 2:, :, ::2]).all() and (got[1, 2:, :, 1] == math.inf).all()
        assert near[1, 2:, :, 3].all()
    assert near_lse[1].all()


@pytest.mark.parametrize("type", ["bf16", "f32"])
def test_large_scores(type):
    """Scores far apart, far from zero, and a maximum that keeps rising along the cache."""
    c = ref.Cache(2, type=type, K=2, B=2, lens=(700, 400), n_q=4, n_kv=1, D=64)
    q = queries(c, 1.0)
    for b, L in ((0, 700), (1, 400)):
        for t in range(L + 3):
            c.pools[0][c.slot(b, t)] *= 0.1 + t / 100.0
    c.pools[0].add_(5.0)
    kw = dict(scale=3.0)
    check(c, q, *run(c, q, **kw), **kw)


def test_rows_apart():
    c = ref.Cache(6, K=7, B=2, lens=(100, 20), n_q=4, n_kv=2, D=64)
    poison(c)
    q = queries(c)
    kw = dict(scale=0.125)
    check(c, q, *run(c, q, q_stride=4 * 64 + 24, **kw), **kw)


def test_offsets_beyond_32_bits():
    """A pool of 5 GB whose pages lie at both ends."""
    import paper_2504_20039_amd as aj
    D, page, n_pages = 128, 16, 1 << 19
    k, v = (torch.empty(n_pages, page, 2, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g = torch.Generator().manual_seed(1)
    table = torch.tensor([[0, n_pages - 1, 7, n_pages - 2, n_pages // 2 + 1]], dtype=torch.int32)
    small = ref.Cache(1, B=1, K=1, lens=(70,), n_q=4, n_kv=2, D=D, page=page, extra_pages=0)
    small.table = torch.arange(5, dtype=torch.int32)[None]
    for i, p in enumerate(table[0].tolist()):
        k[p], v[p] = small.pools[0][i].cuda(), small.pools[1][i].cuda()
    q = torch.randn(1, 2, 4, D, generator=g).to(torch.bfloat16)
    out = torch.zeros(1, 2, 4 * D, dtype=torch.bfloat16, device="cuda")
    h = aj.aj_cache_create(1, 1, 4, 2, D, page, n_pages, 5)
    aj.aj_cache_attend(h, q.flatten(2).cuda(), k, v, table.cuda(), small.i32([70]), 0.1, out)
    x = torch.randn(1, 2, 2 * D, generator=g).to(torch.bfloat16).cuda()
    aj.aj_cache_append(h, q.flatten(2).cuda(), x, x, None, None, 0.0, None, table.cuda(), small.i32([62]), torch.empty_like(out), k, v)
    torch.cuda.synchronize()
    aj.aj_cache_destroy(h)
    check(small, q, out.cpu().view(1, 2, 4, D).double(), None, scale=0.1)
    assert torch.equal(k[n_pages - 2, 14].flatten(), x[0, 0]) and torch.equal(v[n_pages - 2, 15].flatten(), x[0, 1])


def test_refusals():
    import paper_2504_20039_amd as aj
    c = ref.Cache(6, K=3, B=1, lens=(9,), n_q=4, n_kv=2, D=64)
    h = c.create(aj)
    k, v = c.dev_pools()
    q = torch.zeros(1, 4, 256, dtype=torch.bfloat16, device="cuda")
    out, t, n = torch.full_like(q, 9.0), c.table.cuda(), c.i32(c.lens)
    lib, P = aj.load_library(), lambda x: x.data_ptr()

    def attend(q=P(q), k=P(k), v=P(v), t=P(t), n=P(n), scale=0.1, ks=1.0, vs=1.0, out=P(out)):
        return lib.aj_cache_attend(h, q, k, v, t, n, None, None, None, scale, ks, vs, out, None, None)

    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(t=None), dict(n=None), dict(out=None), dict(q=P(q) + 2), dict(k=P(k) + 8), dict(t=P(t) + 2),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(scale=1e-44), dict(ks=2.0), dict(vs=0.5), dict(vs=math.nan)):
        assert attend(**bad) == -1, bad

    def append(q=P(q), k=P(q), v=P(q), eps=1e-5, t=P(t), n=P(n), out=P(out), kp=P(k), vp=P(v), ks=1.0):
        return lib.aj_cache_append(h, q, k, v, None, None, eps, None, t, n, None, None, ks, 1.0, out, kp, vp, None)

    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(t=None), dict(n=None), dict(out=None), dict(kp=None), dict(vp=None), dict(q=P(q) + 4),
                dict(vp=P(v) + 4), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(ks=0.5), dict(n=P(n) + 1)):
        assert append(**bad) == -1, bad

    def commit(m=P(t), node=P(n), t=P(t), n=P(n), layers=1, stride=0, kp=P(k), vp=P(v), new=P(out)):
        return lib.aj_cache_commit(h, m, node, t, n, layers, stride, kp, vp, new, None)

    for bad in (dict(m=None), dict(node=None), dict(t=None), dict(n=None), dict(layers=-1), dict(layers=2), dict(layers=2, stride=100), dict(layers=2, stride=-64),
                dict(kp=None), dict(vp=P(v) + 8), dict(new=None), dict(new=P(n)), dict(m=P(t) + 1)):
        assert commit(**bad) == -1, bad
    torch.cuda.synchronize()
    assert (out == 9.0).all()
    aj.aj_cache_destroy(h)
    empty = aj.aj_cache_create(0, 3, 4, 2, 64, 16, 1, 1)
    assert lib.aj_cache_attend(empty, None, None, None, None, None, None, None, None, 1.0, 1.0, 1.0, None, None, None) == 0
    assert lib.aj_cache_append(empty, None, None, None, None, None, 0.0, None, None, None, None, None, 1.0, 1.0, None, None, None, None) == 0
    assert lib.aj_cache_commit(empty, None, None, None, None, 1, 0, None, None, None, None) == 0
    aj.aj_cache_destroy(empty)


@pytest.mark.parametrize("B", [128, 129, 256, 257, 600])
def test_many_windows(B):
    """More windows than a workgroup has threads; some without rows."""
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 90, (B,), generator=g).tolist()
    rows = torch.randint(0, 3, (B,), generator=g).tolist()
    c = ref.Cache(B, K=1, B=B, page=8, lens=lens, rows=rows, n_q=2, n_kv=1, D=64)
    poison(c)
    q = queries(c)
    kw = dict(scale=0.2)
    check(c, q, *run(c, q, **kw), **kw)
    c = ref.Cache(B, type="f32", K=20, B=B, page=8, lens=[n % 7 for n in lens], rows=[20 * n for n in rows], n_q=2, n_kv=1, D=16)
    q = queries(c)
    check(c, q, *run(c, q, **kw), **kw)


def test_no_rows_at_all():
    c = ref.Cache(1, K=2, B=3, lens=(4, 0, 9), rows=(0, 0, -2), n_q=2, n_kv=1, D=64)
    q = queries(c)
    check(c, q, *run(c, q, scale=0.2), scale=0.2)

"""The paged cache's operators together, as a server's step runs them: masks of the draft trees, every layer's new rows and attention, the
verification of the trees, the accepted path kept in all layers, and the next token over what was kept; the same under graph capture and on two
streams at once."""
import pytest
import torch

import cache_ref as ref

pytestmark = pytest.mark.gpu
EPS, LAYERS = 1e-5, 2


class Model:
    """Two layers' queries, keys and values for trees of K nodes, and a cache for them with room for what follows."""

    def __init__(self, type, seed=3, B=3, K=12, lens=(40, 0, 131)):
        self.c = c = ref.Cache(seed, type=type, B=B, K=K, n_q=8, n_kv=2, D=64, page=16, lens=lens, layers=LAYERS)
        g = c.g
        self.parent = torch.tensor([ref.random_tree(g, K) for _ in range(B)], dtype=torch.int32)
        self.x = [[torch.randn(B, K + 1, n, 64, generator=g).to(c.dtype) for n in (8, 2, 2)] for _ in range(LAYERS)]
        self.w = [[(1 + 0.2 * torch.randn(64, generator=g)).to(c.dtype) for _ in range(2)] for _ in range(LAYERS)]
        self.inv_freq = (10000.0 ** (-torch.arange(0, 64, 2).double() / 64)).float()

    def layer(self, i):
        """The cache of one layer, as the reference reads it."""
        c = ref.Cache.__new__(ref.Cache)
        c.__dict__.update(self.c.__dict__)
        c.pools = [p[i] for p in self.c.pools]
        return c


def verify(aj, w, hidden, parent, B, K, d_t):
    """aj_verify_tree on the last layer's output: lengths and nodes."""
    V = 512
    g = torch.Generator().manual_seed(8)
    W = (torch.randn(V, d_t, generator=g) * 0.02).to(hidden.dtype).cuda()
    clf = (torch.randn(d_t, generator=g) / d_t**0.5).to(hidden.dtype).cuda()
    h = aj.aj_create(B, K, d_t, 0, V, w)
    out = [torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(3)]
    # half of the nodes carry the greedy token of their parent's row
    logits = hidden.view(B, K + 1, d_t).float() @ W.float().T
    tok = logits.argmax(2)
    rows = (parent.long() + 1).cuda()
    draft = torch.where(torch.rand(B, K, generator=g).cuda() < 0.7, torch.gather(tok, 1, rows), 7).to(torch.int32)
    aj.aj_verify_tree(h, hidden, None, W, draft, parent.cuda(), clf, 0.0, 0.5, *out)
    torch.cuda.synchronize()
    aj.aj_destroy(h)
    return out


@pytest.mark.parametrize("type", ["bf16", "fp8", "f32"])
def test_a_step_of_draft_trees(type):
    import paper_2504_20039_amd as aj
    m = Model(type)
    c = m.c
    B, K, R = c.B, c.K, c.K + 1
    pools = c.dev_pools()
    table, lens = c.table.cuda(), c.i32(c.lens)
    depth = torch.zeros(B, R, dtype=torch.int32, device="cuda")
    mask = torch.zeros(B, R, (R + 31) // 32, dtype=torch.int32, device="cuda")
    aj.aj_tree_mask(B, K, m.parent.cuda(), depth, mask)
    h = c.create(aj, rot_dim=64)
    rows = [ref.tree_rows(p) for p in m.parent.tolist()]
    depths, sets = [r[0] for r in rows], [r[1] for r in rows]
    for i in range(LAYERS):
        q, k, v = (t.flatten(2).cuda() for t in m.x[i])
        wq, wk = (t.cuda() for t in m.w[i])
        q_out, out = torch.empty_like(q), torch.empty_like(q)
        kw = dict(depth=depth, k_scale=c.scales[0], v_scale=c.scales[1])
        aj.aj_cache_append(h, q, k, v, wq, wk, EPS, m.inv_freq.cuda(), table, lens, q_out, pools[0][i], pools[1][i], **kw)
        aj.aj_cache_attend(h, q_out, pools[0][i], pools[1][i], table, lens, 0.125, out, mask=mask, **kw)
        torch.cuda.synchronize()
        # the reference reads what was stored, and the queries that were written
        for n in range(2):
            c.pools[n][i] = c.host(pools[n])[i]
        want, _, tol, _ = ref.attend(m.layer(i), q_out.cpu().view(B, R, 8, 64), 0.125, depth=depths, sets=sets)
        got = out.cpu().view(B, R, 8, 64).double()
        assert ((got - want).abs() <= tol).all()
    out_len, _, out_node = verify(aj, aj.AJ_F32 if type == "f32" else aj.AJ_BF16, out, m.parent, B, K, 512)
    new_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    aj.aj_cache_commit(h, mask, out_node, table, lens, LAYERS, pools[0].stride(0), *pools, new_len)
    torch.cuda.synchronize()
    aj.aj_cache_destroy(h)
    assert torch.equal(new_len, lens + 1 + out_len)
    assert (out_len > 0).any()

    # the next token sees the context and the accepted path, in order
    node = out_node.tolist()
    kept = [sorted(sets[b][node[b] + 1]) for b in range(B)]
    one = ref.Cache.__new__(ref.Cache)
    one.__dict__.update(c.__dict__)
    one.K, one.lens, one.rows = 0, new_len.tolist(), None
    h1 = one.create(aj)
    q = torch.randn(B, 1, 8, 64, generator=c.g).to(c.dtype)
    k, v = (torch.randn(B, 1, 2, 64, generator=c.g).to(c.dtype) for _ in range(2))
    for i in range(LAYERS):
        got, q_out = (torch.empty(B, 1, 512, dtype=c.dtype, device="cuda") for _ in range(2))
        kw = dict(k_scale=c.scales[0], v_scale=c.scales[1])
        aj.aj_cache_append(h1, q.flatten(2).cuda(), k.flatten(2).cuda(), v.flatten(2).cuda(), None, None, 0.0, None, table, new_len, q_out, pools[0][i], pools[1][i], **kw)
        aj.aj_cache_attend(h1, q_out, pools[0][i], pools[1][i], table, new_len, 0.125, got, **kw)
        torch.cuda.synchronize()
        # by hand: the path's rows as they were stored, the new token behind them
        after = [c.host(p)[i] for p in pools]
        bits = lambda t: t.view(torch.uint8) if t.dtype == ref.F8 else t  # noqa: E731
        one.pools = [bits(p[i]).clone().view(p.dtype) for p in c.pools]
        for b in range(B):
            for n in range(2):
                for j, r in enumerate(kept[b]):
                    at = c.slot(b, c.lens[b] + j)
                    bits(one.pools[n])[at] = bits(c.pools[n][i])[c.slot(b, c.lens[b] + r)]
                at = c.slot(b, one.lens[b])
                bits(one.pools[n])[at] = bits(after[n])[at]
                for t in range(one.lens[b] + 1):
                    assert torch.equal(bits(one.pools[n])[one.slot(b, t)], bits(after[n])[one.slot(b, t)])
        want, _, tol, _ = ref.attend(one, q, 0.125)
        assert ((got.cpu().view(B, 1, 8, 64).double() - want).abs() <= tol).all()
    aj.aj_cache_destroy(h1)


@pytest.mark.parametrize("type,K,lens", [("bf16", 12, (40, 0, 131)), ("fp8", 0, (900, 70, 3)), ("f32", 40, (20, 300, 64)), ("bf16", 40, (2000, 5, 700))])
def test_a_captured_step_replays_like_the_eager_one(type, K, lens):
    """Append, attend and commit in one graph; the lengths, the nodes and the rows change between replays, and eager calls of the same handle run in between."""
    import paper_2504_20039_amd as aj
    m = Model(type, K=max(K, 1), lens=lens)
    c = m.c
    c.K = K
    B, R = c.B, K + 1
    pools = c.dev_pools()
    keep = [p.clone() for p in pools]
    table, lens_d = c.table.cuda(), c.i32(c.lens)
    depth = torch.zeros(B, R, dtype=torch.int32, device="cuda")
    mask = torch.ones(B, R, (R + 31) // 32, dtype=torch.int32, device="cuda")
    node = torch.zeros(B, dtype=torch.int32, device="cuda")
    q, k, v = (t[:, :R].flatten(2).contiguous().cuda() for t in m.x[0])
    q_out, out = torch.empty_like(q), torch.empty_like(q)
    new_len = torch.zeros_like(lens_d)
    h = c.create(aj, rot_dim=64)
    inv_freq, w = m.inv_freq.cuda(), [t.cuda() for t in m.w[0]]
    parent = m.parent.cuda()

    def step(o=out, n=new_len):
        kw = dict(depth=depth, k_scale=c.scales[0], v_scale=c.scales[1])
        if K:
            aj.aj_tree_mask(B, K, parent, depth, mask)
        aj.aj_cache_append(h, q, k, v, *w, EPS, inv_freq, table, lens_d, q_out, pools[0][0], pools[1][0], **kw)
        aj.aj_cache_attend(h, q_out, pools[0][0], pools[1][0], table, lens_d, 0.125, o, mask=mask, **kw)
        aj.aj_cache_commit(h, mask, node, table, lens_d, LAYERS, pools[0].stride(0), *pools, n)

    def restore():
        for p, s in zip(pools, keep):
            p.copy_(s)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for rnd in range(4):
        lens_d.copy_(torch.tensor([max(0, n - 17 * rnd) for n in c.lens], dtype=torch.int32))
        node.copy_(torch.tensor([K - 1 - rnd % max(K, 1)] * B, dtype=torch.int32))
        q.add_(0.25)
        parent.copy_(torch.tensor([ref.random_tree(c.g, max(K, 1)) for _ in range(B)], dtype=torch.int32))
        restore()
        eager_out, eager_len = torch.empty_like(out), torch.empty_like(new_len)
        step(eager_out, eager_len)
        torch.cuda.synchronize()
        eager_pools = [p.clone() for p in pools]
        restore()
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        same = lambda a, b: torch.equal(a.view(torch.uint8), b.view(torch.uint8))  # noqa: E731
        assert same(out, eager_out) and torch.equal(new_len, eager_len)
        assert all(same(p.contiguous(), e.contiguous()) for p, e in zip(pools, eager_pools))
    aj.aj_cache_destroy(h)


def test_two_handles_on_two_streams():
    """Calls of different handles that overlap in time; each result is that of the call alone."""
    import paper_2504_20039_amd as aj
    work = []
    for seed, type, K, lens in ((1, "bf16", 0, (3000, 700)), (2, "bf16", 40, (500, 900)), (3, "fp8", 6, (2000, 64)), (4, "f32", 20, (100, 300))):
        c = ref.Cache(seed, type=type, K=K, B=2, lens=lens, n_q=8, n_kv=2, D=128)
        q = torch.randn(2, K + 1, 8 * 128, generator=c.g).to(c.dtype).cuda()
        pools = c.dev_pools()
        kw = dict(k_scale=c.scales[0], v_scale=c.scales[1])
        args = (q, *pools, c.table.cuda(), c.i32(c.lens), 0.1)
        h = c.create(aj)
        alone = torch.empty_like(q)
        aj.aj_cache_attend(h, *args, alone, **kw)
        work.append((h, args, kw, alone, torch.cuda.Stream(), [torch.empty_like(q) for _ in range(6)]))
    torch.cuda.synchronize()
    for i in range(6):
        for h, args, kw, _, stream, outs in work:
            aj.aj_cache_attend(h, *args, outs[i], stream=stream, **kw)
    torch.cuda.synchronize()
    for h, _, _, alone, _, outs in work:
        assert all(torch.equal(alone, o) for o in outs)
        aj.aj_cache_destroy(h)

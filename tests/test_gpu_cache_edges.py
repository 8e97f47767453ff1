"""aj_cache_attend where masks, infinities, scales and lengths are at their edges."""
import copy
import math

import pytest
import torch

import cache_ref as ref
from test_gpu_cache_attend import check, poison, queries, run

pytestmark = pytest.mark.gpu
NAN8 = 0x7F


def put(c, pool, at, x):
    if c.type == "fp8":
        c.pools[pool].view(torch.uint8)[at] = NAN8
    else:
        c.pools[pool][at] = x


@pytest.mark.parametrize("type", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("K,rows", [(0, None), (6, (1, 1, 1, 1)), (6, (1, 7, 1, 3))])
@pytest.mark.parametrize("heads", [(4, 2, 64), (40, 1, 128), (2, 1, 256), (6, 2, 80)], ids=str)
def test_a_lone_row_whose_mask_leaves_out_itself(type, K, rows, heads):
    """One live row, its own bit clear: its slot may hold anything.  It sees the cached tokens, or nothing."""
    n_q, n_kv, D = heads
    c = ref.Cache(31, type=type, K=K, B=4, lens=(0, 64, 1, 900), rows=rows, n_q=n_q, n_kv=n_kv, D=D)
    poison(c)
    for b, bad in enumerate((math.nan, math.inf, -math.inf, math.nan)):
        put(c, 0, c.slot(b, c.lens[b]), math.nan)
        put(c, 1, c.slot(b, c.lens[b]), bad)
    q = queries(c)
    kw = dict(scale=D**-0.5, sets=[[set(range(1, r + 1)) for r in range(K + 1)] for _ in range(4)])
    got, lse = run(c, q, **kw)
    check(c, q, got, lse, **kw)
    assert (got[0, 0] == 0).all() and (lse[0, 0] == -math.inf).all()


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("K,lens", [(0, (70, 1500)), (40, (70, 500))])
@pytest.mark.parametrize("D", [16, 48, 64, 80, 112, 128, 144, 208, 256])
def test_infinite_keys_whose_weight_is_zero(type, K, lens, D):
    """A score of -infinity is a weight of zero at every head size: as if the token were nowhere."""
    c = ref.Cache(32, type=type, K=K, B=2, lens=lens, n_q=4, n_kv=1, D=D, page=1)
    q = queries(c)
    q[..., 0], q[..., D - 1] = q[..., 0].abs() + 0.5, q[..., D - 1].abs() + 0.5
    without = copy.copy(c)
    without.table = c.table.clone()
    for b, t, e in ((0, 3, 0), (0, 66, D - 1), (1, lens[1] // 2, 0), (1, lens[1] - 1, D - 1)):
        c.pools[0][c.slot(b, t)][:, e] = -math.inf
        without.table[b, t] = -1
    got, lse = run(c, q, scale=0.1)
    check(without, q, got, lse, scale=0.1)


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("K,lens", [(0, (70, 1500)), (40, (70, 500))])
@pytest.mark.parametrize("D", [64, 80, 256])
def test_rows_whose_scores_are_all_minus_infinity(type, K, lens, D):
    """Nothing has any weight: zeros, whatever the values are."""
    c = ref.Cache(34, type=type, K=K, B=2, lens=lens, n_q=4, n_kv=1, D=D)
    q = queries(c)
    q[..., 1] = q[..., 1].abs() + 0.5
    c.pools[0][..., 1] = -math.inf
    c.pools[1][c.slot(0, 5)], c.pools[1][c.slot(1, lens[1])] = math.inf, math.nan
    got, lse = run(c, q, scale=0.1)
    assert (got == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("type,scale", [("bf16", 1.6e-38), ("f32", 0.9e-38), ("f32", 1.6e-38), ("fp8", 5e-37)])
@pytest.mark.parametrize("K,lens", [(0, (3000, 20)), (40, (700, 0))])
@pytest.mark.parametrize("D", [64, 256])
def test_the_smallest_scales(type, scale, K, lens, D):
    """Scales at the lower end of the normal numbers: nearly equal weights, and others with large queries and keys.

    (The sums q . k themselves are held in fp32: here 2^118 times sums of D products of deviation 2, up to 6 times 2 sqrt(D) <= 2^7.6 in all.)"""
    c = ref.Cache(33, type=type, K=K, B=2, lens=lens, n_q=4, n_kv=2, D=D)
    q = queries(c)
    check(c, q, *run(c, q, scale=scale), scale=scale)
    if type != "fp8":
        q *= 2.0**58
        c.pools[0] *= 2.0**60
        check(c, q, *run(c, q, scale=scale), scale=scale)


@pytest.mark.parametrize("weight", [0.7, 0.9])
@pytest.mark.parametrize("D,G", [(16, 1), (64, 40), (128, 1), (256, 1)])
def test_long_sums_of_equal_weights(weight, D, G):
    """An uncut item of 131072 tokens in fp32, all but a few of the same weight: sums that take one token at a time drift by 2 10^-4, since in a binade every addition rounds
    the same way.

    A lane's part of the sum: at most 64 weights of a tile, one after another, and tiles with what their additions lost; the weights' argument and exponential:
    within 4 steps; then the logarithm as in the reference: 80 2^-24.  Values: products of a tile one after another, then 2048 or 4096 tiles,
    each addition off by half a step: (tiles / 2 + 80) 2^-24 of the values' size."""
    import paper_2504_20039_amd as aj
    n, page, B = 1 << 17, 1 << 16, 512
    g = torch.Generator().manual_seed(5)
    k = torch.zeros(3, page, 1, D)
    k[..., 0] = math.log(weight)
    k[0, :128, :, 0] = 0.0
    v = 0.5 + torch.rand(3, page, 1, D, generator=g)
    v[..., 1] = 1.0
    q = torch.zeros(B, 1, G, D)
    q[..., 0] = 1.0
    h = aj.aj_cache_create(B, 0, G, 1, D, page, 3, 3, aj.AJ_F32)
    table = torch.tensor([[0, 1, 2]], dtype=torch.int32).expand(B, 3).contiguous().cuda()
    out, lse = torch.empty(B, 1, G * D, device="cuda"), torch.empty(B, 1, G, device="cuda")
    aj.aj_cache_attend(h, q.flatten(2).cuda(), k.cuda(), v.cuda(), table, torch.full((B,), n - 1, dtype=torch.int32, device="cuda"), 1.0, out, lse=lse)
    torch.cuda.synchronize()
    aj.aj_cache_destroy(h)
    w = torch.exp(k.flatten(0, 1)[:n, 0, 0].double())
    want_lse, want = w.sum().log(), (w[:, None] * v.flatten(0, 1)[:n, 0].double()).sum(0) / w.sum()
    assert ((lse.double().cpu() - want_lse).abs() <= 80 * 2.0**-24 + 2.0**-22 * want_lse).all(), (lse.double().cpu() - want_lse).abs().max().item()
    err = (out.double().cpu().view(B, G, D) / want - 1).abs().max().item()
    assert err <= (n / 32 / 2 + 80) * 2.0**-24, err


@pytest.mark.parametrize("type", ["bf16", "fp8"])
@pytest.mark.parametrize("D,G", [(16, 1), (64, 40), (128, 1), (128, 40), (256, 1), (256, 40)])
def test_long_sums_of_equal_weights_in_16_bits(type, D, G):
    """As above: a lane adds at most 2048 tiles, each addition off by half a step, to sums of at most 64 weights.  The weight and the result are rounded to bf16, half a step
    each."""
    import paper_2504_20039_amd as aj
    n, page, B = 1 << 17, 1 << 16, 512
    g = torch.Generator().manual_seed(6)
    kv = ref.TYPES[type][1]
    k = torch.zeros(3, page, 1, D)
    k[..., 0] = math.log(0.7)
    k[0, :128, :, 0] = 0.0
    k, v = k.to(kv), (0.5 + torch.rand(3, page, 1, D, generator=g)).to(kv)
    q = torch.zeros(B, 1, G, D, dtype=torch.bfloat16)
    q[..., 0] = 1.0
    h = aj.aj_cache_create(B, 0, G, 1, D, page, 3, 3, aj.AJ_BF16, aj.AJ_KV_FP8_E4M3 if type == "fp8" else aj.AJ_KV_SAME)
    table = torch.tensor([[0, 1, 2]], dtype=torch.int32).expand(B, 3).contiguous().cuda()
    out, lse = torch.empty(B, 1, G * D, dtype=torch.bfloat16, device="cuda"), torch.empty(B, 1, G, device="cuda")
    aj.aj_cache_attend(h, q.flatten(2).cuda(), k.cuda(), v.cuda(), table, torch.full((B,), n - 1, dtype=torch.int32, device="cuda"), 1.0, out, lse=lse)
    torch.cuda.synchronize()
    aj.aj_cache_destroy(h)
    k, v = (x.float().double().flatten(0, 1)[:n, 0] for x in (k, v))
    w = torch.exp(k[:, 0])
    want_lse, want = w.sum().log(), (w[:, None] * v).sum(0) / w.sum()
    assert ((lse.double().cpu() - want_lse).abs() <= (2048 / 2 + 80) * 2.0**-24 + 2.0**-22 * want_lse).all(), (lse.double().cpu() - want_lse).abs().max().item()
    assert (out.double().cpu().view(B, G, D) / want - 1).abs().max().item() <= 2.0**-7 * 1.01

"""hs_tree_verify_attention_paged where values of very different sizes meet: in tokens of one tile, in tiles of one split, in splits, in nodes that a row's mask hides.  What a row
loses is bounded by what it weighs itself: 2^-24 of its largest product of a weight and that token's largest value, for every key."""
import math

import numpy as np
import pytest
import torch

from oracle import paged
from paged_route import route
from paged_util import attention64, i32, make_trees, masks
from paper_2505_13254_b200 import binding as hb

pytestmark = pytest.mark.gpu

LOG2 = math.log(2.0)
SCALE = 128 ** -0.5


def shared_cache(batch, K, V, page=64):
    """(cache, K, V as the cache holds them): every sequence has the same tokens [n, hkv, 128], in the same pages."""
    n, hkv = K.shape[:2]
    pages = max(1, -(-n // page))
    pools, held = [], []
    for x in (K, V):
        byte, scale = paged.quantise(x)
        held.append(paged.dequantise(byte, scale))
        pad = pages * page - n
        byte, scale = np.concatenate([byte, np.full((pad, hkv, 128), 127, np.uint8)]), np.concatenate([scale, np.full((pad, hkv), 255, np.uint8)])
        pools.append((byte.reshape(pages, page, hkv, 128).transpose(0, 2, 1, 3), scale.reshape(pages, page, hkv).transpose(0, 2, 1)))
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    cache = hb.KvCache(t(pools[0][0]), t(pools[1][0]), t(pools[0][1]), t(pools[1][1]), i32([list(range(pages))] * batch), i32([n] * batch))
    return cache, held[0], held[1]


def check(out, lse, q, K, V, kt, vt, mask, apart=True):
    """The bound, term by term: the bf16 output, half a step of 2^-8; P in f16 and the partials of splits in f16, 2^-11 of the weighted mean of |v| each; scores off by delta change a
    weight by e^delta - 1, and the sum as much, with what fp32 sums and ex2 add, 2^-16; of every key 2^-24 of the row's largest product of a weight and its token's largest value.  Tree values of 2^10 and more are apart: their
    token counts as 2^11 there, and the partials keep 2^-38 of such a product."""
    d = lambda a: torch.as_tensor(np.asarray(a), dtype=torch.float64, device="cuda") if not torch.is_tensor(a) else a.double()
    want, want_lse, mean, delta, _ = attention64(q, K, V, kt, vt, mask, SCALE)
    G, n, cached = q.shape[1] // kt.shape[1], len(q), len(K)
    vis = torch.cat([torch.ones(n, cached, dtype=torch.bool, device="cuda"), torch.as_tensor(mask, device="cuda")], 1)
    s = torch.einsum("nhd,khd->hnk", d(q), torch.cat([d(K), d(kt)]).repeat_interleave(G, 1)) * SCALE
    w = torch.softmax(s.masked_fill(~vis, -math.inf), 2).masked_fill(~vis, 0)
    size, tree = d(V).abs().amax(2), d(vt).abs().amax(2)
    ordinary = torch.cat([size, torch.where(tree >= 2.0 ** 10, 2.0 ** 11, tree)]).repeat_interleave(G, 1).T[:, None]
    top, far = (w * ordinary).amax(2).T, (w * torch.cat([size, tree]).repeat_interleave(G, 1).T[:, None]).amax(2).T
    e = delta[:, :, None]
    bound = 2.0 ** -8 * want.abs() + (2 * 2.0 ** -11 + 2 * torch.expm1(e) + 2.0 ** -16) * mean * (1 + 2.0 ** -8)
    bound += (vis.sum(1)[:, None] * 2.0 ** -24 * top + 2.0 ** -38 * far)[:, :, None]
    err = (out.double() - want).abs()
    assert not torch.isnan(out).any()
    assert (err <= bound).all(), float((err / bound.clamp_min(1e-300)).max())
    assert ((lse.double() - want_lse).abs() <= delta + 2.0 ** -18 + 2.0 ** -22 * want_lse.abs()).all()


def run(ctx, pr, cache, q, k, v, nodes):
    lse = torch.zeros(q.shape[:2], device="cuda")
    out = hb.hs_tree_verify_attention_paged(ctx, pr, cache, q, k, v, max_nodes=max(nodes), max_kv_len=int(cache.kv_len.max()), lse_out=lse)
    assert hb.hs_device_error(ctx) == 0
    return out, lse


def hide(pr, first, nodes, hidden):
    """Node `hidden` of every tree is seen by its own row only."""
    words = pr.anc_mask.clone()
    for f, n in zip(first, nodes):
        own = words[f + hidden].clone()
        words[f:f + n, hidden >> 6] &= ~(1 << (hidden & 63))
        words[f + hidden] = own
    pr.anc_mask.copy_(words)


SHAPES = [  # batch, nodes, hq, hkv, tokens, (rows of a block, splits)
    (1, 5, 4, 1, 3000, (32, 16)), (1, 7, 16, 2, 3000, (64, 16)), (1, 60, 8, 2, 3000, (128, 16)), (10, 60, 32, 8, 4096, (256, 3)), (19, 5, 32, 8, 1000, (32, 1)),
    (16, 60, 32, 8, 300, (256, 1)),
]


def random_case(batch, nodes, hq, hkv, tokens, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    cache, K, V = shared_cache(batch, rng.standard_normal((tokens, hkv, 128)), rng.standard_normal((tokens, hkv, 128)))
    ctx, _, pr = make_trees([nodes] * batch, seed)
    rn = lambda h: torch.randn(batch * nodes, h, 128, device="cuda", generator=g).bfloat16()
    return ctx, pr, cache, K, V, rn(hq), rn(hkv), rn(hkv)


@pytest.mark.parametrize("other", [2.0 ** 40, -2.0 ** 90, 2.0 ** 99])
@pytest.mark.parametrize("batch, nodes, hq, hkv, tokens, how", SHAPES)
def test_a_huge_value_costs_the_rows_that_mask_it_nothing_whatever_they_see(batch, nodes, hq, hkv, tokens, how, other):
    """Nodes 2 and 3 are seen by their own rows only; the rows of 2 see 2^20 beside a sibling that is larger by far."""
    assert route(batch, nodes, hq, hkv, tokens) == how
    ctx, pr, cache, K, V, q, k, v = random_case(batch, nodes, hq, hkv, tokens, 31)
    first = [b * nodes for b in range(batch)]
    hide(pr, first, [nodes] * batch, 2)
    hide(pr, first, [nodes] * batch, 3)
    words = pr.anc_mask.clone()
    for f in first:
        words[f + 2, 0] &= ~8
        words[f + 3, 0] &= ~4
        v[f + 2, :, 5], v[f + 3, :, 7] = 2.0 ** 20, other
    pr.anc_mask.copy_(words)
    out, lse = run(ctx, pr, cache, q, k, v, [nodes] * batch)
    for b, m in list(enumerate(masks(pr, [nodes] * batch)))[::7]:
        r, rows = slice(first[b], first[b] + nodes), [i for i in range(nodes) if i != 3]
        small = v[r].clone()
        small[3] = 0                                                     # (seen by none of the rows that are looked at)
        check(out[r][rows], lse[r][rows], q[r][rows], K, V, k[r], small, m[rows])
    ctx.close()


def level_case(batch, nodes, hq, hkv, tokens, gap, V, levels=None, seed=1):
    """Scores in the hand: queries 1/2 in every place, cached keys `levels` (1) in theirs, the tree's so that their scores lie `gap` binades above a cached one's."""
    K = np.ones((tokens, hkv, 128)) * (1.0 if levels is None else levels[:, None, None])
    cache, K, V = shared_cache(batch, K, V)
    ctx, _, pr = make_trees([nodes] * batch, seed)
    n = batch * nodes
    full = lambda h, x: torch.full((n, h, 128), x, device="cuda").bfloat16()
    return ctx, pr, cache, K, V, full(hq, 0.5), full(hkv, 1.0 + gap * LOG2 / (64 * SCALE)), full(hkv, 1.0)


LONG = [(19, 2, 32, 8, 7680, (32, 1)), (19, 12, 32, 8, 7680, (64, 1)), (19, 30, 32, 8, 7680, (128, 1)), (16, 60, 32, 8, 7680, (256, 1)), (1, 60, 32, 8, 7680, (128, 8))]


@pytest.mark.parametrize("gap, value", [(13, 1e6), (14, -2.0 ** 19 * 1.9), (14, 1000.0), (12, -50.0)])
@pytest.mark.parametrize("batch, nodes, hq, hkv, tokens, how", LONG)
def test_a_hidden_value_costs_the_prefix_nothing(batch, nodes, hq, hkv, tokens, how, gap, value):
    """A few heavy tree keys before thousands of light cached ones that make up half of the sum."""
    assert route(batch, nodes, hq, hkv, tokens) == how
    ctx, pr, cache, K, V, q, k, v = level_case(batch, nodes, hq, hkv, tokens, gap, -np.ones((tokens, hkv, 128)))
    first = [b * nodes for b in range(batch)]
    hide(pr, first, [nodes] * batch, 1)
    for f in first:
        v[f + 1] = value
    out, lse = run(ctx, pr, cache, q, k, v, [nodes] * batch)
    for b, m in list(enumerate(masks(pr, [nodes] * batch)))[::9]:
        rows, r = [i for i in range(nodes) if i != 1], slice(first[b], first[b] + nodes)
        check(out[r][rows], lse[r][rows], q[r][rows], K, V, k[r], v[r], m[rows])
        check(out[r][1:2], lse[r][1:2], q[r][1:2], K, V, k[r], v[r], m[1:2])
    ctx.close()


@pytest.mark.parametrize("size", [2.0 ** 30, -2.0 ** 16, 2.0 ** 90])
@pytest.mark.parametrize("batch, nodes, hq, hkv, tokens, how", LONG)
def test_a_cached_value_of_no_weight_costs_nothing(batch, nodes, hq, hkv, tokens, how, size):
    """One early token of a huge value whose score lies far below the others'."""
    rng = np.random.default_rng(7)
    V, levels = rng.uniform(-1.2, -0.8, (tokens, hkv, 128)), rng.choice([0.875, 1.0, 1.125], tokens)
    V[5], levels[5] = size, -15.0                                       # 16 * 64 / sqrt(128) nats below the others, 2^-130
    ctx, pr, cache, K, V, q, k, v = level_case(batch, nodes, hq, hkv, tokens, 0, V, levels)
    out, lse = run(ctx, pr, cache, q, k, v, [nodes] * batch)
    for b, m in list(enumerate(masks(pr, [nodes] * batch)))[::9]:
        r = slice(b * nodes, (b + 1) * nodes)
        check(out[r], lse[r], q[r], K, V, k[r], v[r], m)
    ctx.close()


@pytest.mark.parametrize("spread", [6, 7, 12, 40])
@pytest.mark.parametrize("batch, nodes, hq, hkv, tokens, how", LONG)
def test_tokens_of_every_size_weigh_as_they_should(batch, nodes, hq, hkv, tokens, how, spread):
    """The larger a token's values, the smaller its weight, so that all of them make up the row, in tiles whose sizes differ by 2^spread."""
    rng = np.random.default_rng(spread)
    exponent = rng.integers(-(spread // 2), spread - spread // 2 + 1, tokens)
    V = rng.uniform(0.5, 1.0, (tokens, hkv, 128)) * rng.choice([-1.0, 1.0], (1, hkv, 128)) * 2.0 ** exponent[:, None, None]
    levels = -exponent * LOG2 / (64 * SCALE)
    ctx, pr, cache, K, V, q, k, v = level_case(batch, nodes, hq, hkv, tokens, 8, V, levels)
    g = torch.Generator(device="cuda").manual_seed(spread)
    v *= torch.exp2(torch.randint(-(spread // 2), min(spread - spread // 2, 9) + 1, (len(v), hkv, 1), device="cuda", generator=g).float()).bfloat16()
    out, lse = run(ctx, pr, cache, q, k, v, [nodes] * batch)
    for b, m in list(enumerate(masks(pr, [nodes] * batch)))[::9]:
        r = slice(b * nodes, (b + 1) * nodes)
        check(out[r], lse[r], q[r], K, V, k[r], v[r], m)
    ctx.close()


@pytest.mark.parametrize("value", [2.0 ** 12, -2.0 ** 62, 2.0 ** 70, 2.0 ** 99])
@pytest.mark.parametrize("places", ["one", "all", "node"])
@pytest.mark.parametrize("batch, nodes, hq, hkv, tokens", [(1, 1, 4, 1, 0), (1, 1, 4, 1, 512), (2, 1, 32, 8, 70), (1, 12, 8, 2, 0), (1, 12, 8, 2, 512), (1, 60, 8, 2, 0), (1, 60, 8, 2, 1000),
                                                            (1, 100, 8, 2, 300), (16, 60, 32, 8, 0)])
def test_huge_values_among_zeros(batch, nodes, hq, hkv, tokens, places, value):
    """Trees whose values are zero, or all apart, but for the huge ones."""
    ctx, pr, cache, K, V, q, k, v = random_case(batch, nodes, hq, hkv, tokens, 41)
    v.zero_()
    if places == "all":
        v[:] = value
    elif places == "one":
        v[::nodes, :, 3] = value
    else:
        v[::nodes] = value
    out, lse = run(ctx, pr, cache, q, k, v, [nodes] * batch)
    assert torch.isfinite(out).all()
    for b, m in list(enumerate(masks(pr, [nodes] * batch)))[::9]:
        r = slice(b * nodes, (b + 1) * nodes)
        check(out[r], lse[r], q[r], K, V, k[r], v[r], m)
    ctx.close()


def test_more_sequences_than_a_block_has_threads():
    batch, hkv, lens = 700, 1, [(37 * b) % 90 for b in range(700)]
    rng = np.random.default_rng(3)
    cache, K, V = shared_cache(batch, rng.standard_normal((96, hkv, 128)), rng.standard_normal((96, hkv, 128)), page=32)
    cache.kv_len.copy_(i32(lens))
    ctx, _, pr = make_trees([1] * batch, 3)
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(batch, h, 128, device="cuda", generator=g).bfloat16() for h in (4, hkv, hkv))
    out, lse = run(ctx, pr, cache, q, k, v, [1] * batch)
    for b in range(batch):
        check(out[b:b + 1], lse[b:b + 1], q[b:b + 1], K[:lens[b]], V[:lens[b]], k[b:b + 1], v[b:b + 1], np.ones((1, 1), dtype=bool))
    ctx.close()

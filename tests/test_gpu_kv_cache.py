"""hs_kv_append, hs_kv_append_path and hs_kv_read against the oracle, byte for byte over the whole pool: rows of every size, strides, ragged batches with empty
sequences, page ends, full tables, bad pages, paths of both layouts."""
import math

import numpy as np
import pytest
import torch

from oracle import paged
from paged_util import i32, make_cache
from paper_2505_13254_b200 import binding as hb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = hb.Context(0, 1 << 20)
    yield c
    c.close()


def fresh():
    return hb.Context(0, 1 << 20)


def host(cache):
    return [t.cpu().numpy().copy() for t in (cache.k, cache.k_scale, cache.v, cache.v_scale)]


def same(cache, want):
    for got, w in zip(host(cache), want):
        assert np.array_equal(got, w)


def strided(x, kind):
    """The same values with other strides: whole, inside the rows of a fused projection, or heads far apart."""
    n, h, d = x.shape
    if kind == "whole":
        return x
    if kind == "fused":
        big = torch.full((n, 3 * h + 5, d), math.nan, dtype=x.dtype, device=x.device)
        big[:, 2 * h:3 * h] = x
        return big[:, 2 * h:3 * h]
    big = torch.full((h, n, d + 8), math.nan, dtype=x.dtype, device=x.device)
    big[:, :, :d] = x.transpose(0, 1)
    return big[:, :, :d].transpose(0, 1)


def values(n, h, dtype, seed):
    """Rows of all sizes: scales between 2^-40 and 2^40, a row of zeros, one of subnormal numbers, one of the largest, ties of the rounding, an infinity and a NaN."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, h, 128, device="cuda", generator=g) * torch.exp2(torch.randint(-40, 41, (n, h, 1), device="cuda", generator=g).float())
    special = [torch.zeros(128), torch.full((128,), 2.0 ** -133), torch.linspace(-3.3e38, 3.3e38, 128), torch.arange(128) * 0.5 + 16.0,
               torch.tensor([math.inf] + [1.0] * 127), torch.tensor([1.0] * 127 + [math.nan]), torch.tensor([448.0] + [17.0] * 127),
               torch.tensor([-450.0] + [-17.0] * 127), torch.tensor([1.75] + [2.0 ** -9 * 1.5] * 127)]
    flat = x.view(n * h, 128)
    for i, s in enumerate(special):
        if i < n * h:
            flat[(i * 7) % (n * h)] = s.cuda()
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("held, new, hkv, page, kind", [
    ([0], [1], 1, 16, "whole"), ([15, 0, 16, 17], [1, 0, 3, 40], 3, 16, "fused"), ([0, 5, 100], [70, 1, 29], 8, 32, "apart"),
    ([1023, 1024], [2, 1500], 2, 1024, "whole"), ([7] * 40, [i % 5 for i in range(40)], 1, 64, "fused"), ([0, 0], [0, 0], 2, 16, "whole"),
    ([64, 3, 0], [600, 0, 900], 8, 64, "fused"), ([30], [333], 7, 128, "apart"),
])
def test_append(ctx, dtype, held, new, hkv, page, kind):
    cache, _, _ = make_cache(held, hkv, page, sum(new) + 1, room=max(new))
    off = np.concatenate([[0], np.cumsum(new)]).tolist()
    n = off[-1] + 4                                                     # rows behind the last sequence are left out
    k, v = values(n, hkv, dtype, 1), values(n, hkv, dtype, 2)
    want, table = host(cache), cache.page_table.tolist()
    for b, m in enumerate(new):
        for pool, sc, x in ((want[0], want[1], k), (want[2], want[3], v)):
            paged.append(pool, sc, table, page, b, held[b], x[off[b]:off[b] + m].double().cpu().numpy())
    length = torch.full((len(new),), -1, dtype=torch.int32, device="cuda")
    hb.hs_kv_append(ctx, cache, strided(k, kind), strided(v, kind), i32(off), len_out=length)
    same(cache, want)
    assert length.tolist() == [a + b for a, b in zip(held, new)] and cache.kv_len.tolist() == held
    assert hb.hs_device_error(ctx) == 0
    # the bytes stand for the same values when they are read back
    cache.kv_len.copy_(length)
    for out_type in (torch.float32, torch.bfloat16):
        ko, vo = strided(torch.full((n, hkv, 128), 9.0, dtype=out_type, device="cuda"), kind), torch.full((n, hkv, 128), 9.0, dtype=out_type, device="cuda")
        vo = strided(vo, kind)
        hb.hs_kv_read(ctx, cache, i32(off), k_out=ko, v_out=vo, first=i32(held))
        for b, m in enumerate(new):
            for o, pool, sc in ((ko, want[0], want[1]), (vo, want[2], want[3])):
                got = o[off[b]:off[b] + m].double().cpu().numpy()
                ref = torch.from_numpy(paged.read(pool, sc, table, page, b, range(held[b], held[b] + m))).to(out_type).double().numpy()
                assert np.array_equal(got, ref, equal_nan=True)
        assert (ko[off[-1]:] == 9).all() and (vo[off[-1]:] == 9).all()
    assert hb.hs_device_error(ctx) == 0


def test_append_into_a_fused_projection_of_one_head():
    """One head: its stride means nothing, whatever a slice reports."""
    ctx = fresh()
    cache, _, _ = make_cache([5], 1, 16, 3, room=20)
    fused = torch.randn(20, 6, 128, device="cuda").bfloat16()
    k, v = fused[:, 4:5], fused[:, 5:6]
    want, table = host(cache), cache.page_table.tolist()
    paged.append(want[0], want[1], table, 16, 0, 5, k.double().cpu().numpy())
    paged.append(want[2], want[3], table, 16, 0, 5, v.double().cpu().numpy())
    hb.hs_kv_append(ctx, cache, k, v, i32([0, 20]))
    same(cache, want)
    ctx.close()


def test_tokens_behind_the_table_are_dropped():
    ctx = fresh()
    held, new, page = [10, 30], [40, 2], 16
    cache, _, _ = make_cache(held, 2, page, 4, room=6)                  # tables: 1 page and a poisoned one; 3 and a poisoned one
    cache.page_table[0, 1:] = cache.page_table[1, 0]                     # sequence 0 may use the page of sequence 1
    k = values(42, 2, torch.bfloat16, 5)
    capacity = cache.max_pages * page
    cache.kv_len.copy_(i32([capacity - 3, 30]))
    want, table = host(cache), cache.page_table.tolist()
    for pool, sc in ((want[0], want[1]), (want[2], want[3])):
        x = k.double().cpu().numpy()
        paged.append(pool, sc, table, page, 0, capacity - 3, x[:3])
        paged.append(pool, sc, table, page, 1, 30, x[40:42])
    length = torch.zeros(2, dtype=torch.int32, device="cuda")
    hb.hs_kv_append(ctx, cache, k, k, i32([0, 40, 42]), len_out=length)
    same(cache, want)
    assert length.tolist() == [capacity, 32] and hb.hs_device_error(ctx) == hb.HS_ERR_BAD_PAGE
    ctx.close()


@pytest.mark.parametrize("bad", [-1, 99999, -(1 << 31)])
def test_bad_pages_and_lengths_write_nothing(bad):
    ctx = fresh()
    cache, _, _ = make_cache([0, 0], 2, 16, 6, room=40)
    cache.page_table[0, 1] = bad
    k = values(60, 2, torch.float32, 7)
    want, table = host(cache), cache.page_table.tolist()
    for pool, sc in ((want[0], want[1]), (want[2], want[3])):
        x = k.double().cpu().numpy()
        paged.append(pool, sc, table, 16, 0, 0, x[:30])                 # (tokens 16 .. 29 have no page)
        paged.append(pool, sc, table, 16, 1, 0, x[30:60])
    hb.hs_kv_append(ctx, cache, k, k, i32([0, 30, 60]))
    same(cache, want)
    assert hb.hs_device_error(ctx) == hb.HS_ERR_BAD_PAGE
    ctx.close()
    ctx = fresh()
    cache.kv_len.copy_(i32([30, -4]))
    ko, vo = torch.full((60, 2, 128), 9.0, device="cuda"), torch.full((60, 2, 128), 9.0, device="cuda")
    hb.hs_kv_read(ctx, cache, i32([0, 30, 60]), k_out=ko, v_out=vo)
    good = paged.read(want[0], want[1], table, 16, 0, range(16))
    assert np.array_equal(ko[:16].double().cpu().numpy(), good, equal_nan=True) and (ko[16:] == 9).all() and (vo[16:] == 9).all()
    assert hb.hs_device_error(ctx) == hb.HS_ERR_BAD_PAGE
    ctx.close()


@pytest.mark.parametrize("first", [None, [3, 0, 60], [-5, 99, 0], [(1 << 31) - 1, -(1 << 31), 63]])
def test_read_leaves_rows_of_other_tokens(ctx, first):
    lens = [40, 0, 64]
    cache, K, V = make_cache(lens, 3, 32, 8)
    off = [2, 30, 31, 100]                                              # two rows ahead of the first sequence, four behind the last
    ko, vo = torch.full((104, 3, 128), 9.0, device="cuda"), torch.full((104, 3, 128), 9.0, device="cuda")
    hb.hs_kv_read(ctx, cache, i32(off), k_out=ko, v_out=vo, first=None if first is None else i32(first))
    want_k, want_v = np.full((104, 3, 128), 9.0), np.full((104, 3, 128), 9.0)
    for b in range(3):
        for r in range(off[b], off[b + 1]):
            t = (first[b] if first else 0) + r - off[b]
            if 0 <= t < lens[b]:
                want_k[r], want_v[r] = K[b][t], V[b][t]
    assert np.array_equal(ko.double().cpu().numpy(), want_k) and np.array_equal(vo.double().cpu().numpy(), want_v)
    assert hb.hs_device_error(ctx) == 0


def path_bundles(batch, n_nodes, cap, seed):
    """Paths of chosen nodes, in both numberings, over trees of which some nodes are kept."""
    rng = np.random.default_rng(seed)
    pr, acc = hb.PrunedTree(batch * n_nodes, batch, "cuda"), hb.AcceptOut(batch, cap, "cuda")
    keep, paths = [], []
    for b in range(batch):
        kept = np.sort(np.concatenate([[0], 1 + rng.permutation(n_nodes - 1)[:rng.integers(1, n_nodes - 1)]]))
        n = int(rng.integers(1, min(cap, len(kept)) + 1))
        paths.append(np.concatenate([[0], np.sort(1 + rng.permutation(len(kept) - 1)[:n - 1])]).astype(int))
        keep.append(kept)
    off = np.concatenate([[0], np.cumsum([len(x) for x in keep])]).tolist()
    pr.n_keep.copy_(i32([len(x) for x in keep]))
    pr.keep_off.copy_(i32(off))
    pr.status.zero_()
    acc.status.zero_()
    acc.accept_len.copy_(i32([len(p) - 1 for p in paths]))
    compact, nodes = np.full((batch, cap), -1), np.full((batch, cap), -1)
    for b, p in enumerate(paths):
        compact[b, :len(p)], nodes[b, :len(p)] = p, keep[b][p]
    acc.path_compact.copy_(torch.from_numpy(compact).int())
    acc.path_nodes.copy_(torch.from_numpy(nodes).int())
    return pr, acc, keep, paths, off


@pytest.mark.parametrize("layout", [hb.HS_ROWS_COMPACT, hb.HS_ROWS_ORIGINAL])
@pytest.mark.parametrize("batch, n_nodes, cap, hkv, page", [(1, 5, 2, 1, 16), (5, 60, 12, 8, 16), (33, 20, 32, 3, 64)])
def test_append_path(ctx, layout, batch, n_nodes, cap, hkv, page):
    pr, acc, keep, paths, off = path_bundles(batch, n_nodes, cap, batch)
    held = [(13 * b) % 50 for b in range(batch)]
    cache, _, _ = make_cache(held, hkv, page, batch, room=cap)
    node_off = i32([b * n_nodes for b in range(batch + 1)])
    rows = off[-1] if layout == hb.HS_ROWS_COMPACT else batch * n_nodes
    k, v = values(rows, hkv, torch.bfloat16, 3), values(rows, hkv, torch.bfloat16, 4)
    if batch > 2:
        pr.status[1], acc.status[2] = 4, 7                              # sequences that were skipped append nothing
    want, table = host(cache), cache.page_table.tolist()
    lengths = list(held)
    for b in range(batch):
        if batch > 2 and b in (1, 2):
            continue
        at = (off[b] + paths[b]) if layout == hb.HS_ROWS_COMPACT else b * n_nodes + keep[b][paths[b]]
        for pool, sc, x in ((want[0], want[1], k), (want[2], want[3], v)):
            paged.append(pool, sc, table, page, b, held[b], x.double().cpu().numpy()[at])
        lengths[b] += len(paths[b])
    new_len = torch.zeros(batch, dtype=torch.int32, device="cuda")
    hb.hs_kv_append_path(ctx, cache, pr, acc, k, v, layout=layout, node_off=node_off if layout == hb.HS_ROWS_ORIGINAL else None, len_out=new_len)
    same(cache, want)
    assert new_len.tolist() == lengths and hb.hs_device_error(ctx) == 0


def test_paths_that_do_not_fit():
    """Longer than path_cap, nodes that are none, rows behind the arrays, a table without room: what there is a place and a row for is written."""
    ctx = fresh()
    pr, acc, keep, paths, off = path_bundles(4, 30, 6, 77)
    acc.accept_len.copy_(i32([9, 2, 2, 2]))                             # sequence 0: ten tokens, six places
    acc.path_compact.copy_(i32([[0, 1, 1, 0, 1, 0], [0, -1, 1, 1, 1, 1], [0, 29, 1, 1, 1, 1], [0, 1, 1, 1, 1, 1]]))
    pr.n_keep.copy_(i32([2, 2, 2, 2]))
    held = [3, 0, 0, 31]                                                # sequence 3: one token more fits
    cache, _, _ = make_cache(held, 2, 16, 5)
    assert cache.max_pages == 3
    cache.page_table.copy_(i32([[0, 1, -7], [2, 3, -7], [4, 0, -7], [1, 2, 3]]))
    capacity = cache.max_pages * 16
    cache.kv_len[3] = capacity - 1
    rows = off[3] + 2
    k = values(rows, 2, torch.bfloat16, 6)
    want, table = host(cache), cache.page_table.tolist()
    x = k.double().cpu().numpy()
    for pool, sc in ((want[0], want[1]), (want[2], want[3])):
        paged.append(pool, sc, table, 16, 0, 3, x[off[0] + np.array([0, 1, 1, 0, 1, 0])])
        for b in (1, 2):                                                # tokens 0 and 2; token 1 is no node of the tree
            paged.append(pool, sc, table, 16, b, 0, x[off[b]][None])
            paged.append(pool, sc, table, 16, b, 2, x[off[b] + 1][None])
        paged.append(pool, sc, table, 16, 3, capacity - 1, x[off[3]][None])
    new_len = torch.zeros(4, dtype=torch.int32, device="cuda")
    hb.hs_kv_append_path(ctx, cache, pr, acc, k, k, len_out=new_len)
    same(cache, want)
    assert new_len.tolist() == [9, 3, 3, capacity] and hb.hs_device_error(ctx) == hb.HS_ERR_BAD_PAGE
    ctx.close()


def test_captured_and_replayed_on_another_stream(ctx):
    cache, _, _ = make_cache([5, 20], 2, 16, 9, room=200)
    k, v, off = values(24, 2, torch.bfloat16, 8), values(24, 2, torch.bfloat16, 9), i32([0, 10, 24])
    new_len = torch.zeros(2, dtype=torch.int32, device="cuda")
    want, table = host(cache), cache.page_table.tolist()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        hb.hs_kv_append(ctx, cache, k, v, off, len_out=new_len)
        cache.kv_len.copy_(new_len)
    for i in range(5):
        for pool, sc, x in ((want[0], want[1], k), (want[2], want[3], v)):
            paged.append(pool, sc, table, 16, 0, 5 + 10 * i, x[:10].double().cpu().numpy())
            paged.append(pool, sc, table, 16, 1, 20 + 14 * i, x[10:].double().cpu().numpy())
        graph.replay()
    torch.cuda.synchronize()
    same(cache, want)
    assert cache.kv_len.tolist() == [55, 90] and hb.hs_device_error(ctx) == 0


def test_refusals(ctx):
    cache, _, _ = make_cache([5], 2, 16, 10, room=20)
    off = i32([0, 4])
    x = lambda *s, **k: torch.zeros(*s, dtype=k.get("dtype", torch.bfloat16), device="cuda")
    before = host(cache)

    def refused(status, call):
        with pytest.raises(hb.HsError) as e:
            call()
        assert e.value.status == status
    # lengths are not advanced in place; rows start on 16 bytes and lie whole vectors apart
    refused(hb.HS_ERR_INVALID_ARG, lambda: hb.hs_kv_append(ctx, cache, x(4, 2, 128), x(4, 2, 128), off, len_out=cache.kv_len))
    flat = x(4 * 256 + 8)
    refused(hb.HS_ERR_INVALID_ARG, lambda: hb.hs_kv_append(ctx, cache, flat[1:1025].view(4, 2, 128), flat[1:1025].view(4, 2, 128), off))
    odd = x(4, 2, 132)[:, :, :128]
    refused(hb.HS_ERR_SHAPE, lambda: hb.hs_kv_append(ctx, cache, odd, odd, off))
    same_row = x(1, 2, 128).expand(4, 2, 128)
    refused(hb.HS_ERR_SHAPE, lambda: hb.hs_kv_read(ctx, cache, off, k_out=same_row, v_out=same_row))
    one_head = x(4, 1, 128).expand(4, 2, 128)
    refused(hb.HS_ERR_SHAPE, lambda: hb.hs_kv_append(ctx, cache, one_head, one_head, off))
    pr, acc, *_ = path_bundles(1, 8, 4, 1)
    k = x(8, 2, 128)
    refused(hb.HS_ERR_INVALID_ARG, lambda: hb.hs_kv_append_path(ctx, cache, pr, acc, k, k, layout=hb.HS_ROWS_ORIGINAL))
    refused(hb.HS_ERR_INVALID_ARG, lambda: hb.hs_kv_append_path(ctx, cache, pr, acc, k, k, layout=5))
    refused(hb.HS_ERR_INVALID_ARG, lambda: hb.hs_kv_append_path(ctx, cache, pr, acc, k, k, len_out=cache.kv_len))
    refused(hb.HS_ERR_INVALID_ARG, lambda: hb.hs_kv_append_path(ctx, cache, pr, acc, x(0, 2, 128), x(0, 2, 128)))
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")
    for page, dim in ((8, 128), (24, 128), (2048, 128), (16, 64)):
        c = hb.KvCache(u8(2, 2, page, dim), u8(2, 2, page, dim), u8(2, 2, page), u8(2, 2, page), i32([[0, 1]]), i32([0]))
        refused(hb.HS_ERR_SHAPE, lambda: hb.hs_kv_append(ctx, c, x(4, 2, dim), x(4, 2, dim), off))
    # no rows: nothing to do, and nothing is refused
    hb.hs_kv_append(ctx, cache, x(0, 2, 128), x(0, 2, 128), i32([0, 0]))
    hb.hs_kv_read(ctx, cache, i32([0, 0]), k_out=x(0, 2, 128), v_out=x(0, 2, 128))
    torch.cuda.synchronize()
    same(cache, before)
    assert hb.hs_device_error(ctx) == 0


def test_the_smallest_values_are_read_as_they_are():
    """All bytes at the smallest scales: fp32 is exact, bf16 from 2^-130 on; below that to a multiple of 2^-133."""
    ctx, cache = fresh(), hb.KvCache.empty(2, 1, 16, i32([[0, 1]]))
    cache.k.copy_(torch.arange(256, device="cuda").to(torch.uint8).view(2, 1, 1, 128).expand(2, 1, 16, 128))
    cache.k_scale.copy_(torch.arange(16, device="cuda").to(torch.uint8).expand(2, 1, 16))
    cache.k.masked_fill_((cache.k & 127) == 127, 0)
    cache.kv_len.fill_(32)
    want = paged.read(cache.k.cpu().numpy(), cache.k_scale.cpu().numpy(), [[0, 1]], 16, 0, range(32))
    out = [torch.zeros(32, 1, 128, dtype=t, device="cuda") for t in (torch.float32, torch.bfloat16)]
    for x in out:
        hb.hs_kv_read(ctx, cache, i32([0, 32]), k_out=x, v_out=torch.zeros_like(x))
    whole, half = (x.double().cpu().numpy() for x in out)
    assert np.array_equal(whole, want)
    large = np.abs(want) >= 2.0 ** -130
    assert large.any() and (~large).any() and np.array_equal(half[large], want[large])
    assert np.array_equal(half[~large], np.rint(want[~large] * 2.0 ** 133) * 2.0 ** -133)
    ctx.close()

"""Appends whose rows are not all there: each alone in a context of its own, so that its own error is the one that is read."""
import numpy as np
import pytest
import torch

from oracle import paged
from paged_util import i32
from paper_2505_13254_b200 import binding as hb

pytestmark = pytest.mark.gpu


def pool(batch, hkv=2, page=16):
    cache = hb.KvCache.empty(batch * 2, hkv, page, i32(np.arange(batch * 2).reshape(batch, 2).tolist()))
    for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        t.fill_(77)
    return cache


def rows(n, hkv=2, seed=0):
    return torch.randn(n, hkv, 128, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).bfloat16()


def bundles(paths, keep, total):
    batch, cap = len(paths), 8
    pr, acc = hb.PrunedTree(total, batch, "cuda"), hb.AcceptOut(batch, cap, "cuda")
    pr.n_keep.copy_(i32(keep))
    pr.keep_off.copy_(i32(np.concatenate([[0], np.cumsum(keep)]).tolist()))
    pr.status.zero_()
    acc.status.zero_()
    acc.accept_len.copy_(i32([len(p) - 1 for p in paths]))
    table = np.full((batch, cap), -1)
    for b, p in enumerate(paths):
        table[b, :len(p)] = p
    for t in (acc.path_compact, acc.path_nodes):
        t.copy_(torch.from_numpy(table).int())
    return pr, acc


@pytest.mark.parametrize("layout, path, keep, max_rows", [
    (hb.HS_ROWS_COMPACT, [0, -1, 2], 5, 10),                             # no node
    (hb.HS_ROWS_COMPACT, [0, 5, 2], 5, 10),                              # behind the kept nodes
    (hb.HS_ROWS_COMPACT, [0, 1, 2], 5, 7),                               # a row behind the arrays (sequence 1 starts at row 5)
    (hb.HS_ROWS_ORIGINAL, [0, -3, 2], 5, 10), (hb.HS_ROWS_ORIGINAL, [0, 9, 2], 5, 10), (hb.HS_ROWS_ORIGINAL, [0, 5, 2], 5, 12),
    (hb.HS_ROWS_COMPACT, [0, 1, (1 << 31) - 1], 5, 10), (hb.HS_ROWS_ORIGINAL, [0, 1, (1 << 31) - 1], 5, 10),
])
def test_an_entry_of_a_path_without_a_row_is_an_error(layout, path, keep, max_rows):
    ctx, cache = hb.Context(0, 1 << 20), pool(2)
    pr, acc = bundles([[0, 1], path], [5, keep], 10)
    k, node_off, length = rows(max_rows), i32([0, 5, 10]), torch.zeros(2, dtype=torch.int32, device="cuda")
    hb.hs_kv_append_path(ctx, cache, pr, acc, k, k, layout=layout, node_off=node_off if layout == hb.HS_ROWS_ORIGINAL else None, len_out=length)
    assert hb.hs_device_error(ctx) == hb.HS_ERR_BAD_PAGE
    want = [t.cpu().numpy() for t in pool(2).__dict__.values() if torch.is_tensor(t)][:4]
    table, x = cache.page_table.tolist(), k.double().cpu().numpy()
    for b, p in enumerate(([0, 1], path)):
        for i, node in enumerate(p):
            if 0 <= node < keep and 5 * b + node < max_rows:
                for data, scale in ((want[0], want[2]), (want[1], want[3])):
                    paged.append(data, scale, table, 16, b, i, x[5 * b + node][None])
    for got, w in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), want):
        assert np.array_equal(got.cpu().numpy(), w)
    assert length.tolist() == [2, 3]
    ctx.close()
    # without the entry: no error
    ctx = hb.Context(0, 1 << 20)
    pr, acc = bundles([[0, 1], [0, 1, 2]], [5, 5], 10)
    hb.hs_kv_append_path(ctx, pool(2), pr, acc, rows(10), rows(10), layout=layout, node_off=node_off if layout == hb.HS_ROWS_ORIGINAL else None)
    assert hb.hs_device_error(ctx) == 0
    # and a sequence that was skipped has no path to look at
    acc.path_compact.fill_(-9)
    acc.path_nodes.fill_(-9)
    acc.status.fill_(3)
    hb.hs_kv_append_path(ctx, pool(2), pr, acc, rows(10), rows(10), layout=layout, node_off=node_off if layout == hb.HS_ROWS_ORIGINAL else None)
    assert hb.hs_device_error(ctx) == 0
    ctx.close()


@pytest.mark.parametrize("with_length", [True, False])
@pytest.mark.parametrize("n_rows, off, lengths", [
    (6, [0, 4, 9], [4, 2]), (4, [0, 4, 9], [4, 0]), (3, [0, 4, 9], [3, 0]), (0, [0, 4, 9], [0, 0]), (6, [2, 4, 9], [2, 2]), (3, [5, 7, 9], [0, 0]),
])
def test_rows_that_the_offsets_name_behind_the_arrays_are_an_error(n_rows, off, lengths, with_length):
    ctx, cache = hb.Context(0, 1 << 20), pool(2)
    x, length = rows(max(n_rows, 1))[:n_rows], torch.full((2,), -1, dtype=torch.int32, device="cuda")
    hb.hs_kv_append(ctx, cache, x, x, i32(off), len_out=length if with_length else None)
    assert hb.hs_device_error(ctx) == hb.HS_ERR_SHAPE
    want = [t.cpu().numpy() for t in pool(2).__dict__.values() if torch.is_tensor(t)][:4]
    table, host = cache.page_table.tolist(), x.double().cpu().numpy()
    for b in range(2):
        part = host[min(off[b], n_rows):min(off[b + 1], n_rows)]
        assert len(part) == lengths[b]
        for data, scale in ((want[0], want[2]), (want[1], want[3])):
            paged.append(data, scale, table, 16, b, 0, part)
    for got, w in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), want):
        assert np.array_equal(got.cpu().numpy(), w)
    assert length.tolist() == (lengths if with_length else [-1, -1])
    ctx.close()


def test_rows_of_the_arrays_behind_the_offsets_are_none():
    ctx, cache = hb.Context(0, 1 << 20), pool(2)
    length = torch.zeros(2, dtype=torch.int32, device="cuda")
    hb.hs_kv_append(ctx, cache, rows(12), rows(12), i32([0, 4, 9]), len_out=length)
    hb.hs_kv_append(ctx, cache, rows(9), rows(9), i32([0, 4, 9]))
    assert hb.hs_device_error(ctx) == 0 and length.tolist() == [4, 5]
    ctx.close()


def test_one_tensor_in_host_memory_is_refused():
    ctx, cache, rope = hb.Context(0, 1 << 20), pool(1), hb.make_rope(128)
    pr, acc = bundles([[0, 1]], [4], 4)
    k, q, off, length = rows(4), rows(4, 8), i32([0, 4]), i32([0])
    host = hb.KvCache(*(t.cpu() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.page_table, cache.kv_len)))
    tree = dict(max_nodes=4, max_kv_len=9)
    for call in (lambda: hb.hs_kv_append(ctx, cache, k.cpu(), k, off), lambda: hb.hs_kv_append(ctx, cache, k, k.cpu(), off),
                 lambda: hb.hs_kv_append(ctx, cache, k, k, off.cpu()), lambda: hb.hs_kv_append(ctx, cache, k, k, off, len_out=length.cpu()),
                 lambda: hb.hs_kv_append(ctx, host, k, k, off), lambda: hb.hs_kv_append_path(ctx, cache, pr, acc, k, k.cpu()),
                 lambda: hb.hs_kv_append_path(ctx, host, pr, acc, k, k), lambda: hb.hs_kv_read(ctx, cache, off, k_out=k, v_out=k.cpu()),
                 lambda: hb.hs_kv_read(ctx, cache, off, k_out=k, v_out=k, first=length.cpu()), lambda: hb.hs_rotary(ctx, rope, i32([0] * 4).cpu(), q),
                 lambda: hb.hs_rotary(ctx, rope, i32([0] * 4), q, k.cpu()), lambda: hb.hs_rotary_tree(ctx, rope, pr, length.cpu(), q, k, max_nodes=4),
                 lambda: hb.hs_tree_verify_attention_paged(ctx, pr, cache, q, k.cpu(), k, **tree), lambda: hb.hs_tree_verify_attention_paged(ctx, pr, host, q, k, k, **tree),
                 lambda: hb.hs_tree_verify_attention_paged(ctx, pr, cache, q, k, k, lse_out=torch.zeros(4, 8), **tree)):
        with pytest.raises(ValueError):
            call()
    torch.cuda.synchronize()
    assert hb.hs_device_error(ctx) == 0
    ctx.close()

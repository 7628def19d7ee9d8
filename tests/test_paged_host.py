"""The paged cache, rotary positions and the attention over the cache, as far as they need no device: layouts of the structures, frequencies, refusals of
the binding, the rule that cuts the attention's launch, and what the sources must say."""
import ctypes
import os
import re
import shutil

import numpy as np
import pytest
import torch

from oracle import paged
from paged_route import route
from paper_2505_13254_b200 import binding as hb
from paper_2505_13254_b200 import build


def test_struct_sizes_match_the_header():
    assert ctypes.sizeof(hb._KvCache) == 6 * 4 + 6 * 8
    assert ctypes.sizeof(hb._PagedAttnDesc) == 5 * 4 + 4 + 8 + 8
    assert ctypes.sizeof(hb._RopeConfig) == 4 * 4 + 8 * 8 + 8
    assert ctypes.sizeof(hb._Rope) == 4 * 4 + 128 * 8
    assert ctypes.sizeof(hb._Heads) == 2 * 8 + 8 + 4 * 8
    assert hb.lib().hs_status_string(hb.HS_ERR_BAD_PAGE) not in (b"", b"ok", hb.lib().hs_status_string(99))


@pytest.mark.parametrize("dim, config", [
    (128, {}), (16, {}), (256, dict(base=500000.0)), (64, dict(scaling="linear", factor=4.0)), (128, dict(scaling="ntk", factor=2.5, base=1e6)),
    (128, dict(scaling="llama3", base=500000.0, factor=8.0, low_freq_factor=1.0, high_freq_factor=4.0, original_len=8192)),
    (64, dict(scaling="yarn", factor=16.0, original_len=4096)), (128, dict(scaling="yarn", factor=4.0, original_len=32768, attn_factor=1.25, beta_fast=16.0)),
    (32, dict(scaling="table", inv_freq=[0.0, 7.0, 6.283185307179586, 1e-9, 3.5] + [0.25] * 11)),
])
def test_frequencies(dim, config):
    rope = hb.make_rope(max(dim, 32), dim, **config)
    f, scale = paged.frequencies(dim, **config)
    assert (rope.head_dim, rope.rotary_dim) == (max(dim, 32), dim)
    assert abs(rope.table.scale - scale) <= 2.0 ** -24 * scale
    got = np.array([float(rope.table.turns[i]) for i in range(dim // 2)]) / 2.0 ** 64
    want = f / (2 * np.pi) % 1.0
    # two ways of a dozen fp64 operations each, at most 2^-53 of a frequency apiece; a whole turn more or less is the same
    off = np.abs(got - want)
    assert (np.minimum(off, 1 - off) <= 2.0 ** -48 * np.maximum(1.0, f)).all()


@pytest.mark.parametrize("change", [
    dict(head_dim=120), dict(head_dim=272), dict(rotary_dim=144), dict(rotary_dim=8), dict(rotary_dim=40), dict(base=1.0), dict(base=float("nan")),
    dict(scaling="linear", factor=0.0), dict(scaling="linear", factor=float("inf")), dict(scaling="llama3", factor=8.0),
    dict(scaling="llama3", factor=8.0, original_len=8192, high_freq_factor=1.0), dict(scaling="yarn", factor=4.0),
    dict(scaling="yarn", factor=4.0, original_len=4096, beta_slow=0.0), dict(scaling="yarn", factor=4.0, original_len=4096, beta_fast=0.5),
    dict(scaling="yarn", factor=4.0, original_len=4096, attn_factor=-1.0), dict(scaling="table"), dict(scaling="table", inv_freq=[-1.0] * 64),
    dict(scaling="table", inv_freq=[float("nan")] * 64),
])
def test_a_bad_configuration_is_refused(change):
    with pytest.raises(hb.HsError):
        hb.make_rope(**dict(dict(head_dim=128), **change))


def test_a_bad_table_or_name_is_a_python_error():
    with pytest.raises(ValueError):
        hb.make_rope(128, scaling="table", inv_freq=[1.0] * 63)
    with pytest.raises(ValueError):
        hb.make_rope(128, scaling="dynamic")


def cache(batch=2, hkv=2, page=16, pages=3):
    return hb.KvCache.empty(batch * pages, hkv, page, torch.arange(batch * pages, dtype=torch.int32).view(batch, pages))


@pytest.mark.parametrize("edit, error", [
    (lambda t: t.update(k=t["k"].float()), TypeError), (lambda t: t.update(page_table=t["page_table"].long()), TypeError),
    (lambda t: t.update(kv_len=t["kv_len"][:1]), ValueError), (lambda t: t.update(v=t["v"][:-1]), ValueError),
    (lambda t: t.update(k_scale=t["k_scale"][:, :1]), ValueError), (lambda t: t.update(k=t["k"].transpose(1, 2), v=t["v"].transpose(1, 2)), ValueError),
    (lambda t: t.update(page_table=t["page_table"].t().contiguous().t()), ValueError),
])
def test_a_cache_of_other_tensors_is_refused(edit, error):
    c = cache()
    t = dict(k=c.k, v=c.v, k_scale=c.k_scale, v_scale=c.v_scale, page_table=c.page_table, kv_len=c.kv_len)
    edit(t)
    with pytest.raises(error):
        hb.KvCache(**t)


def test_a_cache_takes_tensors_like_its_own_only():
    c = cache()
    c.kv_len = torch.ones(2, dtype=torch.int32)
    assert c.kv_len.tolist() == [1, 1]
    for name, value in (("kv_len", torch.ones(2, dtype=torch.int64)), ("kv_len", torch.ones(3, dtype=torch.int32)),
                        ("page_table", torch.zeros(2, 6, dtype=torch.int32)[:, ::2]), ("k", c.k[:-1])):
        with pytest.raises(ValueError):
            setattr(c, name, value)
    with pytest.raises(AttributeError):
        c.page_size = 32


def rows(n=4, heads=2, dim=128, dtype=torch.bfloat16):
    return torch.zeros(n, heads, dim, dtype=dtype)


def test_calls_reach_the_library():
    nat, c, off = hb.native(), cache(), torch.zeros(3, dtype=torch.int32)
    pr, acc, rope = hb.PrunedTree(4, 2, "cpu"), hb.AcceptOut(2, 4, "cpu"), hb.make_rope(128)
    q, k = rows(heads=4), rows()
    bad = hb.HS_ERR_INVALID_ARG                                        # (of the missing context)
    assert nat.kv_append(0, c, k, k, off, None, 0) == bad
    assert nat.kv_append(0, c, rows(0), rows(0), off, off[:2], 0) == bad
    assert nat.kv_append_path(0, c, pr, acc, 0, None, k, k, None, 0) == bad
    assert nat.kv_read(0, c, off, None, k, k, 0) == bad
    assert nat.tree_verify_attention_paged(0, pr, c, q, k, k, 4, 100, 0, None, None, q, None, 0) == bad
    assert nat.rotary(0, rope, off, rows(3), rows(3), None, None, 0) == bad
    assert nat.rotary_tree(0, rope, pr, c.kv_len, 4, 0, None, q, q, k, k, 0) == bad


@pytest.mark.parametrize("call", [
    lambda n, c, pr, acc, o: n.kv_append(0, c, rows(), rows(5), o, None, 0),                               # shapes differ
    lambda n, c, pr, acc, o: n.kv_append(0, c, rows(heads=3), rows(heads=3), o, None, 0),                  # not the cache's heads
    lambda n, c, pr, acc, o: n.kv_append(0, c, rows(dim=64), rows(dim=64), o, None, 0),
    lambda n, c, pr, acc, o: n.kv_append(0, c, rows().transpose(1, 2).contiguous().transpose(1, 2), rows(), o, None, 0),
    lambda n, c, pr, acc, o: n.kv_append(0, c, rows(8)[::2], rows(), o, None, 0),                          # strides differ
    lambda n, c, pr, acc, o: n.kv_append(0, c, rows()[0], rows()[0], o, None, 0),                          # two dimensions
    lambda n, c, pr, acc, o: n.kv_append(0, c, rows(), rows(dtype=torch.float32), o, None, 0),
    lambda n, c, pr, acc, o: n.kv_read(0, c, o, None, rows(), rows(5), 0),
    lambda n, c, pr, acc, o: n.kv_append(0, c, rows(), rows(), o[:2], None, 0),                            # offsets of another batch
    lambda n, c, pr, acc, o: n.kv_append(0, c, rows(), rows(), o, o, 0),
    lambda n, c, pr, acc, o: n.kv_read(0, c, o[:2], None, rows(), rows(), 0),
    lambda n, c, pr, acc, o: n.kv_read(0, c, o, o, rows(), rows(), 0),
    lambda n, c, pr, acc, o: n.kv_append_path(0, c, pr, acc, 1, o[:2], rows(), rows(), None, 0),
    lambda n, c, pr, acc, o: n.kv_append_path(0, c, pr, acc, 0, None, rows(), rows(), o, 0),
    lambda n, c, pr, acc, o: n.tree_verify_attention_paged(0, pr, c, rows(), rows(), rows(), 4, 9, 1, o[:2], None, rows(), None, 0),
    lambda n, c, pr, acc, o: n.tree_verify_attention_paged(0, pr, c, rows(), rows(), rows(), 4, 9, 0, None, None, rows(), torch.zeros(4, 3), 0),
    lambda n, c, pr, acc, o: n.tree_verify_attention_paged(0, pr, c, rows(), rows(), rows(), 4, 9, 0, None, None, rows(), torch.zeros(3, 2), 0),
    lambda n, c, pr, acc, o: n.rotary_tree(0, hb.make_rope(128), pr, c.kv_len, 4, 1, o[:2], rows(), rows(), None, None, 0),
    lambda n, c, pr, acc, o: n.kv_append_path(0, c, pr, acc, 0, None, rows(8)[::2], rows(), None, 0),      # the tree's rows are contiguous
    lambda n, c, pr, acc, o: n.kv_append_path(0, c, pr, acc, 0, None, rows(), rows(5), None, 0),
    lambda n, c, pr, acc, o: n.kv_append_path(0, c, hb.PrunedTree(4, 3, "cpu"), acc, 0, None, rows(), rows(), None, 0),    # another batch
    lambda n, c, pr, acc, o: n.kv_append_path(0, c, pr, hb.AcceptOut(1, 4, "cpu"), 0, None, rows(), rows(), None, 0),
    lambda n, c, pr, acc, o: n.tree_verify_attention_paged(0, pr, c, rows(), rows(), rows(5), 4, 9, 0, None, None, rows(), None, 0),
    lambda n, c, pr, acc, o: n.tree_verify_attention_paged(0, pr, c, rows(), rows(heads=1), rows(heads=1), 4, 9, 0, None, None, rows(), None, 0),
    lambda n, c, pr, acc, o: n.tree_verify_attention_paged(0, hb.PrunedTree(4, 1, "cpu"), c, rows(), rows(), rows(), 4, 9, 0, None, None, rows(), None, 0),
    lambda n, c, pr, acc, o: n.rotary(0, hb.make_rope(128), o, rows(4), rows(4), None, None, 0),           # three positions, four rows
    lambda n, c, pr, acc, o: n.rotary(0, hb.make_rope(64), o, rows(3), rows(3), None, None, 0),
    lambda n, c, pr, acc, o: n.rotary(0, hb.make_rope(128), o, rows(3), rows(3, heads=3), None, None, 0),
    lambda n, c, pr, acc, o: n.rotary(0, hb.make_rope(128), o, rows(3), rows(3), rows(2), rows(2), 0),
    lambda n, c, pr, acc, o: n.rotary_tree(0, hb.make_rope(128), hb.PrunedTree(4, 5, "cpu"), c.kv_len, 4, 0, None, rows(), rows(), None, None, 0),
])
def test_arguments_that_do_not_fit_are_python_errors(call):
    with pytest.raises(ValueError):
        call(hb.native(), cache(), hb.PrunedTree(4, 2, "cpu"), hb.AcceptOut(2, 4, "cpu"), torch.zeros(3, dtype=torch.int32))


def test_other_types_are_python_errors():
    nat, c, off = hb.native(), cache(), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(TypeError):
        nat.kv_append(0, c, rows(dtype=torch.float16), rows(dtype=torch.float16), off, None, 0)
    with pytest.raises(TypeError):
        nat.kv_read(0, c, off)
    pr, acc, rope, wide = hb.PrunedTree(4, 2, "cpu"), hb.AcceptOut(2, 4, "cpu"), hb.make_rope(128), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: nat.kv_append(0, c, rows(), rows(), wide, None, 0), lambda: nat.kv_append(0, c, rows(), rows(), off, wide[:2], 0),
                 lambda: nat.kv_read(0, c, wide, None, rows(), rows(), 0), lambda: nat.kv_read(0, c, off, wide[:2], rows(), rows(), 0),
                 lambda: nat.kv_append_path(0, c, pr, acc, 1, wide, rows(), rows(), None, 0), lambda: nat.rotary(0, rope, wide, rows(3), rows(3), None, None, 0),
                 lambda: nat.rotary_tree(0, rope, pr, wide[:2], 4, 0, None, rows(), rows(), None, None, 0),
                 lambda: nat.tree_verify_attention_paged(0, pr, c, rows(), rows(), rows(), 4, 9, 0, None, None, rows(), torch.zeros(4, 2).bfloat16(), 0)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(AttributeError):
        nat.kv_read(0, object(), off, None, rows(), rows(), 0)


@pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")
@pytest.mark.parametrize("batch, nodes, hq, hkv, longest, rows, splits", [
    (1, 8, 32, 8, 64, 32, 1), (1, 9, 32, 8, 64, 64, 1), (1, 16, 32, 8, 64, 64, 1), (1, 17, 32, 8, 64, 128, 1),      # 32, 36, 64, 68 rows
    (32, 1, 32, 8, 8192, 32, 1), (1, 128, 64, 4, 2048, 128, 2),
    (8, 62, 64, 8, 4096, 256, 1), (4, 62, 64, 8, 4096, 128, 1),       # 256 blocks of 128 rows: two rounds; 128: one
    (16, 60, 32, 8, 2048, 256, 1), (9, 60, 32, 8, 2048, 128, 1),      # 256 blocks; 144
    (10, 60, 32, 8, 2048, 256, 1), (19, 60, 32, 8, 2048, 128, 1),     # 160: two rounds against one; 304: three against two
    (40, 30, 32, 8, 2048, 128, 1),                                    # 120 rows: one block of a head whatever its size
])
def test_blocks_and_splits(batch, nodes, hq, hkv, longest, rows, splits):
    assert route(batch, nodes, hq, hkv, longest) == (rows, splits)


@pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")
def test_splits_never_outnumber_tiles_or_clusters():
    for batch in (1, 2, 5, 40):
        for nodes in (1, 20, 128):
            for longest in (0, 1, 64, 65, 1000, 40000, 1 << 20):
                r, s = route(batch, nodes, 32, 8, longest)
                assert r in (32, 64, 128, 256) and 1 <= s <= min(16, (longest + 63) // 64 + (nodes + 63) // 64)


def text(name):
    return re.sub(r"//.*", "", open(os.path.join(build.CSRC, name)).read())


def test_tensor_memory_is_freed_behind_a_fenced_barrier():
    body = re.sub(r"\s+", "", text("tree_attn_paged.cu"))
    head = body[:body.rindex("tmem_dealloc(")]
    assert re.search(r"tc_fence_before_sync\(\);named_bar_sync\(1,PG_SM_THREADS\);tc_fence_after_sync\(\);if\(warp==0\)$", head)


def test_lanes_that_waited_alone_meet_again_ahead_of_tensor_memory():
    body = text("tree_attn_paged.cu")
    waits = [m.end() for m in re.finditer(r"if \(!ok_\w+\) mbar_wait\(", body)]
    assert len(waits) >= 4
    for at in waits:
        assert re.search(r"\btmem_\w+\(|\bumma_\w+\(|\belect_one\(|__syncwarp\(\)|__any_sync\(HS_FULL_MASK", body[at:]).group(0).startswith("__")


def test_pages_are_checked_before_they_are_used():
    assert re.search(r"if \(\(unsigned int\)page >= \(unsigned int\)c\.n_pages\) \{\s*kv_bad_page\(c\.err\);\s*return -1;", text("kv_page.cuh"))
    assert re.search(r"if \(\(unsigned int\)id >= \(unsigned int\)p\.c\.n_pages\) \{.*?kv_bad_page\(err\);\s*id = 0;", text("tree_attn_paged.cu"), re.S)


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "llama3", "yarn"])
def test_frequencies_that_would_not_be_read_are_a_python_error(scaling):
    with pytest.raises(ValueError):
        hb.make_rope(32, scaling=scaling, factor=4.0, original_len=4096, inv_freq=[0.25] * 16)


def spread(t):
    """The same entries, not side by side."""
    wide = torch.zeros(*t.shape, 2, dtype=t.dtype)
    wide[..., 0] = t
    return wide[..., 0]


@pytest.mark.parametrize("call", [
    lambda n, c, pr, acc, o: n.kv_append(0, c, rows(), rows(), spread(o), None, 0),
    lambda n, c, pr, acc, o: n.kv_append(0, c, rows(), rows(), o, spread(c.kv_len), 0),
    lambda n, c, pr, acc, o: n.kv_append(0, c, rows(), rows(), o[:1].expand(3), None, 0),                  # one entry, not three
    lambda n, c, pr, acc, o: n.kv_append_path(0, c, pr, acc, 1, spread(o), rows(), rows(), None, 0),
    lambda n, c, pr, acc, o: n.kv_append_path(0, c, pr, acc, 0, None, rows(), rows(), spread(c.kv_len), 0),
    lambda n, c, pr, acc, o: n.kv_read(0, c, spread(o), None, rows(), rows(), 0),
    lambda n, c, pr, acc, o: n.kv_read(0, c, o, spread(c.kv_len), rows(), rows(), 0),
    lambda n, c, pr, acc, o: n.tree_verify_attention_paged(0, pr, c, rows(), rows(), rows(), 4, 9, 1, spread(o), None, rows(), None, 0),
    lambda n, c, pr, acc, o: n.tree_verify_attention_paged(0, pr, c, rows(), rows(), rows(), 4, 9, 0, None, None, rows(), torch.zeros(2, 4).t(), 0),
    lambda n, c, pr, acc, o: n.tree_verify_attention_paged(0, pr, c, rows(), rows(), rows(), 4, 9, 0, None, None, rows(), torch.zeros(1).expand(4, 2), 0),
    lambda n, c, pr, acc, o: n.rotary(0, hb.make_rope(128), spread(o), rows(3), rows(3), None, None, 0),
    lambda n, c, pr, acc, o: n.rotary(0, hb.make_rope(128), o[:1].expand(3), rows(3), rows(3), None, None, 0),
    lambda n, c, pr, acc, o: n.rotary_tree(0, hb.make_rope(128), pr, spread(c.kv_len), 4, 0, None, rows(), rows(), None, None, 0),
    lambda n, c, pr, acc, o: n.rotary_tree(0, hb.make_rope(128), pr, c.kv_len, 4, 1, spread(o), rows(), rows(), None, None, 0),
])
def test_lists_whose_entries_do_not_lie_side_by_side_are_python_errors(call):
    with pytest.raises(ValueError):
        call(hb.native(), cache(), hb.PrunedTree(4, 2, "cpu"), hb.AcceptOut(2, 4, "cpu"), torch.zeros(3, dtype=torch.int32))


def test_lists_of_one_entry_have_no_stride():
    c, off = cache(batch=1), torch.zeros(2, dtype=torch.int32)
    one = torch.zeros(4, 3, dtype=torch.int32)[:1, 1]
    assert one.stride() == (3,)
    assert hb.native().kv_append(0, c, rows(), rows(), off, one, 0) == hb.HS_ERR_INVALID_ARG
    assert hb.native().rotary(0, hb.make_rope(128), one, rows(1), rows(1), None, None, 0) == hb.HS_ERR_INVALID_ARG


@pytest.mark.parametrize("call", [
    lambda n, x, c, pr, acc, o: n.kv_append(x, c, rows(), rows(), o, None, 0),
    lambda n, x, c, pr, acc, o: n.kv_append_path(x, c, pr, acc, 0, None, rows(), rows(), None, 0),
    lambda n, x, c, pr, acc, o: n.kv_read(x, c, o, None, rows(), rows(), 0),
    lambda n, x, c, pr, acc, o: n.tree_verify_attention_paged(x, pr, c, rows(), rows(), rows(), 4, 9, 0, None, None, rows(), None, 0),
    lambda n, x, c, pr, acc, o: n.rotary(x, hb.make_rope(128), o, rows(3), rows(3), rows(3), rows(3), 0),
    lambda n, x, c, pr, acc, o: n.rotary_tree(x, hb.make_rope(128), pr, c.kv_len, 4, 0, None, rows(), rows(), None, None, 0),
])
def test_tensors_in_host_memory_are_python_errors(call):
    context = (ctypes.c_char * 1024)()                                   # of device 0
    with pytest.raises(ValueError):
        call(hb.native(), ctypes.addressof(context), cache(), hb.PrunedTree(4, 2, "cpu"), hb.AcceptOut(2, 4, "cpu"), torch.zeros(3, dtype=torch.int32))

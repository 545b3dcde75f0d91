"""The cache operators' host side: tree tables, descriptor layout, what is refused before any launch (no GPU needed)."""
import ctypes
import os
import re

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2411_05289_b200 as sh  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint32) for n in ("struct_size", "version")] + [
        (n, ctypes.c_int32) for n in ("dtype", "batch", "nodes", "heads", "kv_heads", "head_dim", "page_size", "pages",
                                      "layers", "table_width")] + [
        ("stride_table", ctypes.c_int64), ("table", ctypes.c_void_p), ("lens", ctypes.c_void_p)]


class Pages(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p)] + [(n, ctypes.c_int64) for n in ("layer", "page", "token", "head")]


class Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p)] + [(n, ctypes.c_int64) for n in ("seq", "node", "head")]


def desc(**kw):
    d = Desc(ctypes.sizeof(Desc), 1, 1, 2, 3, 8, 4, 64, 16, 10, 1, 5, 5, 4096, 4096)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def pages(**kw):
    p = Pages(4096, 0, 16 * 4 * 64, 4 * 64, 64)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def heads(**kw):
    p = Heads(4096, 3 * 8 * 64, 8 * 64, 64)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


FAKE = ctypes.c_void_p(4096)   # never followed: every call below is refused on the host or has nothing to do
ref = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731


def append(d=None, q=True, k=None, v=None, kc=None, vc=None, depth=None, depth_stride=0, freq=FAKE, rotated=64, interleaved=0,
           qo=True, offset=0):
    lib = sh.load_library()
    new = lambda x: heads() if x is True else x  # noqa: E731
    return lib.spechub_cache_append(ref(d or desc()), ref(new(q)), ref(k or heads()), ref(v or heads()), ref(kc or pages()),
                                    ref(vc or pages()), depth, ctypes.c_int64(depth_stride), freq, rotated, interleaved,
                                    ctypes.c_int64(offset), ref(new(qo)), None, None)


def attend(d=None, q=None, kc=None, vc=None, mask=FAKE, mask_stride=0, shared=None, width=0, shared_len=0, scale=0.1,
           out=None, workspace=FAKE, nbytes=1 << 40):
    lib = sh.load_library()
    return lib.spechub_tree_attention(ref(d or desc()), ref(q or heads()), ref(kc or pages()), ref(vc or pages()), mask,
                                      ctypes.c_int64(mask_stride), shared, width, ctypes.c_int64(shared_len), ctypes.c_float(scale),
                                      ref(out or heads(data=16384)), None, None, workspace, ctypes.c_size_t(nbytes), None)


def accept(d=None, kc=None, vc=None, path=FAKE, levels=3, lens_out=ctypes.c_void_p(8192)):
    lib = sh.load_library()
    return lib.spechub_cache_accept(ref(d or desc()), ref(kc or pages()), ref(vc or pages()), path, levels, lens_out, None, None)


def test_every_declared_function_is_exported():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "spechub_cache.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(spechub_[a-z_]+)\s*\(", src))
    assert names == {"spechub_cache_append", "spechub_tree_attention", "spechub_tree_attention_workspace_bytes", "spechub_cache_accept"}
    for n in names:
        assert hasattr(sh.load_library(), n)


BAD_DESC = [(dict(struct_size=8), -2), (dict(version=2), -2), (dict(dtype=0), -4), (dict(dtype=3), -4), (dict(batch=-1), -3),
            (dict(nodes=0), -3), (dict(kv_heads=0), -12), (dict(heads=6), -12), (dict(heads=2), -12), (dict(head_dim=96), -12),
            (dict(page_size=4), -12), (dict(page_size=24), -12), (dict(page_size=2048), -12), (dict(pages=0), -12),
            (dict(layers=0), -12), (dict(table_width=0), -12), (dict(stride_table=4), -5), (dict(batch=1 << 30, nodes=1 << 10), -3),
            (dict(table_width=1 << 28, stride_table=1 << 28, page_size=64), -12), (dict(table=None), -1), (dict(lens=None), -1)]


@pytest.mark.parametrize("change,code", BAD_DESC)
def test_bad_descriptors_are_refused(change, code):
    for call in (append, attend, accept):
        assert call(desc(**change)) == code, (call.__name__, change)


@pytest.mark.parametrize("change", [dict(data=4104), dict(page=16 * 4 * 64 + 4), dict(token=20), dict(head=68), dict(head=0), dict(token=-64)])
def test_misplaced_caches_are_refused(change):
    for call in (append, attend, accept):
        assert call(kc=pages(**change)) == -11 and call(vc=pages(**change)) == -11
        assert call(kc=pages(data=None)) == -1


def test_append_refuses():
    for bad in (dict(data=4098), dict(seq=1001), dict(node=4), dict(head=-8)):
        assert append(k=heads(**bad)) == -11 and append(v=heads(**bad)) == -11
        assert append(q=heads(**bad)) == -11 and append(qo=heads(**bad)) == -11
    assert append(qo=heads(head=0)) == -11       # rows that are written may not lie over each other
    assert append(qo=None) == -1
    for rotated in (-16, 8, 72, 80, 128):
        assert append(rotated=rotated) == -13
    assert append(interleaved=2) == -13
    assert append(freq=None) == -1
    assert append(depth=FAKE, depth_stride=2) == -5
    assert append(desc(layers=2)) == -12
    assert append(desc(batch=0)) == 0


def test_attention_refuses():
    assert attend(q=heads(node=4)) == -11 and attend(out=heads(data=4100)) == -11 and attend(out=heads(seq=0)) == -11
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert attend(scale=scale) == -15
    assert attend(shared=FAKE, width=2, shared_len=33) == -14
    assert attend(shared=FAKE, width=2, shared_len=-1) == -14
    assert attend(shared=None, width=2, shared_len=32) == -1
    assert attend(mask=None) == -1
    assert attend(mask_stride=2) == -5
    assert attend(desc(layers=2)) == -12
    assert attend(desc(heads=4 * 129)) == -12                # more query heads per cache head than a tile has rows
    assert attend(q=heads(head=0)) == -11                    # (queries are copied as a tensor: rows lie apart)
    same = heads(data=12288)
    assert attend(q=same, out=same) == -11
    lib = sh.load_library()
    lib.spechub_tree_attention_workspace_bytes.restype = ctypes.c_size_t
    need = lib.spechub_tree_attention_workspace_bytes(ref(desc()), ctypes.c_int64(0))
    if need:
        assert attend(nbytes=need - 1) == -7
        assert attend(workspace=None) == -1
        assert attend(workspace=ctypes.c_void_p(4104)) == -11
    assert attend(desc(batch=0)) == 0
    assert lib.spechub_tree_attention_workspace_bytes(ref(desc(nodes=0)), ctypes.c_int64(0)) == 0


def test_accept_refuses():
    assert accept(levels=0) == -3
    assert accept(path=None) == -1 and accept(lens_out=None) == -1
    assert accept(lens_out=ctypes.c_void_p(4096)) == -1   # the lengths themselves
    assert accept(desc(batch=0)) == 0


def test_status_strings():
    for code, word in ((-11, "16 bytes"), (-12, "head_dim"), (-13, "rotated"), (-14, "shared"), (-15, "scale")):
        assert word in sh.status_string(code)


def brute(parents):
    n = len(parents)
    sees = np.eye(n, dtype=bool)
    for i in range(n):
        j = parents[i]
        while j >= 0:
            sees[i, j] = True
            j = parents[j]
    return sees


def as_bits(mask, n):
    words = mask.numpy().view(np.uint32)
    return np.array([[bool(words[i, j // 32] >> (j % 32) & 1) for j in range(32 * words.shape[1])] for i in range(n)])


@pytest.mark.parametrize("k,n", [(1, 1), (1, 40), (2, 1), (2, 7), (2, 31), (3, 13), (2, 63), (4, 100)])
def test_tables_of_complete_trees(k, n):
    t = sh.spechub_tree_tables(sh.Tree(levels=1, k=k), n, device="cpu")
    parents = [-1] + [(i - 1) // k for i in range(1, n)]
    bits = as_bits(t["mask"], n)
    np.testing.assert_array_equal(bits[:, :n], brute(parents))
    assert not bits[:, n:].any()
    np.testing.assert_array_equal(t["depth"].numpy(), brute(parents).sum(1) - 1)


def test_tables_of_a_listed_tree():
    parents = [-1, 0, 0, 1, 1, 2, 3]
    t = sh.spechub_tree_tables(sh.Tree.from_parents(parents, device="cpu"), 7, device="cpu")
    np.testing.assert_array_equal(as_bits(t["mask"], 7)[:, :7], brute(parents))
    with pytest.raises(ValueError):
        sh.spechub_tree_tables(sh.Tree.from_parents(parents, device="cpu"), 8, device="cpu")
    with pytest.raises(ValueError):
        sh.spechub_tree_tables(sh.Tree.heap(7), 0, device="cpu")


def test_tensors_off_the_device_are_refused():
    z = torch.zeros((4, 8, 1, 64), dtype=torch.bfloat16)
    one = torch.zeros((1, 1), dtype=torch.int32)
    with pytest.raises(ValueError):
        sh.spechub_cache_accept(z, z, one, one[0], one)
    with pytest.raises(ValueError):
        sh.spechub_tree_attention(z, z, z, one, one[0], one)
    with pytest.raises(ValueError):
        sh.spechub_cache_append(z, z, z, z, z, one, one[0])
    with pytest.raises(TypeError):
        sh.spechub_cache_accept(None, z, one, one[0], one)


def test_no_workspace_for_what_is_refused():
    lib = sh.load_library()
    lib.spechub_tree_attention_workspace_bytes.restype = ctypes.c_size_t
    need = lambda d, shared=0: lib.spechub_tree_attention_workspace_bytes(ref(d), ctypes.c_int64(shared))  # noqa: E731
    assert need(desc(heads=128, kv_heads=1)) > 0 and need(desc(heads=129, kv_heads=1)) == 0 and need(desc(heads=4096, kv_heads=2)) == 0
    assert need(desc(), -1) == 0 and need(desc(), 1 << 30) == 0 and need(desc(), 1 << 40) == 0


def test_a_scale_whose_exponent_of_two_is_no_number():
    assert attend(scale=3.0e38) == -15
    assert attend(scale=2.3e38, nbytes=0) == -7   # (the next check)


def test_rows_that_are_written_over_each_other():
    """Each stride is long enough for a row, and rows meet all the same."""
    for bad in (dict(node=64), dict(node=7 * 64), dict(seq=64), dict(seq=2 * 8 * 64), dict(head=128), dict(head=96), dict(node=24 * 64 - 8)):
        assert append(qo=heads(**bad)) == -11, bad
        assert attend(out=heads(data=1 << 20, **bad)) == -11, bad
    for bad in (dict(page=64), dict(token=64), dict(token=3 * 64), dict(page=15 * 4 * 64), dict(head=16 * 4 * 64), dict(head=128)):
        for call in (append, accept):
            assert call(kc=pages(**bad)) == -11 and call(vc=pages(data=1 << 30, **bad)) == -11, (call.__name__, bad)
    assert accept(desc(layers=3), kc=pages(layer=64)) == -11
    assert accept(desc(layers=3), kc=pages(layer=9 * 16 * 4 * 64), vc=pages(layer=10 * 16 * 4 * 64)) == -11


def test_outputs_over_inputs():
    """Rows of 128 bytes, nodes of 8 rows, sequences of 3 nodes."""
    for far in (128, 1024, 16, 5 * 1024 + 7 * 128 + 112, -16):
        assert attend(q=heads(data=1 << 20), out=heads(data=(1 << 20) + far)) == -11, far
        assert append(q=heads(data=1 << 20), qo=heads(data=(1 << 20) + far)) == -11, far
    assert attend(q=heads(data=1 << 20), out=heads(data=1 << 20, head=72, node=8 * 72, seq=3 * 8 * 72)) == -11   # other strides
    assert append(q=heads(data=1 << 20), qo=heads(data=1 << 20, head=72, node=8 * 72, seq=3 * 8 * 72)) == -11
    packed = dict(node=16 * 64, seq=3 * 16 * 64)      # 8 heads of q, 4 of k, 4 of v
    at = lambda head: heads(data=(1 << 20) + 128 * head, **packed)  # noqa: E731
    assert append(q=at(0), k=at(8), v=at(12), qo=at(1)) == -11      # over q, not q itself
    assert append(q=at(0), k=at(8), v=at(12), qo=at(4)) == -11
    assert append(q=heads(data=1 << 24), k=at(8), v=heads(data=1 << 22), qo=at(1)) == -11      # the last head lies on k's first
    assert append(q=heads(data=1 << 24), k=heads(data=1 << 22), v=at(12), qo=at(6)) == -11


def test_accept_refuses_keys_that_are_values():
    """Two threads would move the same entries, one perhaps after the other has replaced what it reads."""
    far = 10 * 16 * 4 * 128                             # bytes of the keys
    assert accept(vc=pages()) == -11                    # the keys themselves
    assert accept(vc=pages(data=4096 + far - 128)) == -11
    assert accept(vc=pages(data=4096 + far - 16)) == -11
    assert accept(kc=pages(head=16 * 64, token=64)) == -11                                    # the other order of a page, of the same bytes
    side = dict(page=16 * 4 * 128, token=4 * 128, head=128)
    assert accept(kc=pages(**side), vc=pages(data=4096 + 112, **side)) == -11                 # side by side, but for 16 bytes
    assert accept(desc(layers=2), kc=pages(layer=1 << 20), vc=pages(data=4096 + (1 << 21), layer=1 << 20)) == -11   # the values are the second layer


def test_accept_refuses_new_lengths_over_the_old_ones():
    for at in (4096, 4100, 4092):                       # two lengths of 4 bytes
        assert accept(lens_out=ctypes.c_void_p(at)) == -1, at
    assert "lens_out" in sh.status_string(-1)
    assert accept(lens_out=ctypes.c_void_p(4104), kc=pages(token=64)) == -11      # (the next check)
    assert accept(lens_out=ctypes.c_void_p(4088), kc=pages(token=64)) == -11


def test_more_work_than_a_call_counts():
    """By the table's width and the prefix alone, the same for the workspace's size and for the call, whatever the strides."""
    lib = sh.load_library()
    lib.spechub_tree_attention_workspace_bytes.restype = ctypes.c_size_t
    need = lambda d, shared=0: lib.spechub_tree_attention_workspace_bytes(ref(d), ctypes.c_int64(shared))  # noqa: E731
    rows = lambda d, gap, at: heads(data=at, seq=d.nodes * d.heads * 64 + gap, node=d.heads * 64)  # noqa: E731
    wide = dict(batch=128, nodes=8192, heads=64, kv_heads=8, table_width=8192, stride_table=8192)
    for shared, taken, d in ((0, False, desc(**wide)), (0, True, desc(**{**wide, "table_width": 80})),
                             (6400000, False, desc(batch=1024, nodes=65, heads=8, kv_heads=8)),      # 65 rows in a tile, or 128
                             (3200000, True, desc(batch=1024, nodes=65, heads=8, kv_heads=8))):
        assert (need(d, shared) > 0) == taken
        for gap in (0, 64):
            args = dict(q=rows(d, gap, 1 << 30), out=rows(d, gap, 1 << 45), shared=FAKE, width=400000, shared_len=shared)
            assert attend(d, nbytes=0, **args) == (-7 if taken else -16), (taken, gap)
    assert "table" in sh.status_string(-16)


def test_tables_refuse_what_is_no_tree_in_order():
    make = lambda rows, kind=None: sh.Tree(levels=3, child=torch.tensor(rows, dtype=torch.int32),  # noqa: E731
                                           node_kind=None if kind is None else torch.tensor(kind, dtype=torch.uint8))
    none = [-1, -1]
    for rows, word in (([[2, -1], none, [1, -1], none], "later"),          # node 1 comes before its parent
                       ([[1, 2], [1, -1], none, none], "later"),           # ... is its own
                       ([[1, 2], none, [0, -1], none], "later"),
                       ([[1, 2], [3, -1], [3, -1], none], "child of nodes 1 and 2")):
        with pytest.raises(ValueError, match=word):
            sh.spechub_tree_tables(make(rows), 4, device="cpu")
    # children behind the last node are none; both drafts may lead to one node; a leaf's row may hold anything that is not behind it
    t = sh.spechub_tree_tables(make([[1, 2], [3, 3], [9, -1], [0, 0]], [0, 0, 0, 1]), 4, device="cpu")
    np.testing.assert_array_equal(as_bits(t["mask"], 4)[:, :4], brute([-1, 0, 0, 1]))
    assert t["depth"].tolist() == [0, 1, 1, 2]


def test_tables_of_a_long_chain():
    """A prompt's chunk: the mask is a triangle; made in bytes, not number by number."""
    n = 4099
    t = sh.spechub_tree_tables(sh.Tree(levels=n, k=1), n, device="cpu")
    words = t["mask"].numpy().view(np.uint8)
    assert t["mask"].shape == (n, 129) and t["mask"].dtype == torch.int32 and t["mask"].is_contiguous()
    np.testing.assert_array_equal(np.unpackbits(words, axis=1, bitorder="little")[:, :n], np.tri(n, dtype=np.uint8))
    assert not np.unpackbits(words, axis=1, bitorder="little")[:, n:].any()
    assert t["depth"].tolist() == list(range(n))


def test_positions_that_64_bits_do_not_hold():
    for offset in ((1 << 53) + 1, -(1 << 53) - 1, (1 << 63) - 1, -(1 << 63)):
        assert append(offset=offset) == -13, offset
        assert append(offset=offset, rotated=0, qo=heads(head=128)) == -11    # (nothing is rotated; the next check)
    assert append(offset=1 << 53, qo=heads(head=128)) == -11 and append(offset=-(1 << 53), qo=heads(head=128)) == -11
    assert "pos_offset" in sh.status_string(-13)

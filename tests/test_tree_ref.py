"""The plain implementations that the cache-row and tree operators are tested against,
checked on the CPU against torch's own formats and by hand; and the operators' refusals,
which need no GPU."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_37532_amd as dsv
import tree_ref as T
from paper_2609_37532_amd import _lib


# -------------------------------------------------------------------- the reference
def test_e4m3_values_are_torchs():
    codes = np.arange(256, dtype=np.uint8)
    ours = T.e4m3_value(codes)
    theirs = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ours, theirs, equal_nan=True)


def test_e4m3_codes_are_torchs_with_ties_to_even():
    rng = np.random.default_rng(0)
    mids = (T.E4M3[1:] + T.E4M3[:-1]) / 2  # exact ties
    x = np.concatenate([rng.normal(size=4000) * 30, mids, -mids, T.E4M3, [0.0, -0.0, 448.0]])
    x = np.clip(x, -448, 448).astype(np.float32)
    theirs = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(T.e4m3_code(x), theirs)


def test_bf16_rounding_is_torchs():
    x = np.random.default_rng(1).normal(size=4000).astype(np.float32) * 7
    assert np.array_equal(T.bf16_round(x), torch.from_numpy(x).bfloat16().double().numpy())


@pytest.mark.parametrize("top,e", [(448.0, 0), (448.0 * (1 + 2 ** -20), 1), (0.0, -60),
                                   (1.75, -8), (1.7500001, -7), (2.0 ** -80, -60)])
def test_row_exponent(top, e):
    assert T.row_exponent(np.array([0.0, -top])) == e


def test_layouts_cover_a_tile():
    for dim in (64, 128):
        s, d = np.meshgrid(np.arange(16), np.arange(dim), indexing="ij")
        for at in (T.k_offset(s, d, True), T.k_offset(s, d, False), T.v_offset(s, d)):
            assert np.array_equal(np.sort(at.ravel()), np.arange(16 * dim))


def test_masks_and_walk_by_hand():
    parents = [-1, 0, 0, 1, 2, 4]
    masks, depth = T.masks_of(parents)
    assert masks == [1, 0b11, 0b101, 0b1011, 0b10101, 0b110101] and depth == [0, 1, 1, 2, 2, 3]
    #          root chooses 7 (node 2), node 2 chooses 9 (node 4), node 4 chooses 1: none
    assert T.walk([7, 0, 9, 0, 1, 0], [5, 3, 7, 9, 9, 2], parents) == [0, 2, 4]


# ------------------------------------------------------------------------- refusals
FAKE = 4096  # never dereferenced: every call below is refused before a launch


def append_dims(**kw):
    d = dict(rows=4, num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16, num_pages=9,
             in_dtype=dsv.DSV_BF16, kv_dtype=dsv.DSV_FP8, rotary_dim=128, interleaved=0,
             rope_scale=1.0, q_stride=1024, k_stride=256, v_stride=256)
    d.update(kw)
    return dsv.AppendDims(**d)


def append_call(dims, **kw):
    p = dict(q=FAKE, k=FAKE, v=FAKE, pos=FAKE, inv=FAKE, refs=FAKE, live=None, q_out=FAKE,
             pages=FAKE, scales=FAKE)
    p.update(kw)
    return dsv.load().dsv_rope_append(*p.values(), ctypes.byref(dims) if dims else None, None)


@pytest.mark.parametrize("field,value,status", [
    ("rows", 0, -2), ("num_q_heads", -1, -2), ("num_kv_heads", 0, -2), ("head_dim", 96, -3),
    ("page_size", 32, -3), ("num_pages", 0, -2), ("num_pages", 2 ** 27, -2), ("in_dtype", 2, -3),
    ("kv_dtype", 0, -3), ("rotary_dim", 130, -2), ("rotary_dim", 7, -2), ("interleaved", 2, -2),
    ("rope_scale", float("nan"), -2), ("q_stride", 1016, -2), ("q_stride", 1028, -3),
    ("rows", 2 ** 24 + 1, -2), ("num_kv_heads", 2 ** 27, -2), ("num_kv_heads", -1, -2),
    ("k_stride", 248, -2), ("v_stride", 260, -3), ("k_stride", 2 ** 41, -2)])
def test_append_refuses_dims(field, value, status):
    assert append_call(append_dims(**{field: value})) == status


def test_append_refuses_pointers():
    for name in ("q", "k", "v", "pos", "inv", "refs", "q_out", "pages", "scales"):
        assert append_call(append_dims(), **{name: None}) == -1, name
    for name in ("q", "k", "v", "q_out", "pages", "scales"):
        assert append_call(append_dims(), **{name: FAKE + 8}) == -3, name
    assert append_call(None) == -1
    # a bf16 cache has no scales
    assert append_call(append_dims(kv_dtype=dsv.DSV_BF16)) == -3


def read_call(**kw):
    p = dict(pages=FAKE, scales=FAKE, kv_dtype=dsv.DSV_FP8, refs=FAKE, k=FAKE, v=FAKE, out=1,
             rows=5, hkv=2, dim=64, page=16, pages_n=7)
    p.update(kw)
    return dsv.load().dsv_kv_read(*p.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(pages=None), -1), (dict(scales=None), -1), (dict(refs=None), -1), (dict(k=None), -1),
    (dict(v=None), -1), (dict(kv_dtype=0), -3), (dict(kv_dtype=1), -3), (dict(out=2), -3),
    (dict(rows=0), -2), (dict(hkv=0), -2), (dict(rows=2 ** 26 + 1), -2), (dict(dim=80), -3), (dict(page=8), -3),
    (dict(pages_n=0), -2), (dict(v=FAKE + 2), -3), (dict(scales=FAKE + 4), -3)])
def test_read_refuses(kw, status):
    assert read_call(**kw) == status


def tree_dims(**kw):
    d = dict(num_reqs=3, capacity=64, num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16,
             max_pages_per_req=10, num_pages=40, max_kv_len=160, max_nodes=20,
             kv_dtype=dsv.DSV_FP8, scale=0.1)
    d.update(kw)
    return dsv.TreeDims(**d)


def tree_call(dims, ws=FAKE, nbytes=1 << 40, **kw):
    p = dict(q=FAKE, cu=FAKE, masks=None, pages=FAKE, scales=FAKE, table=FAKE, ctx=FAKE, out=FAKE)
    p.update(kw)
    return dsv.load().dsv_tree_attn(*p.values(), ctypes.byref(dims) if dims else None, ws, nbytes,
                                    None)


@pytest.mark.parametrize("field,value,status", [
    ("num_reqs", 0, -2), ("capacity", 0, -2), ("num_q_heads", 7, -2), ("num_q_heads", 6, -3),
    ("head_dim", 32, -3), ("page_size", 64, -3), ("max_kv_len", 161, -2), ("max_nodes", 0, -2),
    ("max_nodes", 65, -2), ("kv_dtype", 0, -3), ("scale", 0.0, -2), ("num_pages", 0, -2)])
def test_tree_attn_refuses_dims(field, value, status):
    d = tree_dims(**{field: value})
    assert dsv.tree_attn_workspace_bytes(d) == 0
    assert tree_call(d) == status


def test_tree_attn_refuses_pointers_and_workspaces():
    assert tree_call(None) == -1
    for name in ("q", "cu", "pages", "scales", "table", "ctx", "out"):
        assert tree_call(tree_dims(), **{name: None}) == -1, name
    for name in ("q", "pages", "scales", "out"):
        assert tree_call(tree_dims(), **{name: FAKE + 4}) == -3, name
    assert tree_call(tree_dims(kv_dtype=dsv.DSV_BF16)) == -3  # scales without codes
    need = dsv.tree_attn_workspace_bytes(tree_dims())
    assert need > 0
    for ws, nbytes in ((None, need), (FAKE + 16, need), (FAKE, need - 1)):
        assert tree_call(tree_dims(), ws=ws, nbytes=nbytes) == -4


def test_tree_work_is_indexed_with_int32():
    # 16 heads of 64 nodes: row groups multiply the segments
    big = dict(num_reqs=1024, num_kv_heads=8, num_q_heads=128, max_nodes=64,
               max_pages_per_req=4096, max_kv_len=65536)
    assert dsv.tree_attn_workspace_bytes(tree_dims(**big)) == 0
    assert dsv.tree_attn_workspace_bytes(tree_dims(**dict(big, num_reqs=16))) > 0


def test_tree_masks_accept_commit_refuse():
    lib = dsv.load()
    m = lambda *a: lib.dsv_tree_masks(*a, None)
    assert m(None, FAKE, FAKE, FAKE, None, 1, 1) == -1 and m(FAKE, FAKE, FAKE, None, None, 1, 1) == -1
    assert m(FAKE, FAKE, FAKE, FAKE, None, 0, 1) == -2 and m(FAKE, FAKE, FAKE, FAKE, None, 1, 0) == -2
    good = dict(lo=FAKE, dt=1, cu=FAKE, draft=FAKE, parents=FAKE, a=FAKE, path=FAKE, nxt=FAKE, b=2,
                cap=9, vocab=100, ws=FAKE, nbytes=1 << 30)
    for kw, status in ((dict(lo=None), -1), (dict(parents=None), -1), (dict(path=None), -1),
                       (dict(b=0), -2), (dict(cap=65536), -2), (dict(vocab=0), -2),
                       (dict(dt=2), -3), (dict(ws=FAKE + 1), -4), (dict(nbytes=8), -4)):
        assert lib.dsv_tree_accept(*dict(good, **kw).values(), None) == status, kw
    good = dict(pages=FAKE, scales=FAKE, dt=2, cu=FAKE, ctx=FAKE, table=FAKE, path=FAKE, b=2, cap=9,
                hkv=2, dim=128, page=16, pmax=4, pages_n=9)
    for kw, status in ((dict(pages=None), -1), (dict(scales=None), -1), (dict(path=None), -1),
                       (dict(dt=1), -3), (dict(b=0), -2), (dict(b=65536), -2), (dict(cap=0), -2),
                       (dict(hkv=0), -2), (dict(dim=100), -3), (dict(page=32), -3),
                       (dict(pmax=0), -2), (dict(pages_n=0), -2), (dict(pages=FAKE + 8), -3)):
        assert lib.dsv_tree_commit(*dict(good, **kw).values(), None) == status, kw


def test_binding_refuses_host_tensors_and_wrong_shapes():
    x = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    pages = torch.zeros((3, 2, 2, 2048), dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: dsv.rope_append(None, x, x, None, None, i, None, pages),
                 lambda: dsv.kv_read(pages, i, x, x),
                 lambda: dsv.tree_masks(i, i, i, i.long()),
                 lambda: dsv.tree_attn(x, i, None, pages, i[:, None], i, x),
                 lambda: dsv.tree_accept(x[0], i, i, i, i, i, i),
                 lambda: dsv.tree_commit(pages, i, i, i[:, None], i)):
        with pytest.raises(ValueError):
            call()


# --------------------------------------------------------------- rotary frequencies
def test_rope_frequencies():
    inv, s = dsv.rope_frequencies(8, 10000.0, device="cpu")
    assert s == 1.0 and np.allclose(inv.numpy(), [1, 0.1, 0.01, 0.001])
    lin, _ = dsv.rope_frequencies(8, scaling="linear", factor=4, device="cpu")
    assert np.allclose(lin.numpy(), inv.numpy() / 4)
    ntk, _ = dsv.rope_frequencies(8, scaling="ntk", factor=4, device="cpu")
    assert np.isclose(ntk[0], inv[0]) and np.isclose(ntk[-1], inv[-1] / 4)
    yarn, s = dsv.rope_frequencies(64, scaling="yarn", factor=4, original_len=4096, device="cpu")
    full = dsv.rope_frequencies(64, device="cpu")[0]
    ratio = (yarn / full).numpy()
    turns = 4096 * full.numpy() / (2 * np.pi)
    assert np.allclose(ratio[turns > 40], 1) and np.allclose(ratio[turns < 0.7], 0.25)
    assert (np.diff(ratio) <= 1e-6).all() and np.isclose(s, 0.1 * np.log(4) + 1)
    for bad in (dict(rotary_dim=7), dict(rotary_dim=8, scaling="else"),
                dict(rotary_dim=8, scaling="yarn"), dict(rotary_dim=8, factor=0.5),
                dict(rotary_dim=2, scaling="ntk")):
        with pytest.raises(ValueError):
            dsv.rope_frequencies(**bad, device="cpu")


def test_structs_match_the_header():
    # rows .. rope_scale are 11 words, padded to the 64-bit strides
    assert ctypes.sizeof(dsv.AppendDims) == 48 + 24 and ctypes.sizeof(dsv.TreeDims) == 48
    assert _lib.AppendDims.q_stride.offset == 48

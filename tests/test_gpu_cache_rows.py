"""GPU: rope_append, kv_read and tree_commit against plain 64-bit implementations.

The cache is exact: k is rotated in double precision and rounded once, so its codes,
scales and bf16 cells equal the 64-bit reference's bit for bit (a value would have to lie
within 2^-40 of a rounding border to differ).  q is rotated in fp32, each output within
half a bf16 step (2^-8 of it) plus three fp32 roundings of its two terms.
"""
import numpy as np
import pytest
import torch

import paper_2609_37532_amd as dsv
import tree_ref as T
from gpu_util import DEV, i32_dev, say

pytestmark = pytest.mark.gpu


def f32_dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEV)


class Pool:
    """A cache on the device with random contents (codes without NaN)."""

    def __init__(self, rng, pages, hkv, dim, fp8):
        self.fp8 = fp8
        shape = (pages, 2, hkv, 16 * dim)
        if fp8:
            cells = rng.integers(0, 127, shape).astype(np.uint8) | (rng.integers(0, 2, shape) * 128).astype(np.uint8)
            self.cells = torch.from_numpy(cells).to(DEV)
            self.scales = torch.from_numpy(rng.integers(110, 130, (pages, hkv, 2, 16)).astype(np.uint8)).to(DEV)
        else:
            self.cells = torch.from_numpy(rng.normal(size=shape).astype(np.float32)).to(DEV).bfloat16()
            self.scales = None

    def host(self):
        if self.fp8:
            return T.Cache(self.cells.cpu().numpy(), self.scales.cpu().numpy())
        return T.Cache(self.cells.double().cpu().numpy())

    def assert_is(self, ref):
        got = self.host()
        assert np.array_equal(got.cells, ref.cells, equal_nan=True)
        if self.fp8:
            assert np.array_equal(got.scales, ref.scales)


def slots(rng, pattern, rows, pages):
    """Distinct slots of `rows` rows: whole pages, prompts from inside a page, a step's
    few rows for each request, or any."""
    if pattern == "scattered":
        return rng.permutation(pages * 16)[:rows]
    ids, refs, pos = list(rng.permutation(pages)), [], 0
    while len(refs) < rows:
        if pattern == "steps":
            first, n = int(rng.integers(0, 16)), int(rng.integers(1, 9))
        elif pattern == "prompts":
            first, n = (int(rng.integers(0, 16)), int(rng.integers(20, 60)))
        else:
            first, n = 0, rows
        page = ids.pop()
        for t in range(first, first + n):
            if t > first and t % 16 == 0:
                page = ids.pop()
            refs.append(page * 16 + t % 16)
    return np.array(refs[:rows])


def projection(rng, rows, hq, hkv, dim, f32):
    x = rng.normal(size=(rows, hq + 2 * hkv, dim)).astype(np.float32)
    x[:, hq:hq + hkv, 3:dim:29] *= 12
    t = torch.from_numpy(x).to(DEV)
    t = t if f32 else t.bfloat16()
    return t, t.double().cpu().numpy()


def check_append(name, seed, rows, hq, hkv, dim, rot, interleaved, f32, fp8, pattern,
                 scale=1.0, start=0, live=None, bad=0):
    say(name, seed, rows, hq, hkv, dim, rot, interleaved, f32, fp8, pattern)
    rng = np.random.default_rng(seed)
    pages = rows // 2 + 70
    pool = Pool(rng, pages, hkv, dim, fp8)
    ref = pool.host()
    x, xh = projection(rng, rows, hq, hkv, dim, f32)
    refs = slots(rng, pattern, rows, pages)
    for r in rng.permutation(rows)[:bad]:
        refs[r] = rng.choice([-1, -7, pages * 16, 2 ** 31 - 1])
    pos = (start + rng.integers(0, 4000, rows)).astype(np.int32)
    inv = None
    if rot:
        inv = (10000.0 ** (-np.arange(rot // 2) / (rot // 2))).astype(np.float32)
    q_out = torch.full((rows, hq, dim), -77.0, dtype=torch.bfloat16, device=DEV)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    dsv.rope_append(q if hq else None, k, v, i32_dev(pos) if rot else None,
                    f32_dev(inv) if rot else None, i32_dev(refs), q_out if hq else None, pool.cells,
                    pool.scales, interleaved=interleaved, rope_scale=scale,
                    num_live=None if live is None else i32_dev([live]))
    torch.cuda.synchronize()
    n = rows if live is None else min(max(live, 0), rows)
    freq = np.zeros(0) if inv is None else inv
    turned = T.rotate(xh, pos, freq, interleaved, np.float64(np.float32(scale)))
    for r in range(n):
        if 0 <= refs[r] < pages * 16:
            ref.write(refs[r], turned[r, hq:hq + hkv], xh[r, hq + hkv:])
    pool.assert_is(ref)
    got = q_out.double().cpu().numpy()
    assert (got[n:] == -77).all()
    if hq and n:
        # both terms of a pair, each with its product and factor rounded, and their sum
        mag = np.abs(xh[:n, :hq]).max(-1, keepdims=True) * 2 * max(scale, 1)
        off = np.abs(got[:n] - turned[:n, :hq])
        assert (off <= 2.0 ** -8 * np.abs(turned[:n, :hq]) + 4 * 2.0 ** -24 * mag).all()
    return pool, ref


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("pattern,rows", [("pages", 1), ("pages", 16), ("pages", 77), ("prompts", 131),
                                          ("steps", 53), ("scattered", 40)])
def test_append_slot_patterns(fp8, pattern, rows):
    check_append("append", rows, rows, 8, 2, 128, 128, False, False, fp8, pattern)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rot,interleaved", [(0, False), (2, False), (20, False), (20, True), (32, False),
                                             (48, True), (64, False), (64, True)])
@pytest.mark.parametrize("f32,fp8", [(False, True), (True, False), (True, True)])
def test_append_layouts(dim, rot, interleaved, f32, fp8):
    check_append("layout", rot + dim, 37, 4, 4, dim, rot, interleaved, f32, fp8, "prompts")


@pytest.mark.parametrize("hq,hkv", [(0, 1), (1, 1), (40, 8), (16, 16), (7, 3)])
def test_append_heads(hq, hkv):
    check_append("heads", 5, 33, hq, hkv, 128, 128, False, False, True, "prompts")


def test_append_many_rows_and_heads_together():
    # more than 1,024 (chunk, head) pairs: several heads to a workgroup, four q rows to one
    check_append("many", 6, 2100, 3, 9, 64, 64, False, False, True, "prompts")
    check_append("many", 7, 2049, 2, 10, 64, 64, True, False, False, "steps")


@pytest.mark.parametrize("live", [0, 1, 17, 50, 99, -4])
def test_append_live_rows(live):
    check_append("live", 8, 50, 4, 2, 128, 128, False, False, True, "prompts", live=live)


@pytest.mark.parametrize("fp8", [False, True])
def test_append_skips_slots_out_of_range(fp8):
    check_append("bad", 9, 60, 4, 2, 64, 64, False, False, fp8, "prompts", bad=13)
    check_append("all bad", 10, 20, 4, 2, 64, 64, False, False, fp8, "pages", bad=20)


@pytest.mark.parametrize("start", [1_000_000, 2 ** 31 - 5000, -3000])
def test_append_far_positions(start):
    check_append("far", 11, 24, 2, 2, 128, 128, False, True, True, "pages", start=start, scale=1.25)


def test_append_values_that_are_not_finite_and_rows_of_nothing():
    dim, hkv = 64, 1
    for fp8 in (True, False):
        rng = np.random.default_rng(12)
        pool = Pool(rng, 4, hkv, dim, fp8)
        ref = pool.host()
        x = rng.normal(size=(6, 2 * hkv, dim)).astype(np.float32)
        x[0] = 0.0
        x[1, :, 3] = np.inf
        x[2, :, 5] = np.nan
        x[3] = -np.inf
        x[4] *= 1e-30
        x[5] *= 1e30
        t = torch.from_numpy(x).to(DEV)
        refs = np.arange(17, 23)
        dsv.rope_append(None, t[:, :1], t[:, 1:], None, None, i32_dev(refs), None, pool.cells, pool.scales)
        for r in range(6):
            ref.write(refs[r], x[r, :1].astype(np.float64), x[r, 1:].astype(np.float64))
        if fp8:  # NaN codes may carry either sign
            got = pool.host()
            assert np.array_equal(got.scales, ref.scales)
            assert np.array_equal(T.e4m3_value(got.cells), T.e4m3_value(ref.cells), equal_nan=True)
        else:
            pool.assert_is(ref)


def test_append_q_in_place_and_graph_replays():
    rng = np.random.default_rng(13)
    rows, hq, hkv, dim = 29, 8, 2, 128
    pool = Pool(rng, 40, hkv, dim, True)
    refs = i32_dev(slots(rng, "prompts", rows, 40))
    inv = dsv.rope_frequencies(dim)[0]
    q = torch.zeros((rows, hq, dim), dtype=torch.bfloat16, device=DEV)
    kv = torch.zeros((rows, 2 * hkv, dim), dtype=torch.bfloat16, device=DEV)
    pos = i32_dev(np.zeros(rows))
    k_out = torch.empty((rows, hkv, dim), dtype=torch.bfloat16, device=DEV)
    v_out = torch.empty_like(k_out)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = dsv.Graph().capture(lambda: (
        dsv.rope_append(q, kv[:, :hkv], kv[:, hkv:], pos, inv, refs, q, pool.cells, pool.scales, stream=s),
        dsv.kv_read(pool.cells, refs, k_out, v_out, pool.scales, stream=s)), s)
    for step in range(3):
        qs = torch.randn(q.shape, device=DEV).bfloat16()
        kvs = torch.randn(kv.shape, device=DEV).bfloat16()
        at = i32_dev(rng.integers(0, 9000, rows))
        q.copy_(qs), kv.copy_(kvs), pos.copy_(at)
        torch.cuda.synchronize()
        g.replay(s)
        torch.cuda.synchronize()
        other, k2, v2 = torch.empty_like(q), torch.empty_like(k_out), torch.empty_like(v_out)
        dsv.rope_append(qs, kvs[:, :hkv], kvs[:, hkv:], at, inv, refs, other, pool.cells, pool.scales)
        dsv.kv_read(pool.cells, refs, k2, v2, pool.scales)
        torch.cuda.synchronize()
        assert torch.equal(other, q) and torch.equal(k2, k_out) and torch.equal(v2, v_out)
    g.close()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("pattern,rows,dim", [("pages", 1, 128), ("pages", 100, 64), ("prompts", 90, 128),
                                              ("steps", 61, 64), ("scattered", 70, 128), ("again", 40, 64)])
def test_read(fp8, f32, pattern, rows, dim):
    say("read", fp8, f32, pattern, rows, dim)
    rng = np.random.default_rng(rows)
    pages, hkv = 80, 3
    pool = Pool(rng, pages, hkv, dim, fp8)
    refs = rng.integers(0, 40, rows) if pattern == "again" else slots(rng, pattern, rows, pages)
    if rows > 8:  # entries outside the cache are zeros
        refs[rng.permutation(rows)[:5]] = [-1, pages * 16, -2 ** 31, 2 ** 31 - 1, pages * 16 + 3]
    dtype = torch.float32 if f32 else torch.bfloat16
    out = [torch.full((rows, hkv, dim), float("nan"), dtype=dtype, device=DEV) for _ in range(2)]
    dsv.kv_read(pool.cells, i32_dev(refs), *out, pool.scales)
    ok = (refs >= 0) & (refs < pages * 16)
    want = pool.host().read(np.where(ok, refs, 0))
    for got, w in zip(out, want):
        assert np.array_equal(got.double().cpu().numpy(), np.where(ok[:, None, None], w, 0.0))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("dim,k", [(128, 1), (128, 64), (64, 17), (64, 64)])
def test_commit(fp8, dim, k):
    say("commit", fp8, dim, k)
    rng = np.random.default_rng(k + dim)
    B, hkv = 5, 2
    ctx = rng.integers(0, 50, B)
    ctx[0] = 0
    nodes = np.array([k, max(1, k // 2), 0, k, k])
    pmax = (int(ctx.max()) + k) // 16 + 1
    pages = B * pmax + 3
    pool = Pool(rng, pages, hkv, dim, fp8)
    ref = pool.host()
    table = rng.permutation(pages)[:B * pmax].reshape(B, pmax)
    cu = np.concatenate([[0], np.cumsum(nodes)])
    cap = int(cu[-1]) + 3
    path = np.full(cap, 12345)
    moved = ref.cells.copy(), None if ref.scales is None else ref.scales.copy()
    src = T.Cache(*moved)
    for i in range(B):
        n = int(nodes[i])
        if not n:
            continue
        # all nodes (a chain), the last ones, a random path, and one cut by a bad entry
        mine = [list(range(n)), list(range(n))[-(n // 2 + 1):], [], None, None][i]
        if mine is None:
            mine = [0] + sorted(rng.permutation(np.arange(1, n))[:n // 3].tolist())
        row = mine + [-1] * (n - len(mine))
        if i == 4 and len(mine) > 2:
            row[2] = n  # not a node: the path ends here
            mine = mine[:2]
        path[cu[i]:cu[i + 1]] = row
        slot = lambda t: int(table[i, t // 16]) * 16 + t % 16
        for m, node in enumerate(mine):
            a, b = slot(int(ctx[i]) + node), slot(int(ctx[i]) + m)
            d = np.arange(dim)
            for kind in (0, 1):
                at = (lambda s: T.k_offset(s, d, fp8)) if kind == 0 else (lambda s: T.v_offset(s, d))
                ref.cells[b // 16, kind][:, at(b % 16)] = src.cells[a // 16, kind][:, at(a % 16)]
            if fp8:
                ref.scales[b // 16, :, :, b % 16] = src.scales[a // 16, :, :, a % 16]
    dsv.tree_commit(pool.cells, i32_dev(cu), i32_dev(ctx), i32_dev(table), i32_dev(path), pool.scales)
    pool.assert_is(ref)


def test_commit_skips_bad_metadata():
    rng = np.random.default_rng(3)
    pool = Pool(rng, 12, 1, 64, True)
    ref = pool.host()
    table = np.arange(12).reshape(4, 3)
    table[0, 0] = 99   # a page outside the pool: its rows are not moved
    cu = [0, 5, 10, 15, 20]
    ctx = [0, -1, 45, 0]  # negative; past the page table
    path = [0, 2, 4, -1, -1] * 3 + [-1] * 5
    dsv.tree_commit(pool.cells, i32_dev(cu), i32_dev(ctx), i32_dev(table), i32_dev(path), pool.scales)
    pool.assert_is(ref)


def test_slots_past_32_bits_of_cells():
    """A pool of more than 2^32 cells: the last pages are written, read and moved."""
    pages, hkv, dim = 1_060_000, 1, 128
    cells = torch.zeros((pages, 2, hkv, 16 * dim), dtype=torch.uint8, device=DEV)
    scales = torch.zeros((pages, hkv, 2, 16), dtype=torch.uint8, device=DEV)
    assert cells.numel() > 2 ** 32
    rows = 40
    refs = np.concatenate([np.arange(20), pages * 16 - 20 + np.arange(20)])
    x = torch.randn((rows, 2, dim), device=DEV).bfloat16()
    inv, _ = dsv.rope_frequencies(dim)
    pos = i32_dev(np.arange(rows))
    dsv.rope_append(None, x[:, :1], x[:, 1:], pos, inv, i32_dev(refs), None, cells, scales)
    k, v = (torch.empty((rows, 1, dim), dtype=torch.float32, device=DEV) for _ in range(2))
    dsv.kv_read(cells, i32_dev(refs), k, v, scales)
    xh = x.double().cpu().numpy()
    want = T.Cache(np.zeros((3, 2, 1, 16 * dim), np.uint8), np.zeros((3, 1, 2, 16), np.uint8))
    turned = T.rotate(xh[:, :1], np.arange(rows), inv.double().cpu().numpy(), False)
    for r in range(rows):
        want.write(r, turned[r], xh[r, 1:])
    wk, wv = want.read(np.arange(rows))
    assert np.array_equal(k.double().cpu().numpy(), wk)
    assert np.array_equal(v.double().cpu().numpy(), wv)
    # the last page: node 3 to position 1
    table = i32_dev([[pages - 1]])
    dsv.tree_commit(cells, i32_dev([0, 4]), i32_dev([0]), table, i32_dev([0, 3, -1, -1]), scales)
    at = i32_dev([pages * 16 - 16 + 1, pages * 16 - 16 + 3])
    k, v = k[:2].clone(), v[:2].clone()
    dsv.kv_read(cells, at, k, v, scales)
    assert torch.equal(k[0], k[1]) and torch.equal(v[0], v[1])


def test_binding_refuses():
    rng = np.random.default_rng(1)
    pool = Pool(rng, 4, 2, 64, True)
    x = torch.zeros((3, 6, 64), dtype=torch.bfloat16, device=DEV)
    q, k, v = x[:, :2], x[:, 2:4], x[:, 4:]
    out, refs = torch.zeros_like(q).contiguous(), i32_dev([0, 1, 2])
    inv, _ = dsv.rope_frequencies(64)
    pos = i32_dev([0, 1, 2])
    good = dict(q=q, k=k, v=v, positions=pos, inv_freq=inv, kv_refs=refs, q_out=out,
                kv_pages=pool.cells, kv_scales=pool.scales)
    dsv.rope_append(**good)
    bad = [dict(k=k[:2]), dict(v=v.float()), dict(q=q.transpose(0, 1)), dict(q_out=out[:, :1]),
           dict(positions=pos[:2]), dict(positions=pos.long()), dict(inv_freq=inv.double()),
           dict(kv_refs=refs.long()), dict(kv_scales=pool.scales[:2]), dict(kv_scales=None),
           dict(k=x[:, 2:3]), dict(num_live=i32_dev([1, 2])), dict(k=k[..., ::2])]
    for kw in bad:
        with pytest.raises(ValueError):
            dsv.rope_append(**{**good, **kw})
    odd = torch.zeros(3 * 6 * 64 + 4, dtype=torch.bfloat16, device=DEV)[4:].view(3, 6, 64)
    with pytest.raises(dsv.DSVError):  # rows off 16 bytes
        dsv.rope_append(**{**good, "k": odd[:, 2:4]})
    with pytest.raises(dsv.DSVError):  # more frequencies than pairs
        dsv.rope_append(**{**good, "inv_freq": dsv.rope_frequencies(66)[0]})
    torch.cuda.synchronize()

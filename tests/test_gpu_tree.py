"""GPU: tree_masks, tree_attn and tree_accept against plain 64-bit implementations, and
the operators of a tree step together.

Attention tolerance: the output is rounded once to bf16 (2^-8 of it).  Before that, a
score is an fp32 dot product, off by at most dim * 2^-24 of the sum of its terms'
magnitudes (|q| |k| is at most 14 * 14 for the rows here, so 2^-12 of a scaled score's
unit), a weight carries that twice (itself and in the sum) and 2^-17 of its pair of bf16
parts, and the outputs are averages of values of magnitude `top`: 2^-10 * top together.
"""
import numpy as np
import pytest
import torch

import paper_2609_37532_amd as dsv
import tree_ref as T
from gpu_util import DEV, i32_dev, say

pytestmark = pytest.mark.gpu


def signed(masks):
    return torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64, device=DEV)


class Case:
    """A random batch: trees (or causal chains without masks) over a paged cache."""

    def __init__(self, seed, ctx, nodes, hkv=2, group=4, dim=128, fp8=False, masks="tree", extra=3,
                 max_nodes=None):
        rng = self.rng = np.random.default_rng(seed)
        self.ctx, self.nodes, self.hkv, self.dim, self.fp8 = list(ctx), list(nodes), hkv, dim, fp8
        B = len(ctx)
        self.cu = np.concatenate([[0], np.cumsum(nodes)])
        self.live = int(self.cu[-1])
        cap = max(1, self.live + extra)
        self.max_len = max(1, max(c + k for c, k in zip(ctx, nodes)))
        pmax = -(-self.max_len // 16)
        pages = B * pmax + 2
        self.table = rng.permutation(pages)[:B * pmax].reshape(B, pmax)
        self.q = torch.from_numpy(rng.normal(size=(cap, hkv * group, dim)).astype(np.float32)).to(DEV).bfloat16()
        shape = (pages, 2, hkv, 16 * dim)
        if fp8:  # normal values under scales of 2^-6 .. 2^-4
            x = torch.from_numpy((rng.normal(size=shape) * 40).astype(np.float32)).to(DEV)
            self.pages = x.to(torch.float8_e4m3fn).view(torch.uint8)
            self.scales = torch.from_numpy(rng.integers(121, 124, (pages, hkv, 2, 16)).astype(np.uint8)).to(DEV)
        else:
            self.pages = torch.from_numpy(rng.normal(size=shape).astype(np.float32)).to(DEV).bfloat16()
            self.scales = None
        self.parents = [p for k in nodes for p in T.random_tree(rng, k)]
        self.masks = None
        if masks == "tree":
            self.masks = [m for i in range(B) for m in T.masks_of(self.parents[self.cu[i]:self.cu[i + 1]])[0]]
        elif masks == "any":  # any bits, also past the nodes; some rows see no node
            self.masks = [int(x) for x in rng.integers(0, 2 ** 63, self.live, dtype=np.uint64)]
            for j in range(0, self.live, 3):
                self.masks[j] = 0
        self.max_nodes = max_nodes or max(1, max(nodes))
        self.out = torch.full((cap, hkv * group, dim), float("nan"), dtype=torch.bfloat16, device=DEV)

    def run(self, stream=None, workspace=None):
        masks = None
        if self.masks is not None:
            masks = torch.cat([signed(self.masks), torch.zeros(self.q.shape[0] - self.live, dtype=torch.int64, device=DEV)])
        dsv.tree_attn(self.q, i32_dev(self.cu), masks, self.pages, i32_dev(self.table), i32_dev(self.ctx),
                      self.out, self.scales, max_nodes=self.max_nodes, max_kv_len=self.max_len,
                      workspace=workspace, stream=stream)
        return self

    def sees(self, i):
        k, c = self.nodes[i], self.ctx[i]
        s = np.ones((k, c + k), bool)
        for j in range(k):
            m = (1 << j + 1) - 1 if self.masks is None else self.masks[self.cu[i] + j]
            s[j, c:] = [(m >> n & 1) == 1 for n in range(k)]
        return s

    def cells(self):
        if self.fp8:
            return T.Cache(self.pages.cpu().numpy(), self.scales.cpu().numpy())
        return T.Cache(self.pages.double().cpu().numpy())

    def want(self):
        cache, q = self.cells(), self.q.double().cpu().numpy()
        out = np.zeros(q.shape)
        for i, (c, k) in enumerate(zip(self.ctx, self.nodes)):
            if k:
                t = np.arange(c + k)
                keys, values = cache.read(self.table[i][t // 16].astype(np.int64) * 16 + t % 16)
                o = self.cu[i]
                out[o:o + k] = T.attend(q[o:o + k], keys, values, self.sees(i), self.dim ** -0.5)
        return out

    def check(self, name):
        say(name, self.ctx[:4], self.nodes[:4], self.hkv, self.q.shape, self.fp8)
        self.run()
        got, want = self.out.double().cpu().numpy(), self.want()
        assert not got[self.live:].any(), "tail rows are zeros"
        assert np.array_equal(np.isnan(got), np.isnan(want))
        finite = np.isfinite(want)
        assert np.array_equal(got[~finite], want[~finite], equal_nan=True)
        off = np.abs(got[finite] - want[finite])
        top = np.abs(want[finite]).max(initial=0) + 4.0  # values are normal
        bound = 2.0 ** -8 * np.abs(want[finite]) + 2.0 ** -10 * top
        assert (off <= bound).all(), "off by up to %.3g" % (off - bound).max()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 2, 4, 8, 16])
def test_head_groups_and_tree_sizes(group, dim, fp8):
    """Every form: from one row tile to several row groups, ragged trees in one batch."""
    for most in (1, 5, 16, 33, 64):
        nodes = [most, max(1, most // 2), 0, 1, most]
        Case(most + group, [70, 300, 40, 1, 515], nodes, group=group, dim=dim, fp8=fp8).check("group")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("masks", ["tree", "any", None])
@pytest.mark.parametrize("ctx", [0, 1, 15, 16, 31, 32, 33, 64])
def test_contexts_and_page_edges(ctx, masks, fp8):
    Case(ctx, [ctx, ctx, 0], [64, 19, 3], hkv=1, fp8=fp8, masks=masks).check("edge")


def test_rows_that_see_nothing_are_zero():
    c = Case(3, [0, 0, 40], [5, 33, 4], masks="any")
    c.masks = [0] * c.live
    c.run()
    got = c.out.double().cpu().numpy()
    assert not got[:38].any() and got[38:42].all()
    c.check("nothing")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("reqs,hkv,ctx,nodes", [(1, 8, 900, 16), (3, 2, 5000, 40), (40, 2, 700, 12),
                                                (2, 1, 20000, 64), (70, 4, 130, 7), (300, 1, 60, 5)])
def test_work_splits(reqs, hkv, ctx, nodes, fp8):
    """Pieces of segments, stream-K shares, more than one request to a planning thread."""
    rng = np.random.default_rng(reqs)
    ctxs = rng.integers(ctx // 2, ctx + 1, reqs).tolist()
    ks = rng.integers(1, nodes + 1, reqs).tolist()
    Case(reqs, ctxs, ks, hkv=hkv, group=4 if reqs < 100 else 1, dim=64 if reqs > 50 else 128,
         fp8=fp8).check("split")


@pytest.mark.parametrize("dim", [64, 128])
def test_many_requests_of_several_row_groups(dim):
    """More requests than a planning thread's one, some of them cut into row groups."""
    rng = np.random.default_rng(dim)
    nodes = rng.integers(0, 4, 530)
    nodes[rng.permutation(530)[:12]] = rng.integers(17, 40, 12)
    ctx = rng.integers(0, 60, 530)
    Case(dim, ctx.tolist(), nodes.tolist(), hkv=1, group=16, dim=dim, fp8=dim == 128).check("many")


def test_two_streams_at_once():
    """Calls that overlap, each with its own workspace."""
    cases = [Case(31, [900, 40, 3000], [40, 64, 9], fp8=True), Case(32, [2000, 700], [33, 64], group=8)]
    base = [c.run().out.clone() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(4):
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                c.out.fill_(float("nan"))
                c.run()
        torch.cuda.synchronize()
        for c, b in zip(cases, base):
            assert torch.equal(c.out, b)


@pytest.mark.parametrize("as_handle", [False, True])
def test_a_workspace_of_the_calls_own_on_another_stream(as_handle):
    """Without a workspace argument the call's own is ordered with its stream, whatever
    the current stream allocates and writes meanwhile."""
    c = Case(33, [5000, 3000, 40], [64, 20, 9])
    base = c.run().out.clone()
    masks = torch.cat([signed(c.masks), torch.zeros(3, dtype=torch.int64, device=DEV)])
    cu, table, ctx = i32_dev(c.cu), i32_dev(c.table), i32_dev(c.ctx)
    dims = dsv.tree_attn_dims(c.q, c.pages, table, max_nodes=64, max_kv_len=c.max_len)
    nbytes = dsv.tree_attn_workspace_bytes(dims)
    s = torch.cuda.Stream()
    for _ in range(4):
        c.out.fill_(float("nan"))
        torch.cuda.synchronize()
        for _ in range(3):
            dsv.tree_attn(c.q, cu, masks, c.pages, table, ctx, c.out, dims=dims,
                          stream=int(s.cuda_stream) if as_handle else s)
            torch.full((nbytes + 256,), 255, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        assert torch.equal(c.out, base)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("group", [1, 4, 16])
def test_values_that_are_not_finite_in_unseen_nodes(group, fp8):
    """Infinities and NaN in K and V of nodes reach the rows that see them, and no other."""
    c = Case(7, [37, 0, 100], [30, 64, 11], hkv=1, group=group, dim=64, fp8=fp8)
    for i, node, kind, dims, bits in ((0, 4, 1, [3], 0x7F80), (0, 9, 1, [3, 60], 0xFF80),
                                      (0, 20, 1, [17], 0x7FC0), (1, 50, 0, [1], 0x7FC0),
                                      (1, 63, 1, [0, 33], 0x7F80), (2, 10, 1, [5], 0xFFC0)):
        t = c.ctx[i] + node
        page, slot = int(c.table[i][t // 16]), t % 16
        for d in dims:
            at = T.v_offset(slot, d) if kind else T.k_offset(slot, d, fp8)
            if fp8:
                c.pages[page, kind, 0, at] = 0x7F
            else:
                c.pages.view(torch.int16)[page, kind, 0, at] = bits - 65536 if bits > 32767 else bits
    c.check("not finite")


def test_what_lies_past_the_nodes_is_not_read_as_keys():
    for fp8 in (False, True):
        c = Case(8, [20, 3], [5, 9], fp8=fp8, masks="any")
        c.masks = [2 ** 64 - 1] * c.live  # bits past the nodes too
        for i in range(2):
            for t in range(c.ctx[i] + c.nodes[i], c.table.shape[1] * 16):
                page, slot, d = int(c.table[i][t // 16]), t % 16, torch.arange(c.dim, device=DEV)
                for kind, at in ((0, T.k_offset(slot, d, fp8)), (1, T.v_offset(slot, d))):
                    c.pages[page, kind, :, at] = 0x7F if fp8 else float("nan")
                if fp8:
                    c.scales[page, :, :, slot] = 255
        c.check("past")


def test_bad_metadata_is_skipped():
    c = Case(9, [30, 40, 50, 60], [4, 6, 5, 3], max_nodes=5)
    before = c.out.clone()
    c.run()
    got, want = c.out.double().cpu().numpy(), c.want()
    assert torch.equal(c.out[4:10].isnan(), before[4:10].isnan())  # six nodes of at most five: left
    for a, b in ((0, 4), (10, 18)):
        assert np.abs(got[a:b] - want[a:b]).max() < 0.05
    c = Case(10, [30, 40], [4, 6])
    c.table[0, 1] = 10 ** 6  # outside the pool: unspecified for this request, fine for the next
    c.ctx = [30, 40]
    c.run()
    c.table[0, 1] = 0
    assert np.abs(c.out.double().cpu().numpy()[4:10] - c.want()[4:10]).max() < 0.05


def test_causal_block_is_verify_attention():
    """Without masks and with a bf16 cache: the same rows as verify_attn's."""
    c = Case(11, [500, 33, 1200], [16, 9, 1], masks=None, hkv=4).run()
    other = torch.empty_like(c.out)
    dsv.verify_attn(c.q, i32_dev(c.cu), c.pages, i32_dev(c.table), i32_dev(c.ctx), other,
                    max_kv_len=c.max_len)
    d = (other.double() - c.out.double()).abs()
    assert (d <= 2.0 ** -7 * other.double().abs() + 2.0 ** -12).all()


def test_deterministic_on_another_stream_and_in_replays():
    c = Case(12, [900, 30, 2000], [40, 64, 7], fp8=True, group=8)
    c.run()
    base = c.out.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        c.out.fill_(float("nan"))
        c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.out, base)
    # two graphs that share a workspace, replayed in turn with eager work between
    dims = dsv.tree_attn_dims(c.q, c.pages, i32_dev(c.table), c.scales, max_nodes=64, max_kv_len=c.max_len)
    ws = dsv.alloc_workspace(dsv.tree_attn_workspace_bytes(dims))
    masks = torch.cat([signed(c.masks), torch.zeros(3, dtype=torch.int64, device=DEV)])
    cu, table, ctx = i32_dev(c.cu), i32_dev(c.table), i32_dev(c.ctx)
    q2, out2 = torch.randn(c.q.shape, device=DEV).bfloat16(), torch.empty_like(c.out)
    call = lambda q, out, **kw: dsv.tree_attn(q, cu, masks, c.pages, table, ctx, out, c.scales, dims=dims,
                                              workspace=ws, **kw)
    call(q2, out2)
    base2 = out2.clone()
    torch.cuda.synchronize()
    g1 = dsv.Graph().capture(lambda: call(c.q, c.out, stream=side), side)
    g2 = dsv.Graph().capture(lambda: call(q2, out2, stream=side), side)
    for _ in range(3):
        c.out.fill_(float("nan")), out2.fill_(float("nan"))
        torch.cuda.synchronize()
        g1.replay(side), g2.replay(side)
        torch.cuda.synchronize()
        assert torch.equal(c.out, base) and torch.equal(out2, base2)
        dsv.tree_attn(q2, cu, None, c.pages, table, ctx, torch.empty_like(out2), c.scales, dims=dims, workspace=ws)
    torch.cuda.synchronize()
    g1.close(), g2.close()


# ------------------------------------------------------------------ masks and acceptance
def test_masks():
    rng = np.random.default_rng(0)
    nodes = [64, 1, 0, 33, 2, 64, 65, 64]  # one tree too large: left as it was
    cu = np.concatenate([[0], np.cumsum(nodes)])
    parents = np.concatenate([T.random_tree(rng, k, p) for k, p in zip(nodes, [0.2, 1, 1, 0.5, 0, 1, 0, 0.9])]).astype(np.int64)
    parents[cu[3] + 5], parents[cu[3] + 9] = 5, 40  # not before their nodes: roots
    parents = np.append(parents, [7, 7])
    cap = len(parents)
    ctx = rng.integers(0, 5000, len(nodes))
    masks = torch.full((cap,), -5, dtype=torch.int64, device=DEV)
    pos = torch.full((cap,), -5, dtype=torch.int32, device=DEV)
    dsv.tree_masks(i32_dev(parents), i32_dev(cu), i32_dev(ctx), masks, pos)
    wm, wp = np.full(cap, -5, np.int64), np.full(cap, -5, np.int32)
    for i, k in enumerate(nodes):
        if k <= 64:
            m, d = T.masks_of(parents[cu[i]:cu[i + 1]])
            wm[cu[i]:cu[i + 1]] = np.array(m, np.uint64).view(np.int64)
            wp[cu[i]:cu[i + 1]] = ctx[i] + np.array(d, int)
    assert np.array_equal(masks.cpu().numpy(), wm) and np.array_equal(pos.cpu().numpy(), wp)
    again = torch.full_like(masks, -5)
    dsv.tree_masks(i32_dev(parents), i32_dev(cu), i32_dev(ctx), again)
    assert torch.equal(masks, again)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("vocab,most", [(7, 64), (1000, 13), (50257, 40), (131073, 64)])
def test_accept(vocab, most, bf16):
    """Random trees; small vocabularies make ties, equal siblings and wrong turns common."""
    say("accept", vocab, most, bf16)
    rng = np.random.default_rng(most)
    nodes = rng.integers(1, most + 1, 9).tolist() + [0, 1, most]
    cu = np.concatenate([[0], np.cumsum(nodes)])
    live, cap = int(cu[-1]), int(cu[-1]) + 4
    parents = np.concatenate([T.random_tree(rng, k, 0.5) for k in nodes if k] + [[0] * 4]).astype(np.int64)
    parents[cu[0]], parents[cu[4] + nodes[4] - 1] = 3, 64  # a root's entry is not used
    logits = torch.from_numpy(rng.integers(-3, 3, (cap, vocab)).astype(np.float32)).to(DEV)
    draft = rng.integers(0, vocab, cap)
    for i, k in enumerate(nodes):
        for j in range(1, k):
            p = parents[cu[i] + j]
            if 0 <= p < j and rng.random() < 0.6:
                logits[cu[i] + p, draft[cu[i] + j]] = 9.0
    logits = logits.bfloat16() if bf16 else logits
    choice = logits.float().cpu().numpy().argmax(1)
    n = len(nodes)
    a, nxt = (torch.full((n,), -9, dtype=torch.int32, device=DEV) for _ in range(2))
    path = torch.full((cap,), -9, dtype=torch.int32, device=DEV)
    dsv.tree_accept(logits, i32_dev(cu), i32_dev(draft), i32_dev(parents), a, path, nxt)
    wa, wn, wp = np.zeros(n, int), np.full(n, -1), np.full(cap, -9)
    for i, k in enumerate(nodes):
        if not k:
            continue
        rows = slice(cu[i], cu[i + 1])
        w = T.walk(choice[rows], draft[rows], parents[rows])
        wa[i], wn[i] = len(w) - 1, choice[cu[i] + w[-1]]
        wp[rows] = w + [-1] * (k - len(w))
    assert np.array_equal(a.cpu().numpy(), wa) and np.array_equal(nxt.cpu().numpy(), wn)
    assert np.array_equal(path.cpu().numpy(), wp)
    assert wa.max() > 1 or most < 5


def test_a_chain_is_accepts_prefix():
    rng = np.random.default_rng(5)
    nodes = [16, 1, 0, 9]
    cu = np.concatenate([[0], np.cumsum(nodes)])
    cap, vocab = 30, 333
    logits = torch.randn((cap, vocab), device=DEV)
    draft = rng.integers(0, vocab, cap)
    for r in (0, 1, 2, 17, 18, 19, 20):
        logits[r, draft[r + 1]] = 20.0
    parents = np.concatenate([np.arange(k) - 1 for k in nodes] + [[0] * (cap - int(cu[-1]))])
    make = lambda: [torch.zeros(4, dtype=torch.int32, device=DEV) for _ in range(2)]
    (a, t), (b, u) = make(), make()
    path = torch.zeros(cap, dtype=torch.int32, device=DEV)
    dsv.accept(logits, i32_dev(cu), i32_dev(draft), a, t)
    dsv.tree_accept(logits, i32_dev(cu), i32_dev(draft), i32_dev(parents), b, path, u)
    assert torch.equal(a, b) and torch.equal(t, u)


# --------------------------------------------------------------------------- a step
@pytest.mark.parametrize("fp8", [False, True])
def test_a_tree_step(fp8):
    """Prompt, tree, acceptance and commit: afterwards the cache is what a linear decode
    of the accepted tokens would have left, and attention over it agrees."""
    rng = np.random.default_rng(21)
    B, hkv, group, dim, vocab, most = 3, 2, 4, 128, 500, 20
    hq = hkv * group
    ctx, nodes = [45, 0, 130], [20, 13, 7]
    pmax = 12
    table = rng.permutation(B * pmax + 4)[:B * pmax].reshape(B, pmax)
    shape = (B * pmax + 4, 2, hkv, 16 * dim)
    pages = torch.zeros(shape, dtype=torch.uint8 if fp8 else torch.bfloat16, device=DEV)
    scales = torch.zeros((shape[0], hkv, 2, 16), dtype=torch.uint8, device=DEV) if fp8 else None
    inv, rs = dsv.rope_frequencies(dim, scaling="yarn", factor=4, original_len=4096)
    slot = lambda i, t: table[i, t // 16] * 16 + t % 16
    tab, cxd = i32_dev(table), i32_dev(ctx)
    # the prompts, packed
    pos = np.concatenate([np.arange(c) for c in ctx])
    refs = np.concatenate([[slot(i, t) for t in range(c)] for i, c in enumerate(ctx)])
    x = torch.randn((len(pos), hq + 2 * hkv, dim), device=DEV).bfloat16()
    q_out = torch.empty((len(pos), hq, dim), dtype=torch.bfloat16, device=DEV)
    put = lambda x, pos, refs, q_out, live=None: dsv.rope_append(
        x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], pos, inv, refs, q_out, pages, scales, rope_scale=rs,
        num_live=live)
    put(x, i32_dev(pos), i32_dev(refs), q_out)
    # the trees
    cu = np.concatenate([[0], np.cumsum(nodes)])
    cap = B * most
    cud = i32_dev(cu)
    parents = np.concatenate([T.random_tree(rng, k, 0.5) for k in nodes] + [[0] * (cap - int(cu[-1]))])
    masks = torch.zeros(cap, dtype=torch.int64, device=DEV)
    posd = torch.zeros(cap, dtype=torch.int32, device=DEV)
    dsv.tree_masks(i32_dev(parents), cud, cxd, masks, posd)
    refs = np.zeros(cap, int)
    for i, k in enumerate(nodes):
        refs[cu[i]:cu[i + 1]] = [slot(i, ctx[i] + n) for n in range(k)]
    y = torch.randn((cap, hq + 2 * hkv, dim), device=DEV).bfloat16()
    q = torch.zeros((cap, hq, dim), dtype=torch.bfloat16, device=DEV)
    put(y, posd, i32_dev(refs), q, cud[B:])  # rows past the trees name slot 0 and are not written
    out = torch.empty_like(q)
    dsv.tree_attn(q, cud, masks, pages, tab, cxd, out, scales, max_nodes=most)
    draft = rng.permutation(vocab)[:cap]
    logits = torch.randn((cap, vocab), device=DEV).bfloat16()
    for i, k in enumerate(nodes):
        for j in range(1, k):
            if parents[cu[i] + j] == 0 or rng.random() < 0.7:
                logits[cu[i] + parents[cu[i] + j], draft[cu[i] + j]] = 12.0
    a, nxt = (torch.zeros(B, dtype=torch.int32, device=DEV) for _ in range(2))
    path = torch.zeros(cap, dtype=torch.int32, device=DEV)
    dsv.tree_accept(logits, cud, i32_dev(draft), i32_dev(parents), a, path, nxt)
    dsv.tree_commit(pages, cud, cxd, tab, path, scales)
    accepted, path = a.cpu().numpy(), path.cpu().numpy()
    assert accepted.max() >= 2
    # a linear decode of the same tokens, into another cache
    pages2, scales2 = torch.zeros_like(pages), None if scales is None else torch.zeros_like(scales)
    rows, pos, refs2, keep = [], [], [], []
    for i in range(B):
        for t in range(ctx[i]):
            keep.append((i, t))
        for m in range(accepted[i] + 1):
            rows.append(cu[i] + path[cu[i] + m]), pos.append(ctx[i] + m), refs2.append(slot(i, ctx[i] + m))
            keep.append((i, ctx[i] + m))
    xy = torch.cat([x, y[torch.tensor(rows, device=DEV)]])
    first = np.concatenate([[slot(i, t) for t in range(c)] for i, c in enumerate(ctx)])
    all_pos = i32_dev(np.concatenate([np.concatenate([np.arange(c) for c in ctx]), pos]))
    all_refs = i32_dev(np.concatenate([first, refs2]))
    other = torch.empty((len(xy), hq, dim), dtype=torch.bfloat16, device=DEV)
    dsv.rope_append(xy[:, :hq], xy[:, hq:hq + hkv], xy[:, hq + hkv:], all_pos, inv, all_refs, other, pages2,
                    scales2, rope_scale=rs)
    refs = i32_dev([slot(i, t) for i, t in keep])
    got, want = ([torch.empty((len(keep), hkv, dim), dtype=torch.float32, device=DEV) for _ in range(2)]
                 for _ in range(2))
    dsv.kv_read(pages, refs, *got, scales)
    dsv.kv_read(pages2, refs, *want, scales2)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # the last accepted node saw the context and its path: a causal block over the linear cache
    k2 = accepted + 1
    cu2 = np.concatenate([[0], np.cumsum(k2)])
    rows = torch.tensor(rows, device=DEV)
    lin = torch.empty((len(rows), hq, dim), dtype=torch.bfloat16, device=DEV)
    dsv.tree_attn(q[rows].contiguous(), i32_dev(cu2), None, pages2, tab, cxd, lin, scales2)
    d = (lin.double() - out[rows].double()).abs()
    assert (d <= 2.0 ** -7 * lin.double().abs() + 2.0 ** -10).all()
    if not fp8:  # the block's own attention reads the cache that rope_append wrote
        assert k2.max() <= dsv.MAX_QLEN
        other = torch.empty_like(lin)
        dsv.verify_attn(q[rows].contiguous(), i32_dev(cu2), pages2, tab, cxd, other)
        d = (lin.double() - other.double()).abs()
        assert (d <= 2.0 ** -7 * lin.double().abs() + 2.0 ** -10).all()

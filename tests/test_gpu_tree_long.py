"""GPU: tree attention over long contexts, so that a key counted twice or left out shows,
and over pieces longer than the page ids that a wave holds at a time.

Random keys and values average out: at 20,000 keys a lost block of 32 moves the outputs by
less than a bf16 step.  Here every block has one key with K = 0 (score 0) whose V is large in one
dim, the block's number modulo D, and 0 elsewhere, so that each block makes up a good part of
an output of its own.

Tolerance, with A = sum w |v| / sum w of a row and dim: the rounding to bf16 (2^-8 of the
output), and relative to A: a score is an fp32 sum of D exact products, off by D * 2^-24 *
|q| |k| * scale, which a weight carries twice (itself and in the sum); 2^-17 for the weight's
pair of bf16 parts; 2^-22 for exp2, its argument and the quotient; and the sums over n keys, of
weights and of products, n * 2^-24 each.  That a block shows is asserted: it moves its output
by more than twice the bound.
"""
import math

import numpy as np
import pytest
import torch

import paper_2609_37532_amd as dsv
from gpu_util import DEV, i32_dev, say
from test_gpu_tree import signed
import tree_ref as T

pytestmark = pytest.mark.gpu

LEAD, SKEW_PCT = 6 * 32, 6  # the plan's lead-in per segment and the shares' alternation


class Long:
    """A batch over a pool drawn on the device, with a marked key in every block."""

    def __init__(self, seed, ctx, nodes, hkv, group, dim, fp8):
        rng = np.random.default_rng(seed)
        self.ctx, self.nodes, self.hkv, self.group, self.dim, self.fp8 = ctx, nodes, hkv, group, dim, fp8
        B = len(ctx)
        keys = np.asarray(ctx) + np.asarray(nodes)
        self.max_len = int(keys.max())
        need = -(-keys // 16)
        self.total = int(need.sum()) + 3
        ids, at = rng.permutation(self.total), 0
        table = np.full((B, int(need.max())), -1, np.int64)
        for i in range(B):
            table[i, :need[i]] = ids[at:at + need[i]]
            at += need[i]
        self.table = table
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        shape = (self.total, 2, hkv, 16 * dim)
        self.scales = None
        if fp8:
            self.pages = torch.empty(shape, dtype=torch.uint8, device=DEV)
            for a in range(0, self.total, 4096):
                x = torch.randn((min(4096, self.total - a),) + shape[1:], generator=g, device=DEV)
                self.pages[a:a + 4096] = x.mul_(64).to(torch.float8_e4m3fn).view(torch.uint8)
            self.scales = torch.full((self.total, hkv, 2, 16), 121, dtype=torch.uint8, device=DEV)
        else:
            self.pages = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
        # the marked keys: (request, block) -> position
        req = np.repeat(np.arange(B), [c // 32 for c in ctx])
        blk = np.concatenate([np.arange(c // 32) for c in ctx])
        t = 32 * blk + (7 * blk + req) % 32
        page, slot = torch.tensor(table[req, t // 16], device=DEV), torch.tensor(t % 16, device=DEV)
        dims = torch.tensor(blk % dim, device=DEV)
        chunk = 16 if fp8 else 8
        self.pages.view(self.total, 2, hkv, dim // chunk, 16, chunk)[page, 0, :, :, slot] = 0
        v = self.pages.view(self.total, 2, hkv, dim, 16)
        v[page, 1, :, :, slot] = 0
        v[page, 1, :, dims, slot] = 0x7E if fp8 else 1792.0
        if fp8:
            self.scales[page, :, 1, slot] = 129
        self.cu = np.concatenate([[0], np.cumsum(nodes)])
        cap = int(self.cu[-1]) + 2
        self.q = torch.randn((cap, hkv * group, dim), generator=g, device=DEV, dtype=torch.bfloat16)
        self.masks = [m for k in nodes for m in T.masks_of(T.random_tree(rng, k))[0]]
        self.out = torch.full_like(self.q, float("nan"))

    def run(self):
        masks = torch.cat([signed(self.masks), torch.zeros(2, dtype=torch.int64, device=DEV)])
        table = i32_dev(self.table)
        dims = dsv.tree_attn_dims(self.q, self.pages, table, self.scales, max_nodes=max(self.nodes),
                                  max_kv_len=self.max_len)
        self.ws = dsv.alloc_workspace(dsv.tree_attn_workspace_bytes(dims))
        dsv.tree_attn(self.q, i32_dev(self.cu), masks, self.pages, table, i32_dev(self.ctx), self.out,
                      self.scales, dims=dims, workspace=self.ws)
        torch.cuda.synchronize()
        B = len(self.ctx)
        return self.ws[:4 * (2 * B + 3)].view(torch.int32).cpu().numpy()

    def rows(self, i, g):
        """K and V of request i's keys, in 64 bits."""
        n, dim = self.ctx[i] + self.nodes[i], self.dim
        ids = torch.tensor(self.table[i, :-(-n // 16)], device=DEV)
        chunk = 16 if self.fp8 else 8
        x = self.pages[ids, :, g]
        x = x.view(torch.float8_e4m3fn).float().double() if self.fp8 else x.double()
        k = x[:, 0].view(-1, dim // chunk, 16, chunk).transpose(1, 2).reshape(-1, dim)
        v = x[:, 1].view(-1, dim, 16).transpose(1, 2).reshape(-1, dim)
        if self.fp8:
            e = torch.exp2(self.scales[ids, g].double() - 127).transpose(0, 1).reshape(2, -1)
            k, v = k * e[0, :, None], v * e[1, :, None]
        return k[:n].contiguous(), v[:n].contiguous()

    def check(self, i, g):
        ctx, k, dim = self.ctx[i], self.nodes[i], self.dim
        o, n = int(self.cu[i]), ctx + k
        keys, values = self.rows(i, g)
        heads = slice(g * self.group, (g + 1) * self.group)
        q = self.q[o:o + k, heads].double().reshape(-1, dim)
        x = torch.mm(q, keys.t().contiguous()) / math.sqrt(dim)
        sees = torch.ones((k, n), dtype=torch.bool, device=DEV)
        bits = signed(self.masks[o:o + k])[:, None] >> torch.arange(k, device=DEV)
        sees[:, ctx:] = (bits & 1).bool()
        x = x.view(k, self.group, n).masked_fill(~sees[:, None], -math.inf).view(-1, n)
        w = torch.softmax(x, -1)
        want, size = torch.mm(w, values), torch.mm(w, values.abs())
        norm = float(q.norm(dim=1).max() * keys.norm(dim=1).max()) / math.sqrt(dim)
        eps = 2 * dim * 2.0 ** -24 * norm + 2.0 ** -17 + 2.0 ** -22 + 2 * n * 2.0 ** -24
        bound = 2.0 ** -8 * want.abs() + eps * size
        # what each block's marked key adds to its output
        blk = torch.arange(ctx // 32, device=DEV)
        t = 32 * blk + (7 * blk + i) % 32
        share = w[:, t] * 1792.0
        assert bool((share > 2 * bound[:, blk % dim]).all())
        got = self.out[o:o + k, heads].double().reshape(-1, dim)
        worst = float(((got - want).abs() / bound).max())
        say("request %d head %d: %d keys, %.2f of the bound" % (i, g, n, worst))
        assert worst <= 1


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("ctx,nodes,hkv,group,dim", [
    ([15000, 19000], [64, 64], 1, 4, 128), ([20000, 300], [33, 5], 1, 16, 128), ([20000], [9], 2, 1, 128),
    ([9000, 4000, 70], [64, 20, 64], 2, 16, 64), ([5000] * 9, [12] * 9, 4, 4, 64)])
def test_every_block_counts_once(ctx, nodes, hkv, group, dim, fp8):
    say("long", ctx, nodes, hkv, group, dim, fp8)
    c = Long(len(ctx) + dim, ctx, nodes, hkv, group, dim, fp8)
    c.run()
    for i in range(min(len(ctx), 4)):
        for g in range(hkv):
            c.check(i, g)


# stage_keys: of the form that these sizes take; a wave holds the page ids of 256 stages
@pytest.mark.parametrize("stage_keys,B,ctx,nodes,hkv,group,dim,fp8", [
    (32, 64, 12000, 2, 8, 1, 128, False), (32, 64, 12000, 3, 8, 4, 128, True),
    (32, 64, 12000, 25, 8, 4, 128, True), (32, 24, 12000, 40, 8, 16, 64, True),
    (64, 16, 19000, 64, 8, 16, 128, False), (64, 16, 19000, 64, 8, 16, 128, True)])
def test_pieces_longer_than_the_page_ids_of_a_wave(stage_keys, B, ctx, nodes, hkv, group, dim, fp8):
    window = 256 * stage_keys
    rng = np.random.default_rng(ctx + nodes)
    ctxs = rng.integers(ctx * 5 // 6, ctx * 7 // 6, B).tolist()
    ks = rng.integers(max(1, nodes - 2), nodes + 1, B).tolist()
    say("window", stage_keys, B, ctx, nodes, hkv, group, dim, fp8)
    c = Long(ctx + dim, ctxs, ks, hkv, group, dim, fp8)
    say("pool %.2f GB" % (c.pages.numel() * c.pages.element_size() / 1e9))
    plan = c.run()
    share = int(plan[B + 1])
    assert share > window
    # segments of the plan (a request, a KV head, up to `group_rows` rows) and their pieces
    rows = group * max(ks)
    group_rows = 64 if rows <= 64 else 128 if rows <= 128 else 256
    skew = share * SKEW_PCT // 100 // 32 * 32
    begin = lambda b: b * share + (b & 1) * skew
    total = int(plan[B])
    starts = [begin(b) for b in range(total // share + 2)]
    whole, cut = [], []
    for i in range(B):
        groups = -(-group * ks[i] // group_rows)
        segv = -(-(ctxs[i] + ks[i]) // 32) * 32 + LEAD
        for g in range(hkv):
            for r in range(groups):
                s0 = int(plan[i]) + (g * groups + r) * segv + LEAD
                inner = [b for b in starts if s0 < b < s0 + segv - LEAD]
                edges = [s0] + inner + [s0 + segv - LEAD]
                if max(b - a for a, b in zip(edges, edges[1:])) > window:
                    (cut if inner else whole).append((i, g))
    assert whole and cut
    live = int(c.cu[-1])
    assert bool(c.out[:live].isfinite().all()) and not bool(c.out[live:].any())
    mid = lambda x: x[len(x) // 2]
    for i, g in sorted({whole[0], mid(whole), whole[-1], cut[0], mid(cut), cut[-1]}):
        c.check(i, g)

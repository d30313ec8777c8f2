"""GPU: rope_append and kv_read of so many rows that a workgroup takes several KV heads
(cache.hip's kManyBlocks: from 1,024 (16 rows, head) pairs on two, for rope_append four from
2,048 on; kv_read 256 dims' worth), with head counts that leave the last group short."""
import numpy as np
import pytest
import torch

import paper_2609_37532_amd as dsv
from gpu_util import DEV, i32_dev, say
from test_gpu_cache_rows import Pool, check_append, slots

pytestmark = pytest.mark.gpu


def pairs(rows, hkv):
    return -(-rows // 16) * hkv


@pytest.mark.parametrize("rows,hkv,dim,rot,interleaved,f32,fp8,pattern,kw", [
    (4700, 7, 64, 64, False, False, True, "prompts", {}),
    (4691, 7, 128, 128, False, True, False, "steps", {}),
    (3700, 9, 64, 32, True, True, True, "scattered", {}),
    (3650, 9, 128, 128, False, False, False, "pages", dict(bad=300)),
    (4700, 7, 64, 20, False, False, True, "steps", dict(live=4333)),
    (5500, 6, 64, 64, True, False, False, "prompts", dict(scale=1.25, start=200000))])
def test_append_four_heads_to_a_workgroup(rows, hkv, dim, rot, interleaved, f32, fp8, pattern, kw):
    assert pairs(rows, hkv) >= 2048 and hkv % 4
    check_append("four heads", rows, rows, 2, hkv, dim, rot, interleaved, f32, fp8, pattern, **kw)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("dim,hkv", [(64, 5), (64, 7), (128, 5)])
@pytest.mark.parametrize("pattern", ["pages", "prompts", "steps", "scattered", "again"])
def test_read_several_heads_to_a_workgroup(pattern, dim, hkv, fp8, f32):
    rows = 3301
    say("read many", pattern, dim, hkv, fp8, f32)
    assert pairs(rows, hkv) >= 1024 and hkv % (256 // dim)
    rng = np.random.default_rng(dim + hkv)
    pages = 1300
    pool = Pool(rng, pages, hkv, dim, fp8)
    refs = rng.integers(0, pages * 16, rows) if pattern == "again" else slots(rng, pattern, rows, pages)
    bad = rng.permutation(rows)[:90]
    refs[bad] = rng.choice([-1, pages * 16, -2 ** 31, 2 ** 31 - 1, pages * 16 + 3], 90)
    dtype = torch.float32 if f32 else torch.bfloat16
    out = [torch.full((rows, hkv, dim), float("nan"), dtype=dtype, device=DEV) for _ in range(2)]
    dsv.kv_read(pool.cells, i32_dev(refs), *out, pool.scales)
    ok = (refs >= 0) & (refs < pages * 16)
    want = pool.host().read(np.where(ok, refs, 0))
    for got, w in zip(out, want):
        assert np.array_equal(got.double().cpu().numpy(), np.where(ok[:, None, None], w, 0.0))

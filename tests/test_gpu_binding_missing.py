"""GPU: a required tensor that is None is refused with its name, before anything runs."""
import pytest
import torch

import paper_2609_37532_amd as dsv
from gpu_util import DEV, i32_dev

pytestmark = pytest.mark.gpu


def calls():
    """(function, its arguments by name, those that may be None)"""
    hkv, dim, cap, B, vocab = 2, 64, 3, 1, 100
    pages = torch.zeros((4, 2, hkv, 16 * dim), dtype=torch.bfloat16, device=DEV)
    rows = torch.zeros((cap, 2, dim), dtype=torch.bfloat16, device=DEV)
    i3, i1, cu = i32_dev([0, 1, 2]), i32_dev([0]), i32_dev([0, 3])
    table, masks = i32_dev([[0, 1]]), torch.tensor([1, 3, 5], device=DEV)
    inv = torch.ones(dim // 2, device=DEV)
    out = lambda: torch.zeros_like(rows)
    return [
        (dsv.rope_append, dict(q=rows, k=rows, v=rows, positions=i3, inv_freq=inv, kv_refs=i3, q_out=out(),
                               kv_pages=pages, kv_scales=None, num_live=None), ("q", "inv_freq")),
        (dsv.kv_read, dict(kv_pages=pages, kv_refs=i3, k_out=out(), v_out=out()), ()),
        (dsv.tree_masks, dict(parents=i3, cu_qlens=cu, ctx_lens=i1, masks=masks.clone(), positions=i3.clone()),
         ("positions",)),
        (dsv.tree_attn, dict(q_packed=rows, cu_qlens=cu, masks=masks, kv_pages=pages, page_table=table,
                             ctx_lens=i1, out=out()), ("masks",)),
        (dsv.tree_accept, dict(logits_packed=torch.zeros((cap, vocab), device=DEV), cu_qlens=cu,
                               draft_tokens=i3, parents=i3, accept_len=i1.clone(), path=i3.clone(),
                               next_token=i1.clone()), ()),
        (dsv.tree_commit, dict(kv_pages=pages, cu_qlens=cu, ctx_lens=i1, page_table=table, path=i3), ()),
    ]


@pytest.mark.parametrize("n", range(6))
def test_missing(n):
    fn, good, optional = calls()[n]
    fn(**good)
    for name, value in good.items():
        if value is None:
            continue
        if name in optional:
            fn(**{**good, name: None})
            continue
        with pytest.raises(ValueError, match=name):
            fn(**{**good, name: None})
    torch.cuda.synchronize()


def test_missing_with_what_needs_it():
    fn, good, _ = calls()[0]
    fn(**{**good, "inv_freq": None, "positions": None})
    fn(**{**good, "q": None, "q_out": None})
    fn(**{**good, "inv_freq": None, "positions": None, "q": None, "q_out": None})
    torch.cuda.synchronize()

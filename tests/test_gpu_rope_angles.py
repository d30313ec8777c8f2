"""GPU: rope_append's angles at far positions, where position * inv_freq no longer fits a
double (31 bits times 24), and k's rotation where the terms of a pair cancel.

The reference takes the product and its remainder modulo 2 pi in whole numbers.  k before
its one rounding is within 2^-50 * (|a| + |b|) * |rope_scale| of the exact value: sin and
cos carry the reduction's three roundings and the sum's one (at most 2.5 * 2^-53), their
factor one, the product and the sum one each, 5.5 * 2^-53 in all.  The reference's own sin and
cos are within 2^-52.  The cell is within half a bf16 step (2^-8 of it) of that.
"""
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2609_37532_amd as dsv
from gpu_util import DEV, i32_dev, say

pytestmark = pytest.mark.gpu

PI = Fraction(314159265358979323846264338327950288419716939937510582097494459, 10 ** 62)


def angle(position, freq):
    """position * freq modulo 2 pi, within [-pi, pi], correctly rounded."""
    theta = int(position) * Fraction(float(freq))
    return float(theta - 2 * PI * round(theta / (2 * PI)))


FAR = [2 ** 31 - 1, 2 ** 31 - 12345, 2 ** 30 + 7, -2 ** 31, -2 ** 31 + 3, 2 ** 29 + 1, 2 ** 29, 123457, 1, 0]


def frequencies(kind, half, rng):
    if kind == "plain":
        return (10000.0 ** (-np.arange(half) / half)).astype(np.float32)
    lo, hi = {"fast": (0.5, 1.0), "wide": (2.0 ** -20, 512.0)}[kind]
    return np.exp(rng.uniform(np.log(lo), np.log(hi), half)).astype(np.float32)


@pytest.mark.parametrize("kind", ["plain", "fast", "wide"])
@pytest.mark.parametrize("cancel", [False, True])
@pytest.mark.parametrize("scale", [1.0, 1.25])
def test_k_at_far_positions(kind, cancel, scale):
    dim, half, rows = 128, 64, len(FAR)
    rng = np.random.default_rng(4)
    freq = frequencies(kind, half, rng)
    theta = np.array([[angle(p, f) for f in freq] for p in FAR])
    c, s = np.cos(theta) * scale, np.sin(theta) * scale
    x = rng.normal(size=(rows, dim)).astype(np.float32)
    if cancel:  # a cos - b sin is what fp32 left of a and b
        x[:, :half], x[:, half:] = np.sin(theta), np.cos(theta)
    a, b = x[:, :half].astype(np.float64), x[:, half:].astype(np.float64)
    say("far", kind, cancel, scale)
    pages = torch.zeros((1, 2, 1, 16 * dim), dtype=torch.bfloat16, device=DEV)
    k = torch.from_numpy(x).to(DEV)[:, None]
    refs = i32_dev(np.arange(rows))
    dsv.rope_append(None, k, torch.zeros_like(k), i32_dev(FAR), torch.from_numpy(freq).to(DEV), refs, None,
                    pages, rope_scale=scale)
    out = [torch.empty((rows, 1, dim), dtype=torch.float32, device=DEV) for _ in range(2)]
    dsv.kv_read(pages, refs, *out)
    got = out[0][:, 0].double().cpu().numpy()
    eps = 2.0 ** -50 + 2.0 ** -51
    for at, want in ((slice(0, half), a * c - b * s), (slice(half, dim), b * c + a * s)):
        off = np.abs(got[:, at] - want)
        bound = 2.0 ** -8 * np.abs(want) + eps * (np.abs(a) + np.abs(b)) * scale
        worst = float((off / bound).max())
        assert worst <= 1


def test_q_at_far_positions():
    """q turns in fp32: the two products' factors are rounded, a product, and the sum."""
    dim, half, rows = 64, 32, len(FAR)
    rng = np.random.default_rng(5)
    freq = frequencies("fast", half, rng)
    theta = np.array([[angle(p, f) for f in freq] for p in FAR])
    c, s = np.cos(theta)[:, None], np.sin(theta)[:, None]
    q = torch.from_numpy(rng.normal(size=(rows, 3, dim)).astype(np.float32)).to(DEV)
    k = torch.zeros((rows, 1, dim), device=DEV)
    pages = torch.zeros((1, 2, 1, 16 * dim), dtype=torch.bfloat16, device=DEV)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
    dsv.rope_append(q, k, k, i32_dev(FAR), torch.from_numpy(freq).to(DEV), i32_dev(np.arange(rows)), out, pages)
    x, got = q.double().cpu().numpy(), out.double().cpu().numpy()
    a, b = x[..., :half], x[..., half:]
    for at, want in ((slice(0, half), a * c - b * s), (slice(half, dim), b * c + a * s)):
        bound = 2.0 ** -8 * np.abs(want) + 3 * 2.0 ** -24 * (np.abs(a) + np.abs(b))
        worst = float((np.abs(got[..., at] - want) / bound).max())
        assert worst <= 1

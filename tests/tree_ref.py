"""Plain 64-bit implementations of the cache-row and tree operators (numpy), for their
tests: written from the definitions, element by element where that is affordable."""
import numpy as np

PAGE = 16
MIN_EXP = -60

# ------------------------------------------------------------------ number formats
E4M3 = np.array([(c % 8) / 8 * 2.0 ** -6 if c < 8 else (1 + c % 8 / 8) * 2.0 ** (c // 8 - 7)
                 for c in range(127)])


def e4m3_value(code):
    """Values of e4m3 codes."""
    code = np.asarray(code, np.uint8)
    table = np.append(E4M3, np.nan)
    return np.where(code & 128, -1.0, 1.0) * table[code & 127]


def e4m3_code(y):
    """Nearest codes (ties to the even one) of values within +-448; NaN for what is not
    finite."""
    y = np.asarray(y, np.float64)
    a = np.where(np.isfinite(y), np.abs(y), 0.0)
    middle = (E4M3[1:] + E4M3[:-1]) / 2
    at = np.searchsorted(middle, a, side="left")  # a tie stays with the lower code
    tie = (at < 126) & (a == middle[np.minimum(at, 125)]) & (at % 2 == 1)
    code = (at + tie).astype(np.uint8) | np.where(np.signbit(y), 128, 0).astype(np.uint8)
    return np.where(np.isfinite(y), code, np.uint8(127))


def row_exponent(x):
    """Least e >= MIN_EXP with every finite |x| <= 448 * 2^e (last axis)."""
    a = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    e = np.full(a.shape, MIN_EXP, np.int64)
    while True:
        more = a > 448.0 * np.ldexp(1.0, e)
        if not more.any():
            return e
        e += more


def bf16_round(x):
    """64-bit values to the nearest bf16 (ties to even), as 64-bit values."""
    x = np.asarray(x, np.float64)
    m, e = np.frexp(np.where(np.isfinite(x), x, 0.0))
    step = np.ldexp(1.0, np.maximum(e, -125) - 8)
    y = np.rint(x / step) * step
    y = np.where(np.abs(y) > 3.3895313892515355e38, np.copysign(np.inf, y), y)
    return np.where(np.isfinite(x), y, x)


# -------------------------------------------------------------------------- layouts
def k_offset(slot, d, fp8):
    c = 16 if fp8 else 8
    return (d // c * PAGE + slot) * c + d % c


def v_offset(slot, d):
    return d * PAGE + slot


class Cache:
    """A host copy of a cache: `cells` [P][2][Hkv][16*D] of codes (uint8) or of bf16 values
    (64-bit), `scales` [P][Hkv][2][16] or None."""

    def __init__(self, cells, scales=None):
        self.cells, self.scales = cells, scales
        self.dim = cells.shape[3] // PAGE

    def write(self, ref, k, v):
        """k, v [Hkv, D] to slot `ref`."""
        page, slot, d = ref // PAGE, ref % PAGE, np.arange(self.dim)
        for kind, x, at in ((0, k, k_offset(slot, d, self.scales is not None)),
                            (1, v, v_offset(slot, d))):
            if self.scales is None:
                self.cells[page, kind][:, at] = bf16_round(x)
            else:
                e = row_exponent(x)
                self.cells[page, kind][:, at] = e4m3_code(x * np.ldexp(1.0, -e)[:, None])
                self.scales[page, :, kind, slot] = e + 127

    def read(self, refs):
        """K and V [rows, Hkv, D] of slots in range."""
        refs = np.asarray(refs, np.int64)
        page, slot, d = refs[:, None] // PAGE, refs[:, None] % PAGE, np.arange(self.dim)
        out = []
        for kind, at in ((0, k_offset(slot, d, self.scales is not None)), (1, v_offset(slot, d))):
            x = np.swapaxes(self.cells[page, kind, :, at], 1, 2)
            if self.scales is not None:
                e = self.scales[refs // PAGE, :, kind, refs % PAGE].astype(np.int64) - 127
                x = e4m3_value(x) * np.ldexp(1.0, e)[:, :, None]
            out.append(x)
        return out


# ------------------------------------------------------------------------ operators
def rotate(x, positions, inv_freq, interleaved, scale=1.0):
    """Rotary positions on x [rows, heads, D] in 64 bits."""
    x = np.array(x, np.float64)
    half = len(inv_freq)
    theta = np.asarray(positions, np.float64)[:, None] * np.asarray(inv_freq, np.float64)
    c, s = scale * np.cos(theta)[:, None], scale * np.sin(theta)[:, None]
    a = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    b = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    xa, xb = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = xa * c - xb * s, xb * c + xa * s
    return x


def masks_of(parents):
    """(masks, depths) of one tree."""
    masks, depth = [], []
    for j, p in enumerate(parents):
        ok = 0 <= p < j
        masks.append((masks[p] if ok else 0) | 1 << j)
        depth.append(depth[p] + 1 if ok else 0)
    return masks, depth


def attend(q, keys, values, sees, scale):
    """q [rows, Hq, D], keys/values [len, Hkv, D], sees [rows, len] -> [rows, Hq, D]; a key
    that a row does not see has no part in it, whatever it holds."""
    rows, hq, dim = q.shape
    hkv = keys.shape[1]
    out = np.zeros((rows, hkv, hq // hkv, dim))
    q = q.reshape(rows, hkv, -1, dim)
    finite = np.isfinite(keys).all() and np.isfinite(values).all()
    for g in range(hkv):
        # all rows at once, or row by row over the keys that each sees
        for part in [np.arange(rows)] if finite else np.arange(rows)[:, None]:
            at = np.flatnonzero(sees[part].any(0))
            if not len(at):
                continue
            with np.errstate(invalid="ignore", over="ignore"):
                x = q[part, g] @ keys[at, g].T * scale  # [rows, group, keys]
                x = np.where(sees[part][:, at][:, None], x, -np.inf)
                w = np.exp(x - np.maximum(x.max(-1, keepdims=True), -1e300))
                total = w.sum(-1, keepdims=True)
                out[part, g] = w @ values[at, g] / np.where(total == 0, 1.0, total)
    return out.reshape(rows, hq, dim)


def walk(choice, draft, parents):
    """Greedy acceptance of one tree: the accepted nodes (the root first)."""
    path, at = [0], 0
    while True:
        n = next((n for n in range(at + 1, len(draft))
                  if parents[n] == at and draft[n] == choice[at]), None)
        if n is None:
            return path
        path.append(n)
        at = n


def random_tree(rng, k, chain=0.35):
    return [-1 if j == 0 else j - 1 if rng.random() < chain else
            int(rng.integers(max(0, j - 8), j)) for j in range(k)]

"""The operators around a verified tree of drafted tokens, as timed cases.

Five kinds of pass:

  append   ``rope_append``: rotary positions on a step's (or a prompt's) q and k, and
           its k and v written to the paged cache in bf16 or quantised to 8 bits.  A
           pass over a quantised cache also reads the rows back (``kv_read``), so that
           it returns the values the cache stands for
  read     ``kv_read``: cache rows gathered into dense bf16 tensors
  attn     ``tree_attn``: attention of packed tree nodes over the paged cache
  accept   ``tree_accept``: greedy acceptance of drafted trees
  commit   ``tree_commit``: the accepted path's cache rows moved into place (again read
           back where the cache is quantised)

With ``own`` false a pass computes the same in elementary torch operations.  Inputs are
drawn on the device from the seed.
"""
import math
import random

import torch

own = False

PAGE = 16     # tokens per cache page
ROOT = -1     # parent of a tree's first node
FP8_MAX = 448.0
MIN_EXP = -60  # least exponent of a quantised row's scale
LARGEST = {"bytes": 600_000_000, "flops": 220_000_000_000}  # of a drawn case


# ------------------------------------------------------------------- the cases
def listed():
    return [
        # one token of one request, as a plain decode step writes it: latency alone
        {"name": "append_one_token", "kind": "append", "reqs": 1, "rows": 1, "hq": 32, "hkv": 8,
         "dim": 128, "rot": 128, "interleaved": False, "yarn": 1, "dtype": "bf16",
         "cache": "fp8", "start": 5000},
        # a long prompt's chunk, far positions under scaled frequencies, into a bf16 cache
        {"name": "append_prompt_8k", "kind": "append", "reqs": 3, "rows": 8191, "hq": 32,
         "hkv": 8, "dim": 128, "rot": 128, "interleaved": False, "yarn": 4, "dtype": "bf16",
         "cache": "bf16", "start": 100000},
        # a step of 32 ragged requests, half of each head rotated in pairs, fp32 projections
        {"name": "append_step_partial_f32", "kind": "append", "reqs": 32, "rows": 739, "hq": 16,
         "hkv": 2, "dim": 64, "rot": 32, "interleaved": True, "yarn": 1, "dtype": "f32",
         "cache": "fp8", "start": 8000},
        # some scattered rows of a bf16 cache (a few requests' shared prefix tails)
        {"name": "read_bf16_300", "kind": "read", "rows": 300, "hkv": 8, "dim": 64,
         "cache": "bf16", "scattered": True},
        # long contexts handed to another engine: quantised pages into dense rows
        {"name": "read_fp8_60k", "kind": "read", "rows": 60001, "hkv": 8, "dim": 128,
         "cache": "fp8", "scattered": False},
        # one interactive request, a small tree: latency alone
        {"name": "attn_b1_n16_ctx700", "kind": "attn", "reqs": 1, "hkv": 8, "group": 4,
         "dim": 128, "ctx_lo": 700, "ctx_hi": 700, "nodes": 16, "tree": "wide", "cache": "bf16"},
        # the ordinary serving step: 32 requests, ragged trees, contexts to 8K, 8-bit cache
        {"name": "attn_b32_n26_fp8", "kind": "attn", "reqs": 32, "hkv": 8, "group": 4,
         "dim": 128, "ctx_lo": 1024, "ctx_hi": 8192, "nodes": 26, "tree": "wide", "cache": "fp8"},
        # the largest: full trees under 64 query heads and long contexts, bf16 cache
        {"name": "attn_b16_n64_g8_ctx16k", "kind": "attn", "reqs": 16, "hkv": 8, "group": 8,
         "dim": 128, "ctx_lo": 2000, "ctx_hi": 16300, "nodes": 64, "tree": "wide",
         "cache": "bf16"},
        # drafted trees of one small batch, fp32 logits of a vocabulary with odd rows
        {"name": "accept_b2_n13_f32", "kind": "accept", "reqs": 2, "nodes": 13, "vocab": 50257,
         "dtype": "f32"},
        # full trees of eight requests at the flagship's vocabulary
        {"name": "accept_b8_n64", "kind": "accept", "reqs": 8, "nodes": 64, "vocab": 151936,
         "dtype": "bf16"},
        # the accepted rows of one interactive request's tree, one layer: latency alone
        {"name": "commit_b1_bf16", "kind": "commit", "reqs": 1, "nodes": 16, "hkv": 8,
         "dim": 128, "ctx_lo": 700, "ctx_hi": 700, "cache": "bf16"},
        # the accepted rows of a serving step's trees, one layer, 8-bit cache
        {"name": "commit_b32_fp8", "kind": "commit", "reqs": 32, "nodes": 26, "hkv": 8,
         "dim": 128, "ctx_lo": 1000, "ctx_hi": 2000, "cache": "fp8"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "read", "attn", "attn", "attn", "accept", "commit"])
    c = {"kind": kind, "cache": rng.choice(["bf16", "fp8"])}
    if kind == "append":
        c["reqs"] = _log_int(rng, 1, 64)
        c["rows"] = max(c["reqs"], _log_int(rng, 1, 8191))
        c["hkv"] = rng.choice([1, 2, 4, 8])
        c["hq"] = c["hkv"] * rng.choice([1, 2, 4, 8])
        c["dim"] = rng.choice([64, 128])
        c["rot"] = rng.choice([c["dim"], c["dim"], c["dim"] // 2, c["dim"] // 4, 20, 48])
        c["interleaved"] = rng.random() < 0.4
        c["yarn"] = rng.choice([1, 1, 4, 32])
        c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
        c["start"] = rng.choice([0, _log_int(rng, 1, 1000000)])
    elif kind == "read":
        c["rows"] = _log_int(rng, 1, 60000)
        c["hkv"] = rng.choice([1, 2, 4, 8])
        c["dim"] = rng.choice([64, 128])
        c["scattered"] = rng.random() < 0.4
        if c["scattered"]:  # each row costs the pages that it lies in
            c["rows"] = max(1, c["rows"] // 8)
    elif kind == "attn":
        hi = _log_int(rng, 64, 16384)
        c.update(reqs=_log_int(rng, 1, 64), hkv=rng.choice([1, 2, 4, 8]),
                 group=rng.choice([1, 2, 4, 8, 16]), dim=rng.choice([64, 128, 128]),
                 ctx_lo=int(hi * rng.uniform(0.0, 0.9)), ctx_hi=hi, nodes=_log_int(rng, 1, 64),
                 tree=rng.choice(["wide", "wide", "chain"]))
    elif kind == "accept":
        c.pop("cache")
        c.update(reqs=_log_int(rng, 1, 32), nodes=_log_int(rng, 1, 64),
                 vocab=rng.choice([32000, 50257, 65537, 151936, _log_int(rng, 1000, 262144)]),
                 dtype=rng.choice(["bf16", "bf16", "f32"]))
    else:
        hi = _log_int(rng, 64, 4096)
        c.update(reqs=_log_int(rng, 1, 64), nodes=_log_int(rng, 2, 64),
                 hkv=rng.choice([1, 2, 4, 8]), dim=rng.choice([64, 128]),
                 ctx_lo=int(hi * rng.uniform(0.1, 0.9)), ctx_hi=hi)
    while any(work(c)[k] > LARGEST[k] for k in LARGEST):
        if c["kind"] == "read":
            c["rows"] = c["rows"] * 3 // 4
        else:
            c["reqs"] = max(1, c["reqs"] * 3 // 4)
            if c["reqs"] == 1:
                c["nodes"] = max(1, c["nodes"] * 3 // 4)
    return c


# --------------------------------------------------------------------- lengths
def _spread(lo, hi, n):
    return [lo + int((hi - lo) * (i + 0.5) / n) for i in range(n)]


def _contexts(case):
    return _spread(case["ctx_lo"], case["ctx_hi"], case["reqs"])


def _nodes(case):
    """Nodes of each request's tree: from half of the largest to the largest."""
    most = case["nodes"]
    return _spread(max(1, most // 2), most + 1, case["reqs"])[:-1] + [most]


def _rows_of(case):
    """Rows of each request of an append: ragged, `rows` together."""
    n, rows = case["reqs"], case["rows"]
    cut = [rows * i // n + (rows // (3 * n) if i % 2 else 0) for i in range(n)] + [rows]
    return [b - a for a, b in zip(cut, cut[1:])]


def _offsets(k):
    cu = [0]
    for x in k:
        cu.append(cu[-1] + x)
    return cu


def _dealt(seed, values):
    values = list(values)
    random.Random(seed).shuffle(values)
    return values


def _dense(rows, dim, heads, size):
    return rows * heads * dim * size


def _cache_row(case):
    """Bytes of one token's K and V in the cache."""
    dim, heads = case["dim"], case["hkv"]
    return heads * 2 * (dim + 1) if case["cache"] == "fp8" else heads * 2 * dim * 2


def work(case):
    kind, dim = case["kind"], case.get("dim")
    if kind == "append":
        heads = case["hq"] + 2 * case["hkv"]
        size = 4 if case["dtype"] == "f32" else 2
        read = _dense(case["rows"], dim, heads, size) + 8 * case["rows"]
        moved = _dense(case["rows"], dim, case["hq"], 2) + case["rows"] * _cache_row(case)
        if case["cache"] == "fp8":  # read back
            moved += case["rows"] * (_cache_row(case) + 2 * case["hkv"] * dim * 2)
        return {"bytes": read + moved,
                "flops": case["rows"] * (3 * case["rot"] * heads + 40 * case["rot"])}
    if kind == "read":
        rows = case["rows"] * (_cache_row(case) + 4)
        return {"bytes": rows + case["rows"] * case["hkv"] * dim * 4, "flops": 0}
    nodes = _nodes(case)
    if kind == "attn":
        hq, ctx = case["hkv"] * case["group"], _contexts(case)
        keys = sum(c + k for c, k in zip(ctx, nodes))
        live = sum(nodes)
        seen = sum(c * k + k * (k + 1) // 2 for c, k in zip(ctx, nodes))
        return {"bytes": keys * _cache_row(case) + (live + case["reqs"] * case["nodes"]) * hq * dim * 2
                + keys // 4, "flops": 4 * dim * hq * seen}
    if kind == "accept":
        live = sum(nodes)
        return {"bytes": live * case["vocab"] * (4 if case["dtype"] == "f32" else 2) + 16 * live,
                "flops": live * case["vocab"]}
    moved = sum(min(k, 1 + k // 4) for k in nodes) * _cache_row(case)
    back = sum(nodes) * (_cache_row(case) + 2 * case["hkv"] * dim * 2) if case["cache"] == "fp8" else 0
    return {"bytes": 2 * moved + back + 16 * sum(nodes), "flops": 0}


# ---------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * int(seed) + 29)
    return g


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _frequencies(case):
    """Inverse frequencies of base 10,000 and the factor on cos and sin.  `yarn` > 1
    stretches the slow ones by that factor for a model trained to 32,768 positions."""
    half, factor = case["rot"] // 2, case["yarn"]
    inv = 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    if factor > 1:
        turns = 32768 * inv / (2 * math.pi)
        keep = ((torch.log2(turns) - 0) / 5).clamp(0, 1)  # 1 turn .. 32 turns
        inv = inv * keep + inv / factor * (1 - keep)
    return inv.float().cuda(), torch.tensor(0.1 * math.log(factor) + 1.0).item()  # an fp32 value


def _pool(case, total, g):
    """A cache pool of `total` pages with rows of normal values (a few large dims)."""
    hkv, dim = case["hkv"], case["dim"]
    shape = (total, 2, hkv, PAGE * dim)
    if case["cache"] == "bf16":
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16), None
    pages = torch.empty(shape, device="cuda", dtype=torch.uint8)
    scales = torch.empty((total, hkv, 2, PAGE), device="cuda", dtype=torch.uint8)
    for at in range(0, total, 2048):
        n = min(2048, total - at)
        code = torch.randn((n,) + shape[1:], generator=g, device="cuda").mul_(100).clamp_(-448, 448)
        pages[at:at + n] = code.to(torch.float8_e4m3fn).view(torch.uint8)
    scales.copy_(torch.randint(118, 123, scales.shape, generator=g, device="cuda", dtype=torch.uint8))
    return pages, scales


def _table(lengths, g, spare=8):
    """A page table for requests of these lengths, their pages scattered over the pool."""
    pages = [max(1, -(-x // PAGE)) for x in lengths]
    total = sum(pages) + spare
    ids = torch.randperm(total, generator=g, device="cuda", dtype=torch.int32)
    table = torch.zeros((len(pages), max(pages)), dtype=torch.int32, device="cuda")
    at = 0
    for i, p in enumerate(pages):
        table[i, :p] = ids[at:at + p]
        at += p
    return table, total


def _refs(table, req, pos):
    """Cache slots (page * 16 + slot) of positions `pos` of requests `req`."""
    return table[req, pos // PAGE] * PAGE + pos % PAGE


def _prepare_append(case, seed, g):
    n, rows, dim, hq, hkv = case["reqs"], case["rows"], case["dim"], case["hq"], case["hkv"]
    k = _dealt(seed, _rows_of(case))
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    # the projections of q, k and v come out of one matrix product, side by side; k has
    # a few large channels
    x = torch.randn((rows, hq + 2 * hkv, dim), generator=g, device="cuda")
    x[:, hq:hq + hkv, 5:dim:41] *= 9.0
    x = x.to(dtype)
    req = torch.repeat_interleave(torch.arange(n, device="cuda"),
                                  torch.tensor(k, device="cuda"), output_size=rows)
    at = torch.arange(rows, device="cuda") - torch.tensor(_offsets(k), device="cuda")[req]
    first = case["start"] % PAGE  # a prompt's chunk goes on where the last one ended
    table, total = _table([first + c for c in k], g)
    inv, factor = _frequencies(case)
    pages, scales = _pool(case, total, g)
    return {"q": x[:, :hq], "k": x[:, hq:hq + hkv], "v": x[:, hq + hkv:],
            "positions": (case["start"] + at).to(torch.int32), "inv_freq": inv, "factor": factor,
            "refs": _refs(table, req, first + at).to(torch.int32),
            "q_out": torch.zeros((rows, hq, dim), dtype=torch.bfloat16, device="cuda"),
            "pages": pages, "scales": scales, "interleaved": case["interleaved"],
            "k_out": torch.empty((rows, hkv, dim), dtype=torch.bfloat16, device="cuda"),
            "v_out": torch.empty((rows, hkv, dim), dtype=torch.bfloat16, device="cuda")}


def _prepare_read(case, seed, g):
    rows, dim, hkv = case["rows"], case["dim"], case["hkv"]
    if case["scattered"]:
        total = -(-rows // 2) + 8
        refs = torch.randperm(total * PAGE, generator=g, device="cuda")[:rows]
    else:  # whole contexts, each from its first position
        lengths = _dealt(seed, _spread(rows // 8, rows // 3, 4)) if rows >= 64 else [rows]
        if rows >= 64:
            lengths.append(rows - sum(lengths))
        table, total = _table(lengths, g)
        refs = torch.cat([_refs(table, torch.tensor(i, device="cuda"),
                                torch.arange(x, device="cuda")) for i, x in enumerate(lengths)])
    pages, scales = _pool(case, total, g)
    out = [torch.empty((rows, hkv, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    return {"pages": pages, "scales": scales, "refs": refs.to(torch.int32), "k_out": out[0],
            "v_out": out[1]}


def _trees(case, seed, nodes):
    """Parents of each request's nodes (a node comes after its parent), and the masks of
    what each node sees: itself and its ancestors."""
    r = random.Random(seed)
    parents, masks = [], []
    for k in nodes:
        mine = []
        for j in range(k):
            chain = case.get("tree") == "chain" or r.random() < 0.35
            p = ROOT if j == 0 else j - 1 if chain else r.randrange(max(0, j - 8), j)
            parents.append(p)
            mine.append((mine[p] if j else 0) | 1 << j)
        masks += [m - (1 << 64) if m >> 63 else m for m in mine]
    return parents, masks


def _prepare_attn(case, seed, g):
    n, dim, hkv = case["reqs"], case["dim"], case["hkv"]
    hq, cap = hkv * case["group"], case["reqs"] * case["nodes"]
    nodes, ctx = _dealt(2 * seed, _nodes(case)), _dealt(2 * seed + 1, _contexts(case))
    table, total = _table([c + k for c, k in zip(ctx, nodes)], g)
    pages, scales = _pool(case, total, g)
    masks = _trees(case, seed, nodes)[1]
    masks += [0] * (cap - len(masks))
    return {"q": torch.randn((cap, hq, dim), generator=g, device="cuda", dtype=torch.bfloat16),
            "cu": _i32(_offsets(nodes)), "ctx": _i32(ctx), "table": table, "pages": pages,
            "scales": scales, "masks": torch.tensor(masks, dtype=torch.int64, device="cuda"),
            "out": torch.empty((cap, hq, dim), dtype=torch.bfloat16, device="cuda"),
            "max_nodes": case["nodes"], "max_len": case["ctx_hi"] + case["nodes"]}


def _prepare_accept(case, seed, g):
    """Logits that repeat a random part of each tree: every node's token is drafted by its
    parent's row, and about two thirds of the first children are what the target chose."""
    n, vocab, cap = case["reqs"], case["vocab"], case["reqs"] * case["nodes"]
    nodes = _dealt(2 * seed, _nodes(case))
    parents = _trees(case, seed, nodes)[0]
    r, cu = random.Random(seed + 1), _offsets(nodes)
    draft = r.sample(range(vocab), cap) if vocab >= cap else [r.randrange(vocab) for _ in range(cap)]
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    logits = torch.randn((cap, vocab), generator=g, device="cuda", dtype=dtype)
    rows, ids = [], []
    for i in range(n):
        taken = set()
        for j in range(1, nodes[i]):
            p = cu[i] + parents[cu[i] + j]
            if p not in taken and r.random() < 0.65:
                taken.add(p)
                rows.append(p)
                ids.append(draft[cu[i] + j])
    if rows:
        logits[torch.tensor(rows, device="cuda"), torch.tensor(ids, device="cuda")] = 14.0
    parents += [ROOT] * (cap - len(parents))
    return {"logits": logits, "cu": _i32(cu), "draft": _i32(draft), "parents": _i32(parents),
            "accept_len": _i32([0] * n), "next_token": _i32([0] * n), "path": _i32([0] * cap),
            "max_nodes": case["nodes"]}


def _prepare_commit(case, seed, g):
    nodes, ctx = _dealt(2 * seed, _nodes(case)), _dealt(2 * seed + 1, _contexts(case))
    cap = case["reqs"] * case["nodes"]
    table, total = _table([c + k for c, k in zip(ctx, nodes)], g)
    pages, scales = _pool(case, total, g)
    r, path = random.Random(seed), []
    for k in nodes:  # about a quarter of the nodes lie on the accepted path
        mine = [0] + sorted(r.sample(range(1, k), min(k - 1, k // 4)))
        path += mine + [-1] * (k - len(mine))
    live = len(path)
    path += [-1] * (cap - live)
    req = torch.repeat_interleave(torch.arange(len(nodes), device="cuda"),
                                  torch.tensor(nodes, device="cuda"), output_size=live)
    at = torch.arange(live, device="cuda") - torch.tensor(_offsets(nodes), device="cuda")[req]
    refs = _refs(table, req, torch.tensor(ctx, device="cuda")[req] + at)
    s = {"pages": pages, "scales": scales, "cu": _i32(_offsets(nodes)), "ctx": _i32(ctx),
         "table": table, "path": _i32(path), "max_nodes": case["nodes"],
         "refs": refs.to(torch.int32)}
    for name in ("k_out", "v_out"):
        s[name] = torch.empty((live, case["hkv"], case["dim"]), dtype=torch.bfloat16, device="cuda")
    return s


def prepare(case, seed):
    make = {"append": _prepare_append, "read": _prepare_read, "attn": _prepare_attn,
            "accept": _prepare_accept, "commit": _prepare_commit}[case["kind"]]
    return dict(make(case, seed, _generator(seed)), kind=case["kind"])


# ------------------------------------------------------------------ plain forms
def _k_rows(pages):
    """K of a pool by page and slot: [pages, 16, heads, dims cut into the tile's chunks]."""
    chunk = 8 if pages.dtype == torch.bfloat16 else 16
    dim = pages.shape[-1] // PAGE
    x = pages[:, 0].unflatten(-1, (dim // chunk, PAGE, chunk))
    return x.permute(0, 3, 1, 2, 4)


def _v_rows(pages):
    return pages[:, 1].unflatten(-1, (pages.shape[-1] // PAGE, PAGE)).permute(0, 3, 1, 2)


def _plain_write(pages, refs, k, v):
    page, slot = refs.long() // PAGE, refs.long() % PAGE
    rows = _k_rows(pages)
    rows[page, slot] = k.unflatten(-1, rows.shape[-2:])
    _v_rows(pages)[page, slot] = v


def _plain_read(pages, scales, refs):
    """K and V of these slots in fp32."""
    page, slot = refs.long() // PAGE, refs.long() % PAGE
    k, v = _k_rows(pages)[page, slot].flatten(-2), _v_rows(pages)[page, slot]
    if scales is None:
        return k.float(), v.float()
    # a power of two is its exponent's bits
    exp = (scales[page, :, :, slot].int() << 23).view(torch.float32).unsqueeze(-1)
    return (k.contiguous().view(torch.float8_e4m3fn).float() * exp[:, :, 0],
            v.contiguous().view(torch.float8_e4m3fn).float() * exp[:, :, 1])


def _plain_rotate(x, cos, sin, rot, interleaved):
    cos, sin = cos.to(x.dtype)[:, None], sin.to(x.dtype)[:, None]
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else r.chunk(2, -1)
    a, b = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([r, x[..., rot:]], -1)


def _power(exp):
    """2^exp in 64 bits, exactly."""
    return (exp.long() + 1023 << 52).view(torch.float64)


def _plain_quantise(x):
    """Rows of 64-bit values: their e4m3 values (as fp32, exact) and scale exponents."""
    mant, exp = torch.frexp(x.abs().amax(-1))
    exp = (exp - 9 + (mant > 0.875)).clamp_min(MIN_EXP)  # amax <= 448 * 2^exp
    y = x * _power(-exp.unsqueeze(-1))
    step = _power((torch.frexp(y)[1] - 1).clamp_min(-6) - 3)
    return (torch.round(y / step) * step).float(), exp


def _plain_append(s):
    # in 64 bits: the angles of far positions, and k, whose values are cut to 8 bits
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle) * s["factor"], torch.sin(angle) * s["factor"]
    rot = 2 * s["inv_freq"].numel()
    s["q_out"].copy_(_plain_rotate(s["q"].float(), cos, sin, rot, s["interleaved"]))
    k = _plain_rotate(s["k"].double(), cos, sin, rot, s["interleaved"])
    if s["scales"] is None:
        _plain_write(s["pages"], s["refs"], k.to(torch.bfloat16), s["v"].to(torch.bfloat16))
        return s["q_out"], s["pages"]
    page, slot = s["refs"].long() // PAGE, s["refs"].long() % PAGE
    (k, ke), (v, ve) = _plain_quantise(k), _plain_quantise(s["v"].double())
    cells = [x.to(torch.float8_e4m3fn).view(torch.uint8) for x in (k, v)]
    _plain_write(s["pages"], s["refs"], *cells)
    s["scales"][page, :, :, slot] = (torch.stack([ke, ve], -1) + 127).to(torch.uint8)
    k, v = _plain_read(s["pages"], s["scales"], s["refs"])
    return s["q_out"], k.to(torch.bfloat16), v.to(torch.bfloat16)


def _plain_attn(s):
    cu, ctx = s["cu"].long(), s["ctx"].long()
    n, nodes, most = ctx.numel(), s["max_nodes"], s["max_len"]
    hq, dim = s["q"].shape[1:]
    hkv = s["pages"].shape[2]
    count = cu[1:] - cu[:-1]
    j = torch.arange(nodes, device="cuda")
    row = (cu[:-1, None] + j).clamp_max(s["q"].shape[0] - 1)
    t = torch.arange(most, device="cuda")
    refs = s["table"].long()[:, (t // PAGE).clamp_max(s["table"].shape[1] - 1)] * PAGE + t % PAGE
    k, v = _plain_read(s["pages"], s["scales"], refs.flatten())
    k = k.view(n, most, hkv, dim).permute(0, 2, 3, 1).contiguous()
    v = v.view(n, most, hkv, dim).transpose(1, 2)
    inside = t < (ctx + count)[:, None]
    v = torch.where(inside[:, None, :, None], v, v.new_zeros(()))
    node = t - ctx[:, None]  # of each key, negative in the context
    bit = s["masks"][row][:, :, None] >> node.clamp(0, 63)[:, None, :] & 1
    sees = ((node < 0)[:, None, :] | (bit == 1)) & inside[:, None, :]
    q = s["q"][row].float().view(n, nodes, hkv, -1, dim).permute(0, 2, 3, 1, 4)
    x = torch.matmul(q.flatten(2, 3) * dim ** -0.5, k).view(n, hkv, -1, nodes, most)
    x = torch.where(sees[:, None, None], x, x.new_full((), -math.inf))
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = x.sum(-1, keepdim=True)
    x = torch.matmul(x.flatten(2, 3), v).view(n, hkv, -1, nodes, dim)
    x = x / torch.where(total > 0, total, torch.ones_like(total))
    out = x.permute(0, 3, 1, 2, 4).reshape(n, nodes, hq, dim).to(torch.bfloat16)
    s["out"].zero_()
    live = j < count[:, None]
    s["out"][row[live]] = out[live]
    return s["out"]


def _plain_accept(s):
    """A node is accepted if it and all its ancestors are what their parents' rows chose."""
    cu = s["cu"].long()
    n, nodes, cap = cu.numel() - 1, s["max_nodes"], s["logits"].shape[0]
    top = s["logits"].amax(-1, keepdim=True)
    vocab = s["logits"].shape[1]
    ids = torch.arange(vocab, device="cuda", dtype=torch.int32)
    choice = torch.where(s["logits"] == top, ids, vocab).amin(-1)
    j = torch.arange(nodes, device="cuda")
    row = (cu[:-1, None] + j).clamp_max(cap - 1)
    inside = j < (cu[1:] - cu[:-1])[:, None]
    parent = torch.where(inside, s["parents"].long()[row], ROOT)
    at = parent.clamp_min(0)
    match = (choice[row].gather(1, at) == s["draft"][row]) & (parent >= 0) | (j == 0)
    # up[i, j, m]: m is j or an ancestor of j; squaring the parent relation closes it
    up = (torch.nn.functional.one_hot(at, nodes) * (parent >= 0)[..., None]).float()
    up = up + torch.eye(nodes, device="cuda")
    hops = max(1, (nodes - 1).bit_length())
    for _ in range(hops):
        up = (torch.matmul(up, up) > 0).float()
    good = ~((up > 0) & ~match[:, None, :]).any(-1) & inside
    count = good.sum(-1)
    order = torch.where(good, j, nodes).sort(-1).values
    order = torch.where(order < nodes, order, -1)
    s["path"][row[inside]] = order[inside].to(torch.int32)
    last = (cu[:-1] + order.amax(-1).clamp_min(0)).clamp_max(cap - 1)
    s["accept_len"].copy_((count - 1).clamp_min(0))
    s["next_token"].copy_(choice[last])
    return s["accept_len"], s["path"], s["next_token"]


def _plain_commit(s):
    cu, ctx, path = s["cu"].long(), s["ctx"].long(), s["path"].long()
    r = torch.arange(path.numel(), device="cuda")
    req = torch.searchsorted(cu, r, right=True) - 1
    keep = (r < cu[-1]) & (path >= 0)
    r, req, node = r[keep], req[keep], path[keep]
    table, base = s["table"].long(), ctx[req]
    src, dst = _refs(table, req, base + node), _refs(table, req, base + r - cu[req])
    k, v = _k_rows(s["pages"]), _v_rows(s["pages"])
    at, to = (src // PAGE, src % PAGE), (dst // PAGE, dst % PAGE)
    k[to], v[to] = k[at], v[at]
    if s["scales"] is None:
        return s["pages"]
    x = s["scales"].permute(0, 3, 1, 2)
    x[to] = x[at]
    return tuple(y.to(torch.bfloat16) for y in _plain_read(s["pages"], s["scales"], s["refs"]))


# ------------------------------------------------------------------------- run
def _own_run(s):
    import paper_2609_37532_amd as dsv
    kind = s["kind"]
    if kind == "append":
        dsv.rope_append(s["q"], s["k"], s["v"], s["positions"], s["inv_freq"], s["refs"],
                        s["q_out"], s["pages"], s["scales"], interleaved=s["interleaved"],
                        rope_scale=s["factor"])
        if s["scales"] is None:
            return s["q_out"], s["pages"]
        dsv.kv_read(s["pages"], s["refs"], s["k_out"], s["v_out"], s["scales"])
        return s["q_out"], s["k_out"], s["v_out"]
    if kind == "read":
        dsv.kv_read(s["pages"], s["refs"], s["k_out"], s["v_out"], s["scales"])
        return s["k_out"], s["v_out"]
    if kind == "attn":
        if "ws" not in s:  # kept by the program from step to step
            # no request is longer than its row of the page table
            most = min(s["max_len"], PAGE * s["table"].shape[1])
            s["dims"] = dsv.tree_attn_dims(s["q"], s["pages"], s["table"], s["scales"],
                                           max_nodes=s["max_nodes"], max_kv_len=most)
            s["ws"] = dsv.alloc_workspace(dsv.tree_attn_workspace_bytes(s["dims"]))
        dsv.tree_attn(s["q"], s["cu"], s["masks"], s["pages"], s["table"], s["ctx"], s["out"],
                      s["scales"], dims=s["dims"], workspace=s["ws"])
        return s["out"]
    if kind == "accept":
        if "ws" not in s:
            s["ws"] = dsv.alloc_workspace(dsv.accept_workspace_bytes(
                s["logits"].shape[0], s["accept_len"].numel(), s["logits"].shape[1]))
        dsv.tree_accept(s["logits"], s["cu"], s["draft"], s["parents"], s["accept_len"],
                        s["path"], s["next_token"], workspace=s["ws"])
        return s["accept_len"], s["path"], s["next_token"]
    dsv.tree_commit(s["pages"], s["cu"], s["ctx"], s["table"], s["path"], s["scales"])
    if s["scales"] is None:
        return s["pages"]
    dsv.kv_read(s["pages"], s["refs"], s["k_out"], s["v_out"], s["scales"])
    return s["k_out"], s["v_out"]


def run(state):
    if own:
        return _own_run(state)
    kind = state["kind"]
    if kind == "append":
        return _plain_append(state)
    if kind == "read":
        k, v = _plain_read(state["pages"], state["scales"], state["refs"])
        state["k_out"].copy_(k)
        state["v_out"].copy_(v)
        return state["k_out"], state["v_out"]
    return {"attn": _plain_attn, "accept": _plain_accept, "commit": _plain_commit}[kind](state)


# ----------------------------------------------------------------------- exact
def _e4m3_table():
    """The values of the 127 finite codes from 0 up."""
    values = [(c % 8) / 8 * 2.0 ** -6 if c < 8 else (1 + c % 8 / 8) * 2.0 ** (c // 8 - 7)
              for c in range(127)]
    return torch.tensor(values, dtype=torch.float64, device="cuda")


def _powers(exp):
    table = torch.tensor([2.0 ** e for e in range(-160, 161)], dtype=torch.float64, device="cuda")
    return table[exp.long() + 160]


def _exact_quantise(x):
    """The values that rows of x stand for in the cache: the least power of two that
    brings them to 448, and the nearest code (the even one of two)."""
    values = _e4m3_table()
    top = x.abs().amax(-1, keepdim=True).clamp_min(1e-300)
    exp = torch.ceil(torch.log2(top / FP8_MAX)).clamp_min(MIN_EXP)
    exp = exp + (top > FP8_MAX * _powers(exp)).long() - (top <= FP8_MAX * _powers(exp - 1)).long()
    scale = _powers(exp.clamp_min(MIN_EXP))
    y = x.abs() / scale
    middle = (values[1:] + values[:-1]) / 2
    at = torch.bucketize(y, middle)
    at = at + ((at < 126) & (y == middle[at.clamp_max(125)]) & (at % 2 == 1)).long()
    return torch.copysign(values[at] * scale, x)


def _exact_rows(pages, scales, refs):
    """K and V of the slots `refs` in 64 bits, element by element."""
    total, _, hkv, tile = pages.shape
    dim = tile // PAGE
    d = torch.arange(dim, device="cuda")
    page, slot = refs.long()[:, None, None] // PAGE, refs.long()[:, None, None] % PAGE
    base = (page * 2 * hkv + torch.arange(hkv, device="cuda")[:, None]) * tile
    chunk = 8 if scales is None else 16
    k_at = base + (d // chunk * PAGE + slot) * chunk + d % chunk
    v_at = base + hkv * tile + d * PAGE + slot
    k, v = pages.reshape(-1)[k_at], pages.reshape(-1)[v_at]
    if scales is None:
        return k.double(), v.double()
    values = _e4m3_table()
    values = torch.cat([values, values.new_tensor([math.nan])])
    e = _powers(scales.permute(0, 3, 2, 1)[page[:, 0, 0], slot[:, 0, 0]].int() - 127)
    sign = lambda c: 1.0 - 2.0 * (c >> 7).double()  # noqa: E731
    return (sign(k) * values[(k & 127).long()] * e[:, 0, :, None],
            sign(v) * values[(v & 127).long()] * e[:, 1, :, None])


def _exact_append(s):
    rot = 2 * s["inv_freq"].numel()
    turn = torch.polar(torch.full((), s["factor"], dtype=torch.float64, device="cuda"),
                       s["positions"].double()[:, None, None] * s["inv_freq"].double())

    def rotated(x):
        x = x.double().clone()
        if s["interleaved"]:
            z = torch.complex(x[..., 0:rot:2], x[..., 1:rot:2]) * turn
            x[..., 0:rot:2], x[..., 1:rot:2] = z.real, z.imag
        else:
            z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
            x[..., :rot // 2], x[..., rot // 2:rot] = z.real, z.imag
        return x

    q, k, v = rotated(s["q"]), rotated(s["k"]), s["v"].double()
    if s["scales"] is not None:
        return q, _exact_quantise(k), _exact_quantise(v)
    pages = s["pages"].double().reshape(-1)
    _, _, hkv, tile = s["pages"].shape
    dim = tile // PAGE
    d, refs = torch.arange(dim, device="cuda"), s["refs"].long()[:, None, None]
    base = (refs // PAGE * 2 * hkv + torch.arange(hkv, device="cuda")[:, None]) * tile
    pages[base + (d // 8 * PAGE + refs % PAGE) * 8 + d % 8] = k
    pages[base + hkv * tile + d * PAGE + refs % PAGE] = v
    return q, pages.view(s["pages"].shape)


def _exact_attn(s):
    cu, ctx = s["cu"].tolist(), s["ctx"].tolist()
    hkv, dim = s["pages"].shape[2], s["q"].shape[2]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for i, c in enumerate(ctx):
        o, k = cu[i], cu[i + 1] - cu[i]
        t = torch.arange(c + k, device="cuda")
        refs = s["table"][i].long()[t // PAGE] * PAGE + t % PAGE
        keys, values = _exact_rows(s["pages"], s["scales"], refs)
        sees = torch.ones((k, c + k), dtype=torch.bool, device="cuda")
        bits = s["masks"][o:o + k, None].bitwise_right_shift(torch.arange(k, device="cuda"))
        sees[:, c:] = bits.bitwise_and(1).bool()
        for h in range(hkv):
            q = s["q"][o:o + k].double().view(k, hkv, -1, dim)[:, h].reshape(-1, dim)
            x = torch.mm(q, keys[:, h].t().contiguous()) / math.sqrt(dim)
            x = x.view(k, -1, c + k).masked_fill(~sees[:, None], -math.inf)
            x = torch.softmax(x, -1).nan_to_num(0.0)
            y = torch.mm(x.view(-1, c + k), values[:, h].contiguous())
            out.view(-1, hkv, s["q"].shape[1] // hkv, dim)[o:o + k, h] = y.view(k, -1, dim)
    return out


def _exact_commit(s):
    if s["scales"] is None:
        return None  # the moved rows are copies
    cu, ctx, path = s["cu"].tolist(), s["ctx"].tolist(), s["path"].tolist()
    k, v = _exact_rows(s["pages"], s["scales"], s["refs"])
    took = list(range(cu[-1]))
    for i in range(len(ctx)):
        for j in range(cu[i + 1] - cu[i]):
            if path[cu[i] + j] >= 0:
                took[cu[i] + j] = cu[i] + path[cu[i] + j]
    took = torch.tensor(took, device="cuda")
    return k[took], v[took]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(s)
    if case["kind"] == "read":
        return _exact_rows(s["pages"], s["scales"], s["refs"])
    if case["kind"] == "attn":
        return _exact_attn(s)
    return _exact_commit(s) if case["kind"] == "commit" else None

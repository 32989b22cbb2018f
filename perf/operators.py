"""Cases of the operators on microscaled 4-bit rows and of drawing from scores, as a user's program calls them.

Five kinds of pass:
  quantize  rows to 4-bit codes with a scale per 32 elements, the rows' squared norms, and the values read back
  product   rows of 16 or 32 bits times all 4-bit rows: the scores of a batch
  product4  the same with the batch taken to 4 bits first
  search    a batch taken to 4 bits, and its k nearest among all 4-bit rows
  sample    one id for each row of scores, by temperature, top-k, top-p and min-p from given random numbers
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"u8": torch.uint8, "i8": torch.int8, "f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"u8": 1, "i8": 1, "f32": 4, "f16": 2, "bf16": 2}
DEV = "cuda"
STEP = 128  # a 4-bit row is stored in steps of 128 elements: 64 bytes of codes and 4 of scales
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MIDDLES = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)


def listed():
    return [
        # the questions of a few users, taken to 4 bits: latency alone
        {"name": "quantize-queries", "op": "quantize", "n": 37, "d": 200, "dtype": "f32", "pad": 0},
        # a million int8 embeddings taken to 4 bits
        {"name": "quantize-points", "op": "quantize", "n": 1_000_000, "d": 100, "dtype": "i8", "pad": 0},
        # one state of a decoder against all rows of its output layer
        {"name": "product-one", "op": "product", "nx": 1, "n": 131_072, "d": 4096, "dtype": "bf16", "out": "f32", "pad": 0},
        # a small batch of float questions against all points, scores in full; rows that are slices of wider ones
        {"name": "product-33", "op": "product", "nx": 33, "n": 500_001, "d": 200, "dtype": "f32", "out": "f32", "pad": 5},
        # a long prompt's states through a layer of 4-bit weights
        {"name": "product-many", "op": "product", "nx": 2048, "n": 16_384, "d": 4096, "dtype": "bf16", "out": "bf16", "pad": 0},
        # a thousand questions against a small collection, scores in full
        {"name": "product4-1k", "op": "product4", "nx": 1000, "n": 10_000, "d": 128, "dtype": "u8", "out": "f32", "pad": 0},
        # the same with long rows: matrix work
        {"name": "product4-many", "op": "product4", "nx": 4096, "n": 65_536, "d": 2048, "dtype": "bf16", "out": "bf16", "pad": 0},
        # one question to a million points
        {"name": "search-one", "op": "search", "nq": 1, "n": 1_000_000, "d": 128, "dtype": "u8", "metric": "l2", "k": 10},
        # ten thousand questions to a million float embeddings under the inner product
        {"name": "search-10k", "op": "search", "nq": 10_000, "n": 1_000_000, "d": 200, "dtype": "f32", "metric": "ip", "k": 10},
        # the next token of one user
        {"name": "sample-one", "op": "sample", "rows": 1, "n": 128_000, "dtype": "bf16", "filters": "p", "masked": 0.0, "empty": False, "pad": 0},
        # a serving batch, odd rows, part of the entries masked
        {"name": "sample-64", "op": "sample", "rows": 64, "n": 50_001, "dtype": "f32", "filters": "kpm", "masked": 0.2, "empty": True, "pad": 0},
        # many rows, each with settings of its own
        {"name": "sample-500", "op": "sample", "rows": 500, "n": 128_000, "dtype": "f16", "filters": "each", "masked": 0.0, "empty": False, "pad": 8},
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    v = min(max(v, lo), hi)
    return v + 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(("quantize", "product", "product4", "search", "sample"))
    if op == "quantize":
        d = _log(rng, 16, 4096)
        return {"op": op, "n": _log(rng, 1, min(1_000_000, 100_000_000 // d)), "d": d, "dtype": rng.choice(sorted(TYPES)),
                "pad": rng.choice((0, 0, 3, 8))}
    if op in ("product", "product4"):
        d = _log(rng, 16, 4096)
        n = _log(rng, 100, min(500_000, 500_000_000 // d))
        most = 40_000_000_000 if op == "product" else 200_000_000_000
        nx = _log(rng, 1, max(1, min(4096, most // (n * d), 200_000_000 // n)))
        dtype = rng.choice(("f32", "f16", "bf16") if op == "product" else sorted(TYPES))
        # (products of bytes leave the range of f16)
        return {"op": op, "nx": nx, "n": n, "d": d, "dtype": dtype, "out": rng.choice(("f32", "bf16") if SIZE[dtype] == 1 else ("f32", "f16", "bf16")),
                "pad": rng.choice((0, 0, 3, 8))}
    if op == "search":
        d = rng.choice((96, 100, 128, 200, _log(rng, 16, 512), _log(rng, 16, 512)))
        n = _log(rng, 100, 1_000_000)
        nq = _log(rng, 1, max(1, min(10_000, 2_000_000_000 // n, 400_000_000_000 // (n * d))))
        return {"op": op, "nq": nq, "n": n, "d": d, "dtype": rng.choice(("u8", "i8", "f32")), "metric": rng.choice(("l2", "ip")),
                "k": _log(rng, 1, 100)}
    n = _log(rng, 100, 200_000)
    return {"op": op, "rows": _log(rng, 1, min(2000, 60_000_000 // n)), "n": n, "dtype": rng.choice(("f32", "f16", "bf16")),
            "filters": rng.choice(("", "k", "p", "m", "kpm", "each")), "masked": rng.choice((0.0, 0.2, 0.9)), "empty": rng.random() < 0.5,
            "pad": rng.choice((0, 0, 3, 8))}


# ---------------------------------------------------------------- inputs

def _rows(g, n, d, dtype, turn=False):
    """n rows of d: the distributions of workloads.py for bytes and 32-bit floats, states of a model with a few
    large channels for 16 bits.  `turn`: rows that come from the same centres moved a little (questions)."""
    if n * d > 64_000_000:  # in parts, each drawn like the whole
        return torch.cat([_rows(g, min(n - i, 64_000_000 // d), d, dtype, turn) for i in range(0, n, 64_000_000 // d)])
    c = torch.Generator(device=DEV)
    c.manual_seed(2305)
    x = torch.randn((n, d), device=DEV, generator=g)
    if dtype in ("f16", "bf16"):
        x *= torch.where(torch.rand(d, device=DEV, generator=c) < 0.01, 12.0, 1.0)
        return x.to(TYPES[dtype])
    which = torch.randint(0, 512, (n,), device=DEV, generator=g)
    if dtype == "u8":
        centres = 40.0 * torch.empty((512, d), device=DEV).exponential_(1.0, generator=c) - 16.0
        return torch.clamp(torch.round(centres[which] + 12.0 * x), 0, 255).to(torch.uint8)
    centres = torch.randn((512, d), device=DEV, generator=c)
    if dtype == "i8":
        return torch.clamp(torch.round(40.0 * centres[which] + 25.0 * x), -127, 127).to(torch.int8)
    centres /= centres.norm(dim=1, keepdim=True)
    if turn:
        centres = centres * math.cos(math.pi / 6) + centres.roll(1, 1) * math.sin(math.pi / 6)
    x = centres[which] + 0.05 * x
    return x / x.norm(dim=1, keepdim=True)


def _wider(x, pad):
    """The same rows as a slice of a tensor whose rows are `pad` elements longer."""
    if not pad:
        return x
    wide = torch.empty((x.shape[0], x.shape[1] + pad), dtype=x.dtype, device=x.device)
    wide.copy_(torch.nn.functional.pad(x, (0, pad)))
    return wide[:, :x.shape[1]]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    op = case["op"]
    s = {"case": dict(case)}
    if op == "quantize":
        s["x"] = _wider(_rows(g, case["n"], case["d"], case["dtype"]), case["pad"])
    elif op in ("product", "product4"):
        weights = "bf16" if case["dtype"] == "f16" else case["dtype"]
        s["codes"], s["scales"], s["norms"] = _stored(_rows(g, case["n"], case["d"], weights))
        s["x"] = _wider(_rows(g, case["nx"], case["d"], case["dtype"], turn=True), case["pad"])
    elif op == "search":
        s["codes"], s["scales"], s["norms"] = _stored(_rows(g, case["n"], case["d"], case["dtype"]))
        s["x"] = _rows(g, case["nq"], case["d"], case["dtype"], turn=True)
    else:
        rows, n = case["rows"], case["n"]
        z = 2.5 * torch.randn((rows, n), device=DEV, generator=g)
        top = torch.randint(0, n, (rows, 40), device=DEV, generator=g)
        # (an entry that is drawn twice gets the larger value: which of two writes comes last is not the seed's)
        z.scatter_reduce_(1, top, 8.0 + 4.0 * torch.rand((rows, 40), device=DEV, generator=g), "amax")
        if case["masked"]:
            z.masked_fill_(torch.rand((rows, n), device=DEV, generator=g) < case["masked"], -math.inf)
        if case["empty"]:
            z[torch.randint(0, rows, (1,), device=DEV, generator=g)] = -math.inf
        s["x"] = _wider(z.to(TYPES[case["dtype"]]), case["pad"])
        s["u"] = torch.rand(rows, device=DEV, generator=g)
        f = case["filters"]
        s["t"], s["k"], s["p"], s["m"] = 0.8, 50 if "k" in f else 0, 0.9 if "p" in f else 1.0, 0.05 if "m" in f else 0.0
        if f == "each":
            r = torch.rand((4, rows), device=DEV, generator=g)
            s["t"] = 0.3 + 1.2 * r[0]
            s["k"] = torch.where(r[1] < 0.5, 0, (r[1] * 200).to(torch.int32)).to(torch.int32)
            s["p"] = torch.where(r[2] < 0.3, 1.0, r[2]).contiguous()
            s["m"] = torch.where(r[3] < 0.5, 0.0, 0.1 * r[3]).contiguous()
    return s


# ---------------------------------------------------------------- plain forms

def _codes(x):
    """4-bit codes (n, d padded to steps of 128) and scale bytes of rows, by the formulas."""
    n, d = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -d % STEP)).view(n, -1, 32)
    amax = x.abs().amax(2)
    fine = amax < math.inf
    byte = torch.clamp(((amax.view(torch.int32) >> 23) & 255) - 2, min=0)
    # times 2^(127 - byte)
    y = x * ((254 - byte) << 23).view(torch.float32)[..., None]
    mag = y.abs()
    code = torch.zeros_like(mag, dtype=torch.uint8)
    for i, m in enumerate(MIDDLES):  # ties to the even code
        code += (mag >= m if i % 2 else mag > m).to(torch.uint8)
    code |= torch.signbit(y).to(torch.uint8) << 3
    code = torch.where(fine[..., None], code, torch.zeros_like(code))
    byte = torch.where(fine, byte, torch.full_like(byte, 255)).to(torch.uint8)
    return code.view(n, -1), byte


def _values(code, byte):
    """What codes and scale bytes stand for, in 32 bits."""
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=code.device)
    v = table[code.int()].view(code.shape[0], -1, 32)
    b = byte.int()
    scale = torch.where(b == 0, torch.full_like(b, 1 << 22), b << 23)  # 2^-127 is a subnormal number
    scale = torch.where(b == 255, torch.full_like(b, 0x7FC00000), scale).view(torch.float32)
    return (v * scale[..., None]).view(code.shape[0], -1)


def _stored(x):
    """Rows as a program holds them: packed codes, scale bytes, squared norms."""
    parts = []
    for i in range(0, x.shape[0], 65536):
        code, byte = _codes(x[i:i + 65536])
        parts.append((code[:, 0::2] | code[:, 1::2] << 4, byte, _values(code, byte).square().sum(1)))
    return tuple(torch.cat(p).contiguous() for p in zip(*parts))


def _unpacked(codes, scales):
    return _values(torch.stack((codes & 15, codes >> 4), dim=2).view(codes.shape[0], -1), scales)


def _plain_search(s, case):
    qc, qb = _codes(s["x"])
    q, v = _values(qc, qb), _unpacked(s["codes"], s["scales"])
    ids = torch.arange(v.shape[0], device=DEV)
    k = min(case["k"], v.shape[0])
    out_i = torch.full((q.shape[0], case["k"]), -1, dtype=torch.int32, device=DEV)
    out_d = torch.full((q.shape[0], case["k"]), math.inf, device=DEV)
    part = max(1, 1_000_000_000 // v.shape[0])
    for i in range(0, q.shape[0], part):
        t = q[i:i + part] @ v.T
        if case["metric"] == "l2":
            t = q[i:i + part].square().sum(1, keepdim=True) + (s["norms"] - 2.0 * t)
        else:
            t = 0.0 - t
        # one whole number that sorts as (distance, id)
        b = t.view(torch.int32)
        key = (torch.where(b < 0, b ^ 0x7FFFFFFF, b).long() << 32) | ids
        best = torch.topk(key, k, dim=1, largest=False, sorted=True).values
        out_i[i:i + part, :k] = (best & 0xFFFFFFFF).int()
        out_d[i:i + part, :k] = t.gather(1, best & 0xFFFFFFFF)
    return {"ids": out_i, "dists": out_d}


def _column(v, rows):
    return (v if isinstance(v, torch.Tensor) else torch.full((rows,), v, device=DEV)).double().unsqueeze(1)


def _plain_sample(s):
    z = s["x"].double()
    rows, n = z.shape
    t, k, p, m = (_column(v.float() if isinstance(v, torch.Tensor) else torch.tensor(v).float().item(), rows) for v in (s["t"], s["k"], s["p"], s["m"]))
    z = torch.where(z.isnan(), -math.inf, z)
    z, order = torch.sort(z, dim=1, descending=True, stable=True)
    best = z[:, :1]
    w = torch.where(z == best, 1.0, torch.exp((z - best) / t))
    there = z > -math.inf
    w = torch.where(there, w, 0.0)
    at = torch.arange(n, device=DEV)
    w = torch.where((k > 0) & (at >= k), 0.0, w)
    run_mass = torch.cumsum(w, 1)
    before = run_mass - w
    before[:, 1:] = run_mass[:, :-1]
    w = torch.where((p > 0) & (p < 1) & (before >= p * run_mass[:, -1:]), 0.0, w)
    w = torch.where((m > 0) & (w < torch.clamp(m, max=1.0)), 0.0, w)
    kept = torch.zeros_like(w).scatter_(1, order, w)  # back in the order of ids
    run_mass = torch.cumsum(kept, 1)
    mass = run_mass[:, -1:]
    aim = s["u"].double().unsqueeze(1) * mass
    last = n - 1 - (kept > 0).flip(1).int().argmax(1)
    at = torch.minimum(torch.searchsorted(run_mass, aim, right=True).squeeze(1), last)
    empty = ~there.any(1)
    # log(w / mass) as -log(1 + others / w): a mass that is nearly all the drawn one's loses nothing
    drawn = kept.gather(1, at.unsqueeze(1))
    logprob = -torch.log1p(kept.scatter(1, at.unsqueeze(1), 0.0).sum(1, keepdim=True) / drawn).squeeze(1)
    return {"ids": torch.where(empty, -1, at).int(), "logprobs": torch.where(empty, -math.inf, logprob).float()}


# ---------------------------------------------------------------- one pass

def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        from paper_2305_04359_amd import binding as A
        if op == "quantize":
            rows = A.ann_mx_quantize(state["x"], norms=True)
            return {"values": A.ann_mx_dequantize(rows), "norms": rows.norms}
        if op == "sample":
            ids, logprobs = A.ann_sample(state["x"], state["u"], temperature=state["t"], top_k=state["k"], top_p=state["p"], min_p=state["m"])
            return {"ids": ids, "logprobs": logprobs}
        rows = A.MxRows(state["codes"], state["scales"], case["d"], state["norms"])
        if op == "search":
            queries = A.ann_mx_quantize(state["x"], norms=True)
            ids, dists = A.ann_mx_search(rows, queries, case["k"], metric=A.L2SQ if case["metric"] == "l2" else A.MIPS)
            return {"ids": ids, "dists": dists}
        x = A.ann_mx_quantize(state["x"]) if op == "product4" else state["x"]
        return A.ann_mx_product(x, rows, dtype=TYPES[case["out"]])
    if op == "quantize":
        v = _values(*_codes(state["x"]))
        return {"values": v[:, :case["d"]].contiguous(), "norms": v.square().sum(1)}
    if op == "sample":
        return _plain_sample(state)
    if op == "search":
        return _plain_search(state, case)
    v = _unpacked(state["codes"], state["scales"])
    x = state["x"]
    x = _values(*_codes(x)) if op == "product4" else torch.nn.functional.pad(x.float(), (0, v.shape[1] - x.shape[1]))
    return (x @ v.T).to(TYPES[case["out"]])


def work(case):
    op = case["op"]
    if op == "sample":
        size = case["rows"] * case["n"]
        return {"bytes": size * SIZE[case["dtype"]] + 12 * case["rows"], "flops": 4 * size}
    d = case["d"]
    row4 = 17 * -(-d // 32)  # 16 bytes of codes and one of scale for 32 elements
    n = case["n"]
    if op == "quantize":
        return {"bytes": n * (d * SIZE[case["dtype"]] + 2 * row4 + 4 * d + 4), "flops": 4 * n * d}
    if op == "search":
        return {"bytes": n * (row4 + 4) + case["nq"] * (d * SIZE[case["dtype"]] + 8 * case["k"]), "flops": 2 * case["nq"] * n * d}
    nx = case["nx"]
    return {"bytes": n * row4 + nx * d * SIZE[case["dtype"]] + nx * n * SIZE[case["out"]], "flops": 2 * nx * n * d}


# ---------------------------------------------------------------- the definitions, in 64 bits

def _exact_values(x):
    """What the 4-bit form of rows stands for, from the definition: the shared exponent by frexp, and the rounding by
    whole steps of the level's own spacing."""
    n, d = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -d % 32)).view(n, -1, 32)
    amax = x.abs().amax(2, keepdim=True)
    e = torch.where(amax > 0, torch.frexp(amax).exponent - 3, -127).clamp(min=-127).double()
    y = x / torch.exp2(e)
    spacing = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    y = (torch.round(y / spacing) * spacing).clamp(-6, 6)
    y = torch.where(amax < math.inf, y * torch.exp2(e), math.nan)
    return y.view(n, -1)[:, :d]


def _exact_stored(codes, scales, d):
    nibbles = torch.stack((codes & 15, codes >> 4), dim=2).view(codes.shape[0], -1)
    e, m = (nibbles >> 1 & 3).double(), (nibbles & 1).double()
    v = torch.where(e > 0, torch.exp2(e - 1) * (1 + m / 2), m / 2) * torch.where(nibbles >= 8, -1.0, 1.0)
    return (v.view(codes.shape[0], -1, 32) * torch.exp2(scales.double() - 127)[..., None]).view(codes.shape[0], -1)[:, :d]


def _exact_draw(z, u, t, k, p, m):
    """One row of scores (64 bits, on the host): the id drawn and its log-probability, candidate by candidate."""
    ids = np.flatnonzero(z > -math.inf)
    if not len(ids):
        return -1, -math.inf
    ids = ids[np.argsort(-z[ids], kind="stable")]
    best = z[ids[0]]
    w = np.where(z[ids] == best, 1.0, np.exp((z[ids] - best) / t))
    if k > 0:
        ids, w = ids[:int(k)], w[:int(k)]
    if 0 < p < 1:
        keep = 1 + int(np.searchsorted(np.cumsum(w), p * math.fsum(w), side="left"))
        ids, w = ids[:keep], w[:keep]
    if m > 0:
        keep = int((w >= min(m, 1.0)).sum())
        ids, w = ids[:keep], w[:keep]
    by_id = np.argsort(ids)
    ids, w = ids[by_id], w[by_id]
    mass = math.fsum(w)
    at = min(int(np.searchsorted(np.cumsum(w), u * mass, side="right")), len(ids) - 1)
    return int(ids[at]), -math.log1p(math.fsum(np.delete(w, at)) / w[at])


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        v = _exact_values(s["x"])
        return {"values": v, "norms": v.square().sum(1)}
    if op == "sample":
        rows = case["rows"]
        z = s["x"].double().cpu().numpy()
        u = s["u"].double().cpu().numpy()
        t, k, p, m = (v.double().cpu().numpy() if isinstance(v, torch.Tensor) else np.full(rows, np.float32(v), np.float64) for v in (s["t"], s["k"], s["p"], s["m"]))
        got = [_exact_draw(z[i], u[i], t[i], k[i], p[i], m[i]) for i in range(rows)]
        return {"ids": torch.tensor([a for a, _ in got], dtype=torch.int32), "logprobs": torch.tensor([b for _, b in got], dtype=torch.float64)}
    v = _exact_stored(s["codes"], s["scales"], case["d"])
    if op == "search":
        q = _exact_values(s["x"])
        out = torch.full((q.shape[0], case["k"]), math.inf, dtype=torch.float64, device=DEV)
        part = max(1, 500_000_000 // v.shape[0])
        norms = v.square().sum(1)
        for i in range(0, q.shape[0], part):
            t = q[i:i + part] @ v.T
            t = q[i:i + part].square().sum(1, keepdim=True) + norms - 2 * t if case["metric"] == "l2" else -t
            k = min(case["k"], v.shape[0])
            out[i:i + part, :k] = torch.topk(t, k, dim=1, largest=False, sorted=True).values
        return {"ids": None, "dists": out}  # which of several equal ones is a matter of order, not of numbers
    x = _exact_values(s["x"]) if op == "product4" else s["x"].double()
    return x @ v.T

"""The token-row operators (``umap_rows``), as cases to be timed and compared.

Kinds of case, one public call each (an 8-bit result is also read back, as the program that keeps it does):

* ``lookup``       rows of a learned table by id, times a scale (``umap_rows_lookup``);
* ``lookup_grad``  the table's gradient, summed by id (``umap_rows_lookup_grad``);
* ``norm``         root-mean-square norm of rows, of gathered rows or of rows plus a residual, into a float type or
                   into 8 bits with scales (``umap_rows_norm``);
* ``norm_grad``    its gradient for the rows and the weight (``umap_rows_norm_grad``).

Ids follow Zipf's law (id v about in proportion to 1 / (v + 1), as tokens numbered by frequency do); `absent` of a
thousand are -1 (padding). `pad` columns lie between the rows of an input that is part of a wider buffer.
"""

from __future__ import annotations

import math

import torch

own = False   # False: the plain form; True: the library's calls
DEV = "cuda"
EPS = 1e-6
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8,
         "f8": torch.float8_e4m3fn}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "i8": 1, "f8": 1}
LARGEST = {"i8": 127.0, "f8": 448.0}


def listed() -> list[dict]:
    return [
        # serving: the row of one new token
        dict(name="lookup_one", kind="lookup", n=1, rows=32_000, dim=2048, table="bf16", out="bf16", ids="i64",
             absent=0, scale=45.25, group=0),
        # word vectors (300 entries) of a data set's 70,000 words out of a million, for the kNN in front of a layout
        dict(name="lookup_words", kind="lookup", n=70_000, rows=1_000_000, dim=300, table="f16", out="f32", ids="i32",
             absent=0, scale=1.0, group=0),
        # rows kept in 8 bits (784 features, one scale a row), read back for a ragged batch
        dict(name="lookup_8bit", kind="lookup", n=20_011, rows=70_000, dim=784, table="i8", out="bf16", ids="i32",
             absent=0, scale=1.0, group=0),
        # the tokens of a large training batch, some of it padding
        dict(name="lookup_batch", kind="lookup", n=32_768, rows=128_000, dim=4096, table="bf16", out="bf16",
             ids="i64", absent=20, scale=64.0, group=0),
        # the smallest training step: a small table, fp32
        dict(name="lookup_grad_small", kind="lookup_grad", n=77, rows=2000, dim=64, dy="f32", out="f32", ids="i32",
             absent=0, scale=8.0, pad=0),
        # an ordinary step
        dict(name="lookup_grad_step", kind="lookup_grad", n=8192, rows=32_000, dim=1024, dy="bf16", out="f32",
             ids="i64", absent=10, scale=32.0, pad=0),
        # a large batch into a large table; the most frequent id has some 11,000 of the rows
        dict(name="lookup_grad_batch", kind="lookup_grad", n=131_072, rows=128_000, dim=2048, dy="bf16", out="f32",
             ids="i64", absent=20, scale=1.0, pad=0),
        # serving: one token's row read, normalised and stored in 8 bits
        dict(name="norm_one", kind="norm", n=1, dim=4096, x="bf16", w="bf16", out="i8", group=0, residual=False,
             gather=32_000, pad=0),
        # a data set's points (70,000 x 784) normalised into an 8-bit table with a scale per 128 columns
        dict(name="norm_points", kind="norm", n=70_000, dim=784, x="f32", w="f32", out="f8", group=128, residual=False,
             gather=0, pad=0),
        # a long prompt's rows: residual added, normalised, the product's input in 8 bits with a scale per row
        dict(name="norm_prompt", kind="norm", n=32_768, dim=4096, x="bf16", w="bf16", out="i8", group=0, residual=True,
             gather=0, pad=0),
        # training: a ragged batch of odd rows inside a wider buffer
        dict(name="norm_grad_odd", kind="norm_grad", n=1023, dim=1001, x="f16", w="f32", upstream=False, pad=7),
        # training: a large batch, the residual's gradient added
        dict(name="norm_grad_batch", kind="norm_grad", n=32_768, dim=4096, x="bf16", w="bf16", upstream=True, pad=0),
    ]


def _log_int(rng, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _dim(rng, most: int) -> int:
    """Row lengths: any number, or one that divides well."""
    d = _log_int(rng, 16, most)
    step = rng.choice([1, 1, 4, 8, 64, 128])
    d = max(step, d // step * step)
    return d if d != 3072 else d + step


def draw(rng) -> dict:
    kind = rng.choice(["lookup", "lookup_grad", "norm", "norm_grad"])
    dim = _dim(rng, 8192)
    n = _log_int(rng, 1, max(2, min(131_072, 100_000_000 // dim)))
    pad = rng.choice([0, 0, 0, 8, 7])
    if kind == "lookup":
        table = rng.choice(["f32", "f16", "bf16", "bf16", "i8", "f8"])
        return dict(kind=kind, n=n, rows=_log_int(rng, 100, min(1_000_000, 400_000_000 // dim)), dim=dim, table=table,
                    out=rng.choice(["bf16", "bf16", "f16", "f32"]), ids=rng.choice(["i32", "i64"]),
                    absent=rng.choice([0, 0, 20, 500]), scale=rng.choice([1.0, math.sqrt(dim)]),
                    group=rng.choice([0, 0, 32, 128]) if table in LARGEST else 0)
    if kind == "lookup_grad":
        return dict(kind=kind, n=n, rows=_log_int(rng, 100, min(500_000, 200_000_000 // dim)), dim=dim,
                    dy=rng.choice(["bf16", "bf16", "f16", "f32"]), out=rng.choice(["f32", "f32", "bf16"]),
                    ids=rng.choice(["i32", "i64"]), absent=rng.choice([0, 0, 20, 500]),
                    scale=rng.choice([1.0, math.sqrt(dim)]), pad=pad)
    x = rng.choice(["bf16", "bf16", "f16", "f32"])
    w = rng.choice([x, x, "f32"])
    if kind == "norm":
        out = rng.choice(["i8", "i8", "f8", "bf16", "f32"])
        gather = rng.choice([0, 0, 0, 10_007])
        return dict(kind=kind, n=n, dim=dim, x=x, w=w, out=out, group=rng.choice([0, 0, 32, 128]) if out in LARGEST else 0,
                    residual=not gather and rng.random() < 0.6, gather=gather, pad=0 if gather else pad)
    return dict(kind=kind, n=n, dim=dim, x=x, w=w, upstream=rng.random() < 0.5, pad=pad)


def _rand(gen, n: int, dim: int, kind: str, pad: int = 0, spread: float = 1.0) -> torch.Tensor:
    """n x dim normal values, as the left columns of rows that are dim + pad long."""
    x = torch.empty((n, dim + pad), dtype=TYPES[kind], device=DEV)
    return x.normal_(0.0, spread, generator=gen)[:, :dim]


def _ids(gen, n: int, rows: int, kind: str, absent: int) -> torch.Tensor:
    u = torch.rand(n, generator=gen, device=DEV, dtype=torch.float64)
    ids = (torch.exp(u * math.log(rows + 1)) - 1).long().clamp(0, rows - 1)
    if absent:
        gone = torch.rand(n, generator=gen, device=DEV) < absent / 1000.0
        ids = torch.where(gone, -1, ids)
    return ids.to(torch.int32 if kind == "i32" else torch.int64)


def _groups(dim: int, group: int) -> int:
    return -(-dim // group) if group else 1


def prepare(case: dict, seed: int) -> dict:
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    kind, n, dim = case["kind"], case["n"], case["dim"]
    s = dict(case)
    if kind == "lookup":
        rows, t = case["rows"], case["table"]
        if t in LARGEST:
            values = _rand(gen, rows, dim, "bf16", spread=0.25 * LARGEST[t]).clamp_(-LARGEST[t], LARGEST[t])
            s["T"] = (values.round_() if t == "i8" else values).to(TYPES[t])
            s["scales"] = torch.rand((rows, _groups(dim, case["group"])), generator=gen, device=DEV) * 0.02 + 0.001
        else:
            s["T"], s["scales"] = _rand(gen, rows, dim, t), None
        s["tokens"] = _ids(gen, n, rows, case["ids"], case["absent"])
        s["y"] = torch.empty((n, dim), dtype=TYPES[case["out"]], device=DEV)
    elif kind == "lookup_grad":
        s["dY"] = _rand(gen, n, dim, case["dy"], case["pad"])
        s["tokens"] = _ids(gen, n, case["rows"], case["ids"], case["absent"])
        s["G"] = torch.empty((case["rows"], dim), dtype=TYPES[case["out"]], device=DEV)
    else:
        # the weight of a trained norm: around one
        s["W"] = (1.0 + 0.2 * torch.randn(dim, generator=gen, device=DEV)).to(TYPES[case["w"]])
        if kind == "norm":
            s["X"] = _rand(gen, case["gather"] or n, dim, case["x"], case["pad"])
            s["tokens"] = _ids(gen, n, case["gather"], "i64", 0) if case["gather"] else None
            s["R"] = _rand(gen, n, dim, case["x"], case["pad"], 2.0) if case["residual"] else None
            s["H"] = torch.empty((n, dim), dtype=TYPES[case["x"]], device=DEV) if case["residual"] or case["gather"] else None
            s["y"] = torch.empty((n, dim), dtype=TYPES[case["out"]], device=DEV)
            if case["out"] in LARGEST:
                s["y_scales"] = torch.empty((n, _groups(dim, case["group"])), dtype=torch.float32, device=DEV)
                s["back"] = torch.empty((n, dim), dtype=torch.bfloat16, device=DEV)
        else:
            s["X"] = _rand(gen, n, dim, case["x"], case["pad"], 2.0)
            s["dY"] = _rand(gen, n, dim, case["x"], case["pad"])
            s["dH"] = _rand(gen, n, dim, case["x"], case["pad"]) if case["upstream"] else None
            s["dX"] = torch.empty((n, dim), dtype=TYPES[case["x"]], device=DEV)
            s["dW"] = torch.empty(dim, dtype=torch.float32, device=DEV)
    return s


# ---- plain form ------------------------------------------------------------------------------------------------


def _spread(scales: torch.Tensor, dim: int, group: int) -> torch.Tensor:
    """A scale for each column, or one for all of them."""
    return scales.repeat_interleave(group, dim=1)[:, :dim] if group else scales


def _plain_rows(table, ids, scale, scales=None, group=0):
    there = (ids >= 0) & (ids < table.shape[0])
    at = torch.where(there, ids, 0).long()
    rows = table[at].float()
    if scales is not None:
        rows = rows * _spread(scales[at], table.shape[1], group)
    return torch.where(there[:, None], rows * scale, 0.0)


def _plain_lookup(s):
    return _plain_rows(s["T"], s["tokens"], s["scale"], s["scales"], s["group"]).to(TYPES[s["out"]])


def _plain_lookup_grad(s):
    ids, rows = s["tokens"], s["rows"]
    there = (ids >= 0) & (ids < rows)
    total = torch.zeros((rows, s["dim"]), dtype=torch.float32, device=DEV)
    total.index_add_(0, torch.where(there, ids, 0).long(), torch.where(there[:, None], s["dY"].float(), 0.0))
    return (total * s["scale"]).to(TYPES[s["out"]])


def _plain_norm(s):
    h = s["X"].float() if s["tokens"] is None else _plain_rows(s["X"], s["tokens"], 1.0)
    if s["R"] is not None:
        h = h + s["R"].float()
    y = h * (1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)) * s["W"].float()
    found = {} if s["H"] is None else {"h": h.to(s["H"].dtype)}
    if s["out"] not in LARGEST:
        return found | {"y": y.to(TYPES[s["out"]])}
    dim, group = s["dim"], s["group"] or s["dim"]
    count = _groups(dim, group)
    most = torch.nn.functional.pad(y.abs(), (0, count * group - dim)).view(-1, count, group).amax(2)
    scales = most / LARGEST[s["out"]]
    each = scales.repeat_interleave(group, dim=1)[:, :dim]
    q = torch.where(each > 0, y / each, 0.0)
    q = q.round().to(torch.int8) if s["out"] == "i8" else q.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return found | {"scales": scales, "y": (q.float() * each).to(torch.bfloat16)}


def _plain_norm_grad(s):
    h, dy = s["X"].float(), s["dY"].float()
    rho = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    g = dy * s["W"].float()
    dx = g * rho - h * ((g * h).mean(1, keepdim=True) * rho * rho * rho)
    if s["dH"] is not None:
        dx = dx + s["dH"].float()
    return {"dx": dx.to(s["dX"].dtype), "dw": (dy * h * rho).sum(0)}


# ---- the library's calls ---------------------------------------------------------------------------------------


def _own(s):
    from paper_2008_00325_amd import umap_rows as R

    kind = s["kind"]
    if kind == "lookup":
        R.umap_rows_lookup(s["T"], s["tokens"], s["y"], scale=s["scale"], table_scales=s["scales"], group=s["group"])
        return s["y"]
    if kind == "lookup_grad":
        if "work" not in s:
            need = R.umap_rows_lookup_grad_workspace(s["n"], s["rows"], s["dim"])
            s["work"] = torch.empty(need, dtype=torch.uint8, device=DEV)
        R.umap_rows_lookup_grad(s["dY"], s["tokens"], s["G"], s["work"], scale=s["scale"])
        return s["G"]
    if kind == "norm":
        eight = s["out"] in LARGEST
        R.umap_rows_norm(s["X"], s["y"], weight=s["W"], residual=s["R"], h=s["H"], ids=s["tokens"],
                         y_scales=s["y_scales"] if eight else None, group=s["group"], eps=EPS)
        found = {} if s["H"] is None else {"h": s["H"]}
        if not eight:
            return found | {"y": s["y"]}
        R.umap_rows_lookup(s["y"], None, s["back"], table_scales=s["y_scales"], group=s["group"])
        return found | {"scales": s["y_scales"], "y": s["back"]}
    if "work" not in s:
        s["work"] = torch.empty(R.umap_rows_norm_grad_workspace(s["n"], s["dim"]), dtype=torch.uint8, device=DEV)
    R.umap_rows_norm_grad(s["dY"], s["X"], s["dX"], weight=s["W"], dh=s["dH"], dweight=s["dW"], workspace=s["work"],
                          eps=EPS)
    return {"dx": s["dX"], "dw": s["dW"]}


PLAIN = {"lookup": _plain_lookup, "lookup_grad": _plain_lookup_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad}


def run(state: dict):
    return _own(state) if own else PLAIN[state["kind"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------


def _distinct(n: float, rows: int) -> float:
    """Different ids among n draws: sum over v of 1 - (1 - p_v)^n with p_v = ln((v + 2) / (v + 1)) / ln(rows + 1)."""
    v = torch.arange(rows, dtype=torch.float64)
    p = torch.log1p(1.0 / (v + 1.0)) / math.log(rows + 1)
    return float((1.0 - torch.exp(n * torch.log1p(-p.clamp(max=1 - 1e-12)))).sum())


def work(case: dict) -> dict:
    kind, n, dim = case["kind"], case["n"], case["dim"]
    if kind == "lookup":
        m = n * (1 - case["absent"] / 1000.0)
        row = dim * SIZE[case["table"]] + (4 * _groups(dim, case["group"]) if case["table"] in LARGEST else 0)
        ids = n * (4 if case["ids"] == "i32" else 8)
        return {"bytes": _distinct(m, case["rows"]) * row + ids + n * dim * SIZE[case["out"]], "flops": m * dim}
    if kind == "lookup_grad":
        m = n * (1 - case["absent"] / 1000.0)
        ids = n * (4 if case["ids"] == "i32" else 8)
        return {"bytes": m * dim * SIZE[case["dy"]] + ids + case["rows"] * dim * SIZE[case["out"]], "flops": m * dim}
    if kind == "norm":
        x = SIZE[case["x"]]
        total = (_distinct(n, case["gather"]) * dim * x + 8 * n) if case["gather"] else n * dim * x
        total += (n * dim * x if case["residual"] else 0) + dim * SIZE[case["w"]]
        total += n * dim * x if case["residual"] or case["gather"] else 0
        if case["out"] in LARGEST:   # the values in 8 bits and their scales, and the rows that are read back
            total += n * dim * 3 + n * _groups(dim, case["group"]) * 4
        else:
            total += n * dim * SIZE[case["out"]]
        return {"bytes": total, "flops": 6 * n * dim}
    total = n * dim * SIZE[case["x"]] * (4 if case["upstream"] else 3) + dim * (SIZE[case["w"]] + 4)
    return {"bytes": total, "flops": 12 * n * dim}


# ---- from the definitions, in 64 bits --------------------------------------------------------------------------


def _nearest_f8(v: torch.Tensor) -> torch.Tensor:
    """The nearest multiple of the spacing that a 4-bit exponent and 3-bit mantissa give at v (ties to even)."""
    _, e = torch.frexp(v)   # |v| in [2^(e-1), 2^e)
    unit = torch.exp2(((e - 1).clamp(min=-6) - 3).double())
    return ((v / unit).round() * unit).clamp(-448.0, 448.0)


def exact(case: dict, seed: int):
    s = prepare(case, seed)
    kind, n, dim, f64 = case["kind"], case["n"], case["dim"], torch.float64
    if kind == "lookup":
        y = torch.zeros((n, dim), dtype=f64, device=DEV)
        here = torch.nonzero(s["tokens"] >= 0)[:, 0]
        at = s["tokens"][here].long()
        got = s["T"].index_select(0, at).to(f64) if case["table"] != "f8" else s["T"].float().index_select(0, at).to(f64)
        if s["scales"] is not None:
            column = torch.arange(dim, device=DEV) // (case["group"] or dim)
            got *= s["scales"].index_select(0, at).to(f64)[:, column]
        y[here] = got * case["scale"]
        return y
    if kind == "lookup_grad":
        # rows in the order of their ids: a row of the gradient is the difference of two running sums
        order = torch.argsort(s["tokens"], stable=True)
        ends = torch.searchsorted(s["tokens"][order].long().contiguous(),
                                  torch.arange(-1, case["rows"], device=DEV), right=True)
        g = torch.empty((case["rows"], dim), dtype=f64, device=DEV)
        for c in range(0, dim, 256):
            part = s["dY"][:, c:c + 256][order].to(f64)
            running = torch.cat([torch.zeros_like(part[:1]), part.cumsum(0)])
            at = running[ends]
            g[:, c:c + 256] = (at[1:] - at[:-1]) * case["scale"]
        return g
    W = s["W"].to(f64)
    if kind == "norm":
        h = s["X"].to(f64) if s["tokens"] is None else s["X"].to(f64).index_select(0, s["tokens"])
        if s["R"] is not None:
            h = h + s["R"].to(f64)
        y = h / torch.sqrt(h.pow(2).sum(1) / dim + EPS)[:, None] * W
        found = {} if s["H"] is None else {"h": h}
        if case["out"] not in LARGEST:
            return found | {"y": y}
        group = case["group"] or dim
        scales = torch.stack([y[:, c:c + group].abs().max(1).values for c in range(0, dim, group)], 1)
        scales = scales / LARGEST[case["out"]]
        each = scales[:, torch.arange(dim, device=DEV) // group]
        v = y / each.clamp(min=1e-300)
        v = v.round() if case["out"] == "i8" else _nearest_f8(v)
        return found | {"scales": scales, "y": v * each}
    h, dy = s["X"].to(f64), s["dY"].to(f64)
    unit = h / torch.sqrt(h.pow(2).sum(1) / dim + EPS)[:, None]      # dy/dh = W / norm * (I - unit unit^T / dim)
    back = dy * W
    dx = (back - unit * ((back * unit).sum(1) / dim)[:, None]) / torch.sqrt(h.pow(2).sum(1) / dim + EPS)[:, None]
    if s["dH"] is not None:
        dx = dx + s["dH"].to(f64)
    return {"dx": dx, "dw": (dy * unit).sum(0)}

"""Performance cases of the row operators around a sparse convolution: linear layers with an epilogue, products
grouped by expert or by kernel offset, and the norm and three-axis rotation of queries and keys.

A case is a dict of plain values:

  op       "linear", "linear_bwd", "grouped", "grouped_bwd", "rope", "rope_bwd"
  rows     rows of features (linear, rope) or entries of all groups together (grouped)
  dtype    of features, weights, gradients and outputs
  c_in, c_out, act ("none", "relu", "gelu", "silu"), bias, residual, save (the product before the activation is
           an output too), pad (the rows of x are that many elements farther apart than c_in)
  groups   number of groups; skew: how unequal they are (standard deviation of the logarithm of their shares);
           table: rows of x that the entries refer to, 0 where entry p is row p; pairs: entries are the pairs of a
           rulebook, so gradients are gathered too; grads: which gradients are asked for
  hq, hk, d heads of queries and keys, channels of a head; sections: pairs of channels that each axis turns; pairing:
           "halves" (j, j + d/2) or "adjacent" (2j, 2j + 1); norm: queries and keys are normalised first

Inputs are made on the GPU from the seed alone: features ~ N(0, 1), weights ~ N(0, 1/sqrt(c_in)), gradients ~ N(0, 1/16),
coordinates those of voxels in a box of 1408 x 1600 x 41 cells.
"""
from __future__ import annotations

import functools
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}
DEVICE = "cuda:0"
BOX = (1408, 1600, 41)
BASE, EPS = 10000.0, 1e-6


def _linear(name, rows, c_in, c_out, dtype, act="none", *, bias=True, residual=False, save=False, pad=0):
    return {"name": name, "op": "linear", "rows": rows, "c_in": c_in, "c_out": c_out, "dtype": dtype, "act": act, "bias": bias,
            "residual": residual, "save": save, "pad": pad}


def _linear_bwd(name, rows, c_in, c_out, dtype, act="none", *, bias=True, pad=0):
    return {"name": name, "op": "linear_bwd", "rows": rows, "c_in": c_in, "c_out": c_out, "dtype": dtype, "act": act, "bias": bias, "pad": pad}


def _grouped(name, rows, groups, c_in, c_out, dtype, act="none", *, bias=True, table=0, skew=0.7, save=False):
    return {"name": name, "op": "grouped", "rows": rows, "groups": groups, "c_in": c_in, "c_out": c_out, "dtype": dtype, "act": act,
            "bias": bias, "table": table, "skew": skew, "pairs": False, "save": save}


def _grouped_bwd(name, rows, groups, c_in, c_out, dtype, act="none", *, bias=True, table=0, skew=0.7, pairs=False, grads="xw"):
    return {"name": name, "op": "grouped_bwd", "rows": rows, "groups": groups, "c_in": c_in, "c_out": c_out, "dtype": dtype, "act": act,
            "bias": bias, "table": table, "skew": skew, "pairs": pairs, "grads": grads}


def _rope(name, op, rows, hq, hk, d, sections, dtype, *, pairing="halves", norm=True):
    return {"name": name, "op": op, "rows": rows, "hq": hq, "hk": hk, "d": d, "sections": ",".join(map(str, sections)), "dtype": dtype,
            "pairing": pairing, "norm": norm}


def listed():
    return [
        # one row through the wide half of a feed-forward block: a single token or voxel query; the weights are all there is to read
        _linear("linear one row bf16", 1, 1024, 4096, "bf16", "gelu"),
        # a first layer on raw point attributes in single precision: few channels, odd numbers of them
        _linear("linear small odd f32", 2000, 19, 37, "f32", "relu"),
        # feed-forward block over the voxels of one sweep, kept for the backward pass
        _linear("linear sweep f16", 53373, 64, 256, "f16", "gelu", save=True),
        # a projection back into the residual stream of a wide model: the largest product
        _linear("linear wide bf16", 32768, 2048, 2048, "bf16", residual=True),
        # training step of a feed-forward layer over three sweeps
        _linear_bwd("linear bwd sweeps bf16", 110545, 128, 512, "bf16", "gelu"),
        # a few voxels of a late frame dealt to many experts, most of which get none
        _grouped("experts few rows bf16", 48, 64, 512, 1024, "bf16", "silu"),
        # a sweep's voxels dealt to eight experts
        _grouped("experts sweep f16", 53373, 8, 128, 512, "f16", "silu", table=53373),
        # the weight gradient of a 3x3x3 layer, 64 -> 64, from its rulebook
        _grouped_bwd("rulebook gradient f16", 360625, 27, 64, 64, "f16", bias=False, table=53373, pairs=True, grads="w"),
        # training step of a wide model's experts
        _grouped_bwd("experts bwd wide bf16", 16384, 16, 512, 2048, "bf16", "silu", table=8192),
        # queries and keys of one new row
        _rope("rope one row bf16", "rope", 1, 16, 4, 128, (20, 22, 22), "bf16"),
        # four scenes in one batch
        _rope("rope batch4 bf16", "rope", 261574, 8, 8, 32, (6, 5, 5), "bf16", pairing="adjacent"),
        # training step over three sweeps, grouped keys
        _rope("rope bwd sweeps f16", "rope_bwd", 110545, 8, 2, 64, (10, 11, 11), "f16"),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _channels(rng, lo, hi):
    c = _between(rng, lo, hi)
    return rng.choice([c, max(16, (c + 15) // 16 * 16), max(32, (c + 31) // 32 * 32), max(64, (c + 63) // 64 * 64)])


def _draw_once(rng):
    op = rng.choice(["linear", "linear", "linear_bwd", "grouped", "grouped_bwd", "rope", "rope_bwd"])
    dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
    act = rng.choice(["none", "relu", "gelu", "silu"])
    pad = rng.choice([0, 0, 0, 8, 64, 5])
    if op in ("linear", "linear_bwd"):
        rows, c_in, c_out = _between(rng, 1, 300000), _channels(rng, 8, 4096), _channels(rng, 8, 4096)
        if op == "linear":
            return _linear("", rows, c_in, c_out, dtype, act, bias=rng.random() < 0.7, residual=rng.random() < 0.4, save=rng.random() < 0.3, pad=pad)
        return _linear_bwd("", rows, c_in, c_out, dtype, act, bias=rng.random() < 0.7, pad=pad)
    if op in ("grouped", "grouped_bwd"):
        rows, groups = _between(rng, 1, 400000), rng.choice([1, 2, 4, 8, 16, 27, 32, 64, 125])
        c_in, c_out = _channels(rng, 8, 2048), _channels(rng, 8, 2048)
        bias, skew = rng.random() < 0.5, rng.uniform(0.0, 1.5)
        table = rng.choice([0, rows, _between(rng, 1, rows)])
        if op == "grouped":
            return _grouped("", rows, groups, c_in, c_out, dtype, act, bias=bias, table=table, skew=skew, save=rng.random() < 0.3)
        if rng.random() < 0.4:
            return _grouped_bwd("", rows, groups, c_in, c_out, dtype, bias=False, table=max(1, table), skew=skew, pairs=True, grads=rng.choice(["w", "xw"]))
        return _grouped_bwd("", rows, groups, c_in, c_out, dtype, act, bias=bias, table=table, skew=skew, grads=rng.choice(["xw", "xw", "w", "x"]))
    hk = rng.choice([1, 2, 4, 8])
    hq = hk * rng.choice([1, 1, 2, 4, 8])
    d = rng.choice([16, 32, 64, 64, 96, 128, 128, 256, 2 * rng.randint(4, 80)])
    third = d // 6
    sections = rng.choice([(d // 2,), (d // 2 - 2 * third, third, third), (third, third, third)])
    return _rope("", op, _between(rng, 1, 300000), hq, hk, d, sections, dtype, pairing=rng.choice(["halves", "adjacent"]), norm=rng.random() < 0.75)


def draw(rng):
    """One more case: an operator, then sizes spread over the logarithm of their ranges, as far as they cost no more than listed ones."""
    while True:
        case = _draw_once(rng)
        need = work(case)
        most = 1.0e10 if case["dtype"] == "f32" else 1.0e11
        if need["flops"] <= most and need["bytes"] <= 5.0e8:
            del case["name"]
            return case


# ---- inputs ----------------------------------------------------------------------------------------------
def _sizes(case, rng):
    """Entries of each group: shares of unequal size, summing to rows; some groups of a skewed set get nothing."""
    share = [math.exp(case["skew"] * rng.gauss(0.0, 1.0)) * (0.0 if rng.random() < 0.05 else 1.0) for _ in range(case["groups"])]
    share[rng.randrange(case["groups"])] += 1e-3
    if case["rows"] < 8 * case["groups"]:
        sizes = [0] * case["groups"]
        for g in rng.choices(range(case["groups"]), weights=share, k=case["rows"]):
            sizes[g] += 1
        return sizes
    total = sum(share)
    sizes = [int(case["rows"] * s / total) for s in share]
    sizes[max(range(case["groups"]), key=lambda g: share[g])] += case["rows"] - sum(sizes)
    return sizes


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    rows = case["rows"]

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device=DEVICE) * scale).to(dt)

    if case["op"].startswith("rope"):
        hq, hk, d = case["hq"], case["hk"], case["d"]
        sections = [int(s) for s in case["sections"].split(",")]
        qkv = normal(rows, (hq + 2 * hk) * d)                       # the projection's output: queries, keys, values
        s = {"q": qkv[:, :hq * d].unflatten(1, (hq, d)), "k": qkv[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d)), "sections": sections}
        coords = torch.stack([torch.randint(0, n, (rows,), generator=gen, device=DEVICE) for n in (4, *BOX)], 1).to(torch.int32)
        s["pos"] = coords[:, 1:1 + len(sections)]
        s["gain_q"] = (1.0 + normal(d, scale=0.1).float()).to(dt) if case["norm"] else None
        s["gain_k"] = (1.0 + normal(d, scale=0.1).float()).to(dt) if case["norm"] else None
        if case["op"] == "rope_bwd":
            s["grad_q"], s["grad_k"] = normal(rows, hq, d, scale=1 / 16), normal(rows, hk, d, scale=1 / 16)
        return s

    c_in, c_out = case["c_in"], case["c_out"]
    scale = 1.0 / math.sqrt(c_in)
    if case["op"].startswith("linear"):
        s = {"x": normal(rows, c_in + case["pad"])[:, :c_in], "weight": normal(c_in, c_out, scale=scale)}
        s["bias"] = normal(c_out, scale=0.5) if case["bias"] else None
        if case["op"] == "linear":
            s["residual"] = normal(rows, c_out) if case["residual"] else None
        else:
            s["pre"] = normal(rows, c_out) if case["act"] != "none" else None
            s["grad"] = normal(rows, c_out, scale=1 / 16)
        return s

    groups, table = case["groups"], case["table"]
    sizes = _sizes(case, random.Random(f"{seed} {groups} {rows}"))
    bounds = [0]
    for n in sizes:
        bounds.append(bounds[-1] + n)
    s = {"bounds": bounds, "starts": torch.tensor(bounds, dtype=torch.int32, device=DEVICE), "weight": normal(groups, c_in, c_out, scale=scale)}
    s["x"] = normal(table if table else rows, c_in)

    def list_of_rows():
        """Rows of the table, ascending inside each group, as a rulebook or a stable sort by expert leaves them."""
        key = torch.randint(0, table, (rows,), generator=gen, device=DEVICE)
        owner = torch.repeat_interleave(torch.arange(groups, device=DEVICE), torch.tensor(sizes, device=DEVICE), output_size=rows)
        return ((owner * table + key).sort().values % table).to(torch.int32)

    s["rows"] = list_of_rows() if table else None
    s["bias"] = normal(groups, c_out, scale=0.5) if case["bias"] else None
    if case["op"] == "grouped_bwd":
        s["pre"] = normal(rows, c_out) if case["act"] != "none" else None
        s["grad_rows"] = list_of_rows() if case["pairs"] else None
        s["grad"] = normal(table if case["pairs"] else rows, c_out, scale=1 / 16)
    return s


@functools.lru_cache(maxsize=4)
def _turns(sections, d):
    """cos and sin of every position of every axis, [axis][position][pair] (what a program without the operator keeps)."""
    tables = []
    for axis, n in enumerate(sections):
        freq = BASE ** (-torch.arange(n, dtype=torch.float64, device=DEVICE) / max(n, 1))
        angle = torch.arange(BOX[axis], dtype=torch.float64, device=DEVICE)[:, None] * freq
        tables.append((angle.cos().float(), angle.sin().float()))
    return tables


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    dt, rows = DTYPES[case["dtype"]], case["rows"]
    if case["op"].startswith("rope") and not own:
        s["turns"] = _turns(tuple(s["sections"]), case["d"])
    if not own:
        return s
    from paper_2402_07710_amd import binding as sc

    def empty(*shape):
        return torch.empty(shape, dtype=dt, device=DEVICE)

    def workspace(n):
        return torch.empty(max(n, 16), dtype=torch.uint8, device=DEVICE)

    op = case["op"]
    if op.startswith("rope"):
        hq, hk, d = case["hq"], case["hk"], case["d"]
        s["table"] = sc.sc_rope_table(d, s["sections"], base=BASE, device=DEVICE)
        s["out_q"], s["out_k"] = empty(rows, hq, d), empty(rows, hk, d)
        if op == "rope_bwd":
            s["grad_gain_q"], s["grad_gain_k"] = (empty(d), empty(d)) if case["norm"] else (None, None)
            s["workspace"] = workspace(sc.sc_qk_rope_workspace_bytes(rows, hq, hk, d))
    elif op in ("linear", "grouped"):
        s["out"] = empty(rows, case["c_out"])
        s["kept"] = empty(rows, case["c_out"]) if case["save"] else None
    elif op == "linear_bwd":
        s["grad_x"], s["grad_weight"] = empty(rows, case["c_in"]), torch.empty_like(s["weight"])
        s["grad_bias"] = empty(case["c_out"]) if case["bias"] else None
        s["workspace"] = workspace(sc.sc_linear_workspace_bytes(rows, case["c_in"], case["c_out"], dt))
    else:
        s["grad_x"] = empty(rows, case["c_in"]) if "x" in case["grads"] else None
        s["grad_weight"] = torch.empty_like(s["weight"]) if "w" in case["grads"] else None
        s["grad_bias"] = empty(case["groups"], case["c_out"]) if case["bias"] and "w" in case["grads"] else None
        s["workspace"] = workspace(sc.sc_grouped_workspace_bytes(rows, case["groups"], case["c_in"], case["c_out"], dt))
    return s


# ---- one pass ----------------------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2402_07710_amd import binding as sc
    case = s["case"]
    op = case["op"]
    if op == "linear":
        sc.sc_linear_fwd(s["x"], s["weight"], s["out"], bias=s["bias"], act=case["act"], residual=s["residual"], pre=s["kept"])
        return [s["out"], s["kept"]] if case["save"] else [s["out"]]
    if op == "linear_bwd":
        sc.sc_linear_bwd(s["grad"], s["x"], s["weight"], grad_x=s["grad_x"], grad_weight=s["grad_weight"], grad_bias=s["grad_bias"],
                         pre=s["pre"], act=case["act"], workspace=s["workspace"])
        return [t for t in (s["grad_x"], s["grad_weight"], s["grad_bias"]) if t is not None]
    if op == "grouped":
        sc.sc_grouped_fwd(s["x"], s["weight"], s["starts"], s["out"], rows=s["rows"], bias=s["bias"], act=case["act"], pre=s["kept"])
        return [s["out"], s["kept"]] if case["save"] else [s["out"]]
    if op == "grouped_bwd":
        sc.sc_grouped_bwd(s["grad"], s["x"], s["weight"], s["starts"], grad_x=s["grad_x"], grad_weight=s["grad_weight"],
                          grad_bias=s["grad_bias"], rows=s["rows"], grad_rows=s["grad_rows"], pre=s["pre"], act=case["act"],
                          workspace=s["workspace"])
        return [t for t in (s["grad_x"], s["grad_weight"], s["grad_bias"]) if t is not None]
    if op == "rope":
        sc.sc_qk_rope_fwd(s["q"], s["k"], s["pos"], s["table"], s["out_q"], s["out_k"], gain_q=s["gain_q"], gain_k=s["gain_k"], eps=EPS,
                          pairing=case["pairing"])
        return [s["out_q"], s["out_k"]]
    sc.sc_qk_rope_bwd(s["grad_q"], s["grad_k"], s["q"], s["k"], s["pos"], s["table"], s["out_q"], s["out_k"], gain_q=s["gain_q"],
                      gain_k=s["gain_k"], grad_gain_q=s["grad_gain_q"], grad_gain_k=s["grad_gain_k"], eps=EPS, pairing=case["pairing"],
                      workspace=s["workspace"])
    return [t for t in (s["out_q"], s["out_k"], s["grad_gain_q"], s["grad_gain_k"]) if t is not None]


def _activate(v, act):
    if act == "relu":
        return v.clamp(min=0.0)
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "silu":
        return v * torch.sigmoid(v)
    return v


def _slope(v, act):
    if act == "relu":
        return (v > 0.0).to(v.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "silu":
        sig = torch.sigmoid(v)
        return sig * (1.0 + v * (1.0 - sig))
    return torch.ones_like(v)


def _run_plain(s):
    case = s["case"]
    op, dt, act = case["op"], DTYPES[case["dtype"]], case.get("act")
    if op == "linear":
        pre = s["x"].float() @ s["weight"].float()
        if s["bias"] is not None:
            pre = pre + s["bias"].float()
        out = _activate(pre, act)
        if s["residual"] is not None:
            out = out + s["residual"].float()
        return [out.to(dt), pre.to(dt)] if case["save"] else [out.to(dt)]
    if op == "linear_bwd":
        grad = s["grad"].float()
        if act != "none":
            grad = grad * _slope(s["pre"].float(), act)
        out = [(grad @ s["weight"].float().t()).to(dt), (s["x"].float().t() @ grad).to(dt)]
        return out + [grad.sum(0).to(dt)] if case["bias"] else out
    if op == "grouped":
        x = s["x"].float() if s["rows"] is None else s["x"].index_select(0, s["rows"]).float()
        pre = torch.empty((case["rows"], case["c_out"]), device=DEVICE)
        for g in range(case["groups"]):
            a, b = s["bounds"][g], s["bounds"][g + 1]
            if a < b:
                torch.mm(x[a:b], s["weight"][g].float(), out=pre[a:b])
                if s["bias"] is not None:
                    pre[a:b] += s["bias"][g].float()
        out = _activate(pre, act).to(dt)
        return [out, pre.to(dt)] if case["save"] else [out]
    if op == "grouped_bwd":
        grad = s["grad"].float() if s["grad_rows"] is None else s["grad"].index_select(0, s["grad_rows"]).float()
        if act != "none":
            grad = grad * _slope(s["pre"].float(), act)
        out = []
        parts = [(g, s["bounds"][g], s["bounds"][g + 1]) for g in range(case["groups"]) if s["bounds"][g] < s["bounds"][g + 1]]
        if "x" in case["grads"]:
            grad_x = torch.empty((case["rows"], case["c_in"]), device=DEVICE)
            for g, a, b in parts:
                torch.mm(grad[a:b], s["weight"][g].float().t(), out=grad_x[a:b])
            out.append(grad_x.to(dt))
        if "w" in case["grads"]:
            x = s["x"].float() if s["rows"] is None else s["x"].index_select(0, s["rows"]).float()
            grad_w = torch.zeros((case["groups"], case["c_in"], case["c_out"]), device=DEVICE)
            for g, a, b in parts:
                torch.mm(x[a:b].t(), grad[a:b], out=grad_w[g])
            out.append(grad_w.to(dt))
            if case["bias"]:
                grad_b = torch.zeros((case["groups"], case["c_out"]), device=DEVICE)
                for g, a, b in parts:
                    grad_b[g] = grad[a:b].sum(0)
                out.append(grad_b.to(dt))
        return out
    # rope, rope_bwd
    half, pairing = case["d"] // 2, case["pairing"]
    turned = sum(s["sections"])
    cos = torch.cat([t[0][s["pos"][:, a].long()] for a, t in enumerate(s["turns"])], 1)[:, None, :]
    sin = torch.cat([t[1][s["pos"][:, a].long()] for a, t in enumerate(s["turns"])], 1)[:, None, :]

    def rotate(v, sine):
        if pairing == "halves":
            a, b = v[..., :turned], v[..., half:half + turned]
            return torch.cat([a * cos - b * sine, v[..., turned:half], a * sine + b * cos, v[..., half + turned:]], -1)
        a, b = v[..., 0:2 * turned:2], v[..., 1:2 * turned:2]
        return torch.cat([torch.stack([a * cos - b * sine, a * sine + b * cos], -1).flatten(-2), v[..., 2 * turned:]], -1)

    if op == "rope":
        out = []
        for v, gain in ((s["q"], s["gain_q"]), (s["k"], s["gain_k"])):
            v = v.float()
            if gain is not None:
                v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * gain.float()
            out.append(rotate(v, sin).to(dt))
        return out
    grads, gains = [], []
    for grad, v, gain in ((s["grad_q"], s["q"], s["gain_q"]), (s["grad_k"], s["k"], s["gain_k"])):
        turned_back = rotate(grad.float(), -sin)
        if gain is None:
            grads.append(turned_back.to(dt))
            continue
        v = v.float()
        scale = torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
        unit = v * scale
        gains.append((turned_back * unit).sum((0, 1)).to(dt))
        u = turned_back * gain.float()
        grads.append(((u - unit * (u * unit).mean(-1, keepdim=True)) * scale).to(dt))
    return grads + gains


# ---- what a pass needs, and what it should give ----------------------------------------------------------------
def work(case):
    """Bytes: every input once, every output once.  Operations: the products (of the rotation: five a channel, ten backwards)."""
    size, rows, op = SIZES[case["dtype"]], case["rows"], case["op"]
    if op.startswith("rope"):
        values = rows * (case["hq"] + case["hk"]) * case["d"]
        coords = 4 * rows * len(case["sections"].split(","))
        passes = 2 if op == "rope" else 3
        return {"bytes": passes * values * size + coords, "flops": 5 * (passes - 1) * values}
    c_in, c_out = case["c_in"], case["c_out"]
    has_act, bias = case["act"] != "none", case["bias"]
    if op == "linear":
        values = rows * (c_in + c_out * (1 + case["residual"] + case["save"])) + c_in * c_out + c_out * bias
        return {"bytes": values * size, "flops": 2 * rows * c_in * c_out}
    if op == "linear_bwd":
        values = rows * (c_out * (1 + has_act) + 2 * c_in) + 2 * c_in * c_out + c_out * bias
        return {"bytes": values * size, "flops": 4 * rows * c_in * c_out}
    groups = min(case["groups"], rows)
    read = min(rows, case["table"]) if case["table"] else rows
    lists = 4 * (case["groups"] + 1) + (4 * rows if case["table"] else 0)
    if op == "grouped":
        values = read * c_in + rows * c_out * (1 + case["save"]) + groups * (c_in * c_out + c_out * bias)
        return {"bytes": values * size + lists, "flops": 2 * rows * c_in * c_out}
    grads = case["grads"]
    values = (read if case["pairs"] else rows) * c_out + (rows * c_out if has_act else 0)
    if "x" in grads:
        values += groups * c_in * c_out + rows * c_in
    if "w" in grads:
        values += read * c_in + case["groups"] * (c_in * c_out + c_out * bias)
    return {"bytes": values * size + lists + (4 * rows if case["pairs"] else 0), "flops": 2 * rows * c_in * c_out * len(grads)}


def exact(case, seed):
    """The definitions in 64 bits; gradients by differentiating them."""
    s = _inputs(case, seed)
    op = case["op"]
    wide = {key: (v.double() if torch.is_tensor(v) and v.is_floating_point() else v) for key, v in s.items()}

    def activation(v):
        kinds = {"none": lambda t: t, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}
        return kinds[case["act"]](v)

    def through_activation(pre, grad):
        if pre is None:
            return grad
        at = pre.detach().requires_grad_(True)
        activation(at).backward(grad)
        return at.grad

    if op == "linear":
        pre = wide["x"].matmul(wide["weight"])
        if s["bias"] is not None:
            pre += wide["bias"]
        out = activation(pre)
        if s["residual"] is not None:
            out = out + wide["residual"]
        return [out, pre] if case["save"] else [out]
    if op == "linear_bwd":
        grad = through_activation(wide["pre"], wide["grad"])
        out = [grad.matmul(wide["weight"].t().contiguous()), wide["x"].t().contiguous().matmul(grad)]
        return out + [grad.sum(0)] if case["bias"] else out
    if op in ("grouped", "grouped_bwd"):
        rows, groups, c_in, c_out = case["rows"], case["groups"], case["c_in"], case["c_out"]
        x = wide["x"] if s["rows"] is None else wide["x"][s["rows"].long()]
        member = [slice(s["bounds"][g], s["bounds"][g + 1]) for g in range(groups)]
        if op == "grouped":
            pre = torch.cat([x[m].matmul(wide["weight"][g]) + (wide["bias"][g] if s["bias"] is not None else 0.0) for g, m in enumerate(member)])
            return [activation(pre), pre] if case["save"] else [activation(pre)]
        grad = wide["grad"] if s["grad_rows"] is None else wide["grad"][s["grad_rows"].long()]
        grad = through_activation(wide["pre"], grad)
        out = []
        if "x" in case["grads"]:
            out.append(torch.cat([grad[m].matmul(wide["weight"][g].t().contiguous()) for g, m in enumerate(member)]))
        if "w" in case["grads"]:
            out.append(torch.stack([x[m].t().contiguous().matmul(grad[m]) for m in member]))
            if case["bias"]:
                out.append(torch.stack([grad[m].sum(0) for m in member]))
        return out
    d = case["d"]
    index = torch.arange(d // 2, device=DEVICE)
    low = index if case["pairing"] == "halves" else 2 * index
    high = index + d // 2 if case["pairing"] == "halves" else 2 * index + 1
    angle = torch.zeros((case["rows"], d // 2), dtype=torch.float64, device=DEVICE)
    at = 0
    for axis, n in enumerate(s["sections"]):
        for i in range(n):
            angle[:, at] = s["pos"][:, axis].double() * BASE ** (-i / n)
            at += 1
    turn = torch.polar(torch.ones_like(angle), angle)[:, None, :]

    def forward(v, gain):
        if gain is not None:
            v = v / torch.sqrt(v.square().mean(-1, keepdim=True) + EPS) * gain
        z = torch.complex(v[..., low], v[..., high]) * turn
        out = torch.empty_like(v)
        out[..., low], out[..., high] = z.real, z.imag
        return out

    if op == "rope":
        return [forward(wide["q"], wide["gain_q"]), forward(wide["k"], wide["gain_k"])]
    grads, gains = [], []
    for name in ("q", "k"):
        v = wide[name].detach().clone().requires_grad_(True)
        gain = wide["gain_" + name]
        gain = gain.detach().clone().requires_grad_(True) if gain is not None else None
        forward(v, gain).backward(wide["grad_" + name])
        grads.append(v.grad)
        if gain is not None:
            gains.append(gain.grad)
    return grads + gains

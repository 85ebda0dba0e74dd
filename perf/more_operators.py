"""Performance cases of attention over packed scenes and of the group norm with an activation, forward and backward.

A case is a dict of plain values:

  op       "attention", "attention_bwd", "norm", "norm_bwd"
  rows     rows of features (norm) or of queries (attention), of all scenes together
  scenes   how many scenes the rows are packed from; skew: how unequal they are (standard deviation of the logarithm of their shares)
  dtype    of rows, outputs and gradients
  keys     rows of keys and values of all scenes together; 0: the queries' own rows, slices of one projection
  hq, hk, d  heads of queries and of keys, channels of a head
  causal   queries and keys of a scene end together, and a query sees no key behind it
  c, groups, act ("none", "relu", "gelu", "silu"), save (mean and 1/deviation are outputs too)   of the norm

How long the scenes are follows from the case, what the rows hold from the seed: queries, keys, values and features ~ N(0, 1), features with
a mean of their own in every channel, gradients ~ N(0, 1/16).
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}
DEVICE = "cuda:0"
EPS = 1e-5


def _attention(name, op, rows, scenes, hq, hk, d, dtype, *, keys=0, causal=False, skew=0.5):
    return {"name": name, "op": op, "rows": rows, "scenes": scenes, "keys": keys, "hq": hq, "hk": hk, "d": d, "dtype": dtype, "causal": causal, "skew": skew}


def _norm(name, op, rows, scenes, c, groups, dtype, act, *, save=False, skew=0.3):
    return {"name": name, "op": op, "rows": rows, "scenes": scenes, "c": c, "groups": groups, "dtype": dtype, "act": act, "save": save, "skew": skew}


def listed():
    return [
        # one new row asks a short history: nothing but latency
        _attention("attention one row bf16", "attention", 1, 1, 8, 8, 32, "bf16", keys=77, causal=True),
        # the next row of eight long sequences, grouped heads: the cache is all there is to read
        _attention("attention next rows f16", "attention", 8, 8, 16, 4, 128, "f16", keys=262144, causal=True, skew=0.3),
        # the voxels of one sweep in windows of some 48
        _attention("attention windows f16", "attention", 53373, 1112, 8, 8, 16, "f16"),
        # whole sequences of serialised voxels, packed, causal, grouped heads: the largest products
        _attention("attention sequences bf16", "attention", 16384, 3, 16, 4, 128, "bf16", causal=True),
        # a few odd scenes in single precision, queries of one set over the keys of another, more queries than keys in some
        _attention("attention odd f32", "attention", 1501, 7, 6, 2, 20, "f32", keys=2103, causal=True, skew=0.9),
        # training step over the windows of three sweeps
        _attention("attention bwd windows f16", "attention_bwd", 110545, 2303, 8, 8, 16, "f16"),
        # training step over packed sequences, grouped heads
        _attention("attention bwd sequences bf16", "attention_bwd", 16384, 4, 16, 4, 64, "bf16", causal=True),
        # odd scenes in single precision
        _attention("attention bwd odd f32", "attention_bwd", 1501, 7, 6, 2, 20, "f32", skew=0.9),
        # a late, small scene in the deepest stage
        _norm("norm few rows bf16", "norm", 33, 1, 256, 32, "bf16", "silu"),
        # four scenes in one batch, first stage, kept for the backward pass
        _norm("norm batch4 f16", "norm", 261574, 4, 64, 8, "f16", "relu", save=True),
        # training step over three sweeps, a wide stage
        _norm("norm bwd sweeps bf16", "norm_bwd", 110545, 3, 256, 32, "bf16", "silu"),
        # odd channels in single precision
        _norm("norm bwd odd f32", "norm_bwd", 3001, 5, 45, 9, "f32", "gelu", skew=0.9),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    op = rng.choice(["attention", "attention", "attention_bwd", "norm", "norm_bwd"])
    dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
    skew = rng.uniform(0.0, 1.0)
    if op.startswith("norm"):
        rows, groups = _between(rng, 1, 300000), rng.choice([1, 2, 4, 8, 16, 32, 32, rng.randint(1, 48)])
        c = groups * rng.choice([1, 2, 4, 4, 8, 8, 16, 16, 32, rng.randint(1, 40)])
        scenes = rng.choice([1, 2, 4, rng.randint(1, 16), _between(rng, 1, max(1, rows // 20))])
        # the slope of the rectifier jumps where a value is next to zero, so its gradient is none to compare with
        act = rng.choice(["none", "relu", "gelu", "silu"] if op == "norm" else ["none", "gelu", "silu"])
        return _norm("", op, rows, min(scenes, rows), c, groups, dtype, act, save=op == "norm" and rng.random() < 0.5, skew=skew)
    hk = rng.choice([1, 2, 4, 8])
    hq = hk * rng.choice([1, 1, 1, 2, 3, 4, 8])
    d = rng.choice([16, 32, 32, 64, 64, 128, 128, rng.randint(4, 160), 256])
    kind = rng.choice(["windows", "scenes", "scenes", "other keys", "next rows"] if op == "attention" else ["windows", "scenes", "scenes", "other keys"])
    if kind == "windows":
        rows = _between(rng, 100, 150000)
        return _attention("", op, rows, max(1, rows // _between(rng, 9, 300)), hq, hk, d, dtype, causal=rng.random() < 0.3, skew=min(skew, 0.6))
    scenes = rng.choice([1, 1, 2, 3, 4, rng.randint(1, 32)])
    if kind == "next rows":
        rows = scenes * rng.choice([1, 1, 1, rng.randint(2, 8)])
        return _attention("", op, rows, scenes, hq, hk, d, dtype, keys=_between(rng, 1, 300000), causal=rng.random() < 0.7, skew=min(skew, 0.3) if rows == scenes else skew)
    rows = _between(rng, 1, 20000)
    keys = _between(rng, 1, 20000) if kind == "other keys" else 0
    return _attention("", op, rows, min(scenes, rows), hq, hk, d, dtype, keys=keys, causal=rng.random() < 0.5, skew=skew)


def draw(rng):
    """One more case: an operator, then sizes spread over the logarithm of their ranges, as far as they cost no more than listed ones."""
    while True:
        case = _draw_once(rng)
        if case["op"].endswith("bwd") or "c" in case:                   # gradients and deviations of next to nothing are rounding alone
            if min(case["rows"], case.get("keys") or case["rows"]) * case.get("c", 1) < 8 * case["scenes"] * case.get("groups", 1):
                continue
        need = work(case)
        most = 1.0e10 if case["dtype"] == "f32" else 2.0e11
        lens, key_lens = _lengths(case)
        wide = case["c"] if "c" in case else case["hq"] * max(max(key_lens), case["d"])
        if need["flops"] <= most and need["bytes"] <= 4.0e8 and len(lens) * max(max(lens), 1) * wide <= 2.0e9:
            del case["name"]
            return case


# ---- inputs ----------------------------------------------------------------------------------------------
def _shares(rows, scenes, skew, rng):
    """Rows of each scene: shares of unequal size, summing to rows; of many scenes some get nothing."""
    if rows == scenes and skew <= 0.31:                                # a row each: the next one of every sequence
        return [1] * scenes
    share = [math.exp(skew * rng.gauss(0.0, 1.0)) * (0.0 if rng.random() < 0.03 else 1.0) for _ in range(scenes)]
    share[rng.randrange(scenes)] += 1e-3
    total, passed, lens = sum(share), 0.0, []
    for part in share:
        passed += part
        lens.append(int(rows * passed / total + 0.5))                   # where the scene ends
    return [stop - first for first, stop in zip([0] + lens, lens)]


def _lengths(case):
    """Rows, or queries, and keys of every scene."""
    rng = random.Random(f"{case['rows']} {case['scenes']} {case['skew']}")
    lens = _shares(case["rows"], case["scenes"], case["skew"], rng)
    return lens, _shares(case["keys"], case["scenes"], case["skew"], rng) if case.get("keys") else lens


def _starts(lens):
    bounds = [0]
    for n in lens:
        bounds.append(bounds[-1] + n)
    return torch.tensor(bounds, dtype=torch.int32, device=DEVICE)


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    rows = case["rows"]

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device=DEVICE) * scale).to(dt)

    lens, key_lens = _lengths(case)
    s = {"lens": lens, "key_lens": key_lens, "starts": _starts(lens)}
    if case["op"].startswith("norm"):
        c = case["c"]
        s["x"] = (torch.randn((rows, c), generator=gen, device=DEVICE) + torch.randn(c, generator=gen, device=DEVICE)).to(dt)
        s["gain"] = (1.0 + normal(c, scale=0.2).float()).to(dt)
        s["bias"] = normal(c, scale=0.2)
        if case["op"] == "norm_bwd":
            s["grad"] = normal(rows, c, scale=1 / 16)
        return s
    hq, hk, d, keys = case["hq"], case["hk"], case["d"], case["keys"]
    if keys:
        s["q"], s["k"], s["v"] = normal(rows, hq, d), normal(keys, hk, d), normal(keys, hk, d)
        s["key_starts"] = _starts(key_lens)
    else:                                                               # the projection's output: queries, keys, values
        qkv = normal(rows, (hq + 2 * hk) * d)
        s["q"], s["k"], s["v"] = (part.unflatten(1, (-1, d)) for part in qkv.split([hq * d, hk * d, hk * d], 1))
        s["key_starts"] = s["starts"]
    if case["op"] == "attention_bwd":
        s["grad"] = normal(rows, hq, d, scale=1 / 16)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    dt, rows = DTYPES[case["dtype"]], case["rows"]
    op = case["op"]
    if op == "attention_bwd":                                           # what the forward pass left
        out, lse = _attend(s)
        s["out"], s["lse"] = out.to(dt), lse
    if op == "norm_bwd":
        s["stats"] = torch.stack(_moments(s), -1).float()
    if own:
        from paper_2402_07710_amd import binding as sc

        def empty(*shape):
            return torch.empty(shape, dtype=dt, device=DEVICE)

        def workspace(n):
            return torch.empty(max(n, 16), dtype=torch.uint8, device=DEVICE)

        if op.startswith("norm"):
            c, groups = case["c"], case["groups"]
            s["workspace"] = workspace(sc.sc_group_norm_workspace_bytes(rows, case["scenes"], c, groups))
            s["new"] = empty(rows, c)
            if op == "norm":
                s["stats"] = torch.empty((case["scenes"], groups, 2), device=DEVICE) if case["save"] else None
            else:
                s["grad_gain"], s["grad_bias"] = empty(c), empty(c)
            return s
        hq, hk, d, keys = case["hq"], case["hk"], case["d"], case["keys"]
        sizes = (rows, keys if keys else rows, case["scenes"], hq, hk, d, dt)
        if op == "attention":
            s["out"] = empty(rows, hq, d)
            s["workspace"] = workspace(sc.sc_attention_workspace_bytes(*sizes))
        else:
            s["workspace"] = workspace(sc.sc_attention_bwd_workspace_bytes(*sizes))
            if keys:
                s["grads"] = [empty(rows, hq, d), empty(keys, hk, d), empty(keys, hk, d)]
            else:
                s["grads"] = [part.unflatten(1, (-1, d)) for part in empty(rows, (hq + 2 * hk) * d).split([hq * d, hk * d, hk * d], 1)]
    return s


# ---- one pass ----------------------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2402_07710_amd import binding as sc
    case = s["case"]
    op = case["op"]
    if op == "attention":
        sc.sc_attention_fwd(s["q"], s["k"], s["v"], s["out"], q_starts=s["starts"], k_starts=s["key_starts"], causal=case["causal"], workspace=s["workspace"])
        return [s["out"]]
    if op == "attention_bwd":
        sc.sc_attention_bwd(s["grad"], s["q"], s["k"], s["v"], s["out"], s["lse"], *s["grads"], q_starts=s["starts"], k_starts=s["key_starts"],
                            causal=case["causal"], workspace=s["workspace"])
        return s["grads"]
    if op == "norm":
        sc.sc_group_norm_fwd(s["x"], s["new"], case["groups"], starts=s["starts"], gain=s["gain"], bias=s["bias"], act=case["act"], eps=EPS, stats=s["stats"],
                             workspace=s["workspace"])
        return [s["new"], s["stats"]] if case["save"] else [s["new"]]
    sc.sc_group_norm_bwd(s["grad"], s["x"], s["stats"], s["new"], case["groups"], starts=s["starts"], gain=s["gain"], bias=s["bias"], act=case["act"],
                         grad_gain=s["grad_gain"], grad_bias=s["grad_bias"], workspace=s["workspace"])
    return [s["new"], s["grad_gain"], s["grad_bias"]]


def _padding(starts, lens, rows):
    """For scenes padded to the longest: row of every place [scenes, longest], which places are rows, and the place of every row."""
    longest = max(max(lens), 1)
    place = torch.arange(longest, device=DEVICE)
    first, stop = starts[:-1].long()[:, None], starts[1:].long()[:, None]
    there = first + place < stop
    index = torch.where(there, first + place, 0)
    row = torch.arange(rows, device=DEVICE)
    scene = torch.bucketize(row, starts[1:].long(), right=True)
    return index, there, scene * longest + row - starts.long()[scene]


def _scores(s):
    """Padded queries [scenes, hk, hq/hk * longest, d], keys, values in 32 bits, weights of the values, logarithm of their sums, and where the rows are."""
    case = s["case"]
    hq, hk, d = case["hq"], case["hk"], case["d"]
    q_index, q_there, q_place = _padding(s["starts"], s["lens"], case["rows"])
    k_index, k_there, k_place = _padding(s["key_starts"], s["key_lens"], case["keys"] or case["rows"])
    scenes, nq = q_index.shape
    nk = k_index.shape[1]
    grouped = (scenes * hk, hq // hk * nq, d)
    q = s["q"][q_index].float().transpose(1, 2).reshape(grouped)
    k = s["k"][k_index].float().transpose(1, 2).reshape(scenes * hk, nk, d)
    v = s["v"][k_index].float().transpose(1, 2).reshape(scenes * hk, nk, d)
    seen = k_there[:, None, :]
    if case["causal"]:
        ahead = (k_there.sum(1) - q_there.sum(1))[:, None, None]
        seen = seen & (torch.arange(nk, device=DEVICE) <= torch.arange(nq, device=DEVICE)[:, None] + ahead)
    scores = (torch.bmm(q, k.transpose(1, 2)) * d ** -0.5).view(scenes, hq, nq, nk)
    scores = scores.masked_fill_(~seen[:, None], -math.inf)
    most = scores.amax(-1, keepdim=True)
    scores = scores.sub_(torch.where(most > -math.inf, most, 0.0)).exp_()
    total = scores.sum(-1, keepdim=True)
    weights = scores.div_(torch.where(total > 0.0, total, 1.0)).view(scenes * hk, -1, nk)
    lse = (most + total.log())[..., 0].transpose(1, 2).reshape(-1, hq)[q_place]
    return q, k, v, weights, lse, q_index, q_place, k_place


def _rows_of(padded, scenes, heads, place):
    """[scenes * hk, hq/hk * longest, d] -> the scenes' rows [rows, heads, d]."""
    d = padded.shape[-1]
    return padded.view(scenes, heads, -1, d).transpose(1, 2).reshape(-1, heads, d)[place]


def _attend(s):
    case = s["case"]
    _, _, v, weights, lse, _, q_place, _ = _scores(s)
    return _rows_of(torch.bmm(weights, v), case["scenes"], case["hq"], q_place), lse


def _in_groups(s, rows, index):
    """Rows of [scenes, longest, groups, channels of a group] in 32 bits."""
    return rows[index].float().unflatten(2, (s["case"]["groups"], -1))


def _moments(s):
    """Mean and 1/deviation [scenes, groups] of the rows, in two passes."""
    index, there, _ = _padding(s["starts"], s["lens"], s["case"]["rows"])
    x = _in_groups(s, s["x"], index)
    there = there[:, :, None, None]
    count = (there.sum((1, 2, 3)) * x.shape[-1]).clamp(min=1)[:, None]
    mean = (x * there).sum((1, 3)) / count
    square = (x - mean[:, None, :, None]).square() * there
    return mean, torch.rsqrt(square.sum((1, 3)) / count + EPS)


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
    op, dt, scenes = case["op"], DTYPES[case["dtype"]], case["scenes"]
    if op == "attention":
        return [_attend(s)[0].to(dt)]
    if op == "attention_bwd":
        q, k, v, weights, _, q_index, q_place, k_place = _scores(s)
        q_there = torch.arange(q_index.shape[1], device=DEVICE) < (s["starts"][1:] - s["starts"][:-1])[:, None]
        grad = (s["grad"][q_index].float() * q_there[:, :, None, None]).transpose(1, 2).reshape(q.shape)
        grad_v = torch.bmm(weights.transpose(1, 2), grad)
        slope = torch.bmm(grad, v.transpose(1, 2))
        slope = weights.mul_(slope.sub_((weights * slope).sum(-1, keepdim=True))).mul_(case["d"] ** -0.5)
        grad_q, grad_k = torch.bmm(slope, k), torch.bmm(slope.transpose(1, 2), q)
        return [_rows_of(grad_q, scenes, case["hq"], q_place).to(dt), _rows_of(grad_k, scenes, case["hk"], k_place).to(dt),
                _rows_of(grad_v, scenes, case["hk"], k_place).to(dt)]
    index, there, place = _padding(s["starts"], s["lens"], case["rows"])
    mean, scale = _moments(s) if op == "norm" else s["stats"].unbind(-1)
    unit = (_in_groups(s, s["x"], index) - mean[:, None, :, None]) * scale[:, None, :, None]
    gain, bias = s["gain"].float().unflatten(0, (case["groups"], -1)), s["bias"].float().unflatten(0, (case["groups"], -1))
    pre = unit * gain + bias
    if op == "norm":
        out = _activate(pre, case["act"]).flatten(2).flatten(0, 1)[place].to(dt)
        return [out, torch.stack([mean, scale], -1)] if case["save"] else [out]
    grad = _in_groups(s, s["grad"], index) * there[:, :, None, None] * _slope(pre, case["act"])
    along = grad * unit
    grad_gain, grad_bias = along.sum((0, 1)).flatten(), grad.sum((0, 1)).flatten()
    count = (there.sum(1) * unit.shape[-1]).clamp(min=1)[:, None]
    mean_grad, mean_along = (grad * gain).sum((1, 3)) / count, (along * gain).sum((1, 3)) / count
    grad_x = (grad * gain - mean_grad[:, None, :, None] - unit * mean_along[:, None, :, None]) * scale[:, None, :, None]
    return [grad_x.flatten(2).flatten(0, 1)[place].to(dt), grad_gain.to(dt), grad_bias.to(dt)]


# ---- what a pass needs, and what it should give ----------------------------------------------------------------
def _pairs(case):
    """Pairs of a query and a key that it sees."""
    total = 0
    for nq, nk in zip(*_lengths(case)):
        if not case["causal"]:
            total += nq * nk
        else:                                                           # query i sees i + nk - nq + 1 keys, none where that is less
            first = max(0, nq - nk)
            total += (nq - first) * (first + nk - nq + 1 + nk) // 2
    return total


def work(case):
    """Bytes: every input once, every output once.  Operations: of attention the products (two a pair and channel forward, five backward), of
    the norm some ten a value forward and twenty backward."""
    size, rows, op = SIZES[case["dtype"]], case["rows"], case["op"]
    if op.startswith("norm"):
        values = rows * case["c"]
        passes = 2 if op == "norm" else 3
        stats = 8 * case["scenes"] * case["groups"] * (case["save"] or op == "norm_bwd")
        return {"bytes": (passes * values + passes * case["c"]) * size + stats + 4 * (case["scenes"] + 1), "flops": 10 * (passes - 1) * values}
    hq, hk, d, keys = case["hq"], case["hk"], case["d"], case["keys"] or rows
    queries, shared = rows * hq * d, keys * hk * d
    starts = 4 * (case["scenes"] + 1) * (2 if case["keys"] else 1)
    if op == "attention":
        return {"bytes": (2 * queries + 2 * shared) * size + starts, "flops": 4 * _pairs(case) * hq * d}
    return {"bytes": (4 * queries + 4 * shared) * size + 4 * rows * hq + starts, "flops": 10 * _pairs(case) * hq * d}


def exact(case, seed):
    """The definitions in 64 bits, scene by scene; gradients by differentiating them."""
    s = _inputs(case, seed)
    op = case["op"]
    wide = {key: v.double() for key, v in s.items() if torch.is_tensor(v) and v.is_floating_point()}
    lens, key_lens = s["lens"], s["key_lens"]
    if op.startswith("norm"):
        for key in ("x", "gain", "bias"):
            wide[key].requires_grad_(op == "norm_bwd")
        kinds = {"none": lambda t: t, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}
        out, stats = [], []
        for x in wide["x"].split(lens):
            x = x.reshape(len(x), case["groups"], -1)
            if len(x) == 0:
                out.append(x.flatten(1))
                stats.append(torch.tensor([[0.0, EPS ** -0.5]] * case["groups"], dtype=torch.float64, device=DEVICE))
                continue
            mean, var = x.mean((0, 2)), x.var((0, 2), unbiased=False)
            unit = (x - mean[:, None]) / torch.sqrt(var + EPS)[:, None]
            out.append(kinds[case["act"]](unit.flatten(1) * wide["gain"] + wide["bias"]))
            stats.append(torch.stack([mean, 1.0 / torch.sqrt(var + EPS)], -1))
        out = torch.cat(out)
        if op == "norm":
            return [out, torch.stack(stats)] if case["save"] else [out]
        out.backward(wide["grad"])
        return [wide["x"].grad, wide["gain"].grad, wide["bias"].grad]
    per = case["hq"] // case["hk"]
    backward = op == "attention_bwd"
    result = [torch.zeros_like(wide[key]) for key in (("q", "k", "v") if backward else ("q",))]
    at = key_at = 0
    for nq, nk in zip(lens, key_lens):
        mine, theirs = slice(at, at + nq), slice(key_at, key_at + nk)
        at, key_at = at + nq, key_at + nk
        if nq == 0 or nk == 0:
            continue
        hidden = None
        if case["causal"]:
            hidden = torch.ones((nq, nk), dtype=torch.bool, device=DEVICE).triu_(nk - nq + 1)
            blind = hidden.all(1)[:, None]
        step = max(1, int(2 ** 29 // (per * nq * nk)))                  # heads of keys at a time
        for h in range(0, case["hk"], step):
            part = slice(h, min(h + step, case["hk"]))
            heads = slice(part.start * per, part.stop * per)
            q = wide["q"][mine, heads].transpose(0, 1).contiguous().requires_grad_(backward)
            k, v = (wide[key][theirs, part].transpose(0, 1).contiguous().requires_grad_(backward) for key in ("k", "v"))
            score = torch.matmul(q, k.repeat_interleave(per, 0).transpose(1, 2).contiguous()) / math.sqrt(case["d"])
            if hidden is not None:
                score = score.masked_fill(hidden, -math.inf).masked_fill(blind, 0.0)
            weight = score.softmax(-1)
            if hidden is not None:
                weight = weight.masked_fill(blind, 0.0)
            out = torch.matmul(weight, v.repeat_interleave(per, 0))
            if not backward:
                result[0][mine, heads] = out.transpose(0, 1)
                continue
            out.backward(wide["grad"][mine, heads].transpose(0, 1).contiguous())
            result[0][mine, heads] = q.grad.transpose(0, 1)
            result[1][theirs, part] = k.grad.transpose(0, 1)
            result[2][theirs, part] = v.grad.transpose(0, 1)
    return result

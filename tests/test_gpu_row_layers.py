"""GPU tests of the row layers (linear, grouped, norm and rotation of queries and keys) against their definitions in 64 bits on
the CPU.

Bounds are per element and follow from the arithmetic: a sum of K products of the given numbers in 32 bits is off by at most
(K + 8) 2^-23 of the sum of their magnitudes (each product exact or rounded once, each addition rounded or cut), an activation
passes that on with a slope of at most 1.13 and adds 2e-6 of its argument, and the result is rounded once to its type, u = 2^-24,
2^-11, 2^-8 of it (plus half the smallest subnormal of f16).  Where the gradient in front of an activation is rounded to 16 bits before
the products, that is u of every term."""
import math

import pytest
import torch

from paper_2402_07710_amd import binding as sc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
ACT_SLOPE, ACT_ERROR = 1.13, 2e-6


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, dtype=torch.float64) * scale).to(dtype)


def spread(t, pad, shift=0, fill=7.0):
    """`t` on the device as a slice of rows that are `pad` elements wider, from element `shift` on; and the whole."""
    whole = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=t.dtype, device=DEV)
    view = whole[:, shift:shift + t.shape[1]]
    view.copy_(t)
    return view, whole


def untouched(whole, view_cols, shift=0, fill=7.0):
    mask = torch.ones(whole.shape[1], dtype=torch.bool)
    mask[shift:shift + view_cols] = False
    return bool((whole.cpu()[:, mask] == fill).all())


def close(got, want, bound, what=""):
    got = got.double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    err = (got - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float(err[bad].max()):.3e} allowed {float((bound + 0 * err)[bad].min()):.3e}"


def act64(v, act):
    return {"none": lambda t: t, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[act](v)


def slope64(v, act):
    at = v.clone().requires_grad_(True)
    return torch.autograd.grad(act64(at, act).sum(), at)[0]


def forward_bound(want, pre, magnitude, K, act, dtype):
    bound = (K + 8) * 2.0 ** -23 * magnitude
    if act != "none":
        bound = ACT_SLOPE * bound + ACT_ERROR * pre.abs()
    return bound + UNIT[dtype] * (want.abs() + bound) + TINY[dtype]


SHAPES = [(1, 1, 1), (1, 1024, 96), (2, 7, 5), (33, 64, 64), (65, 32, 32), (127, 129, 31), (128, 64, 128), (129, 200, 136), (300, 72, 264),
          (1000, 64, 256), (70, 513, 24), (40, 1, 300), (513, 300, 1)]


# ---- linear ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,c_in,c_out", SHAPES)
def test_linear_forward(rows, c_in, c_out, dtype):
    dt = DT[dtype]
    g = gen(rows * 31 + c_in * 7 + c_out)
    x, w = normal(g, rows, c_in, dtype=dt), normal(g, c_in, c_out, dtype=dt, scale=1 / math.sqrt(c_in))
    b, r = normal(g, c_out, dtype=dt), normal(g, rows, c_out, dtype=dt)
    for act, bias, residual, save, pad, shift, wide in (("none", False, False, False, 0, 0, False), ("relu", True, False, True, 8, 0, False),
                                                        ("gelu", True, True, True, 5, 1, False), ("silu", False, True, False, 3, 0, True)):
        print(f"linear {rows} {c_in} {c_out} {dtype} {act} pad {pad} shift {shift}", flush=True)
        out_dt = torch.float32 if wide else dt
        pre = x.double() @ w.double() + (b.double() if bias else 0.0)
        res = r.to(out_dt)
        want = act64(pre, act) + (res.double() if residual else 0.0)
        size = x.double().abs() @ w.double().abs() + (b.double().abs() if bias else 0.0)
        d_x, _ = spread(x, pad, shift)
        d_out, out_whole = spread(torch.zeros(rows, c_out, dtype=out_dt), pad, shift)
        d_res = spread(res, pad, shift)[0] if residual else None
        d_pre = spread(torch.zeros(rows, c_out, dtype=out_dt), pad, shift)[0] if save else None
        sc.sc_linear_fwd(d_x, w.to(DEV), d_out, bias=b.to(DEV) if bias else None, act=act, residual=d_res, pre=d_pre)
        total = size + (res.double().abs() if residual else 0.0)
        close(d_out, want, forward_bound(want, pre, total, c_in, act, out_dt), "out")
        if save:
            close(d_pre, pre, forward_bound(pre, pre, size, c_in, "none", out_dt), "pre")
        assert untouched(out_whole, c_out, shift)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,c_in,c_out", SHAPES + [(5000, 40, 72), (9000, 128, 64), (2100, 65, 130)])
def test_linear_backward(rows, c_in, c_out, dtype):
    dt = DT[dtype]
    g = gen(rows * 17 + c_in * 3 + c_out)
    x, w = normal(g, rows, c_in, dtype=dt), normal(g, c_in, c_out, dtype=dt, scale=1 / math.sqrt(c_in))
    grad, pre = normal(g, rows, c_out, dtype=dt, scale=1 / 16), normal(g, rows, c_out, dtype=dt)
    ws = torch.empty(max(16, sc.sc_linear_workspace_bytes(rows, c_in, c_out, dt)), dtype=torch.uint8, device=DEV)
    for act, pad, shift, parts in (("none", 0, 0, "xwb"), ("gelu", 8, 0, "xwb"), ("silu", 5, 1, "xw"), ("relu", 0, 0, "b"), ("gelu", 0, 0, "x"), ("none", 3, 0, "wb")):
        print(f"linear bwd {rows} {c_in} {c_out} {dtype} {act} pad {pad} {parts}", flush=True)
        d = grad.double() * slope64(pre.double(), act)
        # error of one element in front of the products: its slope's, and one rounding to 16 bits
        d_err = torch.zeros_like(d) if act == "none" else 2 * ACT_ERROR * grad.double().abs() * (1 + pre.double().abs()) + UNIT[dt] * d.abs() + TINY[dt]
        gx = spread(torch.zeros(rows, c_in, dtype=dt), pad, shift)
        gw, gb = torch.full((c_in, c_out), 7.0, dtype=dt, device=DEV), torch.full((c_out,), 7.0, dtype=dt, device=DEV)
        sc.sc_linear_bwd(spread(grad, pad, shift)[0], spread(x, pad, shift)[0], w.to(DEV), grad_x=gx[0] if "x" in parts else None,
                         grad_weight=gw if "w" in parts else None, grad_bias=gb if "b" in parts else None,
                         pre=spread(pre, pad, shift)[0] if act != "none" else None, act=act, workspace=ws)

        def bound(want, size, err, K):
            off = (K + 8) * 2.0 ** -23 * size + err
            return off + UNIT[dt] * (want.abs() + off) + TINY[dt]
        if "x" in parts:
            wt = w.double().t()
            close(gx[0], d @ wt, bound(d @ wt, d.abs() @ wt.abs(), d_err @ wt.abs(), c_out), "dx")
            assert untouched(gx[1], c_in, shift)
        if "w" in parts:
            xt = x.double().t()
            close(gw, xt @ d, bound(xt @ d, xt.abs() @ d.abs(), xt.abs() @ d_err, rows), "dw")
        if "b" in parts:
            close(gb, d.sum(0), bound(d.sum(0), d.abs().sum(0), d_err.sum(0), rows), "db")


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_linear_gradient_against_differences(act):
    """The kernels' gradient in f32 along random directions, against central differences of the definition in 64 bits."""
    g = gen(5)
    rows, c_in, c_out, h = 37, 24, 19, 1e-5
    x, w, b = (normal(g, *s, dtype=torch.float32).double() for s in ((rows, c_in), (c_in, c_out), (c_out,)))
    c = normal(g, rows, c_out, dtype=torch.float32).double()
    pre = (x @ w + b).float()
    gx, gw, gb = torch.empty(rows, c_in, device=DEV), torch.empty(c_in, c_out, device=DEV), torch.empty(c_out, device=DEV)
    ws = torch.empty(sc.sc_linear_workspace_bytes(rows, c_in, c_out, torch.float32), dtype=torch.uint8, device=DEV)
    sc.sc_linear_bwd(c.float().to(DEV), x.float().to(DEV), w.float().to(DEV), gx, gw, gb, pre=pre.to(DEV), act=act, workspace=ws)
    for name, grad, at in (("x", gx, 0), ("w", gw, 1), ("b", gb, 2)):
        d = [torch.zeros_like(t) for t in (x, w, b)]
        d[at] = normal(g, *d[at].shape, dtype=torch.float64)
        f = [float((act64((x + s * d[0]) @ (w + s * d[1]) + b + s * d[2], act) * c).sum()) for s in (h, -h)]
        want, got = (f[0] - f[1]) / (2 * h), float((grad.double().cpu() * d[at]).sum())
        # f32 gradient: 1e-5 of the sum of magnitudes covers its sums and slopes; a kink of relu within h of one of 703 values moves one term
        scale = float((grad.double().cpu().abs() * d[at].abs()).sum())
        assert abs(want - got) <= 1e-5 * scale, (act, name, want, got, scale)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_linear_no_rows(dtype):
    dt = DT[dtype]
    w, ws = torch.ones(16, 24, dtype=dt, device=DEV), torch.empty(16, dtype=torch.uint8, device=DEV)
    sc.sc_linear_fwd(torch.empty(0, 16, dtype=dt, device=DEV), w, torch.empty(0, 24, dtype=dt, device=DEV))
    gw, gb = torch.full_like(w, 3.0), torch.full((24,), 3.0, dtype=dt, device=DEV)
    sc.sc_linear_bwd(torch.empty(0, 24, dtype=dt, device=DEV), torch.empty(0, 16, dtype=dt, device=DEV), w, torch.empty(0, 16, dtype=dt, device=DEV),
                     gw, gb, workspace=ws)
    assert not gw.any() and not gb.any()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_what_is_not_finite_stays_in_its_row(dtype):
    dt = DT[dtype]
    g = gen(3)
    for rows, c_in, c_out in ((20, 40, 64), (300, 72, 136), (300, 71, 33)):
        x, w = normal(g, rows, c_in, dtype=dt), normal(g, c_in, c_out, dtype=dt)
        x[3, c_in - 1], x[rows - 1, 0] = math.inf, math.nan
        out = torch.empty(rows, c_out, dtype=dt, device=DEV)
        sc.sc_linear_fwd(x.to(DEV), w.to(DEV), out)
        finite = torch.isfinite(out.float()).cpu()
        assert not finite[3].any() and not finite[rows - 1].any()
        finite[3] = finite[rows - 1] = True
        assert finite.all()
        grad = normal(g, rows, c_out, dtype=dt)
        gx = torch.empty(rows, c_in, dtype=dt, device=DEV)
        grad[5] = math.nan
        sc.sc_linear_bwd(grad.to(DEV), x.to(DEV), w.to(DEV), grad_x=gx, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
        finite = torch.isfinite(gx.float()).cpu()
        assert not finite[5].any()
        finite[5] = True
        assert finite.all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_activations_at_their_ends(dtype):
    """One channel, weight one: the activation of given values, the infinities and NaN among them, and its slope."""
    dt = DT[dtype]
    v = torch.tensor([-math.inf, -3.0e4, -100.0, -30.0, -13.0, -6.0, -1.0, -1e-3, -0.0, 0.0, 1e-3, 1.0, 6.0, 13.0, 100.0, 3.0e4, math.inf], dtype=dt)
    one = torch.ones(1, 1, dtype=dt, device=DEV)
    for act, ends in (("relu", (0.0, 1.0)), ("gelu", (0.0, 1.0)), ("silu", (0.0, 1.0))):
        out, gx = torch.empty(len(v), 1, dtype=dt, device=DEV), torch.empty(len(v), 1, dtype=dt, device=DEV)
        sc.sc_linear_fwd(v[:, None].to(DEV), one, out, act=act)
        finite = v[1:-1].double()
        want = act64(finite, act)
        close(out[1:-1, 0], want, forward_bound(want, finite, finite.abs(), 1, act, dt), act)
        assert float(out[0]) == 0.0 and float(out[-1]) == math.inf
        ws = torch.empty(sc.sc_linear_workspace_bytes(len(v), 1, 1, dt), dtype=torch.uint8, device=DEV)
        sc.sc_linear_bwd(torch.ones(len(v), 1, dtype=dt, device=DEV), v[:, None].to(DEV), one, grad_x=gx, pre=v[:, None].to(DEV), act=act, workspace=ws)
        want = slope64(finite, act)
        close(gx[1:-1, 0], want, 2 * ACT_ERROR * (1 + finite.abs()).clamp(max=30.0) + 2 * UNIT[dt] * (want.abs() + 1e-5) + TINY[dt], act + " slope")
        assert float(gx[0]) == ends[0] and float(gx[-1]) == ends[1]
        nan = torch.full((1, 1), math.nan, dtype=dt, device=DEV)
        sc.sc_linear_fwd(nan, one, out[:1], act=act)
        assert math.isnan(float(out[0]))


# rows and channels that take every tile of row_tile and weight_tile in sc_rules.h, in whole chunks of 16 bytes and not
LARGE_SHAPES = [(1900, 1032, 1000), (7000, 131, 521), (8200, 131, 521), (70000, 48, 136), (70001, 136, 45), (140000, 24, 72), (140000, 96, 30), (9000, 600, 1030), (66000, 520, 264),
                (34000, 530, 520), (33000, 513, 777)]


def there(got, want, bound, what):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), bad.numel())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,c_in,c_out", LARGE_SHAPES)
def test_linear_large(rows, c_in, c_out, dtype):
    """Every element of large layers and of their gradients, against products in 64 bits on the device."""
    dt = DT[dtype]
    torch.manual_seed(rows + c_in)
    x, w = torch.randn(rows, c_in, device=DEV).to(dt), (torch.randn(c_in, c_out, device=DEV) / math.sqrt(c_in)).to(dt)
    b, r, grad = torch.randn(c_out, device=DEV).to(dt), torch.randn(rows, c_out, device=DEV).to(dt), (torch.randn(rows, c_out, device=DEV) / 16).to(dt)
    plain, size = x.double() @ w.double(), x.double().abs() @ w.double().abs()
    for act, extra in (("none", False), ("gelu", True)):
        print(f"linear large {rows} {c_in} {c_out} {dtype} {act}", flush=True)
        pre = plain + b.double() if extra else plain
        total = size + b.double().abs() if extra else size
        out, whole = spread(torch.zeros(rows, c_out, dtype=dt), 8)
        kept = torch.zeros(rows, c_out, dtype=dt, device=DEV)
        sc.sc_linear_fwd(x, w, out, bias=b if extra else None, act=act, residual=r if extra else None, pre=kept if extra else None)
        want = act64(pre, act) + (r.double() if extra else 0.0)
        there(out, want, forward_bound(want, pre, total + (r.double().abs() if extra else 0.0), c_in, act, dt), "out")
        assert bool((whole[:, c_out:] == 7.0).all())
        if extra:
            there(kept, pre, forward_bound(pre, pre, total, c_in, "none", dt), "pre")
        d = grad.double() * slope64(kept.double(), act)
        d_err = torch.zeros_like(d) if act == "none" else 2 * ACT_ERROR * grad.double().abs() * (1 + kept.double().abs()) + UNIT[dt] * d.abs() + TINY[dt]
        gx, gx_whole = spread(torch.zeros(rows, c_in, dtype=dt), 5)
        gw, gb = torch.full((c_in, c_out), 7.0, dtype=dt, device=DEV), torch.full((c_out,), 7.0, dtype=dt, device=DEV)
        ws = torch.empty(sc.sc_linear_workspace_bytes(rows, c_in, c_out, dt), dtype=torch.uint8, device=DEV)
        sc.sc_linear_bwd(grad, x, w, gx, gw, gb, pre=kept if extra else None, act=act, workspace=ws)

        def bound(want, size, err, K):
            off = (K + 8) * 2.0 ** -23 * size + err
            return off + UNIT[dt] * (want.abs() + off) + TINY[dt]
        wt, xt = w.double().t(), x.double().t()
        there(gx, d @ wt, bound(d @ wt, d.abs() @ wt.abs(), d_err @ wt.abs(), c_out), "dx")
        assert bool((gx_whole[:, c_in:] == 7.0).all())
        there(gw, xt @ d, bound(xt @ d, xt.abs() @ d.abs(), xt.abs() @ d_err, rows), "dw")
        there(gb, d.sum(0), bound(d.sum(0), d.abs().sum(0), d_err.sum(0), rows), "db")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("c_in,c_out", [(520, 528), (521, 1030)])
def test_grouped_large(c_in, c_out, dtype):
    """Groups that take the large tiles, their last rows among few and many; rows from a list."""
    dt, starts = DT[dtype], [0, 4097, 4098, 9300, 12700]
    torch.manual_seed(c_in)
    n, table = starts[-1], 5000
    x, w = torch.randn(table, c_in, device=DEV).to(dt), (torch.randn(4, c_in, c_out, device=DEV) / math.sqrt(c_in)).to(dt)
    rows, grad = torch.randint(0, table, (n,), device=DEV, dtype=torch.int32), (torch.randn(n, c_out, device=DEV) / 16).to(dt)
    d_starts = torch.tensor(starts, dtype=torch.int32, device=DEV)
    out, gx, gw = torch.zeros(n, c_out, dtype=dt, device=DEV), torch.zeros(n, c_in, dtype=dt, device=DEV), torch.full_like(w, 7.0)
    sc.sc_grouped_fwd(x, w, d_starts, out, rows=rows)
    ws = torch.empty(sc.sc_grouped_workspace_bytes(n, 4, c_in, c_out, dt), dtype=torch.uint8, device=DEV)
    sc.sc_grouped_bwd(grad, x, w, d_starts, gx, gw, rows=rows, workspace=ws)
    for k in range(4):
        m = slice(starts[k], starts[k + 1])
        xs, wk, d = x[rows[m].long()].double(), w[k].double(), grad[m].double()
        for got, a, c, K in ((out[m], xs, wk, c_in), (gx[m], d, wk.t(), c_out), (gw[k], xs.t(), d, starts[k + 1] - starts[k])):
            want, off = a @ c, (K + 8) * 2.0 ** -23 * (a.abs() @ c.abs())
            there(got, want, off + UNIT[dt] * (want.abs() + off) + TINY[dt], (k, K))


# ---- grouped ------------------------------------------------------------------------------------------------
GROUPS = {
    "one": [0, 200],
    "ragged": [0, 130, 131, 131, 260, 261, 517],
    "ends": [3, 40, 40, 90],                                   # entries of no group at both ends
    "empty": [0, 0, 0, 0],
    "many": [0] + [i * 3 // 2 for i in range(1, 151)],         # 150 groups of one or two
    "many uneven": [0] * 70 + [1, 900, 900, 1400] + [1400] * 60 + [1401],
}


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kind", list(GROUPS))
@pytest.mark.parametrize("c_in,c_out,listed", [(64, 64, True), (40, 24, False), (136, 160, True), (33, 7, True)])
def test_grouped(kind, c_in, c_out, listed, dtype):
    dt = DT[dtype]
    starts = GROUPS[kind]
    groups, n = len(starts) - 1, starts[-1] + (5 if kind == "ends" else 0)
    g = gen(len(kind) * 100 + c_in)
    x_rows = 50 if listed else n
    x, w = normal(g, x_rows, c_in, dtype=dt), normal(g, groups, c_in, c_out, dtype=dt, scale=1 / math.sqrt(c_in))
    b, grad, pre_in = normal(g, groups, c_out, dtype=dt), normal(g, n, c_out, dtype=dt, scale=1 / 16), normal(g, n, c_out, dtype=dt)
    rows = torch.randint(0, x_rows, (n,), generator=g).to(torch.int32) if listed else None
    if listed and n > 10:                                      # entries without a row count as zeros
        rows[4], rows[7], rows[9] = -1, x_rows, -(1 << 31)
    owner = torch.full((n,), -1)
    for k in range(groups):
        owner[starts[k]:starts[k + 1]] = k
    xs = x.double() if not listed else torch.cat([x.double(), torch.zeros(1, c_in, dtype=torch.float64)])[
        torch.where((rows >= 0) & (rows < x_rows), rows, x_rows).long()]
    member = owner >= 0
    wo, bo = w.double()[owner.clamp(min=0)], b.double()[owner.clamp(min=0)]
    d_starts = torch.tensor(starts, dtype=torch.int32, device=DEV)
    d_rows = rows.to(DEV) if listed else None

    def rowwise(v, m):                                         # v[p] . m[p], in order of the groups to spare memory
        return torch.bmm(v[:, None], m)[:, 0] if n else v.new_zeros(0, m.shape[2])
    for act, bias, pad in (("none", False, 0), ("gelu", True, 3), ("silu", True, 8)):
        print(f"grouped {kind} {c_in} {c_out} {dtype} {act}", flush=True)
        pre = rowwise(xs, wo) + (bo if bias else 0.0)
        want, size = act64(pre, act), rowwise(xs.abs(), wo.abs()) + (bo.abs() if bias else 0.0)
        out, whole = spread(torch.full((n, c_out), 7.0, dtype=dt), pad)
        kept = torch.full((n, c_out), 7.0, dtype=dt, device=DEV)
        sc.sc_grouped_fwd(spread(x, pad)[0], w.to(DEV), d_starts, out, rows=d_rows, bias=b.to(DEV) if bias else None, act=act, pre=kept)
        close(out[member.to(DEV)], want[member], forward_bound(want, pre, size, c_in, act, dt)[member], "out")
        close(kept[member.to(DEV)], pre[member], forward_bound(pre, pre, size, c_in, "none", dt)[member], "pre")
        assert bool((out.cpu()[~member] == 7.0).all()) and bool((kept.cpu()[~member] == 7.0).all()) and untouched(whole, c_out)

        d = grad.double() * slope64(pre_in.double(), act)
        d_err = torch.zeros_like(d) if act == "none" else 2 * ACT_ERROR * grad.double().abs() * (1 + pre_in.double().abs()) + UNIT[dt] * d.abs() + TINY[dt]
        gx = torch.full((n, c_in), 7.0, dtype=dt, device=DEV)
        gw, gb = torch.full_like(w, 7.0).to(DEV), torch.full_like(b, 7.0).to(DEV)
        ws = torch.empty(max(16, sc.sc_grouped_workspace_bytes(n, groups, c_in, c_out, dt)), dtype=torch.uint8, device=DEV)
        sc.sc_grouped_bwd(spread(grad, pad)[0], spread(x, pad)[0], w.to(DEV), d_starts, gx, gw, gb, rows=d_rows,
                          pre=pre_in.to(DEV) if act != "none" else None, act=act, workspace=ws)

        def bound(want, size, err, K):
            off = (K + 8) * 2.0 ** -23 * size + err
            return off + UNIT[dt] * (want.abs() + off) + TINY[dt]
        wt = wo.transpose(1, 2).contiguous()
        want_x = rowwise(d, wt)
        close(gx[member.to(DEV)], want_x[member], bound(want_x, rowwise(d.abs(), wt.abs()), rowwise(d_err, wt.abs()), c_out)[member], "dx")
        assert bool((gx.cpu()[~member] == 7.0).all())
        for k in range(groups):
            m = slice(starts[k], starts[k + 1])
            xt, dk, ek = xs[m].t(), d[m], d_err[m]
            count = starts[k + 1] - starts[k]
            close(gw[k], xt @ dk, bound(xt @ dk, xt.abs() @ dk.abs(), xt.abs() @ ek, count), f"dw[{k}]")
            close(gb[k], dk.sum(0), bound(dk.sum(0), dk.abs().sum(0), ek.sum(0), count), f"db[{k}]")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c_in,c_out", [(8, 8), (256, 260)])
def test_weight_gradients_of_many_groups_in_parts(c_in, c_out, dtype):
    """140 groups, of which every third is summed in several parts, with whole and empty ones between them: sums by few and by many values a workgroup."""
    dt, g = DT[dtype], gen(c_in)
    sizes = [(400 + k, 1, 128 - k % 3, 0, 300, 64)[k % 6] for k in range(140)]
    starts = [0]
    for e in sizes:
        starts.append(starts[-1] + e)
    n = starts[-1]
    x, grad = normal(g, n, c_in, dtype=dt), normal(g, n, c_out, dtype=dt, scale=1 / 16)
    gw, gb = torch.full((140, c_in, c_out), 7.0, dtype=dt, device=DEV), torch.full((140, c_out), 7.0, dtype=dt, device=DEV)
    ws = torch.empty(sc.sc_grouped_workspace_bytes(n, 140, c_in, c_out, dt), dtype=torch.uint8, device=DEV)
    sc.sc_grouped_bwd(grad.to(DEV), x.to(DEV), None, torch.tensor(starts, dtype=torch.int32, device=DEV), grad_weight=gw, grad_bias=gb, workspace=ws)
    for k, count in enumerate(sizes):
        xt, d = x[starts[k]:starts[k + 1]].double().t(), grad[starts[k]:starts[k + 1]].double()
        for got, want, size in ((gw[k], xt @ d, xt.abs() @ d.abs()), (gb[k], d.sum(0), d.abs().sum(0))):
            off = (count + 8) * 2.0 ** -23 * size
            close(got, want, off + UNIT[dt] * (want.abs() + off) + TINY[dt], f"group {k}")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_weight_gradient_of_a_convolution(dtype):
    """From the rulebook that a kernel map exports: both sides gathered, 27 groups, against the sum over pairs."""
    from paper_2402_07710_amd import synth
    dt = DT[dtype]
    coords = torch.from_numpy(synth.lidar_scene(1)[:6000]).to(DEV)
    n, c_in, c_out, g = len(coords), 32, 48, gen(9)
    buf = sc.LayerBuffers(n, 3, 1, "subm", c_in, c_out, "f32")
    buf.hash_build(coords)
    buf.kmap_build(coords)
    pairs_in, pairs_out, starts = buf.export()
    x, grad = normal(g, n, c_in, dtype=dt), normal(g, n, c_out, dtype=dt, scale=1 / 16)
    gw = torch.empty(27, c_in, c_out, dtype=dt, device=DEV)
    ws = torch.empty(sc.sc_grouped_workspace_bytes(len(pairs_in), 27, c_in, c_out, dt), dtype=torch.uint8, device=DEV)
    sc.sc_grouped_bwd(grad.to(DEV), x.to(DEV), None, starts, grad_weight=gw, rows=pairs_in, grad_rows=pairs_out, workspace=ws)
    first = gw.clone()
    sc.sc_grouped_bwd(grad.to(DEV), x.to(DEV), None, starts, grad_weight=gw, rows=pairs_in, grad_rows=pairs_out, workspace=ws)
    assert torch.equal(first, gw)
    pin, pout, st = pairs_in.cpu().long(), pairs_out.cpu().long(), starts.cpu()
    for k in range(27):
        m = slice(int(st[k]), int(st[k + 1]))
        xt, d = x.double()[pin[m]].t(), grad.double()[pout[m]]
        off = (d.shape[0] + 8) * 2.0 ** -23 * (xt.abs() @ d.abs())
        close(gw[k], xt @ d, off + UNIT[dt] * ((xt @ d).abs() + off) + TINY[dt], f"offset {k}")


def test_starts_that_do_not_ascend_stay_inside():
    """Wrong starts give wrong rows, but nothing outside the arrays is written."""
    n, c = 2000, 32
    x, w = torch.ones(n, c, device=DEV, dtype=torch.float16), torch.ones(5, c, c, device=DEV, dtype=torch.float16)
    out = torch.full((n + 64, c), 7.0, device=DEV, dtype=torch.float16)
    size = sc.sc_grouped_workspace_bytes(n, 5, c, c, torch.float16)
    ws = torch.full((size + 4096,), 77, dtype=torch.uint8, device=DEV)
    gw = torch.zeros(6, c, c, device=DEV, dtype=torch.float16)
    for starts in ([0, 2000, 0, 2000, 0, 2000], [-5, 3000, 1 << 30, -(1 << 31), 7, 100000], [2000, 1500, 1000, 500, 0, 0]):
        s = torch.tensor(starts, dtype=torch.int32, device=DEV)
        sc.sc_grouped_fwd(x, w, s, out[:n])
        sc.sc_grouped_bwd(x, x, w, s, grad_weight=gw[:5], workspace=ws[:size])
        torch.cuda.synchronize()
        assert bool((out[n:] == 7.0).all()) and bool((ws[size:] == 77).all()) and not gw[5].any()


# ---- norm and rotation ------------------------------------------------------------------------------------------
def rope64(v, pos, pairs, base, pairing, gain, eps):
    D = v.shape[-1]
    half = D // 2
    if gain is not None:
        v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps) * gain
    angle = torch.zeros(v.shape[0], 1, half, dtype=torch.float64)
    j = 0
    for a, m in enumerate(pairs):
        for i in range(m):
            angle[:, 0, j] = pos[:, a].double() * base ** (-i / m)
            j += 1
    lo = torch.arange(half) if pairing == "halves" else 2 * torch.arange(half)
    hi = lo + half if pairing == "halves" else lo + 1
    a, b = v[..., lo], v[..., hi]
    out = torch.zeros_like(v)
    out[..., lo], out[..., hi] = a * torch.cos(angle) - b * torch.sin(angle), a * torch.sin(angle) + b * torch.cos(angle)
    return out


# sine and cosine are off by 2e-6 at most (their argument's reduction included), statistics by (D + 8) 2^-23 of themselves, a handful of
# products by 2^-24 each: all relative to the pair's magnitude, for which the head's largest stands
def rope_bound(want, D, dt, terms=1.0):
    off = (2e-6 + (D + 16) * 2.0 ** -23) * terms * want.abs().amax(-1, keepdim=True) * 1.5
    return off + UNIT[dt] * (want.abs() + off) + TINY[dt]


ROPE = [  # D, pairs, q heads, k heads, rows
    (2, (1,), 1, 1, 1), (6, (1, 1, 1), 2, 1, 5), (16, (3, 3, 2), 4, 4, 33), (32, (6, 5, 5), 8, 2, 257), (44, (8, 7, 7), 3, 1, 65), (64, (10, 11, 11), 5, 0, 130),
    (64, (32,), 8, 8, 70), (96, (16, 16, 16), 7, 3, 40), (128, (20, 22, 22), 16, 4, 1), (130, (20, 22, 20), 2, 2, 9), (256, (42, 43), 4, 1, 19),
    (10, (2, 2, 1), 3, 2, 11), (18, (3, 3, 3), 5, 1, 21), (36, (18,), 8, 4, 50), (50, (9, 8, 8), 4, 2, 30),
    (1024, (128, 128, 128, 128), 1, 2, 7), (64, (10, 10, 11), 8, 2, 3000),
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("pairing", ["halves", "adjacent"])
@pytest.mark.parametrize("D,pairs,hq,hk,rows", ROPE)
def test_rope(D, pairs, hq, hk, rows, pairing, dtype):
    dt = DT[dtype]
    g = gen(D * 13 + rows)
    eps, base = 1e-6, 10000.0
    coords = torch.randint(0, 65535, (rows, 1 + len(pairs)), generator=g).to(torch.int32)
    pos = coords.to(DEV)[:, 1:]
    table = sc.sc_rope_table(D, pairs, base)
    for norm, layout in ((True, "projection"), (True, "heads first"), (False, "odd")):
        print(f"rope {D} {hq} {hk} {rows} {pairing} {dtype} norm {norm} {layout}", flush=True)
        q, k = normal(g, rows, hq, D, dtype=dt), normal(g, rows, hk, D, dtype=dt)
        if rows > 4:
            q[2] = 0.0                                         # a row of nothing: its norm is the epsilon's
        gq, gk = (1 + normal(g, D, dtype=torch.float64, scale=0.2)).to(dt), (1 + normal(g, D, dtype=torch.float64, scale=0.2)).to(dt)
        cq, ck = normal(g, rows, hq, D, dtype=dt), normal(g, rows, hk, D, dtype=dt)

        def place(t):
            if layout == "projection":
                wide = torch.full((rows, t.shape[1] * D + 24), 7.0, dtype=dt, device=DEV)
                view = wide[:, 8:8 + t.shape[1] * D].unflatten(1, (t.shape[1], D))
            elif layout == "heads first":
                view = torch.empty(t.shape[1], rows, D, dtype=dt, device=DEV).transpose(0, 1)
            else:
                view = torch.empty(rows, t.shape[1], D + 3, dtype=dt, device=DEV)[:, :, 1:1 + D]
            view.copy_(t)
            return view
        keys = hk > 0
        d_q, d_k = place(q), place(k) if keys else None
        o_q, o_k = place(torch.zeros_like(q)), place(torch.zeros_like(k)) if keys else None
        gains = dict(gain_q=gq.to(DEV), gain_k=gk.to(DEV) if keys else None) if norm else {}
        sc.sc_qk_rope_fwd(d_q, d_k, pos, table, o_q, o_k, eps=eps, pairing=pairing, **gains)
        ws = torch.empty(max(16, sc.sc_qk_rope_workspace_bytes(rows, hq, hk, D)), dtype=torch.uint8, device=DEV)
        grads = dict(grad_gain_q=torch.full((D,), 7.0, dtype=dt, device=DEV),
                     grad_gain_k=torch.full((D,), 7.0, dtype=dt, device=DEV) if keys else None) if norm else {}
        b_q, b_k = place(torch.zeros_like(q)), place(torch.zeros_like(k)) if keys else None
        sc.sc_qk_rope_bwd(place(cq), place(ck) if keys else None, d_q, d_k, pos, table, b_q, b_k, eps=eps, pairing=pairing, workspace=ws, **gains, **grads)
        for name, v, c, gain, out, back, dgain in (("q", q, cq, gq, o_q, b_q, grads.get("grad_gain_q")), ("k", k, ck, gk, o_k, b_k, grads.get("grad_gain_k"))):
            if name == "k" and not keys:
                continue
            v64 = v.double().requires_grad_(True)
            g64 = gain.double().requires_grad_(True)
            want = rope64(v64, coords[:, 1:], pairs, base, pairing, g64 if norm else None, eps)
            want.backward(c.double())
            close(out, want.detach(), rope_bound(want.detach(), D, dt), name)
            # every term of the gradient is at most the turned gradient times the gain, over the row's root mean square
            turned = rope64(c.double(), -coords[:, 1:], pairs, base, pairing, None, eps)
            if norm:
                rms = torch.sqrt((v.double() ** 2).mean(-1, keepdim=True) + eps)
                unit = v.double() / rms
                u = turned * gain.double()
                size = (u.abs().amax(-1, keepdim=True) + unit.abs().amax(-1, keepdim=True) * (u * unit).abs().mean(-1, keepdim=True)) / rms
            else:
                size = turned.abs().amax(-1, keepdim=True)
            off = 3 * (2e-6 + (D + 16) * 2.0 ** -23) * size
            close(back, v64.grad, off + UNIT[dt] * (v64.grad.abs() + off) + TINY[dt], "d" + name)
            if norm:
                terms = turned.abs().amax(-1, keepdim=True).expand_as(turned) * unit.abs()
                off = (4e-6 + (D + 16) * 2.0 ** -23 + (v.shape[0] * v.shape[1] + 8) * 2.0 ** -23) * terms.sum((0, 1))
                close(dgain, g64.grad, off + UNIT[dt] * (g64.grad.abs() + off) + TINY[dt], "dgain " + name)
        # in place
        sc.sc_qk_rope_fwd(d_q, d_k, pos, table, d_q, d_k, eps=eps, pairing=pairing, **gains)
        assert torch.equal(d_q, o_q) and (not keys or torch.equal(d_k, o_k))


def test_rope_gradient_against_differences():
    g = gen(21)
    D, pairs, rows, heads, h = 24, (4, 4, 3), 6, 3, 1e-6
    q, c = normal(g, rows, heads, D, dtype=torch.float32).double(), normal(g, rows, heads, D, dtype=torch.float32).double()
    gain = (1 + 0.3 * normal(g, D, dtype=torch.float32)).double()
    pos = torch.randint(0, 2000, (rows, 3), generator=g).to(torch.int32)
    table = sc.sc_rope_table(D, pairs, 100.0)
    dq, dg = torch.empty(rows, heads, D, device=DEV), torch.empty(D, device=DEV)
    ws = torch.empty(sc.sc_qk_rope_workspace_bytes(rows, heads, 0, D), dtype=torch.uint8, device=DEV)
    sc.sc_qk_rope_bwd(c.float().to(DEV), None, q.float().to(DEV), None, pos.to(DEV), table, dq, None, gain_q=gain.float().to(DEV), grad_gain_q=dg,
                      eps=1e-5, pairing="adjacent", workspace=ws)
    for name, grad, at in (("q", dq, 0), ("gain", dg, 1)):
        d = [torch.zeros_like(q), torch.zeros_like(gain)]
        d[at] = normal(g, *d[at].shape, dtype=torch.float64)
        f = [float((rope64(q + s * d[0], pos, pairs, 100.0, "adjacent", gain + s * d[1], 1e-5) * c).sum()) for s in (h, -h)]
        want, got = (f[0] - f[1]) / (2 * h), float((grad.double().cpu() * d[at]).sum())
        assert abs(want - got) <= 2e-5 * float((grad.double().cpu().abs() * d[at].abs()).sum()), (name, want, got)


# ---- how they are called --------------------------------------------------------------------------------------
def test_other_streams_and_graphs():
    """On a stream that is not the current one, and replayed from a graph between eager work: the same bits every time."""
    g = gen(2)
    dt = torch.bfloat16
    rows, c = 3000, 64
    x, w = normal(g, rows, c, dtype=dt).to(DEV), normal(g, c, c, dtype=dt, scale=0.1).to(DEV)
    grad = normal(g, rows, c, dtype=dt).to(DEV)
    pos = torch.randint(0, 1000, (rows, 3), generator=g).to(torch.int32).to(DEV)
    table, gain = sc.sc_rope_table(32, (5, 5, 6)), torch.ones(32, dtype=dt, device=DEV)
    y, pre, gx, gw, gb = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty(c, dtype=dt, device=DEV)
    q = torch.empty_like(x)
    dg = torch.empty_like(gain)
    starts = torch.tensor([0, 700, 700, rows], dtype=torch.int32, device=DEV)
    w3, gw3 = torch.stack([w, w, w]).contiguous(), torch.empty(3, c, c, dtype=dt, device=DEV)
    ws = torch.empty(sc.sc_grouped_workspace_bytes(rows, 3, c, c, dt) + sc.sc_qk_rope_workspace_bytes(rows, 2, 0, 32), dtype=torch.uint8, device=DEV)

    def step(stream=None):
        sc.sc_linear_fwd(x, w, y, act="gelu", pre=pre, stream=stream)
        sc.sc_qk_rope_fwd(y.unflatten(1, (2, 32)), None, pos, table, q.unflatten(1, (2, 32)), None, gain_q=gain, stream=stream)
        sc.sc_grouped_fwd(q, w3, starts, y, act="silu", stream=stream)
        sc.sc_qk_rope_bwd(grad.unflatten(1, (2, 32)), None, y.unflatten(1, (2, 32)), None, pos, table, gx.unflatten(1, (2, 32)), None, gain_q=gain,
                          grad_gain_q=dg, workspace=ws, stream=stream)
        sc.sc_grouped_bwd(grad, x, w3, starts, grad_weight=gw3, workspace=ws, stream=stream)
        sc.sc_linear_bwd(gx, x, w, grad_weight=gw, grad_bias=gb, grad_x=q, pre=pre, act="gelu", workspace=ws, stream=stream)
    outs = (y, pre, gx, gw, gb, q, dg, gw3)
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    assert all(torch.isfinite(t.float()).all() for t in want)
    side = torch.cuda.Stream()
    for t in outs:
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for replay in range(4):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), replay
        (x @ w).sum().item()                                   # eager work in between


def test_offsets_beyond_32_bits():
    """Rows whose bytes lie past 2^32, and entries that point there."""
    rows, c_in, c_out = (1 << 25) + 77, 80, 16
    x = torch.zeros(rows, c_in, dtype=torch.float16, device=DEV)      # 5 GB
    look = [0, 1, (1 << 32) // (2 * c_in) - 1, (1 << 32) // (2 * c_in), (1 << 32) // (2 * c_in) + 1, rows - 65, rows - 1]
    g = gen(8)
    some = normal(g, len(look), c_in, dtype=torch.float16)
    x[look] = some.to(DEV)
    w = normal(g, c_in, c_out, dtype=torch.float16)
    out = torch.empty(rows, c_out, dtype=torch.float16, device=DEV)
    sc.sc_linear_fwd(x, w.to(DEV), out)
    want = some.double() @ w.double()
    size = some.double().abs() @ w.double().abs()
    close(out[look], want, forward_bound(want, want, size, c_in, "none", torch.float16))
    assert int((out != 0).any(1).sum()) == len(look)
    del out
    few = torch.empty(len(look), c_out, dtype=torch.float16, device=DEV)
    sc.sc_grouped_fwd(x, torch.stack([w, w]).to(DEV), torch.tensor([0, 3, len(look)], dtype=torch.int32, device=DEV), few,
                      rows=torch.tensor(look, dtype=torch.int32, device=DEV))
    close(few, want, forward_bound(want, want, size, c_in, "none", torch.float16))
    grad = torch.zeros(rows, c_out, dtype=torch.float16, device=DEV)
    d = normal(g, len(look), c_out, dtype=torch.float16)
    grad[look] = d.to(DEV)
    gw = torch.empty(c_in, c_out, dtype=torch.float16, device=DEV)
    ws = torch.empty(sc.sc_linear_workspace_bytes(rows, c_in, c_out, torch.float16), dtype=torch.uint8, device=DEV)
    sc.sc_linear_bwd(grad, x, w.to(DEV), grad_weight=gw, workspace=ws)
    want, size = some.double().t() @ d.double(), some.double().abs().t() @ d.double().abs()
    off = 64 * 2.0 ** -23 * size                               # the other terms are zeros
    close(gw, want, off + UNIT[torch.float16] * (want.abs() + off) + TINY[torch.float16])

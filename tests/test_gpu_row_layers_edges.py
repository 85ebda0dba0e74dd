"""GPU tests of the row layers where sizes, lists or values come to an end: no rows, heads that fill no group of lanes, epsilon zero, gradients taken by a
list through an activation, tables with fewer rows than entries, the activation's tail, arguments that a call may leave out.  Against the definitions in 64 bits;
bounds as in test_gpu_row_layers.py unless a test derives its own."""
import ctypes
import math

import pytest
import torch

from paper_2402_07710_amd import binding as sc
from tests.test_gpu_row_layers import (ACT_ERROR, DEV, DT, TINY, UNIT, act64, close, forward_bound, gen, normal, rope64, slope64, spread)

pytestmark = pytest.mark.gpu
EVERY = pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])


def product_bound(want, size, err, K, dt):
    off = (K + 8) * 2.0 ** -23 * size + err
    return off + UNIT[dt] * (want.abs() + off) + TINY[dt]


# ---- norm and rotation ---------------------------------------------------------------------------------------
def check_rope_gradients(D, pairs, heads, rows, pairing, dt, eps, v, c, gain, pos, table, keys):
    """Gradients of `v` [rows, heads, D] (as queries, or as keys behind one head of queries) and of the gain."""
    back, dgain = torch.full((rows, heads, D), 7.0, dtype=dt, device=DEV), torch.full((D,), 7.0, dtype=dt, device=DEV)
    one, one_grad = (v[:, :1] + 1).to(DEV).contiguous(), c[:, :1].to(DEV).contiguous()
    dv, dc, dg = v.to(DEV), c.to(DEV), gain.to(DEV)
    ws = torch.empty(sc.sc_qk_rope_workspace_bytes(rows, 1 if keys else heads, heads if keys else 0, D), dtype=torch.uint8, device=DEV)
    if keys:
        sc.sc_qk_rope_bwd(one_grad, dc, one, dv, pos.to(DEV), table, torch.empty_like(one), back, gain_k=dg, grad_gain_k=dgain, eps=eps, pairing=pairing, workspace=ws)
    else:
        sc.sc_qk_rope_bwd(dc, None, dv, None, pos.to(DEV), table, back, None, gain_q=dg, grad_gain_q=dgain, eps=eps, pairing=pairing, workspace=ws)
    v64, g64 = v.double().requires_grad_(True), gain.double().requires_grad_(True)
    rope64(v64, pos, pairs, 10000.0, pairing, g64, eps).backward(c.double())
    turned = rope64(c.double(), -pos, pairs, 10000.0, pairing, None, eps)
    rms = torch.sqrt((v.double() ** 2).mean(-1, keepdim=True) + eps)
    unit, u = v.double() / rms, turned * gain.double()
    size = (u.abs().amax(-1, keepdim=True) + unit.abs().amax(-1, keepdim=True) * (u * unit).abs().mean(-1, keepdim=True)) / rms
    off = 3 * (2e-6 + (D + 16) * 2.0 ** -23) * size
    close(back, v64.grad, off + UNIT[dt] * (v64.grad.abs() + off) + TINY[dt], "dv")
    terms = turned.abs().amax(-1, keepdim=True).expand_as(turned) * unit.abs()
    off = (4e-6 + (D + 16) * 2.0 ** -23 + (rows * heads + 8) * 2.0 ** -23) * terms.sum((0, 1))
    close(dgain, g64.grad, off + UNIT[dt] * (g64.grad.abs() + off) + TINY[dt], "dgain")


@EVERY
@pytest.mark.parametrize("pairing", ["halves", "adjacent"])
@pytest.mark.parametrize("D,pairs", [(64, (10, 11, 11)), (36, (6, 6, 6)), (6, (1, 1, 1)), (24, (4, 4, 4))])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_rope_gradients_of_heads_that_fill_no_group(D, pairs, pairing, eps, dtype):
    """Heads in odd numbers, one among them, and rows that leave the last lanes without work, also with an epsilon of zero: what has no head adds nothing."""
    dt, table = DT[dtype], sc.sc_rope_table(D, pairs)
    for heads, rows in ((1, 1), (3, 5), (1, 333), (5, 130), (2, 77)):
        g = gen(D + 10 * heads + rows)
        v, c = normal(g, rows, heads, D, dtype=dt), normal(g, rows, heads, D, dtype=dt)
        gain = (1 + normal(g, D, dtype=torch.float64, scale=0.2)).to(dt)
        pos = torch.randint(0, 2000, (rows, 3), generator=g).to(torch.int32)
        for keys in (False, True):
            print(f"rope bwd {D} {heads} {rows} {pairing} {dtype} eps {eps} keys {keys}", flush=True)
            check_rope_gradients(D, pairs, heads, rows, pairing, dt, eps, v, c, gain, pos, table, keys)


@EVERY
def test_rope_of_no_rows(dtype):
    """Nothing to turn: outputs without elements, and gains whose gradients are zeros."""
    dt, D = DT[dtype], 32
    table, pos = sc.sc_rope_table(D, (5, 5, 6)), torch.empty(0, 3, dtype=torch.int32, device=DEV)

    def none(heads):
        return torch.empty(0, heads, D, dtype=dt, device=DEV)
    gain, dgq, dgk = torch.ones(D, dtype=dt, device=DEV), torch.full((D,), 7.0, dtype=dt, device=DEV), torch.full((D,), 7.0, dtype=dt, device=DEV)
    sc.sc_qk_rope_fwd(none(4), none(2), pos, table, none(4), none(2), gain_q=gain, gain_k=gain)
    sc.sc_qk_rope_fwd(none(4), None, pos, table, none(4), None)
    ws = torch.empty(16, dtype=torch.uint8, device=DEV)
    sc.sc_qk_rope_bwd(none(4), none(2), none(4), none(2), pos, table, none(4), none(2), gain_q=gain, gain_k=gain, grad_gain_q=dgq, grad_gain_k=dgk, workspace=ws)
    assert not dgq.any() and not dgk.any()
    dgq.fill_(7.0)
    sc.sc_qk_rope_bwd(none(4), None, none(4), None, pos, table, none(4), None, gain_q=gain, grad_gain_q=dgq, workspace=ws)
    assert not dgq.any()
    sc.sc_qk_rope_bwd(none(4), None, None, None, pos, table, none(4), None)


@EVERY
def test_no_rows_and_their_gradient_alone(dtype):
    """A gradient of rows that has no elements is asked for all the same: nothing is to be done."""
    dt = DT[dtype]
    w = torch.ones(16, 24, dtype=dt, device=DEV)
    x, grad = torch.empty(0, 16, dtype=dt, device=DEV), torch.empty(0, 24, dtype=dt, device=DEV)
    ws, starts = torch.empty(16, dtype=torch.uint8, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    for act in ("none", "gelu"):
        pre = grad if act != "none" else None
        sc.sc_linear_bwd(grad, x, w, grad_x=torch.empty_like(x), pre=pre, act=act, workspace=ws)
        sc.sc_grouped_bwd(grad, x, torch.stack([w, w]), starts, grad_x=torch.empty_like(x), pre=pre, act=act, workspace=ws)


def test_rope_axis_without_a_coordinate():
    """A table of three axes and positions of two: refused; positions of more axes than the table's are not."""
    rows, D, g = 40, 32, gen(6)
    q = normal(g, rows, 3, D, dtype=torch.float32).to(DEV)
    pos = torch.randint(0, 900, (rows, 4), generator=g).to(torch.int32).to(DEV)
    out, want = torch.empty_like(q), torch.empty_like(q)
    table = sc.sc_rope_table(D, (5, 5, 4))
    for axes in (1, 2):
        with pytest.raises(ValueError, match="more axes than pos has"):
            sc.sc_qk_rope_fwd(q, None, pos[:, :axes], table, out, None)
        with pytest.raises(ValueError, match="more axes than pos has"):
            sc.sc_qk_rope_bwd(q, None, None, None, pos[:, :axes], table, out, None)
    sc.sc_qk_rope_fwd(q, None, pos[:, :3], table, want, None)
    sc.sc_qk_rope_fwd(q, None, pos, table, out, None)
    assert torch.equal(out, want)
    sc.sc_rope_table(D, (5, 5), table=table)                   # the same memory, two axes now
    sc.sc_qk_rope_fwd(q, None, pos[:, :2], table, out, None)
    assert bool(torch.isfinite(out).all())


def test_rope_heads_between_each_other():
    """Outputs whose rows and heads interleave without touching are as good as any; those that touch are refused."""
    g, D = gen(4), 8
    pos, table = torch.randint(0, 900, (3, 3), generator=g).to(torch.int32).to(DEV), sc.sc_rope_table(D, (1, 1, 1))
    q = normal(g, 3, 2, D, dtype=torch.float32).to(DEV)
    want = torch.empty_like(q)
    sc.sc_qk_rope_fwd(q, None, pos, table, want, None)
    for row, head in ((16, 8), (8, 24), (16, 40), (24, 16), (20, 50)):
        space = torch.full((200,), 7.0, device=DEV)
        out = space.as_strided((3, 2, D), (row, head, 1))
        sc.sc_qk_rope_fwd(q, None, pos, table, out, None)
        assert torch.equal(out, want), (row, head)
        assert int((space == 7.0).sum()) == 200 - 3 * 2 * D
    for row, head in ((0, 8), (8, 0), (7, 30), (16, 7), (8, 8), (8, 16), (20, 47), (16, 30)):
        out = torch.empty(200, device=DEV).as_strided((3, 2, D), (row, head, 1))
        with pytest.raises(sc.ScError):
            sc.sc_qk_rope_fwd(q, None, pos, table, out, None)
        with pytest.raises(sc.ScError):
            sc.sc_qk_rope_bwd(q, None, None, None, pos, table, out, None)
    # inputs may: one head's gradient for all of them
    c = normal(g, 3, 1, D, dtype=torch.float32).to(DEV)
    back, same = torch.empty_like(q), torch.empty_like(q)
    sc.sc_qk_rope_bwd(c.expand(3, 2, D), None, None, None, pos, table, back, None)
    sc.sc_qk_rope_bwd(c.expand(3, 2, D).contiguous(), None, None, None, pos, table, same, None)
    assert torch.equal(back, same)


# ---- grouped --------------------------------------------------------------------------------------------------
# entries, starts, channels: with c_in = 32 and many entries and with few of both the slopes are inside the product with the weights, otherwise they are a pass of their own
LISTED = [(300, [0, 130, 131, 131, 260, 290], 64, 40), (70000, [0, 40000, 40001, 69990], 32, 24), (70000, [0, 40000, 40001, 69990], 31, 25), (5000, [0, 2100, 2100, 4990], 136, 264)]


@EVERY
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("n,starts,c_in,c_out", LISTED)
def test_gradients_taken_by_a_list(n, starts, c_in, c_out, act, dtype):
    """Output gradients gathered by a list, some rows several times, some that are not there, through an activation whose arguments are one row per entry."""
    dt, groups, g = DT[dtype], len(starts) - 1, gen(n + c_in)
    print(f"listed gradients {n} {c_in} {c_out} {act} {dtype}", flush=True)
    x_rows, dy_rows = 90, 70
    x, w = normal(g, x_rows, c_in, dtype=dt), normal(g, groups, c_in, c_out, dtype=dt, scale=1 / math.sqrt(c_in))
    dy, pre = normal(g, dy_rows, c_out, dtype=dt, scale=1 / 16), normal(g, n, c_out, dtype=dt)
    rows, grad_rows = (torch.randint(0, m, (n,), generator=g).to(torch.int32) for m in (x_rows, dy_rows))
    rows[5], rows[140] = -1, x_rows
    grad_rows[0], grad_rows[7], grad_rows[8], grad_rows[131], grad_rows[starts[-1] - 1] = -1, dy_rows, -(1 << 31), (1 << 31) - 1, dy_rows + 3
    pre[7] = math.inf                                          # of an entry whose gradient is not there: it adds nothing

    def taken(t, list_):
        ok = (list_ >= 0) & (list_ < len(t))
        return t.double()[torch.where(ok, list_, 0).long()] * ok[:, None]
    xs, grad = taken(x, rows), taken(dy, grad_rows)
    slopes = slope64(torch.where(torch.isfinite(pre), pre, 0.0).double(), act)
    d = grad * slopes
    d_err = torch.zeros_like(d) if act == "none" else (2 * ACT_ERROR * grad.abs() * (1 + torch.where(torch.isfinite(pre), pre, 0.0).double().abs()) + UNIT[dt] * d.abs() +
                                                        TINY[dt] * (d != 0))
    gx = torch.full((n, c_in), 7.0, dtype=dt, device=DEV)
    gw, gb = torch.full((groups, c_in, c_out), 7.0, dtype=dt, device=DEV), torch.full((groups, c_out), 7.0, dtype=dt, device=DEV)
    ws = torch.empty(sc.sc_grouped_workspace_bytes(n, groups, c_in, c_out, dt), dtype=torch.uint8, device=DEV)
    sc.sc_grouped_bwd(spread(dy, 8)[0], spread(x, 8)[0], w.to(DEV), torch.tensor(starts, dtype=torch.int32, device=DEV), gx, gw, gb, rows=rows.to(DEV),
                      grad_rows=grad_rows.to(DEV), pre=spread(pre, 8)[0] if act != "none" else None, act=act, workspace=ws)
    for k in range(groups):
        m = slice(starts[k], starts[k + 1])
        xk, dk, ek, wt = xs[m], d[m], d_err[m], w[k].double().t().contiguous()
        close(gx[m], dk @ wt, product_bound(dk @ wt, dk.abs() @ wt.abs(), ek @ wt.abs(), c_out, dt), f"dx[{k}]")
        xt, count = xk.t().contiguous(), starts[k + 1] - starts[k]
        close(gw[k], xt @ dk, product_bound(xt @ dk, xt.abs() @ dk.abs(), xt.abs() @ ek, count, dt), f"dw[{k}]")
        close(gb[k], dk.sum(0), product_bound(dk.sum(0), dk.abs().sum(0), ek.sum(0), count, dt), f"db[{k}]")
    assert bool((gx[starts[-1]:] == 7.0).all())


@EVERY
def test_fewer_rows_than_entries(dtype):
    """At the C boundary entry p reads row p, and rows past the last are zeros: forward and in the weights' gradient."""
    dt, g, n, x_rows, c_in, c_out = DT[dtype], gen(3), 300, 210, 40, 24
    lib, starts = sc.load(), [0, 100, 205, 300]
    x, w, b, grad = normal(g, x_rows, c_in, dtype=dt), normal(g, 3, c_in, c_out, dtype=dt), normal(g, 3, c_out, dtype=dt), normal(g, n, c_out, dtype=dt)
    d_x, d_w, d_b, d_grad, s = x.to(DEV), w.to(DEV), b.to(DEV), grad.to(DEV), torch.tensor(starts, dtype=torch.int32, device=DEV)
    out, gw = torch.empty(n, c_out, dtype=dt, device=DEV), torch.empty_like(d_w)
    ws = torch.empty(sc.sc_grouped_workspace_bytes(n, 3, c_in, c_out, dt), dtype=torch.uint8, device=DEV)
    p, stream = (lambda t: ctypes.c_void_p(t.data_ptr())), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    kind = sc.DTYPES[dt]
    assert lib.sc_grouped_fwd(p(d_x), c_in, x_rows, None, n, p(s), 3, p(d_w), p(d_b), 0, p(out), c_out, None, 0, c_in, c_out, kind, kind, stream) == sc.SC_OK
    assert lib.sc_grouped_bwd(p(d_grad), c_out, n, None, p(d_x), c_in, x_rows, None, n, p(s), 3, None, None, 0, 0, None, 0, p(gw), None, c_in, c_out, kind, p(ws),
                              ws.numel(), stream) == sc.SC_OK
    full = torch.cat([x, torch.zeros(n - x_rows, c_in, dtype=dt)]).double()
    for k in range(3):
        m = slice(starts[k], starts[k + 1])
        want, size = full[m] @ w[k].double() + b[k].double(), full[m].abs() @ w[k].double().abs() + b[k].double().abs()
        close(out[m], want, forward_bound(want, want, size, c_in, "none", dt), f"out[{k}]")
        xt, d = full[m].t(), grad[m].double()
        close(gw[k], xt @ d, product_bound(xt @ d, xt.abs() @ d.abs(), 0.0, starts[k + 1] - starts[k], dt), f"dw[{k}]")


def test_as_many_groups_as_there_may_be():
    """SC_GROUPS_MAX of them, of 0 to 400 entries, some in several parts: forward and both gradients."""
    groups, c, dt = sc.SC_GROUPS_MAX, 16, torch.float32
    torch.manual_seed(4)
    sizes = torch.randint(0, 3, (groups,))
    sizes[[0, 77, 30000, 65535]] = torch.tensor([400, 0, 300, 129])
    starts = torch.cat([torch.zeros(1, dtype=torch.int64), sizes.cumsum(0)])
    n, owner = int(starts[-1]), torch.repeat_interleave(torch.arange(groups), sizes).to(DEV)
    x, grad, w = torch.randn(n, c, device=DEV), torch.randn(n, c, device=DEV), torch.randn(groups, c, c, device=DEV)
    out, gx, gw, gb = torch.empty_like(x), torch.empty_like(x), torch.full_like(w, 7.0), torch.full((groups, c), 7.0, device=DEV)
    d_starts, ws = starts.to(DEV, torch.int32), torch.empty(sc.sc_grouped_workspace_bytes(n, groups, c, c, dt), dtype=torch.uint8, device=DEV)
    sc.sc_grouped_fwd(x, w, d_starts, out)
    sc.sc_grouped_bwd(grad, x, w, d_starts, gx, gw, gb, workspace=ws)

    def by_group(t):
        return torch.zeros(groups, *t.shape[1:], dtype=torch.float64, device=DEV).index_add(0, owner, t)
    x, grad, w = x.double(), grad.double(), w.double()[owner]
    for got, terms, axis, K in ((out, x[:, :, None] * w, 1, c), (gx, grad[:, None, :] * w, 2, c)):
        close(got, terms.sum(axis).cpu(), product_bound(terms.sum(axis), terms.abs().sum(axis), 0.0, K, dt).cpu())
    outer = x[:, :, None] * grad[:, None, :]
    close(gw, by_group(outer).cpu(), product_bound(by_group(outer), by_group(outer.abs()), 0.0, 400, dt).cpu(), "dw")
    close(gb, by_group(grad).cpu(), product_bound(by_group(grad), by_group(grad.abs()), 0.0, 400, dt).cpu(), "db")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("c_in,c_out", [(64, 96), (33, 41)])
def test_wide_outputs_with_the_value_ahead_of_the_activation(c_in, c_out, dtype):
    """Both outputs in 32 bits from 16-bit rows: linear with a residual, and grouped."""
    dt, g, n = DT[dtype], gen(c_in), 333
    x, w, b, r = normal(g, n, c_in, dtype=dt), normal(g, 2, c_in, c_out, dtype=dt, scale=0.2), normal(g, 2, c_out, dtype=dt), normal(g, n, c_out, dtype=torch.float32)
    for act in ("gelu", "silu"):
        out, pre = torch.empty(n, c_out, device=DEV), torch.empty(n, c_out, device=DEV)
        sc.sc_linear_fwd(x.to(DEV), w[0].to(DEV), out, bias=b[0].to(DEV), act=act, residual=r.to(DEV), pre=pre)
        plain, size = x.double() @ w[0].double() + b[0].double(), x.double().abs() @ w[0].double().abs() + b[0].double().abs()
        want = act64(plain, act) + r.double()
        close(out, want, forward_bound(want, plain, size + r.double().abs(), c_in, act, torch.float32), "out")
        close(pre, plain, forward_bound(plain, plain, size, c_in, "none", torch.float32), "pre")
        sc.sc_grouped_fwd(x.to(DEV), w.to(DEV), torch.tensor([0, 120, n], dtype=torch.int32, device=DEV), out, bias=b.to(DEV), act=act, pre=pre)
        for k, m in enumerate((slice(0, 120), slice(120, n))):
            plain, size = x[m].double() @ w[k].double() + b[k].double(), x[m].double().abs() @ w[k].double().abs() + b[k].double().abs()
            want = act64(plain, act)
            close(out[m], want, forward_bound(want, plain, size, c_in, act, torch.float32), "grouped out")
            close(pre[m], plain, forward_bound(plain, plain, size, c_in, "none", torch.float32), "grouped pre")


# starts, channels: the slopes inside the product with the weights in each of its tiles (few rows, thousands, one tile of columns), in whole chunks and not, and ahead of it
BIASES = [([0, 130], 24, 40), ([0, 4001], 128, 64), ([0, 70000], 24, 72), ([0, 70001], 31, 41), ([0, 5000], 200, 264), ([0, 40000], 96, 513), ([0, 300], 512, 9), ([0, 40000], 200, 192), ([0, 3000], 160, 7),
          ([0, 1, 1, 66, 131, 400, 401], 48, 40), ([2, 700, 701, 3801], 130, 72), ([0, 33000, 33000, 33129, 70000], 30, 136), ([0] * 70 + [900, 900, 2400], 40, 1030)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("starts,c_in,c_out", BIASES)
def test_bias_gradient_of_values_before_their_rounding(starts, c_in, c_out, dtype):
    """A group's last gradient takes back the sum of the others, which few rows have: what is left is as small as the rounding of the terms to 16 bits, and the bias'
    gradient is within the error of a sum in 32 bits of it."""
    dt, groups, n, g = DT[dtype], len(starts) - 1, starts[-1] + 3, gen(starts[-1] + c_out)
    print(f"bias {starts[-1]} in {groups} {c_in} {c_out} {dtype}", flush=True)
    pre, grad, taken = normal(g, n, c_out, dtype=dt), torch.zeros(n, c_out, dtype=dt), torch.randperm(n, generator=g).to(torch.int32)
    want, bound = (torch.zeros(groups, c_out, dtype=torch.float64) for _ in range(2))
    for k in range(groups):
        lo, hi = starts[k], starts[k + 1]
        if hi - lo < 2:
            continue
        some = lo + torch.randperm(hi - 1 - lo, generator=g)[:20]
        grad[some] = normal(g, len(some), c_out, dtype=dt)
        d = grad[some].double() * slope64(pre[some].double(), "silu")
        grad[hi - 1], pre[hi - 1] = -d.sum(0).to(dt), 40.0     # where the slope is one
        want[k] = d.sum(0) + grad[hi - 1].double()
        size = d.abs().sum(0) + grad[hi - 1].double().abs()
        off = (len(some) + 9) * 2.0 ** -23 * size + (ACT_ERROR * grad[some].double().abs() * (1 + pre[some].double().abs())).sum(0)
        bound[k] = off + UNIT[dt] * (want[k].abs() + off) + TINY[dt]
    x, w = normal(g, n, c_in, dtype=dt).to(DEV), normal(g, groups, c_in, c_out, dtype=dt, scale=0.1).to(DEV)
    d_grad, d_pre, d_starts = grad.to(DEV), pre.to(DEV), torch.tensor(starts, dtype=torch.int32, device=DEV)
    listed = torch.empty_like(d_grad)
    listed[taken.long()] = d_grad                               # entry p's is row taken[p]
    size = sc.sc_grouped_workspace_bytes(n, groups, c_in, c_out, dt)
    ws = torch.full((size + 4096,), 77, dtype=torch.uint8, device=DEV)
    gx, gw = torch.empty(n, c_in, dtype=dt, device=DEV), torch.empty(groups, c_in, c_out, dtype=dt, device=DEV)
    for rows, kw in ((d_grad, {}), (listed, dict(grad_rows=taken.to(DEV)))):
        for wanted in (dict(grad_x=gx, grad_weight=gw), dict(grad_x=gx), dict(grad_weight=gw), {}):
            gb = torch.full((groups, c_out), 7.0, dtype=dt, device=DEV)
            sc.sc_grouped_bwd(rows, x, w, d_starts, grad_bias=gb, pre=d_pre, act="silu", workspace=ws[:size], **kw, **wanted)
            close(gb, want, bound, f"grouped {sorted(wanted)} {sorted(kw)}")
    assert bool((ws[size:] == 77).all())
    if groups == 1:
        m = slice(starts[0], starts[1])
        size = sc.sc_linear_workspace_bytes(starts[1], c_in, c_out, dt)
        ws = torch.full((size + 4096,), 77, dtype=torch.uint8, device=DEV)
        for wanted in (dict(grad_x=gx[m], grad_weight=gw[0]), dict(grad_x=gx[m]), dict(grad_weight=gw[0]), {}):
            gb = torch.full((c_out,), 7.0, dtype=dt, device=DEV)
            sc.sc_linear_bwd(d_grad[m], x[m], w[0], grad_bias=gb, pre=d_pre[m], act="silu", workspace=ws[:size], **wanted)
            close(gb, want[0], bound[0], f"linear {sorted(wanted)}")
        assert bool((ws[size:] == 77).all())


def test_bias_gradient_of_starts_that_do_not_ascend():
    """Wrong starts give wrong sums, but nothing outside the arrays is written."""
    for n, c_in, c_out in ((2000, 32, 40), (70000, 24, 40), (3000, 160, 40)):
        dt, groups = torch.float16, 5
        x, grad, w = torch.ones(n, c_in, dtype=dt, device=DEV), torch.ones(n, c_out, dtype=dt, device=DEV), torch.ones(groups, c_in, c_out, dtype=dt, device=DEV)
        size = sc.sc_grouped_workspace_bytes(n, groups, c_in, c_out, dt)
        ws, gx = torch.full((size + 4096,), 77, dtype=torch.uint8, device=DEV), torch.full((n + 64, c_in), 7.0, dtype=dt, device=DEV)
        gw, gb = torch.zeros(groups + 1, c_in, c_out, dtype=dt, device=DEV), torch.zeros(groups + 1, c_out, dtype=dt, device=DEV)
        for starts in ([0, n, 0, n, 0, n], [-5, n + 1000, 1 << 30, -(1 << 31), 7, 100000], [n, n // 2, n // 3, n // 4, 0, 0]):
            print(f"starts {n} {starts}", flush=True)
            sc.sc_grouped_bwd(grad, x, w, torch.tensor(starts, dtype=torch.int32, device=DEV), gx[:n], gw[:groups], gb[:groups], pre=grad, act="gelu", workspace=ws[:size])
            torch.cuda.synchronize()
            assert bool((ws[size:] == 77).all()) and bool((gx[n:] == 7.0).all()) and not gw[groups].any() and not gb[groups].any()


# ---- what a call may leave out ----------------------------------------------------------------------------------
@EVERY
def test_rows_gradient_without_the_rows(dtype):
    """The gradient of the rows needs the weights, not the rows: where no weight gradient is asked for, x may be None."""
    dt, g, n, c_in, c_out = DT[dtype], gen(1), 200, 48, 40
    w, grad, pre = (normal(g, *s, dtype=dt).to(DEV) for s in ((2, c_in, c_out), (n, c_out), (n, c_out)))
    x, starts = normal(g, n, c_in, dtype=dt).to(DEV), torch.tensor([0, 90, n], dtype=torch.int32, device=DEV)
    ws = torch.empty(sc.sc_grouped_workspace_bytes(n, 2, c_in, c_out, dt), dtype=torch.uint8, device=DEV)
    for act in ("none", "gelu"):
        got = [torch.full((n, c_in), 7.0, dtype=dt, device=DEV) for _ in range(4)]
        gb = [torch.full((2, c_out), 7.0, dtype=dt, device=DEV) for _ in range(4)]
        kw = dict(pre=pre if act != "none" else None, act=act, workspace=ws)
        for i, rows in enumerate((x, None)):
            sc.sc_linear_bwd(grad, rows, w[0], grad_x=got[i], grad_bias=gb[i][0], **kw)
            sc.sc_grouped_bwd(grad, rows, w, starts, grad_x=got[2 + i], grad_bias=gb[2 + i], **kw)
        assert torch.equal(got[0], got[1]) and torch.equal(got[2], got[3]) and torch.equal(gb[0], gb[1]) and torch.equal(gb[2], gb[3])
        assert bool((got[0] != 7.0).any()) and bool((got[2] != 7.0).any())


# ---- the activation's tail --------------------------------------------------------------------------------------
@EVERY
def test_gelu_in_relative_terms(dtype):
    """v Phi(v) and Phi(v) + v phi(v) down to -12, where 16-bit types still have all their digits.  The weight of the tail is within 2.1e-5 of itself, the
    exponential's argument within 3 2^-24 of itself (v^2 / 2 of at most 72: 1.3e-5): 4e-5 of the terms, and one rounding."""
    dt = DT[dtype]
    v = torch.cat([torch.linspace(-12, 6, 40001, dtype=torch.float64), -torch.logspace(-6, 1, 2000, dtype=torch.float64)]).to(dt)
    one, exact = torch.ones(1, 1, dtype=dt, device=DEV), v.double()
    phi, cdf = torch.exp(-exact ** 2 / 2) / math.sqrt(2 * math.pi), torch.special.erfc(-exact / math.sqrt(2)) / 2
    out, gx = torch.empty(len(v), 1, dtype=dt, device=DEV), torch.empty(len(v), 1, dtype=dt, device=DEV)
    sc.sc_linear_fwd(v[:, None].to(DEV), one, out, act="gelu")
    ws = torch.empty(sc.sc_linear_workspace_bytes(len(v), 1, 1, dt), dtype=torch.uint8, device=DEV)
    sc.sc_linear_bwd(torch.ones(len(v), 1, dtype=dt, device=DEV), v[:, None].to(DEV), one, grad_x=gx, pre=v[:, None].to(DEV), act="gelu", workspace=ws)
    want, off = exact * cdf, 4e-5 * exact.abs() * cdf
    close(out[:, 0], want, off + UNIT[dt] * (want.abs() + off) + TINY[dt], "gelu")
    want, off = cdf + exact * phi, 4e-5 * (cdf + exact.abs() * phi)
    close(gx[:, 0], want, off + UNIT[dt] * (want.abs() + off) + TINY[dt], "gelu's slope")

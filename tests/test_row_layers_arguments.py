"""CPU tests of what the row layers refuse, at the C boundary and in the marshalling of tensors, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2402_07710_amd import binding as sc

F16, F32, BF16 = sc.SC_F16, sc.SC_F32, sc.SC_BF16
EINVAL, ECAP, OK = sc.SC_EINVAL, sc.SC_ECAP, sc.SC_OK


@pytest.fixture(scope="module")
def lib():
    return sc.load()


def linear_fwd(lib, **change):
    a = dict(x=16, ldx=32, rows=10, w=32, b=None, act=0, r=None, ldr=0, y=48, ldy=64, pre=None, ldp=0, c_in=32, c_out=64, dt=F16, out=F16)
    a.update(change)
    return lib.sc_linear_fwd(*a.values(), None)


def linear_bwd(lib, **change):
    a = dict(dy=16, lddy=64, x=32, ldx=32, rows=0, w=48, pre=None, ldp=0, act=0, dx=64, lddx=32, dw=None, db=None, c_in=32, c_out=64, dt=F16, ws=None, bytes=0)
    a.update(change)
    return lib.sc_linear_bwd(*a.values(), None)


def test_linear_refuses(lib):
    assert linear_fwd(lib, rows=0) == OK and linear_fwd(lib, rows=0, x=None, y=None) == OK
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(x=17), dict(w=33), dict(b=49), dict(y=47), dict(r=51, ldr=64), dict(pre=53, ldp=64), dict(ldx=31),
                dict(ldy=63), dict(r=64, ldr=63), dict(pre=64, ldp=63), dict(rows=-1), dict(rows=sc.SC_N_MAX + 1), dict(act=4), dict(act=-1), dict(dt=3),
                dict(out=BF16), dict(dt=F32, out=F16), dict(c_in=0), dict(c_out=0), dict(c_in=65537, ldx=1 << 17), dict(c_out=65537, ldy=1 << 17)):
        assert linear_fwd(lib, **bad) == EINVAL, bad
    assert linear_bwd(lib) == OK
    for bad in (dict(dx=None), dict(rows=5, dy=None), dict(rows=5, dy=17), dict(lddy=63), dict(w=None), dict(w=33), dict(dx=65), dict(lddx=31), dict(dw=65), dict(db=65),
                dict(rows=5, dw=64, x=None), dict(rows=5, act=1), dict(rows=5, act=1, pre=64, ldp=63), dict(act=4), dict(dt=3), dict(c_in=0),
                dict(rows=5, act=1, pre=64, ldp=64), dict(rows=5, act=1, pre=64, ldp=64, ws=24, bytes=1 << 20), dict(rows=-1)):
        assert linear_bwd(lib, **bad) == EINVAL, bad
    need = lib.sc_linear_workspace_bytes(100000, 32, 64, F16)
    assert linear_bwd(lib, rows=100000, act=1, pre=64, ldp=64, dw=128, ws=256, bytes=need - 1) == ECAP
    assert linear_bwd(lib, rows=5, act=1, pre=64, ldp=64, ws=256, bytes=639) == ECAP
    assert lib.sc_linear_workspace_bytes(-1, 32, 64, F16) == 0 and lib.sc_linear_workspace_bytes(sc.SC_N_MAX + 1, 32, 64, F16) == 0
    assert lib.sc_linear_workspace_bytes(10, 0, 64, F16) == 0 and lib.sc_linear_workspace_bytes(10, 32, 64, 7) == 0


def grouped_fwd(lib, **change):
    a = dict(x=16, ldx=32, x_rows=10, rows=None, n=10, starts=16, groups=3, w=32, b=None, act=0, y=48, ldy=64, pre=None, ldp=0, c_in=32, c_out=64, dt=F16, out=F16)
    a.update(change)
    return lib.sc_grouped_fwd(*a.values(), None)


def grouped_bwd(lib, **change):
    a = dict(dy=16, lddy=64, dy_rows=10, grad_rows=None, x=32, ldx=32, x_rows=10, rows=None, n=0, starts=16, groups=3, w=48, pre=None, ldp=0, act=0, dx=64, lddx=32,
             dw=None, db=None, c_in=32, c_out=64, dt=F16, ws=None, bytes=0)
    a.update(change)
    return lib.sc_grouped_bwd(*a.values(), None)


def test_grouped_refuses(lib):
    assert grouped_fwd(lib, n=0) == OK
    for bad in (dict(starts=None), dict(starts=18), dict(rows=18), dict(groups=0), dict(groups=65537), dict(n=-1), dict(n=1 << 31), dict(x_rows=-1), dict(x_rows=sc.SC_N_MAX + 1),
                dict(w=None), dict(act=9), dict(ldx=31), dict(y=None), dict(out=BF16)):
        assert grouped_fwd(lib, **bad) == EINVAL, bad
    assert grouped_bwd(lib) == OK
    for bad in (dict(starts=None), dict(grad_rows=18), dict(rows=18), dict(groups=0), dict(n=-1), dict(dy_rows=-1), dict(dy_rows=sc.SC_N_MAX + 1), dict(dx=None), dict(w=None)):
        assert grouped_bwd(lib, **bad) == EINVAL, bad
    assert lib.sc_grouped_workspace_bytes(10, 0, 32, 64, F16) == 0 and lib.sc_grouped_workspace_bytes(1 << 31, 2, 32, 64, F16) == 0


def heads(data=16, row=128, head=64, n=2):
    return ctypes.byref(sc.ScHeads(data, row, head, n))


def rope_fwd(lib, **change):
    a = dict(q=heads(), k=heads(n=1), rows=0, D=64, pos=16, ld_pos=4, axes=3, table=16, pairing=0, gq=None, gk=None, eps=1e-6, qo=heads(), ko=heads(n=1), dt=F16)
    a.update(change)
    return lib.sc_qk_rope_fwd(*a.values(), None)


def rope_bwd(lib, **change):
    a = dict(dqo=heads(), dko=heads(n=1), q=heads(), k=heads(n=1), rows=0, D=64, pos=16, ld_pos=4, axes=3, table=16, pairing=0, gq=None, gk=None, eps=1e-6, dq=heads(),
             dk=heads(n=1), dgq=None, dgk=None, dt=F16, ws=None, bytes=0)
    a.update(change)
    return lib.sc_qk_rope_bwd(*a.values(), None)


def test_rope_refuses(lib):
    assert rope_fwd(lib) == OK and rope_fwd(lib, k=None, ko=None) == OK and rope_bwd(lib) == OK
    for bad in (dict(q=None), dict(q=heads(data=None)), dict(q=heads(data=17)), dict(q=heads(n=0)), dict(q=heads(n=3)), dict(q=heads(row=-1)), dict(k=heads(n=2)), dict(ko=None),
                dict(D=63), dict(D=0), dict(D=1026), dict(rows=-1), dict(pos=None), dict(pos=18), dict(ld_pos=2), dict(axes=0), dict(axes=5), dict(table=None), dict(table=24),
                dict(pairing=2), dict(gq=17), dict(eps=-1.0), dict(eps=float("nan")), dict(dt=3)):
        assert rope_fwd(lib, **bad) == EINVAL, bad
    for bad in (dict(dq=None), dict(gq=16, q=None), dict(gk=16, k=heads(n=2)), dict(dgq=16), dict(gq=16, dgq=17), dict(gq=16, dgq=16, rows=5), dict(dgk=16, gk=16, dko=None)):
        assert rope_bwd(lib, **bad) == EINVAL, bad
    need = lib.sc_qk_rope_workspace_bytes(5, 2, 1, 64)
    assert need > 0 and rope_bwd(lib, gq=16, dgq=16, rows=5, ws=16, bytes=need - 1) == ECAP
    pairs = (ctypes.c_int32 * 3)(10, 11, 11)
    table = lambda D=64, axes=3, p=pairs, base=1e4, d=16, size=1 << 20: lib.sc_rope_table(D, axes, p, base, d, size, None)   # noqa: E731
    assert table(D=62) == EINVAL and table(axes=0) == EINVAL and table(axes=5) == EINVAL and table(p=None) == EINVAL and table(base=0.0) == EINVAL
    assert table(base=float("nan")) == EINVAL and table(d=None) == EINVAL and table(d=24) == EINVAL and table(size=511) == ECAP
    assert table(p=(ctypes.c_int32 * 3)(40, -10, 2)) == EINVAL
    assert lib.sc_rope_table_bytes(64) == 512 and lib.sc_rope_table_bytes(63) == 0 and lib.sc_rope_table_bytes(2048) == 0


def half(*shape, dtype=torch.float16):
    return torch.zeros(shape, dtype=dtype)


X, W, Y = half(10, 32), half(32, 64), half(10, 64)


@pytest.mark.parametrize("args,kw,what", [
    ((half(10, 32, 1), W, Y), {}, "x must be"), ((X, W, half(640)), {}, "out must be"), ((X, half(31, 64), Y), {}, "weight has"), ((X, W, half(9, 64)), {}, "out has"),
    ((X, W.t().contiguous().t(), Y), {}, "weight must be contiguous"), ((X, W.float(), Y), {}, "weight has the wrong dtype"), ((X, W, Y.bfloat16()), {}, "out must be of"),
    ((X, W, Y), dict(bias=half(63)), "bias has"), ((X, W, Y), dict(bias=half(64, dtype=torch.float32)), "bias has"), ((X, W, Y), dict(residual=half(10, 63)), "residual has"),
    ((X, W, Y), dict(pre=half(10, 64, dtype=torch.float32)), "pre has"), ((half(32, 10).t(), W, Y), {}, "x must be"), ((X.expand(10, 32)[:1].expand(10, 32), W, Y), {}, "x has rows that overlap"),
    ((X, W, Y), {}, "device tensor expected"),
])
def test_linear_tensors(args, kw, what):
    with pytest.raises(ValueError, match=what):
        sc.sc_linear_fwd(*args, stream=0, **kw)


def test_other_tensors():
    starts = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="weight has the wrong shape"):
        sc.sc_grouped_fwd(X, half(2, 32, 64), starts, Y, stream=0)
    with pytest.raises(ValueError, match="device tensor expected"):
        sc.sc_grouped_fwd(X, half(3, 32, 64), starts, Y, stream=0)
    with pytest.raises(ValueError, match="grad_x has the wrong shape"):
        sc.sc_linear_bwd(Y, X, W, grad_x=half(10, 31), stream=0)
    with pytest.raises(ValueError, match="dtype"):
        sc.sc_linear_bwd(Y, X, W, grad_x=half(10, 32, dtype=torch.float32), stream=0)
    q, pos, table = half(5, 2, 64), torch.zeros(5, 3, dtype=torch.int32), torch.zeros(512, dtype=torch.uint8)
    with pytest.raises(ValueError, match="q must be"):
        sc.sc_qk_rope_fwd(half(5, 128), None, pos, table, q, None, stream=0)
    with pytest.raises(ValueError, match="q_out has the wrong shape"):
        sc.sc_qk_rope_fwd(q, None, pos, table, half(5, 2, 32), None, stream=0)
    with pytest.raises(ValueError, match="table is not"):
        sc.sc_qk_rope_fwd(q, None, pos, table[:500], q, None, stream=0)
    with pytest.raises(KeyError):
        sc.sc_linear_fwd(X, W, Y, act="tanh", stream=0)
    with pytest.raises(KeyError):
        sc.sc_qk_rope_fwd(q, None, pos, table, q, None, pairing="thirds", stream=0)
    with pytest.raises(TypeError, match="tensor expected"):
        sc.sc_linear_fwd([[1.0]], W, Y, stream=0)


@pytest.mark.gpu
def test_row_calls_release_the_interpreter_lock():
    lib = sc.load()
    check = ctypes.cast(ctypes.pythonapi.PyGILState_Check, ctypes.c_void_p).value
    sc._native.bind_rows(*[check] * len(sc._NATIVE_ROW_CALLS))
    try:
        x, w, q = X.cuda(), W.cuda(), half(5, 2, 64).cuda()
        y, s, w3 = Y.cuda(), torch.zeros(4, dtype=torch.int32, device="cuda:0"), half(3, 32, 64).cuda()
        pos, table = torch.zeros(5, 3, dtype=torch.int32, device="cuda:0"), torch.zeros(512, dtype=torch.uint8, device="cuda:0")
        sc.sc_linear_fwd(x, w, y)
        sc.sc_linear_bwd(y, x, w, grad_x=x)
        sc.sc_grouped_fwd(x, w3, s, y)
        sc.sc_grouped_bwd(y, x, w3, s, grad_x=x)
        sc.sc_qk_rope_fwd(q, q, pos, table, q, q)
        sc.sc_qk_rope_bwd(q, q, q, q, pos, table, q, q)         # a status other than zero would raise
    finally:
        sc._native.bind_rows(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in sc._NATIVE_ROW_CALLS))

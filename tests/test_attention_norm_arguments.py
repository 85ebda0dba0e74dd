"""CPU tests of what attention and the group norm refuse, at the C boundary and in the marshalling of tensors, before anything is launched; and of their size queries."""
import ctypes
import os
import random
import re

import pytest
import torch

from paper_2402_07710_amd import binding as sc

F16, F32, BF16 = sc.SC_F16, sc.SC_F32, sc.SC_BF16
EINVAL, ECAP, OK = sc.SC_EINVAL, sc.SC_ECAP, sc.SC_OK


@pytest.fixture(scope="module")
def lib():
    return sc.load()


def heads(data=16, row=128, head=64, n=2):
    return ctypes.byref(sc.ScHeads(data, row, head, n))


def fwd(lib, **change):
    a = dict(q=heads(), k=heads(n=1), v=heads(n=1), q_rows=0, k_rows=0, D=64, qs=None, ks=None, kl=None, scenes=1, causal=0, scale=0.125, out=heads(), lse=None, dt=F16,
             ws=None, bytes=0)
    a.update(change)
    return lib.sc_attention_fwd(*a.values(), None)


def bwd(lib, **change):
    a = dict(dout=heads(), q=heads(), k=heads(n=1), v=heads(n=1), out=heads(), lse=16, q_rows=5, k_rows=5, D=64, qs=None, ks=None, kl=None, scenes=1, causal=0, scale=0.125,
             dq=heads(), dk=heads(n=1), dv=heads(n=1), dt=F16, ws=None, bytes=0)
    a.update(change)
    return lib.sc_attention_bwd(*a.values(), None)


def test_attention_refuses(lib):
    assert fwd(lib) == OK and fwd(lib, qs=16, scenes=7) == OK and fwd(lib, qs=16, ks=32, kl=64, scenes=7, causal=1, lse=128) == OK
    common = (dict(q=None), dict(q=heads(data=None)), dict(q=heads(data=17)), dict(q=heads(n=0)), dict(q=heads(n=3), k=heads(n=2), v=heads(n=2)), dict(k=heads(n=0)), dict(v=None),
              dict(v=heads(n=2)), dict(out=heads(n=1)), dict(q=heads(row=-1)), dict(k=heads(row=(1 << 24) + 1)), dict(D=0), dict(D=257), dict(q_rows=-1), dict(k_rows=-1),
              dict(q_rows=sc.SC_N_MAX + 1), dict(k_rows=sc.SC_N_MAX + 1), dict(scenes=0), dict(scenes=-1), dict(scenes=2), dict(ks=16), dict(qs=17), dict(qs=16, ks=18), dict(kl=18),
              dict(qs=16, k_rows=3, q_rows=4), dict(causal=2), dict(causal=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(dt=3),
              dict(lse=18), dict(q=heads(n=64), out=heads(n=64, row=4096), q_rows=1 << 26, k_rows=1 << 26))
    for bad in common:
        assert fwd(lib, **bad) == EINVAL, bad
    assert fwd(lib, q_rows=3, out=heads(row=64)) == EINVAL                     # rows of out overlap
    assert fwd(lib, q_rows=3, out=heads(head=63)) == EINVAL
    for bad in common:
        if "lse" not in bad:
            assert bwd(lib, **bad) == EINVAL, bad
    for bad in (dict(lse=None), dict(dout=None), dict(dout=heads(n=1)), dict(dq=None), dict(dq=heads(n=1)), dict(dk=heads(n=2)), dict(dv=heads(data=17, n=1)), dict(dq=heads(head=63)),
                dict(dk=heads(row=63, n=1)), dict(dv=heads(row=1 << 25, n=1)), dict(ws=None), dict(ws=24, bytes=1 << 20)):
        assert bwd(lib, **bad) == EINVAL, bad
    need = lib.sc_attention_bwd_workspace_bytes(5, 5, 1, 2, 1, 64, F16)
    assert need > 0 and bwd(lib, ws=16, bytes=need - 1) == ECAP


def test_attention_workspaces(lib):
    size, grad = lib.sc_attention_workspace_bytes, lib.sc_attention_bwd_workspace_bytes
    for query in (size, grad):
        for bad in ((-1, 5, 1, 2, 1, 64, F16), (5, -1, 1, 2, 1, 64, F16), (5, 5, 0, 2, 1, 64, F16), (5, 5, 1, 3, 2, 64, F16), (5, 5, 1, 2, 0, 64, F16), (5, 5, 1, 2, 1, 0, F16),
                    (5, 5, 1, 2, 1, 257, F16), (5, 5, 1, 2, 1, 64, 3)):
            assert query(*bad) == 0, bad
    assert size(5, 5, 1, 2, 1, 64, F16) == 0
    many = size(1, 100000, 1, 8, 8, 64, F16)                                    # one row over a long cache: in parts
    parts = many // (8 * (64 * 4 + 8))
    assert 2 <= parts <= 256 and many >= parts * 8 * (64 * 4 + 8)
    assert fwd(lib, q_rows=1, k_rows=100000, q=heads(n=8), k=heads(n=8), v=heads(n=8), out=heads(n=8), ws=16, bytes=many - 1) == ECAP
    assert fwd(lib, q_rows=1, k_rows=100000, q=heads(n=8), k=heads(n=8), v=heads(n=8), out=heads(n=8)) == EINVAL
    assert grad(100, 100, 1, 4, 2, 64, F16) >= 2 * 100 * 4 * 4


def norm_fwd(lib, **change):
    a = dict(x=16, ldx=32, rows=10, starts=None, scenes=1, C=32, groups=4, gain=None, bias=None, eps=1e-5, act=0, y=48, ldy=32, stats=None, dt=F16, ws=16, bytes=1 << 20)
    a.update(change)
    return lib.sc_group_norm_fwd(*a.values(), None)


def norm_bwd(lib, **change):
    a = dict(dy=16, lddy=32, x=16, ldx=32, rows=10, starts=None, scenes=1, C=32, groups=4, gain=None, bias=None, act=0, stats=64, dx=48, lddx=32, dgain=None, dbias=None, dt=F16,
             ws=16, bytes=1 << 20)
    a.update(change)
    return lib.sc_group_norm_bwd(*a.values(), None)


def test_group_norm_refuses(lib):
    common = (dict(x=None), dict(x=17), dict(ldx=31), dict(rows=-1), dict(rows=sc.SC_N_MAX + 1), dict(scenes=0), dict(scenes=2), dict(starts=18), dict(C=0), dict(C=65537, ldx=1 << 17),
              dict(groups=0), dict(groups=5), dict(groups=64), dict(gain=17), dict(bias=17), dict(act=4), dict(act=-1), dict(dt=3), dict(ws=None), dict(ws=24), dict(stats=20),
              dict(starts=16, scenes=1 << 22))
    for bad in common:
        assert norm_fwd(lib, **bad) == EINVAL, bad
        assert norm_bwd(lib, **bad) == EINVAL, bad
    for bad in (dict(y=None), dict(y=49), dict(ldy=31), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert norm_fwd(lib, **bad) == EINVAL, bad
    for bad in (dict(dy=None), dict(lddy=31), dict(stats=None), dict(dx=None), dict(dx=49), dict(lddx=31), dict(dgain=17), dict(dbias=17)):
        assert norm_bwd(lib, **bad) == EINVAL, bad
    need = lib.sc_group_norm_workspace_bytes(10, 1, 32, 4)
    assert need > 0 and norm_fwd(lib, bytes=need - 1) == ECAP and norm_bwd(lib, bytes=need - 1) == ECAP
    for bad in ((-1, 1, 32, 4), (10, 0, 32, 4), (10, 1, 0, 1), (10, 1, 32, 5), (10, 1, 32, 0), (10, 1 << 22, 32, 4)):
        assert lib.sc_group_norm_workspace_bytes(*bad) == 0, bad


def half(*shape, dtype=torch.float16):
    return torch.zeros(shape, dtype=dtype)


Q, K = half(10, 4, 32), half(12, 2, 32)
STARTS = torch.zeros(4, dtype=torch.int32)


@pytest.mark.parametrize("args,kw,what", [
    ((half(10, 128), K, K, Q), {}, "q must be"), ((Q, half(12, 64), K, Q), {}, "k must be"), ((Q, K, half(11, 2, 32), Q), {}, "v has the wrong shape"),
    ((Q, K, half(12, 1, 32), Q), {}, "v has another number"), ((Q, K, K, half(10, 2, 32)), {}, "out has another number"), ((Q, K, K, half(10, 4, 16)), {}, "out has the wrong shape"),
    ((Q, K, None, Q), {}, "v is needed"), ((Q, K, K, None), {}, "out is needed"), ((Q, K.float(), K, Q), {}, "wrong dtype"), ((Q, K, K, Q.float()), {}, "wrong dtype"),
    ((Q, K, K, Q), dict(lse=half(10, 4)), "lse must be float32"), ((Q, K, K, Q), dict(lse=torch.zeros(10, 3)), "lse has the wrong shape"),
    ((Q, K, K, Q), dict(k_starts=STARTS), "k_starts without"), ((Q, K, K, Q), dict(q_starts=STARTS), "as many keys"), ((Q, K, K, Q), dict(q_starts=STARTS[:1], k_starts=STARTS), "scenes"),
    ((Q, K, K, Q), dict(q_starts=STARTS, k_starts=STARTS[:3]), "k_starts has the wrong shape"), ((Q, K, K, Q), dict(q_starts=STARTS.long(), k_starts=STARTS), "q_starts must be int32"),
    ((Q, K, K, Q), dict(k_lens=STARTS), "k_lens has the wrong shape"), ((Q.transpose(1, 2).contiguous().transpose(1, 2), K, K, Q), {}, "channels contiguous"),
    ((Q, K, K, Q), {}, "device tensor expected"),
])
def test_attention_tensors(args, kw, what):
    with pytest.raises(ValueError, match=what):
        sc.sc_attention_fwd(*args, stream=0, **kw)


def test_attention_gradient_tensors():
    lse = torch.zeros(10, 4)
    good = dict(grad_out=Q, q=Q, k=K, v=K, out=Q, lse=lse, grad_q=Q, grad_k=K, grad_v=K)
    for name, value, what in (("grad_out", None, "grad_out is needed"), ("lse", None, "lse is needed"), ("grad_k", half(12, 4, 32), "grad_k has another number"),
                              ("grad_q", half(9, 4, 32), "grad_q has the wrong shape"), ("out", Q.bfloat16(), "out has the wrong dtype"), ("q", Q, "device tensor expected")):
        with pytest.raises(ValueError, match=what):
            sc.sc_attention_bwd(**{**good, name: value}, stream=0)


def test_group_norm_tensors():
    x, c, stats = half(10, 32), half(32), torch.zeros(1, 4, 2)
    for args, kw, what in (((x, half(10, 31), 4), {}, "out has the wrong shape"), ((x, half(10, 32, dtype=torch.float32), 4), {}, "wrong dtype"), ((x, None, 4), {}, "out is needed"),
                           ((x, x, 4), dict(gain=half(31)), "gain has"), ((x, x, 4), dict(bias=c.float()), "wrong dtype"), ((x, x, 4), dict(stats=torch.zeros(4, 2)), "stats has"),
                           ((x, x, 4), dict(stats=half(1, 4, 2)), "stats must be float32"), ((x, x, 4), dict(starts=STARTS[:1]), "starts must be"), ((x, x, 4), dict(starts=STARTS.long()), "starts must be int32"),
                           ((x.t(), x, 4), {}, "x must be"), ((x, x, 4), {}, "device tensor expected")):
        with pytest.raises(ValueError, match=what):
            sc.sc_group_norm_fwd(*args, stream=0, **kw)
    for args, kw, what in (((x, x, None, x, 4), {}, "stats is needed"), ((half(9, 32), x, stats, x, 4), {}, "grad_out has"), ((x, x, stats, half(10, 31), 4), {}, "grad_x has"),
                           ((x, x, stats, x, 4), dict(grad_gain=half(31)), "grad_gain has"), ((x, x, stats, x, 4), {}, "device tensor expected")):
        with pytest.raises(ValueError, match=what):
            sc.sc_group_norm_bwd(*args, stream=0, **kw)
    with pytest.raises(KeyError):
        sc.sc_group_norm_fwd(x, x, 4, act="tanh", stream=0)


def test_attention_refuses_outputs_that_meet_operands(lib):
    """Slices of one row [5][20 heads of 64], 2 bytes a channel: two heads of queries, one of keys.  An output may share no element with what other workgroups still read, or
    with another output."""
    def at(head, n, byte=0):
        return heads(data=(1 << 20) + 128 * head + byte, row=1280, head=64, n=n)
    need = max(lib.sc_attention_bwd_workspace_bytes(5, 5, 1, 2, 1, 64, F16), lib.sc_attention_workspace_bytes(5, 5, 1, 2, 1, 64, F16))
    q, k, v, out, dout, dq, dk, dv = (dict(q=at(0, 2)), dict(k=at(2, 1)), dict(v=at(3, 1)), dict(out=at(4, 2)), dict(dout=at(6, 2)), dict(dq=at(8, 2)), dict(dk=at(10, 1)), dict(dv=at(11, 1)))
    good = dict(**q, **k, **v, **out, q_rows=5, k_rows=5, ws=16, bytes=need)
    for bad in (dict(out=at(2, 2)), dict(out=at(1, 2)), dict(out=at(0, 2, 2)), dict(out=at(2, 2, 64)), dict(out=at(22, 2)), dict(out=heads(data=(1 << 20) + 256, row=2560, head=64))):
        assert fwd(lib, **{**good, **bad}) == EINVAL, bad
    good.update(**dout, **dq, **dk, **dv, lse=16)
    for name in ("q", "dout", "k", "v", "dk", "dv"):
        assert bwd(lib, **{**good, "dq": {**q, **dout, "k": at(1, 2), "v": at(3, 2), "dk": at(9, 2), "dv": at(11, 2)}[name]}) == EINVAL, name
    for name in ("dk", "dv"):
        for other in (at(0, 1), at(1, 1), at(7, 1), at(2, 1, 2), at(3, 1, 126), at(9, 1), at(10 if name == "dv" else 11, 1)):
            assert bwd(lib, **{**good, name: other}) == EINVAL, name
    assert bwd(lib, **{**good, "dq": at(5, 2)}) == EINVAL                        # half of out


def test_attention_refuses_scales_that_are_infinite_to_base_2(lib):
    """Kernels take exponentials to base 2: scale log2(e) is above the largest number of 32 bits, 3.4028e38, from 2.3587e38 on."""
    for call in (fwd, bwd):
        for scale in (2.36e38, 2.9e38, 3.4e38):
            assert call(lib, scale=scale) == EINVAL, scale
    for scale in (1e-45, 1.0, sc.SC_ATTENTION_SCALE_MAX):
        assert fwd(lib, scale=scale) == OK, scale


def test_workspaces_for_all_sizes(lib):
    """Sizes shrink and grow with rows; the bounds, which the header and the binding give alike, hold for all of them."""
    size, grad, norm = lib.sc_attention_workspace_bytes, lib.sc_attention_bwd_workspace_bytes, lib.sc_group_norm_workspace_bytes
    assert size(2048, 2048, 1, 8, 8, 64, F16) > size(8192, 8192, 1, 8, 8, 64, F16) and grad(16384, 16384, 1, 8, 8, 64, F16) > grad(32768, 32768, 1, 8, 8, 64, F16)
    assert norm(32000, 1, 64, 8) > norm(33000, 1, 64, 8)
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "sc.h")).read()

    def macro(name):
        found = re.search(r"#define " + name + r"\(([^)]*)\) (.*)", text)
        return eval(f"lambda {found.group(1)}: " + found.group(2).replace("(size_t)", ""))
    most, most_grad, most_norm = macro("SC_ATTENTION_WORKSPACE_MAX"), macro("SC_ATTENTION_BWD_WORKSPACE_MAX"), macro("SC_NORM_WORKSPACE_MAX")
    rng, nearest = random.Random(3), [0.0, 0.0, 0.0]
    for i in range(200000):
        rows, keys, scenes, k_heads, per, D = (int(2 ** rng.uniform(0, bits)) for bits in (26, 26, 12, 6, 5, 8.001))
        if i % 3 == 0:
            keys = rows
        dt, heads_q, scenes = rng.choice([F16, F32]), k_heads * per, 1 if i % 2 else scenes
        need, need_grad = size(rows, keys, scenes, heads_q, k_heads, D, dt), grad(rows, keys, scenes, heads_q, k_heads, D, dt)
        C, groups = k_heads * per, per
        need_norm = norm(rows, scenes, C, groups)
        for j, (n, m, m2) in enumerate(((need, most(D), sc.sc_attention_workspace_max(D)), (need_grad, most_grad(rows, heads_q, D), sc.sc_attention_bwd_workspace_max(rows, heads_q, D)),
                                        (need_norm, most_norm(scenes, C, groups), sc.sc_group_norm_workspace_max(scenes, C, groups)))):
            assert n <= m == m2, (j, rows, keys, scenes, heads_q, k_heads, D, dt)
            nearest[j] = max(nearest[j], n / m)
    print(nearest)
    assert min(nearest) > 0.5, nearest

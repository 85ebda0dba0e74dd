"""GPU tests of attention over packed scenes, forward and backward, against the definition in 64 bits.

Tolerances follow from the roundings.  u is half a step of the rows' type (2^-9+1 bf16, 2^-11 f16, 2^-24 f32), f = 2^-24.  A score of D products in 32 bits is off by
e = (D + 2) f sum |q k| scale at most, its exponential by e and 4 f (|score| + 1) more, relatively; a weight is rounded once (u).  So out is off by
(u + 2 (e + ...) + n f) sum w |v| and its own rounding u |out|; weights of f16 that are below 2^-14 2^-6 of the largest by 2^-31 of it instead of u.
Backward: dP is off by (D + 2) f sum |do v|, delta by (u + D f) sum |do o| (o is the rounded output), P by e + the error of lse, dS = P (dP - delta) is rounded once.
"""
import math

import pytest
import torch

from paper_2402_07710_amd import binding as sc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F = 2.0 ** -24
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def half_step(dt):
    return torch.finfo(dt).eps / 2


def starts_of(lens, at=0):
    out = [at]
    for n in lens:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device=DEV)


def reference(q, k, v, grad, lens, key_lens, key_starts, q_starts, causal, scale, dt):
    """out, lse, dq, dk, dv in 64 bits and how far each may be off, scene by scene and head by head; NaN where no scene has the row."""
    hq, hk, D = q.shape[1], k.shape[1], q.shape[2]
    u, tiny = half_step(dt), 0.0 if dt == torch.float32 else 2.0 ** -31
    q, k, v, grad = (t.double().cpu() for t in (q, k, v, grad))
    nan = float("nan")
    out, lse, dq = torch.full_like(q, nan), torch.full(q.shape[:2], nan, dtype=torch.float64), torch.full_like(q, nan)
    dk, dv = torch.full_like(k, nan), torch.full_like(v, nan)
    t_out, t_lse, t_dq, t_dk, t_dv = (torch.zeros_like(t) for t in (out, lse, dq, dk, dv))
    for a, nq, b, nk in zip(q_starts, lens, key_starts, key_lens):
        qs, ks = slice(a, a + nq), slice(b, b + nk)
        dk[ks], dv[ks] = 0.0, 0.0
        for h in range(hq):
            j = h // (hq // hk)
            Q, K, V, G = q[qs, h], k[ks, j], v[ks, j], grad[qs, h]
            S = Q @ K.t() * scale
            e = (D + 2) * F * (Q.abs() @ K.abs().t()) * scale + 4 * F * (S.abs() + 1)
            seen = torch.ones(nq, nk, dtype=torch.bool)
            if causal:
                seen = torch.arange(nk)[None, :] - torch.arange(nq)[:, None] <= nk - nq
            S = S.masked_fill(~seen, -math.inf)
            L = S.logsumexp(1) if nk else torch.full((nq,), -math.inf, dtype=torch.float64)
            P = torch.where(seen, (S - torch.where(L > -math.inf, L, 0.0)[:, None]).exp(), 0.0)
            e = torch.where(seen, e, 0.0)
            worst = e.amax(1, keepdim=True) if nk else torch.zeros(nq, 1, dtype=torch.float64)
            rel = e + worst + 2 * (nk + 8) * F                      # of a weight over the sum of all
            O = P @ V
            out[qs, h], lse[qs, h] = O, L
            t_out[qs, h] = (P * (u + rel)) @ V.abs() + u * O.abs() + nk * tiny * (V.abs().amax() if nk else 0.0) + 1e-30
            t_lse[qs, h] = worst[:, 0] + (nk + 8) * F + 8 * F * torch.where(L > -math.inf, L, 0.0).abs()
            # backward: with the rounded output and the 32-bit lse that the call is given
            rel = e + t_lse[qs, h][:, None] + 8 * F * torch.where(L > -math.inf, L, 0.0).abs()[:, None]
            dP = G @ V.t()
            delta = (P * dP).sum(1, keepdim=True)
            dS = P * (dP - delta)
            off_dp = (D + 2) * F * (G.abs() @ V.abs().t())
            off_delta = ((u + (D + 4) * F) * O.abs() + t_out[qs, h]) * G.abs()
            off_s = rel * dS.abs() + P * (1 + rel) * (off_dp + off_delta.sum(1, keepdim=True)) + (u + 4 * F) * dS.abs()
            low = 0.0 if dt != torch.float16 else 2.0 ** -25        # below f16's normal numbers
            off_s = torch.where(seen, off_s * (1 + u) + low, 0.0)
            dq[qs, h] = dS @ K * scale
            t_dq[qs, h] = (off_s + (nk + 4) * F * dS.abs()) @ K.abs() * scale
            off_p = torch.where(seen, P * (u + rel) + low, 0.0)
            dk[ks, j] += dS.t() @ Q * scale
            dv[ks, j] += P.t() @ G
            t_dk[ks, j] += (off_s + (nq * hq // hk + 4) * F * dS.abs()).t() @ Q.abs() * scale
            t_dv[ks, j] += (off_p + (nq * hq // hk + 4) * F * P).t() @ G.abs()
    least = {torch.float32: 1e-37, torch.float16: 2.0 ** -25, torch.bfloat16: 1e-37}[dt]
    for t, r in ((t_dq, dq), (t_dk, dk), (t_dv, dv)):
        t += u * r.abs() + least
    t_out += least
    return (out, lse, dq, dk, dv), (t_out, t_lse, t_dq, t_dk, t_dv)


def check(name, got, want, off, before=None):
    """Inside the tolerance where a scene has the row, as it was before the call elsewhere."""
    got = got.double().cpu()
    none = want.isnan()
    if before is not None:
        assert torch.equal(got[none], before.double().cpu()[none]), f"{name}: rows of no scene were written"
    empty = want == -math.inf
    assert torch.equal(got[empty], want[empty]), name
    there = ~none & ~empty
    far = ((got - want).abs() / off)[there]
    worst = float(far.max()) if far.numel() else 0.0
    print(f"{name} {worst:.3f} of its tolerance", flush=True)
    assert torch.isfinite(got[there]).all() and worst <= 1.0, (name, worst)


def data(rows, keys, hq, hk, D, dt, seed=0, together=False):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device=DEV) * scale).to(dt)
    if together:
        qkv = normal(rows, (hq + 2 * hk) * D)
        q, k, v = (part.unflatten(1, (-1, D)) for part in qkv.split([hq * D, hk * D, hk * D], 1))
    else:
        q, k, v = normal(rows, hq, D), normal(keys, hk, D), normal(keys, hk, D)
    return q, k, v, normal(rows, hq, D, scale=1 / 16)


def forward(q, k, v, *, out=None, lse=True, **kw):
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV) if out is None else out
    sums = torch.full(q.shape[:2], 7.0, device=DEV) if lse else None
    scenes = 1 if kw.get("q_starts") is None else len(kw["q_starts"]) - 1
    need = sc.sc_attention_workspace_bytes(q.shape[0], k.shape[0], scenes, q.shape[1], k.shape[1], q.shape[2], q.dtype)
    sc.sc_attention_fwd(q, k, v, out, lse=sums, workspace=torch.full((max(need, 16),), 0xff, dtype=torch.uint8, device=DEV), **kw)
    return out, sums


def backward(grad, q, k, v, out, lse, *, grads=None, **kw):
    grads = [torch.full(t.shape, 7.0, dtype=q.dtype, device=DEV) for t in (q, k, v)] if grads is None else grads
    scenes = 1 if kw.get("q_starts") is None else len(kw["q_starts"]) - 1
    need = sc.sc_attention_bwd_workspace_bytes(q.shape[0], k.shape[0], scenes, q.shape[1], k.shape[1], q.shape[2], q.dtype)
    sc.sc_attention_bwd(grad, q, k, v, out, lse, *grads, workspace=torch.full((max(need, 16),), 0xff, dtype=torch.uint8, device=DEV), **kw)
    return grads


def both(lens, key_lens, hq, hk, D, dt, causal, *, scale=None, lead=0, trail=0, seed=0, together=False):
    """Forward and backward of scenes behind `lead` rows of none and before `trail` more."""
    rows, keys = lead + sum(lens) + trail, lead + sum(key_lens) + trail
    q, k, v, grad = data(rows, keys, hq, hk, D, dt, seed, together)
    q_starts, k_starts = starts_of(lens, lead), starts_of(key_lens, lead)
    kw = dict(q_starts=q_starts, k_starts=k_starts, causal=causal, scale=scale)
    out, lse = forward(q, k, v, **kw)
    want, off = reference(q, k, v, grad, lens, key_lens, k_starts.tolist(), q_starts.tolist(), causal, D ** -0.5 if scale is None else scale, dt)
    seven = torch.full_like(want[0], 7.0)
    check("out", out, want[0], off[0], seven)
    check("lse", lse, want[1], off[1], seven[..., 0])
    grads = backward(grad, q, k, v, out, lse, **kw)
    for name, got, ref, tol in zip(("dq", "dk", "dv"), grads, want[2:], off[2:]):
        check(name, got, ref, tol, torch.full_like(ref, 7.0))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("D", [1, 8, 16, 20, 32, 33, 64, 77, 128, 130, 256])
def test_head_sizes(D, dt):
    both([37, 70], [37, 70], 2, 2, D, dt, False, together=True)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens,key_lens", [
    ([1], [1]), ([1], [300]), ([300], [1]), ([0, 5, 0], [3, 0, 0]), ([129, 0, 1, 64, 63, 65], [129, 0, 1, 64, 63, 65]),
    ([16, 17, 200], [31, 5, 333]), ([1, 2, 1, 3], [700, 513, 0, 64]), ([40, 300, 7], [300, 40, 0])])
def test_scenes(lens, key_lens, causal, dt):
    both(lens, key_lens, 4, 2, 32, dt, causal, lead=3, trail=5)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("hq,hk,D,causal", [(1, 1, 64, True), (6, 2, 40, True), (16, 1, 64, True), (7, 7, 24, False), (5, 1, 128, False), (64, 2, 16, True), (3, 1, 256, True)])
def test_heads(hq, hk, D, causal, dt):
    both([1, 90, 31], [200, 90, 31], hq, hk, D, dt, causal)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("D", [40, 128, 256])
@pytest.mark.parametrize("causal", [False, True])
def test_few_queries_over_many_keys(D, causal, dt):
    """The keys are cut into parts, forward and backward, some of which a scene does not need."""
    both([1, 2, 1], [1900, 0, 300], 4, 2, D, dt, causal)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("causal", [False, True])
def test_long_scenes(causal, dt):
    """Four wavefronts share the tiles; queries are cut into parts backward."""
    both([2500, 1, 1500], [2500, 1, 1500], 8, 4, 16, dt, causal, together=True)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("lens", [[7, 40, 0, 64, 33] * 60, [1] * 300, [0] * 100 + [50] + [0] * 100, [900] + [3] * 150, [3] * 150 + [900], [40] * 64])
def test_many_scenes(lens, dt):
    """More scenes than one search looks at."""
    both(lens, lens, 3, 3, 24, dt, False, lead=2, trail=1)

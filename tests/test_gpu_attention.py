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


@pytest.mark.parametrize("dt", TYPES)
def test_scenes_do_not_see_each_other(dt):
    """Whatever a scene holds, and whatever lies behind its last counted key, the others' results are the same, bit for bit."""
    lens, D = [50, 33, 140, 64], 24
    q, k, v, grad = data(sum(lens), sum(lens), 2, 2, D, dt, 7)
    starts = starts_of(lens)
    counts = torch.tensor([50, 20, 100, 64], dtype=torch.int32, device=DEV)
    for causal in (False, True):
        kw = dict(q_starts=starts, causal=causal, k_lens=counts)
        clean, clean_lse = forward(q, k, v, **kw)
        clean_grads = backward(grad, q, k, v, clean, clean_lse, **kw)
        bad_k, bad_v = k.clone(), v.clone()
        for a in (50 + 20, 50 + 33 + 100):          # behind the counted keys of scenes 1 and 2
            bad_k[a:a + 13], bad_v[a:a + 13] = float("nan"), float("inf")
        got, got_lse = forward(q, bad_k, bad_v, **kw)
        assert torch.equal(got, clean) and torch.equal(got_lse, clean_lse)
        for a, b in zip(backward(grad, q, bad_k, bad_v, got, got_lse, **kw), clean_grads):
            assert torch.equal(a, b)
        bad_k[:50], bad_v[:50] = float("nan"), float("inf")                      # all of scene 0
        got, _ = forward(q, bad_k, bad_v, **kw)
        assert got[:50].isnan().any() and torch.equal(got[50:], clean[50:])


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("D", [16, 64, 100])
def test_key_counts(D, dt):
    """A cache with room behind its keys: as if the keys were all there is; gradients of the others stay as they were."""
    room, counts, lens = [70, 40, 300, 5], [70, 1, 131, 0], [1, 1, 2, 1]
    q, k, v, grad = data(sum(lens), sum(room), 4, 2, D, dt, 3)
    starts, k_starts = starts_of(lens), starts_of(room)
    k_lens = torch.tensor(counts, dtype=torch.int32, device=DEV)
    kw = dict(q_starts=starts, k_starts=k_starts, k_lens=k_lens, causal=True)
    out, lse = forward(q, k, v, **kw)
    want, off = reference(q, k, v, grad, lens, counts, k_starts.tolist(), starts.tolist(), True, D ** -0.5, dt)
    check("out", out, want[0], off[0])
    check("lse", lse, want[1], off[1])
    for name, got, ref, tol in zip(("dq", "dk", "dv"), backward(grad, q, k, v, out, lse, **kw), want[2:], off[2:]):
        check(name, got, ref, tol, torch.full_like(ref, 7.0))


@pytest.mark.parametrize("dt", TYPES)
def test_large_scores(dt):
    """Scores of hundreds, the largest at the end, a constant among them: weights that grow through the tiles."""
    n, D = 700, 32
    q, k, v, grad = data(n, n, 2, 2, D, dt, 11)
    k = (k.float() * torch.linspace(0, 40, n, device=DEV)[:, None, None]).to(dt)
    out, lse = forward(q, k, v)
    want, off = reference(q, k, v, grad, [n], [n], [0], [0], False, D ** -0.5, dt)
    check("out", out, want[0], off[0])
    check("lse", lse, want[1], off[1])


@pytest.mark.parametrize("dt", TYPES)
def test_orders_of_rows_and_heads_and_unaligned_rows(dt):
    """Heads ahead of rows, rows that start anywhere, gradients into slices: the same values as contiguous tensors give, bit for bit."""
    n, h, D = 130, 3, 40
    q, k, v, grad = data(n, n, h, h, D, dt, 5)
    kw = dict(q_starts=starts_of([60, 70]), causal=True)
    out, lse = forward(q, k, v, **kw)
    grads = backward(grad, q, k, v, out, lse, **kw)
    heads_first = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v, grad)]
    odd = []
    for t in (q, k, v, grad):
        wide = torch.full((n, h, D + 3), float("nan"), dtype=dt, device=DEV)
        wide[:, :, 1:1 + D] = t
        odd.append(wide[:, :, 1:1 + D])
    for a, b, c, g in (heads_first, odd):
        there = torch.full((h, n, D), 7.0, dtype=dt, device=DEV).transpose(0, 1)
        got, got_lse = forward(a, b, c, out=there, **kw)
        assert torch.equal(got, out) and torch.equal(got_lse, lse)
        wide = [torch.full((n, h, D + 5), 7.0, dtype=dt, device=DEV) for _ in range(3)]
        backward(g, a, b, c, got, got_lse, grads=[w[:, :, 2:2 + D] for w in wide], **kw)
        for w, want in zip(wide, grads):
            assert torch.equal(w[:, :, 2:2 + D], want) and (w[:, :, :2] == 7).all() and (w[:, :, 2 + D:] == 7).all()
    # one head of keys for all, and rows that are one row
    shared = k[:, :1].expand(n, h, D)
    one, one_lse = forward(q, shared, v[:, :1].expand(n, h, D), **kw)
    want, want_lse = forward(q, k[:, :1].contiguous(), v[:, :1].contiguous(), **kw)
    assert (one.float() - want.float()).abs().max() <= 8 * torch.finfo(dt).eps * want.float().abs().max() and torch.allclose(one_lse, want_lse, atol=1e-4)


def test_gradient_against_differences():
    """f32: a directional derivative of sum(out * grad) against central differences of the 64-bit definition."""
    lens, D = [20, 35], 16
    q, k, v, grad = data(sum(lens), sum(lens), 2, 1, D, torch.float32, 9)
    kw = dict(q_starts=starts_of(lens), causal=True)
    out, lse = forward(q, k, v, **kw)
    grads = backward(grad, q, k, v, out, lse, **kw)
    gen = torch.Generator().manual_seed(1)
    steps = [torch.randn(t.shape, generator=gen, dtype=torch.float64) for t in (q, k, v)]

    def value(h):
        moved = [t.double().cpu() + h * s for t, s in zip((q, k, v), steps)]
        total, at = 0.0, 0
        for n in lens:
            m = slice(at, at + n)
            at += n
            for head in range(2):
                s = (moved[0][m, head] @ moved[1][m, 0].t() * D ** -0.5).masked_fill(torch.ones(n, n).triu(1).bool(), -math.inf)
                total += float((s.softmax(1) @ moved[2][m, 0] * grad[m, head].double().cpu()).sum())
        return total
    want = (value(1e-4) - value(-1e-4)) / 2e-4
    got = sum(float((g.double().cpu() * s).sum()) for g, s in zip(grads, steps))
    assert abs(got - want) <= 1e-4 * max(1.0, abs(want)), (got, want)         # differences: h^2; 32 bits: some 1e-6 of terms that add up to a few


def test_repeated_streams_and_graphs():
    """The same bits every time: on another stream, and in two captured graphs that share a workspace, replayed between eager calls."""
    lens = [700, 3, 260]
    q, k, v, grad = data(sum(lens), sum(lens), 8, 2, 64, torch.bfloat16, 13)
    starts = starts_of(lens)
    args = (sum(lens), sum(lens), 3, 8, 2, 64, torch.bfloat16)
    need = max(sc.sc_attention_workspace_bytes(*args), sc.sc_attention_bwd_workspace_bytes(*args), 16)
    workspace = torch.empty(need, dtype=torch.uint8, device=DEV)
    kw = dict(q_starts=starts, causal=True, workspace=workspace)

    def step(q, out, lse, grads):
        sc.sc_attention_fwd(q, k, v, out, lse=lse, **kw)
        sc.sc_attention_bwd(grad, q, k, v, out, lse, *grads, **kw)

    def buffers():
        return torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV), [torch.zeros_like(t) for t in (q, k, v)]
    want = buffers()
    step(q, *want)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    there = buffers()
    torch.cuda.synchronize()
    with torch.cuda.stream(other):
        step(q, *there)
    torch.cuda.synchronize()
    for a, b in zip((there[0], there[1], *there[2]), (want[0], want[1], *want[2])):
        assert torch.equal(a, b)
    inputs = [q.clone(), q.clone()]
    held, graphs = [buffers(), buffers()], []
    for x, b in zip(inputs, held):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(x, *b)
        graphs.append(graph)
    for turn in range(3):
        inputs[1].copy_(q * (1 + turn))
        for graph, x, b in zip(graphs, inputs, held):
            for t in (b[0], b[1], *b[2]):
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            eager = buffers()
            step(x, *eager)
            torch.cuda.synchronize()
            for s, t in zip((b[0], b[1], *b[2]), (eager[0], eager[1], *eager[2])):
                assert torch.equal(s, t)


def test_nothing_to_do():
    for rows, keys in ((0, 5), (5, 0), (0, 0)):
        q, k, v, grad = data(rows, keys, 2, 2, 16, torch.float16)
        out, lse = forward(q, k, v)
        assert (out == 0).all() and (lse == -math.inf).all()
        for g in backward(grad, q, k, v, out, lse):
            assert (g == 0).all()


@pytest.mark.parametrize("which", ["dq", "dk"])
@pytest.mark.parametrize("lens", [[4000], [30] * 40])
def test_small_gradients_in_f16(lens, which):
    """Gradients of scores far below f16's normal numbers (2^-14) whose sums are not: some 2^-20 here.  Of a random sum each of whose terms is rounded by half a step at
    most, and which is rounded once, the error is within 2 half steps of its size in the mean square; a term that was rounded as a number of 2^-20, in steps of 2^-24, would be off by a 64th."""
    n, D = sum(lens), 32
    q, k, v, grad = data(n, n, 2, 2, D, torch.float16, 17)
    wide, narrow = (k, q) if which == "dq" else (q, k)
    wide.mul_(32), narrow.mul_(1 / 32)
    grad.mul_(2.0 ** -6 if len(lens) == 1 else 2.0 ** -11)
    grad[0] *= 16                                   # a row of larger ones among them
    starts = starts_of(lens)
    kw = dict(q_starts=starts)
    out, lse = forward(q, k, v, **kw)
    got = backward(grad, q, k, v, out, lse, **kw)[0 if which == "dq" else 1]
    want = torch.zeros(n, 2, D, dtype=torch.float64)
    at = 0
    for m in lens:
        s = slice(at, at + m)
        at += m
        for h in range(2):
            Q, K, V, G = (t[s, h].double().cpu() for t in (q, k, v, grad))
            P = (Q @ K.t() * D ** -0.5).softmax(1)
            dP = G @ V.t()
            dS = P * (dP - (G * out[s, h].double().cpu()).sum(1, keepdim=True)) * D ** -0.5      # of the output as it was given
            want[s, h] = dS @ K if which == "dq" else dS.t() @ Q
    rel = float((got.double().cpu() - want).norm() / want.norm())
    print(f"{rel:.1e}", flush=True)
    assert rel <= 2 * 2.0 ** -11


@pytest.mark.parametrize("which", ["dq", "dk"])
@pytest.mark.parametrize("n", [300, 4000])
@pytest.mark.parametrize("wide", [1, 32])
def test_small_gradients_in_f16_behind_vanishing_ones(n, which, wide):
    """As above, behind 64 rows whose weights are some e^-85, whose gradients are hardly numbers of 32 bits.  The bound is that of the test above, and half a step of f16
    where results are below 2^-14 (all steps there are 2^-24): without the factor of 32 some 10^-5 here."""
    D = 32
    q, k, v, grad = data(n, n, 2, 2, D, torch.float16, 19)
    grad.mul_(2.0 ** -6 if n == 4000 else 2.0 ** -10)
    summed, other = (k, q) if which == "dq" else (q, k)
    summed.mul_(wide), other.mul_(1 / wide)
    q[..., 0], k[..., 0] = 0, 0
    if which == "dq":
        q[..., 0], k[:64, :, 0] = 16, -30           # keys that no query has a weight for
    else:
        q[:64, :, 0], k[-1, :, 0] = 16, 30          # queries that have a weight for the last key only
    out, lse = forward(q, k, v)
    got = backward(grad, q, k, v, out, lse)[0 if which == "dq" else 1].double().cpu()
    want = torch.zeros(n, 2, D, dtype=torch.float64)
    for h in range(2):
        Q, K, V, G, O = (t[:, h].double().cpu() for t in (q, k, v, grad, out))
        P = (Q @ K.t() * D ** -0.5).softmax(1)
        dS = P * (G @ V.t() - (G * O).sum(1, keepdim=True)) * D ** -0.5
        want[:, h] = dS @ K if which == "dq" else dS.t() @ Q
    got, want = got[:-1], want[:-1]                 # of the last key dP is delta but for roundings
    error, bound = float((got - want).norm()), 2 * 2.0 ** -11 * float(want.norm()) + float((want.abs() < 2.0 ** -14).double().sum().sqrt()) * 2.0 ** -25
    print(f"{error / float(want.norm()):.1e} {error / bound:.2f}", flush=True)
    assert error <= bound


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("below", [20, 30, 60])
@pytest.mark.parametrize("lens,key_lens,heads,D", [
    ([10], [10], 2, 16), ([37, 10, 130, 1], [37, 10, 130, 1], 2, 64), ([1, 33, 2], [130, 37, 10], 2, 64), ([1037], [1037], 8, 64), ([2437], [2437], 4, 16)])
def test_scores_far_below_zero(lens, key_lens, heads, D, below, causal, dt):
    """All scores some 20 to 60 below zero, which softmax does not feel: a weight against such a sum that belongs to no key would be e^20 to e^60.  Wavefronts
    alone, shared tiles, and queries in parts; the last block of keys is never full, and is seen whole by single rows behind a causal mask."""
    q, k, v, grad = data(sum(lens), sum(key_lens), heads, heads, D, dt, 23)
    q[..., 0], k[..., 0] = 16, -below * D ** 0.5 / 16
    starts, k_starts = starts_of(lens), starts_of(key_lens)
    kw = dict(q_starts=starts, k_starts=k_starts, causal=causal)
    out, lse = forward(q, k, v, **kw)
    want, off = reference(q, k, v, grad, lens, key_lens, k_starts.tolist(), starts.tolist(), causal, D ** -0.5, dt)
    check("out", out, want[0], off[0])
    check("lse", lse, want[1], off[1])
    for name, got, ref, tol in zip(("dq", "dk", "dv"), backward(grad, q, k, v, out, lse, **kw), want[2:], off[2:]):
        check(name, got, ref, tol)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("lens", [[60, 70], [1, 2, 1], [2100]])
def test_outputs_between_and_in_place_of_operands(lens, dt):
    """Queries, keys and values, and their gradients, one head of each behind the other; results in the place of rows that nothing else reads.  The same bits as in tensors of their own."""
    n, h, D = sum(lens), 4, 16
    q, k, v, grad = data(n, n, h, h, D, dt, 29)
    kw = dict(q_starts=starts_of(lens), causal=True)
    out, lse = forward(q, k, v, **kw)
    grads = backward(grad, q, k, v, out, lse, **kw)
    between, there = torch.stack([q, k, v], 2), torch.full((n, h, 3, D), 7.0, dtype=dt, device=DEV)
    got, got_lse = forward(*between.unbind(2), **kw)
    assert torch.equal(got, out) and torch.equal(got_lse, lse)
    backward(grad, *between.unbind(2), got, lse, grads=list(there.unbind(2)), **kw)
    for a, b in zip(there.unbind(2), grads):
        assert torch.equal(a, b)
    x, y, z = k.clone(), v.clone(), out.clone()
    backward(grad, q, x, y, z, lse, grads=[z, x, y], **kw)
    for a, b in zip((z, x, y), grads):
        assert torch.equal(a, b)
    x = q.clone()
    forward(x, k, v, out=x, **kw)
    assert torch.equal(x, out)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("scale", [1e-45, sc.SC_ATTENTION_SCALE_MAX])
def test_least_and_largest_scale(scale, dt):
    """Scores of zero are zero whatever they are scaled by: every row gets the mean of the values, and the logarithm of their number."""
    lens = [40, 1, 130]
    q, k, v, grad = data(sum(lens), sum(lens), 2, 2, 20, dt, 31)
    kw = dict(q_starts=starts_of(lens), scale=scale)
    out, lse = forward(q * 0, k, v, **kw)
    want, off = reference(q * 0, k, v, grad, lens, lens, kw["q_starts"].tolist(), kw["q_starts"].tolist(), False, 1.0, dt)
    check("out", out, want[0], off[0])
    check("lse", lse, want[1], off[1])


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("lens,more,heads,D", [([130], 1, 1, 32), ([200, 180], 33, 8, 32), ([100] * 10, 1, 8, 32), ([95] * 80, 1, 8, 32), ([1300], 1, 30, 64), ([1300], 5, 30, 64), ([260], 64, 2, 256)])
def test_values_that_are_not_finite_behind_a_causal_mask(lens, more, heads, D, dt):
    """Queries that are further from them than SC_ATTENTION_REACH keys, the columns of a wavefront and the rest of a tile, do not feel them.  `more` keys than queries, so that
    what a wavefront's rows see does not end with tiles; few columns, wavefronts alone with 32 and 64, shared tiles."""
    key_lens = [n + more for n in lens]
    q, k, v, _ = data(sum(lens), sum(key_lens), heads, heads, D, dt, 37)
    starts, k_starts = starts_of(lens), starts_of(key_lens)
    kw = dict(q_starts=starts, k_starts=k_starts, causal=True)
    clean, clean_lse = forward(q, k, v, **kw)
    furthest = 0
    for place in (more, 31, 63, 64, 95, 127, 1023, min(key_lens) - 1):             # the key of every scene; the ends of tiles
        if not more <= place < min(key_lens):
            continue
        bad = v.clone()
        for at in k_starts.tolist()[:-1]:
            bad[at + place] = float("inf")
        got, lse = forward(q, k, bad, **kw)
        assert torch.equal(lse, clean_lse)
        for at, n in zip(starts.tolist(), lens):
            mine = slice(at, at + n)
            assert not got[mine][place - more:].isfinite().any(), "queries that see it"
            reached = (got[mine] != clean[mine]).flatten(1).any(1)
            furthest = max(furthest, place - more - int(reached.nonzero()[0]))     # from the last key that the query sees
    print(f"{furthest} keys behind", flush=True)
    assert furthest <= sc.SC_ATTENTION_REACH


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("hk,D", [(2, 64), (1, 128)])
def test_sequences_of_many_rows(hk, D, causal, dt):
    """20004 rows in two scenes, heads that share keys, all gradients.  Each result is a sum of terms that are rounded by half a step at most, and is rounded once, so as of a random sum its
    error is within 2 half steps of its size in the mean square."""
    lens, hq = [14001, 6003], 4
    q, k, v, grad = data(sum(lens), sum(lens), hq, hk, D, dt, 41)
    kw = dict(q_starts=starts_of(lens), causal=causal)
    out, lse = forward(q, k, v, **kw)
    got = [out, *backward(grad, q, k, v, out, lse, **kw)]
    want, at = [torch.zeros(t.shape, dtype=torch.float64, device=DEV) for t in got], 0
    for n in lens:
        rows = slice(at, at + n)
        at += n
        for h in range(hq):
            j = h // (hq // hk)
            Q, K, V, G = q[rows, h].double(), k[rows, j].double(), v[rows, j].double(), grad[rows, h].double()
            P = Q @ K.t() * D ** -0.5
            if causal:
                P = P.masked_fill_(torch.ones((n, n), dtype=torch.bool, device=DEV).triu_(1), -math.inf)
            P = P.softmax(1)
            dS = G @ V.t()
            dS = P * dS.sub_((P * dS).sum(1, keepdim=True)) * D ** -0.5
            want[0][rows, h] = P @ V
            want[1][rows, h] = dS @ K
            want[2][rows, j] += dS.t() @ Q
            want[3][rows, j] += P.t() @ G
    for name, a, b in zip(("out", "dq", "dk", "dv"), got, want):
        rel = float((a.double() - b).norm() / b.norm())
        print(f"{name} {rel:.1e}", flush=True)
        assert rel <= 2 * half_step(dt), name

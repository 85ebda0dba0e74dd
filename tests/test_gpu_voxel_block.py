"""GPU test of the example block: its output and every gradient, in f32, against the same block written with dense products and
differentiated in 64 bits on the CPU; and its steps in 16 bits go downhill."""
import importlib.util
import os

import pytest
import torch

from paper_2402_07710_amd import synth

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("voxel_block", os.path.join(ROOT, "examples", "voxel_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def scenes(sizes):
    parts = []
    for b, n in enumerate(sizes):
        c = torch.from_numpy(synth.lidar_scene(b)[:n]).clone()
        c[:, 0] = b
        parts.append(c)
    return torch.cat(parts).to(torch.int32)


def plain(block, module, coords, x, params):
    """The block in 64 bits: dense products over explicit neighbours."""
    n, C, H, D = len(coords), block.C, block.H, block.D
    index = {tuple(c): i for i, c in enumerate(coords.tolist())}
    y = torch.zeros(n, C, dtype=torch.float64)
    for k in range(27):
        d = (k // 9 - 1, k // 3 % 3 - 1, k % 3 - 1)
        pairs = [(index.get((b, X + d[0], Y + d[1], Z + d[2]), -1), i) for i, (b, X, Y, Z) in enumerate(coords.tolist())]
        pairs = [(i, o) for i, o in pairs if i >= 0]
        if pairs:
            i, o = torch.tensor(pairs).t()
            y = y.index_add(0, o, x[i] @ params["conv"][k])
    qkv = y @ params["w_qkv"] + params["b_qkv"]
    q, k, v = (t.unflatten(1, (H, D)) for t in qkv.split(C, 1))
    sections = (D // 2 - 2 * (D // 6), D // 6, D // 6)
    angle = torch.cat([coords[:, 1 + a, None].double() * module.BASE ** (-torch.arange(m, dtype=torch.float64) / m) for a, m in enumerate(sections)], 1)[:, None]

    def turned(t, gain):
        t = t / torch.sqrt(t.square().mean(-1, keepdim=True) + module.EPS) * gain
        a, b = t[..., :D // 2], t[..., D // 2:]
        return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1)
    q, k = turned(q, params["gain_q"]), turned(k, params["gain_k"])
    o = []
    for b in range(int(coords[:, 0].max()) + 1):
        m = coords[:, 0] == b
        state = torch.einsum("nhd,nhe->hde", k[m], v[m]) / max(1, int(m.sum()))
        o.append(torch.einsum("nhd,hde->nhe", q[m], state))
    u = torch.cat(o).flatten(1) @ params["w_o"] + params["b_o"] + y
    expert = (coords[:, 3].long() * block.E // 41).clamp(max=block.E - 1)
    mixed = torch.zeros_like(u)
    for e in range(block.E):
        m = (expert == e).nonzero()[:, 0]
        hidden = torch.nn.functional.gelu(u[m] @ params["w_1"][e] + params["b_1"][e])
        mixed = mixed.index_add(0, m, hidden @ params["w_2"][e] + params["b_2"][e])
    return u + mixed


def test_block_against_64_bits():
    module = example()
    coords = scenes([700, 300, 401])
    block = module.VoxelBlock(coords.to("cuda:0"), 32, 2, 4, torch.float32, seed=3)
    gen = torch.Generator()
    gen.manual_seed(4)
    x, grad = torch.randn(len(coords), 32, generator=gen), torch.randn(len(coords), 32, generator=gen)
    z = block.forward(x.to("cuda:0"))
    d_x = block.backward(grad.to("cuda:0"))
    params = {name: p.double().cpu().requires_grad_(True) for name, p in block.params.items()}
    x64 = x.double().requires_grad_(True)
    want = plain(block, module, coords, x64, params)
    want.backward(grad.double())
    # six layers in a row of f32 sums of at most 700 terms: each off by 1e-6 of its largest value or so, passed on by the others' norms
    for name, got, ref in [("z", z, want.detach()), ("x", d_x, x64.grad)] + [(name, block.grads[name], p.grad) for name, p in params.items()]:
        err = float((got.double().cpu() - ref).abs().max() / ref.abs().max())
        print(name, f"{err:.1e}", flush=True)
        assert err < 1e-4, (name, err)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_block_learns(dtype):
    module = example()
    coords = scenes([3000, 2000]).to("cuda:0")
    block = module.VoxelBlock(coords, 64, 4, 8, dtype)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(5)
    x, target = (torch.randn((len(coords), 64), generator=gen, device="cuda:0").to(dtype) for _ in range(2))
    losses = []
    for _ in range(6):
        diff = (block.forward(x) - target).float()
        losses.append(float((diff * diff).mean()))
        block.backward((2.0 * diff / 64).to(dtype))
        for name, p in block.params.items():
            g = block.grads[name].float()
            assert torch.isfinite(g).all(), name
            step = 0.02 * p.float().square().mean().sqrt().clamp(min=0.01) * g / (g.square().mean().sqrt() + 1e-12)
            p.copy_((p.float() - step).to(dtype))
    print(losses, flush=True)
    assert losses[-1] < losses[0]

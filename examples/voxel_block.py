"""A block of a voxel network that learns: a sparse convolution, attention over the voxels of each scene, and experts.

    y = conv(x)                                       3x3x3 submanifold convolution over a kernel map
        (norm)  silu(group norm of it) per scene
    q, k, v = y W_qkv + b_qkv                         linear layer
    q, k    = rotate(norm(q)), rotate(norm(k))        per head, by the voxel's three coordinates
    o       = q (k^T v / n)  per scene and head       attention without softmax: grouped products, the scenes are the groups
        (softmax)  softmax(q k^T / sqrt(D)) v         the scenes packed one behind the other
    u = o W_o + b_o + y                               linear layer with residual
    z = u + experts(u)                                two grouped products, rows dealt by the voxels' height

The convolution's weight gradient is a grouped product as well: the pairs of its rulebook, grouped by kernel offset.

    python examples/voxel_block.py [--voxels N] [--steps S] [--dtype bf16] [--attention softmax] [--norm 8]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2402_07710_amd import binding as sc  # noqa: E402
from paper_2402_07710_amd import synth  # noqa: E402

EPS, BASE = 1e-5, 100.0


class VoxelBlock:
    """Weights, the buffers of one set of voxels, and the two passes over them.  `coords` int32 [n, 4] (b, x, y, z), the
    voxels of a scene together.  attention: "linear" or "softmax"; norm_groups: groups of channels that are normalised behind
    the convolution, 0: none."""

    def __init__(self, coords, channels, heads, experts, dtype, seed=0, attention="linear", norm_groups=0):
        n, dev = coords.shape[0], coords.device
        self.coords, self.n, self.C, self.H, self.D, self.E, self.dtype = coords, n, channels, heads, channels // heads, experts, dtype
        self.softmax, self.G = {"linear": False, "softmax": True}[attention], norm_groups
        gen = torch.Generator()
        gen.manual_seed(seed)

        def weight(*shape):
            return (torch.randn(shape, generator=gen) / shape[-2] ** 0.5).to(dev, dtype)

        def zeros(*shape):
            return torch.zeros(shape, dtype=dtype, device=dev)
        C, D, E = channels, self.D, experts
        self.params = {"conv": weight(27, C, C) * 0.3, "w_qkv": weight(C, 3 * C), "b_qkv": zeros(3 * C), "gain_q": zeros(D) + 1, "gain_k": zeros(D) + 1,
                       "w_o": weight(C, C), "b_o": zeros(C), "w_1": weight(E, C, 2 * C), "b_1": zeros(E, 2 * C), "w_2": weight(E, 2 * C, C), "b_2": zeros(E, C)}
        if norm_groups:
            self.params.update(gain_y=zeros(C) + 1, bias_y=zeros(C))
        self.grads = {name: torch.empty_like(p) for name, p in self.params.items()}
        # kernel map of the convolution and its rulebook, groups of scenes and of experts: the voxels' alone
        self.map = sc.LayerBuffers(n, 3, 1, "subm", C, C, dtype, device=dev)
        self.map.hash_build(coords)
        self.map.kmap_build(coords)
        self.pairs_in, self.pairs_out, self.offsets = self.map.export()
        scene = coords[:, 0].long()
        sizes = torch.bincount(scene)
        self.scenes = torch.cat([sizes.new_zeros(1), sizes.cumsum(0)]).to(torch.int32)
        self.per_scene = (1.0 / sizes.clamp(min=1)).to(dtype)[:, None, None]
        expert = (coords[:, 3].long() * E // 41).clamp(max=E - 1)
        self.rows = expert.sort(stable=True).indices.to(torch.int32)
        self.experts = torch.cat([expert.new_zeros(1), torch.bincount(expert, minlength=E).cumsum(0)]).to(torch.int32)
        self.table = sc.sc_rope_table(D, (D // 2 - 2 * (D // 6), D // 6, D // 6), BASE, device=dev)
        need = max(sc.sc_grouped_workspace_bytes(len(self.pairs_in), 27, C, C, dtype), sc.sc_grouped_workspace_bytes(n, E, C, 2 * C, dtype),
                   sc.sc_grouped_workspace_bytes(n, E, 2 * C, C, dtype), sc.sc_grouped_workspace_bytes(n, len(sizes), D, D, dtype),
                   sc.sc_linear_workspace_bytes(n, C, 3 * C, dtype), sc.sc_linear_workspace_bytes(n, C, C, dtype),
                   sc.sc_qk_rope_workspace_bytes(n, heads, heads, D), 16)
        if self.softmax:
            sizes = (n, n, len(self.scenes) - 1, heads, heads, D, dtype)
            need = max(need, sc.sc_attention_workspace_bytes(*sizes), sc.sc_attention_bwd_workspace_bytes(*sizes))
            self.lse = torch.empty((n, heads), device=dev)
        if norm_groups:
            need = max(need, sc.sc_group_norm_workspace_bytes(n, len(self.scenes) - 1, C, norm_groups))
            self.stats = torch.empty((len(self.scenes) - 1, norm_groups, 2), device=dev)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        rows = lambda c: torch.empty((n, c), dtype=dtype, device=dev)      # noqa: E731
        self.y, self.qkv, self.o, self.u = rows(C), rows(3 * C), rows(C), rows(C)
        self.q, self.k = rows(C).unflatten(1, (heads, D)), rows(C).unflatten(1, (heads, D))
        self.hidden, self.pre, self.mixed = rows(2 * C), rows(2 * C), rows(C)
        self.c, self.d_c = (rows(C), rows(C)) if norm_groups else (self.y, None)      # behind the convolution
        self.states = torch.empty((heads, len(sizes), D, D), dtype=dtype, device=dev)
        self.d_hidden, self.d_rows, self.d_o, self.d_qkv, self.d_y = rows(2 * C), rows(C), rows(C), rows(3 * C), rows(C)
        self.d_q, self.d_k = rows(C).unflatten(1, (heads, D)), rows(C).unflatten(1, (heads, D))

    def heads_of(self, qkv):
        """Queries, keys, values [n, H, D], views of the projection's rows."""
        return [part.unflatten(1, (self.H, self.D)) for part in qkv.split(self.C, 1)]

    def forward(self, x):
        p, self.x = self.params, x
        sc.sc_conv_fwd(x, p["conv"], self.c, self.map.kmap, self.map.counts, 3, 1, "subm", self.map.workspace)
        if self.G:
            sc.sc_group_norm_fwd(self.c, self.y, self.G, self.scenes, p["gain_y"], p["bias_y"], "silu", EPS, self.stats, self.workspace)
        sc.sc_linear_fwd(self.y, p["w_qkv"], self.qkv, bias=p["b_qkv"])
        q, k, v = self.heads_of(self.qkv)
        sc.sc_qk_rope_fwd(q, k, self.coords[:, 1:], self.table, self.q, self.k, gain_q=p["gain_q"], gain_k=p["gain_k"], eps=EPS)
        if self.softmax:
            sc.sc_attention_fwd(self.q, self.k, v, self.o.unflatten(1, (self.H, self.D)), self.scenes, lse=self.lse, workspace=self.workspace)
        for h in range(0 if self.softmax else self.H):
            sc.sc_grouped_bwd(v[:, h], self.k[:, h], None, self.scenes, grad_weight=self.states[h], workspace=self.workspace)     # k^T v of every scene
            self.states[h] *= self.per_scene
            sc.sc_grouped_fwd(self.q[:, h], self.states[h], self.scenes, self.o.unflatten(1, (self.H, self.D))[:, h])
        sc.sc_linear_fwd(self.o, p["w_o"], self.u, bias=p["b_o"], residual=self.y)
        sc.sc_grouped_fwd(self.u, p["w_1"], self.experts, self.hidden, rows=self.rows, bias=p["b_1"], act="gelu", pre=self.pre)
        sc.sc_grouped_fwd(self.hidden, p["w_2"], self.experts, self.mixed, bias=p["b_2"])
        return self.u.index_add(0, self.rows, self.mixed)

    def backward(self, grad):
        """Fills self.grads and returns the gradient of x."""
        p, g, ws = self.params, self.grads, self.workspace
        sc.sc_grouped_bwd(grad, self.hidden, p["w_2"], self.experts, grad_x=self.d_hidden, grad_weight=g["w_2"], grad_bias=g["b_2"], grad_rows=self.rows,
                          workspace=ws)
        sc.sc_grouped_bwd(self.d_hidden, self.u, p["w_1"], self.experts, grad_x=self.d_rows, grad_weight=g["w_1"], grad_bias=g["b_1"], rows=self.rows,
                          pre=self.pre, act="gelu", workspace=ws)
        d_u = grad.index_add(0, self.rows, self.d_rows)
        sc.sc_linear_bwd(d_u, self.o, p["w_o"], grad_x=self.d_o, grad_weight=g["w_o"], grad_bias=g["b_o"], workspace=ws)
        q, k, v = self.heads_of(self.qkv)
        d_q, d_k, d_v = self.heads_of(self.d_qkv)
        d_o, d_state = self.d_o.unflatten(1, (self.H, self.D)), torch.empty_like(self.states[0])
        if self.softmax:
            sc.sc_attention_bwd(d_o, self.q, self.k, v, self.o.unflatten(1, (self.H, self.D)), self.lse, self.d_q, self.d_k, d_v, self.scenes, workspace=ws)
        for h in range(0 if self.softmax else self.H):
            sc.sc_grouped_bwd(d_o[:, h], self.q[:, h], self.states[h], self.scenes, grad_x=self.d_q[:, h], grad_weight=d_state, workspace=ws)
            d_state *= self.per_scene
            sc.sc_grouped_bwd(v[:, h], v[:, h], d_state, self.scenes, grad_x=self.d_k[:, h], workspace=ws)       # v d_state^T
            sc.sc_grouped_fwd(self.k[:, h], d_state, self.scenes, d_v[:, h])
        sc.sc_qk_rope_bwd(self.d_q, self.d_k, q, k, self.coords[:, 1:], self.table, d_q, d_k, gain_q=p["gain_q"], gain_k=p["gain_k"],
                          grad_gain_q=g["gain_q"], grad_gain_k=g["gain_k"], eps=EPS, workspace=ws)
        sc.sc_linear_bwd(self.d_qkv, self.y, p["w_qkv"], grad_x=self.d_y, grad_weight=g["w_qkv"], grad_bias=g["b_qkv"], workspace=ws)
        d_y = self.d_y + d_u
        if self.G:
            sc.sc_group_norm_bwd(d_y, self.c, self.stats, self.d_c, self.G, self.scenes, p["gain_y"], p["bias_y"], "silu", g["gain_y"], g["bias_y"], ws)
            d_y = self.d_c
        sc.sc_grouped_bwd(d_y, self.x, None, self.offsets, grad_weight=g["conv"], rows=self.pairs_in, grad_rows=self.pairs_out, workspace=ws)
        # offset 26 - k leads back where offset k came from
        turned = p["conv"].flip(0).transpose(1, 2).contiguous()
        d_x = torch.empty_like(self.x)
        sc.sc_conv_fwd(d_y, turned, d_x, self.map.kmap, self.map.counts, 3, 1, "subm", self.map.workspace)
        return d_x


def main():
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--voxels", type=int, default=53373)
    parser.add_argument("--steps", type=int, default=5)
    parser.add_argument("--dtype", choices=["f32", "bf16", "f16"], default="bf16")
    parser.add_argument("--attention", choices=["linear", "softmax"], default="linear")
    parser.add_argument("--norm", type=int, default=0, help="groups of channels normalised behind the convolution")
    args = parser.parse_args()
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[args.dtype]
    scenes, n, b = [], 0, 0
    while n < args.voxels:
        coords = torch.from_numpy(synth.lidar_scene(b))[:args.voxels - n].clone()
        coords[:, 0] = b
        scenes.append(coords)
        n, b = n + len(coords), b + 1
    coords = torch.cat(scenes).to("cuda:0", torch.int32)
    block = VoxelBlock(coords, 64, 4, 8, dtype, attention=args.attention, norm_groups=args.norm)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(1)
    x = torch.randn((n, 64), generator=gen, device="cuda:0").to(dtype)
    target = torch.randn((n, 64), generator=gen, device="cuda:0").to(dtype)
    for step in range(args.steps):
        diff = (block.forward(x) - target).float()
        print(f"step {step}: {n} voxels in {b} scenes, loss {float((diff * diff).mean()):.4f}", flush=True)
        block.backward((2.0 * diff / 64).to(dtype))
        for name, p in block.params.items():            # a step of a fiftieth of the weights' size along the gradient
            g, size = block.grads[name].float(), p.float().square().mean().sqrt().clamp(min=0.01)
            p.copy_((p.float() - 0.02 * size * g / (g.square().mean().sqrt() + 1e-12)).to(dtype))


if __name__ == "__main__":
    main()

"""Encode a scene once, then look new images up in it: a stack of attention layers over a kept scene.

    python -m paper_2511_21317_b200.run_lookup [--workload small] [--layers 4] [--images 2] [--steps 3] [--page-size 128]

The scene's frames run through the layers of run_stack (x <- x + W_o . Attn(split(W_qkv . rmsnorm(x))), the attention with head-wise
token merging), with per-head layer norms of queries and keys and the 2-D rotation by patch position in front of the attention; every
layer's keys and values go to the pages of a cache.  Then a batch of images that drift on from the scene's last frame runs through the same layers:
their keys (normed and rotated on the way) and values are appended behind the scene, and each image attends to all of the scene and to itself.
The projections are the library's own GEMM.  Prints one JSON line: the time of encoding, and of looking the images up.
"""
from __future__ import annotations

import argparse
import json
import sys

import torch

from . import binding as hb
from . import kv_cache as kc
from . import synth
from .run_stack import rmsnorm, timed


def patch_positions(wl, frames: int, device: str) -> torch.Tensor:
    """(row, column) of every token of `frames` frames: 0 for special tokens, counted from 1 for patches."""
    p = torch.zeros(wl.tokens_per_frame, 2, dtype=torch.int32, device=device)
    p[wl.n_special:, 0] = torch.arange(wl.grid_h, device=device).repeat_interleave(wl.grid_w) + 1
    p[wl.n_special:, 1] = torch.arange(wl.grid_w, device=device).repeat(wl.grid_h) + 1
    return p.repeat(frames, 1)


class Lookup:
    def __init__(self, wl, layers: int, images: int, page_size: int = 128, device: str = "cuda:0", seed: int = 0):
        self.wl, self.layers, self.images, self.device = wl, layers, images, device
        self.H, self.D = wl.heads, wl.head_dim
        dim = self.H * self.D
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, scale):
            return torch.randn(*shape, generator=g, device=device) * scale

        self.w_qkv = [normal(3 * dim, dim, scale=0.02).to(torch.bfloat16) for _ in range(layers)]
        self.w_o = [normal(dim, dim, scale=0.02).to(torch.bfloat16) for _ in range(layers)]
        self.norms = [{"q_weight": 1.0 + normal(self.D, scale=0.1), "k_weight": 1.0 + normal(self.D, scale=0.1), "q_bias": normal(self.D, scale=0.05),
                       "k_bias": normal(self.D, scale=0.05)} for _ in range(layers)]
        # the scene's frames and, drifting on, the images
        every = wl.replace(frames=wl.frames + images)
        x = hb.bf16_from_bits(synth.make_qkv(every)[0], device).permute(1, 0, 2).reshape(every.n_tokens, dim)
        self.x_scene, self.x_images = x[:wl.n_tokens].contiguous(), x[wl.n_tokens:].contiguous()
        self.ctx = hb.Httm(hb.HttmConfig.of(wl))
        self.rotary = kc.Rotary(head_dim=self.D, n_positions=max(wl.grid_h, wl.grid_w) + 1, axes=2, base=100.0, norm="layer")
        self.pos_scene, self.pos_images = patch_positions(wl, wl.frames, device), patch_positions(wl, images, device)
        # pages: the scene's, then those of every image
        per_image = wl.tokens_per_frame
        n_scene, n_image = -(-wl.n_tokens // page_size), -(-per_image // page_size)
        scene_pages = list(range(n_scene))
        tables = [list(range(n_scene + i * n_image, n_scene + (i + 1) * n_image)) for i in range(images)]
        n_pages = n_scene + images * n_image
        shape = (n_pages, self.H, page_size, self.D)
        self.caches = [kc.KvCache(*(torch.zeros(shape, dtype=torch.bfloat16, device=device) for _ in range(2))) for _ in range(layers)]
        args = dict(heads=self.H, kv_heads=self.H, head_dim=self.D, page_size=page_size, n_pages=n_pages, causal=False)
        self.scene_batch = kc.CacheBatch(**args).set([scene_pages], [wl.n_tokens], [wl.n_tokens])
        self.image_batch = kc.CacheBatch(**args).set(tables, [per_image] * images, [per_image] * images, scene_pages, wl.n_tokens)
        n = max(wl.n_tokens, images * per_image)
        self.qkv = torch.empty(n, 3 * dim, dtype=torch.bfloat16, device=device)
        self.attn = torch.empty(n, dim, dtype=torch.bfloat16, device=device)

    def close(self):
        for handle in (self.ctx, self.rotary, self.scene_batch, self.image_batch):
            handle.close()

    def _project(self, x, layer):
        """Q, K, V as [H][n][64] views of the fused projection output."""
        qkv = self.ctx.linear(rmsnorm(x), self.w_qkv[layer], self.qkv[:len(x)])
        v = qkv.view(len(x), 3, self.H, self.D)
        return [v[:, i].permute(1, 0, 2) for i in range(3)]

    def encode(self) -> torch.Tensor:
        """The scene through all layers; their keys and values are kept."""
        x, attn = self.x_scene.clone(), self.attn[:self.wl.n_tokens]
        for layer in range(self.layers):
            q, k, v = self._project(x, layer)
            self.rotary.norm_rotate(q, k, self.pos_scene, **self.norms[layer], out_q=q, out_k=k)   # in place
            self.caches[layer].append(self.scene_batch, k, v)
            self.ctx.global_attention(q, k, v, attn)
            x = x + self.ctx.linear(attn, self.w_o[layer])
        return x

    def lookup(self) -> torch.Tensor:
        """The images through all layers, each behind the kept scene."""
        x, attn = self.x_images.clone(), self.attn[:len(self.x_images)]
        for layer in range(self.layers):
            q, k, v = self._project(x, layer)
            w = self.norms[layer]
            self.rotary.norm_rotate(q, None, self.pos_images, w["q_weight"], None, w["q_bias"], None, out_q=q)
            self.caches[layer].append(self.image_batch, k, v, rotary=self.rotary, positions=self.pos_images, k_weight=w["k_weight"], k_bias=w["k_bias"])
            self.caches[layer].attention(self.image_batch, q, attn)
            x = x + self.ctx.linear(attn, self.w_o[layer])
        return x


def main() -> int:
    ap = argparse.ArgumentParser()
    ap.add_argument("--workload", default="small", choices=sorted(synth.WORKLOADS))
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--images", type=int, default=2, help="new images that are looked up together")
    ap.add_argument("--steps", type=int, default=3)
    ap.add_argument("--page-size", type=int, default=128)
    args = ap.parse_args()
    if not torch.cuda.is_available():
        raise SystemExit("run_lookup: no CUDA device; the kernels have no CPU fallback")
    wl = synth.WORKLOADS[args.workload]
    st = Lookup(wl, args.layers, args.images, args.page_size)
    try:
        ms_encode, ms_lookup = timed(st.encode, args.steps), timed(st.lookup, args.steps)
        y = st.lookup().float()
        torch.cuda.synchronize()
        status = st.ctx.query(hb.Q_DEVICE_STATUS) or st.rotary.status() or st.image_batch.status()
        print(json.dumps({"workload": wl.name, "layers": args.layers, "scene_tokens": wl.n_tokens, "images": args.images,
                          "image_tokens": args.images * wl.tokens_per_frame, "page_size": args.page_size, "ms_encode_scene": ms_encode,
                          "ms_look_up_images": ms_lookup, "finite": bool(torch.isfinite(y).all()), "device_status": status}))
    finally:
        st.close()
    return 0 if status == 0 else 1


if __name__ == "__main__":
    sys.exit(main())

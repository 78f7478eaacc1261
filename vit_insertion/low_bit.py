"""The ViT encoder with 4-bit linear layers and fused norms.

The same model as ``ViT`` with what lies between its attentions taken over by
the library's encoder-block operators:
  - every linear layer of a block is quantize_mxfp4 of its input and
    matmul_mxfp4 with weights that are laid out in 4 bits once;
  - every residual addition, its gate (a vector of features per branch, as
    LayerScale has) and the norm before the next block is one block_norm.
Embedding, attention, GELU and the dense head are PyTorch's.

``tune_last_gate`` fits the last branch's gate to the full model's features by
gradient descent: what merging and 4 bits shift, feature by feature.

    python vit_insertion/low_bit.py --model vit_b16 --batch 16
"""

from __future__ import annotations

import argparse
import json
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402
import torch.nn.functional as F  # noqa: E402

from vit_insertion.model import VIT_CONFIGS, ViT, synthetic_images, varlen_attention  # noqa: E402

LINEARS = ("qkv", "proj", "fc1", "fc2")
EPS = 1e-5  # torch's layer norm, which the full model calls without one


class LowBitViT(ViT):
    """ViT with MXFP4 linear layers and fused norms; same constructor and seed, same weights before rounding."""

    def __init__(self, cfg, device, dtype=torch.bfloat16, seed: int = 0):
        super().__init__(cfg, device, dtype, seed)
        import paper_2604_05718_gb300 as ops

        self.ops = ops
        for p in self.blocks:
            for name in LINEARS:
                p[name] = ops.quantize_mxfp4(p.pop(name + "_w"))
                p[name + "_b"] = p[name + "_b"].float()
            for name in ("ln1", "ln2"):
                p[name + "_w"], p[name + "_b"] = p[name + "_w"].float(), p[name + "_b"].float()
            p["gate1"] = torch.ones(cfg.dim, device=self.device)
            p["gate2"] = torch.ones(cfg.dim, device=self.device)
        self.head_ln_w, self.head_ln_b = self.head_ln_w.float(), self.head_ln_b.float()
        # Where the kernels report errors of their own; check_status() reads it.
        self.status = torch.zeros(2, dtype=torch.int32, device=self.device)

    def check_status(self) -> None:
        """Waits for the device, and raises what a kernel has reported since the last check."""
        code = int(self.status[0])
        if code != 0:
            self.status.zero_()
            raise self.ops.MPMError("a kernel of the 4-bit encoder", code)

    def linear(self, x: torch.Tensor, p: dict, name: str) -> torch.Tensor:
        return self.ops.matmul_mxfp4(self.ops.quantize_mxfp4(x), p[name], bias=p[name + "_b"], out_dtype=x.dtype,
                                     device_status=self.status)

    def norm(self, x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor) -> torch.Tensor:
        """Layer norm of a stream that no branch is added to: at the start and behind a merge."""
        return F.layer_norm(x, (self.cfg.dim,), weight.to(x.dtype), bias.to(x.dtype), eps=EPS)

    def branches(self, x: torch.Tensor, h: torch.Tensor, p: dict, cu: torch.Tensor, max_len: int):
        """One block from the stream x and its norm h: (stream after attention, output of the MLP branch)."""
        cfg = self.cfg
        s = x.shape[0]
        qkv = self.linear(h, p, "qkv").view(s, 3, cfg.heads, cfg.dim // cfg.heads)
        a = varlen_attention(*(qkv[:, i].contiguous() for i in range(3)), cu, max_len).reshape(s, cfg.dim)
        x, h, _ = self.ops.block_norm(self.linear(a, p, "proj"), x, norm="layer", gate=p["gate1"], pre_weight=p["ln2_w"],
                                      pre_bias=p["ln2_b"], eps=EPS, device_status=self.status)
        return x, self.linear(F.gelu(self.linear(h, p, "fc1")), p, "fc2")

    def run_blocks(self, images: torch.Tensor, mpm=None, workspace=None, insert_at=None):
        """(stream before the last MLP addition, that branch's output, maps, offsets of the patches)."""
        cfg = self.cfg
        b, e, n = images.shape[0], cfg.special, cfg.tokens
        x = self.embed(images)
        off = torch.arange(b + 1, device=self.device, dtype=torch.int64) * n
        longest = n
        maps = []
        points = set(cfg.insert_at if insert_at is None else insert_at) if mpm is not None else set()
        h = None
        for i, p in enumerate(self.blocks):
            if i in points:
                specials, patches = self.split(x, off)
                merged, off1, m = mpm.merge(patches, off, workspace=workspace)
                off1_host = off1.cpu()                       # the merged length decides the next shapes
                longest = int((off1_host[1:] - off1_host[:-1]).max())
                maps.append((m, off))
                off = off1
                x = self.join(specials, merged[:int(off1_host[-1])], off)
                h = None
            if h is None:
                h = self.norm(x, p["ln1_w"], p["ln1_b"])
            cu = (off + e * torch.arange(b + 1, device=self.device)).to(torch.int32)
            x, y = self.branches(x, h, p, cu, longest + e)
            if i + 1 == len(self.blocks):
                return x, y, maps, off
            # The next block's norm comes with the addition, unless a merge changes the rows in between.
            after = None if i + 1 in points else self.blocks[i + 1]
            x, h, _ = self.ops.block_norm(y, x, norm="layer", gate=p["gate2"],
                                          pre_weight=None if after is None else after["ln1_w"],
                                          pre_bias=None if after is None else after["ln1_b"], eps=EPS,
                                          device_status=self.status)
        raise ValueError("a model needs blocks")

    def to_grid(self, rows: torch.Tensor, off: torch.Tensor, maps: list, mpm) -> torch.Tensor:
        """Rows of all tokens -> the patches' rows on the full grid (Eq. 3 and Eq. 4)."""
        _, patches = self.split(rows, off)
        if not maps:
            return patches
        if len(maps) == 1:
            return mpm.unmerge_gather(patches, off, maps[0][0], maps[0][1])
        first, off0 = maps[0]
        for m, off_next in maps[1:-1]:
            first = mpm.compose_maps(first, off0, m, off_next)
        return mpm.compose_gather(patches, off, first, off0, maps[-1][0], maps[-1][1])

    def forward(self, images: torch.Tensor, mpm=None, workspace=None, insert_at=None, trace=None):
        """Dense logits [B*N, classes] on the patch grid.  check_status() says whether a kernel failed on the way."""
        if trace is not None:
            raise ValueError("LowBitViT keeps no trace of its insertions")
        x, y, maps, off = self.run_blocks(images, mpm, workspace, insert_at)
        _, h, _ = self.ops.block_norm(y, x, norm="layer", gate=self.blocks[-1]["gate2"], pre_weight=self.head_ln_w,
                                      pre_bias=self.head_ln_b, eps=EPS, device_status=self.status)
        return F.linear(self.to_grid(h, off, maps, mpm), self.head_w, self.head_b)

    def tune_last_gate(self, images: torch.Tensor, target: torch.Tensor, mpm=None, steps: int = 20, rate: float = 0.5,
                       insert_at=None) -> list:
        """Fits the last branch's gate so that the head's input comes near `target`, step by step; the losses.

        target: [rows, dim] features before the head for the rows that the
        last block works on (the full model's, taken along the merges).  The
        loss is the mean square error; a step is one block_norm and its
        backward pass, since nothing before the gate depends on it.
        """
        x, y, _, _ = self.run_blocks(images, mpm, insert_at=insert_at)
        gate = self.blocks[-1]["gate2"]
        args = dict(norm="layer", gate=gate, pre_weight=self.head_ln_w, pre_bias=self.head_ln_b, eps=EPS,
                    device_status=self.status)
        workspace = self.ops.block_norm_workspace(self.cfg.dim, self.device)
        losses = []
        for _ in range(steps):
            _, h, stats = self.ops.block_norm(y, x, with_stats=True, **args)
            off = h.float() - target
            losses.append(off.square().mean())
            # The mean over rows, so that the rate does not depend on their number.
            grads = self.ops.block_norm_backward(None, (2.0 / h.shape[0] * off).to(h.dtype), y, x, stats,
                                                 workspace=workspace, **args)
            gate -= rate * grads.d_gate
        self.check_status()
        return [float(v) for v in losses]


def main() -> int:
    ap = argparse.ArgumentParser()
    ap.add_argument("--model", default="vit_b16", choices=sorted(VIT_CONFIGS))
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--warmup", type=int, default=3)
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args()
    if not torch.cuda.is_available():
        raise RuntimeError("low_bit.py needs a CUDA device")
    import paper_2604_05718_gb300 as mpm
    from paper_2604_05718_gb300 import build
    from vit_insertion.bench_vit import timed

    build.build()
    dev = torch.device("cuda", 0)
    cfg = VIT_CONFIGS[args.model]
    images = synthetic_images(args.batch, cfg.image, cfg.patch, args.seed, dev)
    full, low = ViT(cfg, dev, seed=args.seed), LowBitViT(cfg, dev, seed=args.seed)
    ws = mpm.new_workspace(args.batch * cfg.tokens, args.batch, cfg.dim, torch.bfloat16, dev)
    with torch.inference_mode():
        want = full.forward(images)
        ms = {"full": timed(lambda: full.forward(images), args.steps, args.warmup),
              "merged": timed(lambda: full.forward(images, mpm=mpm, workspace=ws), args.steps, args.warmup),
              "low_bit": timed(lambda: low.forward(images), args.steps, args.warmup),
              "low_bit_merged": timed(lambda: low.forward(images, mpm=mpm, workspace=ws), args.steps, args.warmup)}
        got = low.forward(images, mpm=mpm, workspace=ws)
        low.check_status()
        likeness = F.cosine_similarity(got.float(), want.float(), dim=1).mean().item()
    print(json.dumps({"metric": "ViT encoder + dense head, 4-bit linear layers and fused norms", "model": cfg.name,
                      "batch": args.batch, "ms": ms, "fps": {k: args.batch / v * 1e3 for k, v in ms.items()},
                      "logit_cosine_to_full": likeness, "data": "synthetic Voronoi images, random-init weights"}),
          flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())

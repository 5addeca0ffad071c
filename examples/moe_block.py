"""A block of a model around the expert layer, served and trained in part:  python examples/moe_block.py

  serve   residual stream -> norm -> cq_moe_forward (+ every request's own low-rank adapter) -> gate, residual sum, next norm,
          for a batch of prompts and then token by token
  train   the experts are clustered and stay as they are; the router and the norm in front of it learn to spread the load: loss and
          counts from cq_balance_loss, gradients back through router, rotation and norm

Weights and tokens are synthetic (the tiny configuration)."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_10496_amd import binding as cq, synth  # noqa: E402


class Block:
    """Norm -> layer beside adapters -> gate, residual sum; the norm in front of the next block belongs to the same call."""

    def __init__(self, layer, norm, adapters):
        self.layer, self.norm, self.adapters = layer, norm, adapters

    def __call__(self, h, x, gate, ids):
        """Residual stream h and this block's input x of a batch of tokens -> the stream and the next block's input."""
        y = cq.cq_moe_forward(self.layer, x)
        cq.cq_adapter_apply(self.adapters, x, ids, base=y, out=y)
        out = cq.cq_block_norm(self.norm, h, y, gate)
        return out["h"], out["x"]


def make_model(n_blocks=2, n_adapters=4, rank=8, cfg=None, seed=7):
    cfg = cfg or synth.CONFIGS["tiny"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    inputs = synth.make_layer(cfg)
    rnd = lambda *shape, scale=1.0, mean=0.0: torch.randn(shape, generator=g, device="cuda") * scale + mean
    blocks = []
    for _ in range(n_blocks):
        norm = cq.BlockNorm(w_pre=rnd(cfg.H, scale=0.1, mean=1.0), w_post=rnd(cfg.H, scale=0.1, mean=1.0), residual_scale=1.0,
                            branch_scale=0.5, gate_sigmoid=True)
        adapters = cq.DeviceAdapters(rnd(n_adapters, rank, cfg.H, scale=cfg.H ** -0.5).bfloat16(),
                                     rnd(n_adapters, cfg.H, rank, scale=0.05).bfloat16(), torch.full((n_adapters,), 2.0, device="cuda"))
        blocks.append(Block(cq.device_layer_from_inputs(inputs), norm, adapters))
    first = cq.BlockNorm(w_pre=rnd(cfg.H, scale=0.1, mean=1.0))
    return inputs, first, blocks


def serve(first, blocks, h, gate, ids):
    """One pass of a batch of tokens: h [T, H] bf16, gate [T] f32, ids [T] i32 (-1: the request has no adapter)."""
    x = cq.cq_block_norm(first, h)["x"]
    for block in blocks:
        h, x = block(h, x, gate, ids)
    return h, x


def train_router(h, Wr, R, w_pre, top_k, steps=60, lr=0.02, alpha=1.0, seq_offsets=None, token_mask=None):
    """Gradient steps on router and norm that lower the balance loss of tokens h [T, H]; returns the losses and the last counts."""
    losses, counts = [], None
    for _ in range(steps):
        norm = cq.BlockNorm(w_pre=w_pre)
        x = cq.cq_block_norm(norm, h)["x"]
        XR = cq.cq_rotate_quant(x, R, 8)["XR"]
        route = cq.cq_route_permute(XR, Wr, None, top_k)
        bal = cq.cq_balance_loss(route["logits"], route["ids"], alpha, seq_offsets, token_mask)
        dz = cq.cq_balance_loss_grad(route["logits"], bal["counts"], bal["tokens"], top_k, alpha, seq_offsets, token_mask)
        dWr, dx = dz.t() @ XR, (dz @ Wr) @ R.t()
        dw = cq.cq_block_norm_grad(norm, h, dx=dx.contiguous())["dw_pre"]
        Wr, w_pre = Wr - lr * dWr, w_pre - lr * dw
        losses.append(bal["loss"])
        counts = bal["counts"]
    return torch.cat(losses).tolist(), counts


def main():
    cfg = synth.CONFIGS["tiny"]
    inputs, first, blocks = make_model()
    g = torch.Generator(device="cuda").manual_seed(1)
    # three prompts, one without an adapter; then four decode steps of one token per request
    lengths, request_adapter = [20, 33, 11], [0, -1, 3]
    T = sum(lengths)
    h = torch.randn((T, cfg.H), generator=g, device="cuda").bfloat16()
    gate = torch.randn(T, generator=g, device="cuda")
    ids = torch.cat([torch.full((n,), a, dtype=torch.int32) for n, a in zip(lengths, request_adapter)]).cuda()
    out, _ = serve(first, blocks, h, gate, ids)
    print(f"prompts: {T} tokens of {len(lengths)} requests, stream norm {out.float().norm().item():.3f}")
    ids = torch.tensor(request_adapter, dtype=torch.int32, device="cuda")
    for step in range(4):
        h = torch.randn((len(lengths), cfg.H), generator=g, device="cuda").bfloat16()
        out, _ = serve(first, blocks, h, torch.randn(len(lengths), generator=g, device="cuda"), ids)
        print(f"decode step {step}: stream norm {out.float().norm().item():.3f}")
    # a router that prefers the first experts
    h = torch.randn((512, cfg.H), generator=g, device="cuda") + 0.5
    Wr = torch.from_numpy(inputs.Wr).cuda()
    R = torch.from_numpy(inputs.R).cuda()
    Wr[0] += 0.5 * (torch.ones(cfg.H, device="cuda") @ R) / cfg.H ** 0.5
    losses, counts = train_router(h, Wr, R, torch.ones(cfg.H, device="cuda"), cfg.top_k)
    print(f"balance loss {losses[0]:.4f} -> {losses[-1]:.4f} (1 is even), counts {counts.tolist()}")


if __name__ == "__main__":
    main()

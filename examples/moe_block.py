"""A block of a model around the expert layer, served and trained in part:  python examples/moe_block.py

  serve   residual stream -> norm -> cq_moe_forward (+ every request's own low-rank adapter) -> gate, residual sum, next norm,
          for a batch of prompts and then token by token
  attend  the half of the block in front of that: clustered Q/K/V projection of rotated, quantized rows -> heads with norm and rotation, keys
          and values into a paged cache -> attention over it -> clustered output projection -> residual sum and norm
  train   the experts are clustered and stay as they are; the router and the norm in front of it learn to spread the load: loss and
          counts from cq_balance_loss, gradients back through router, rotation and norm

Weights and tokens are synthetic (the tiny configuration)."""
import os
import sys

import numpy as np
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


class Attention:
    """A block's first half over a paged cache: x (normed rows) of new tokens -> what is added to the residual stream.

    The projections are clustered weights like the experts', one group that holds every token; their inputs are rotated and quantized
    like the layer's (the output projection's weights are taken to be clustered in the basis of its inputs)."""

    def __init__(self, H, n_heads, n_key_heads, D, pages, page_size, width, n_seqs, R, seed=11):
        rng = np.random.default_rng(seed)

        def clustered(n, k):
            cent = np.sort(rng.standard_normal((1, n, 16)) * k ** -0.5, axis=2).astype(np.float32)
            return cq.DeviceCodebook(rng.integers(0, 256, (1, n, k // 2), dtype=np.uint8), synth.f32_to_bf16_bits(cent))
        self.Hq, self.Hk, self.D, self.R = n_heads, n_key_heads, D, R
        self.w_qkv, self.w_out = clustered((n_heads + 2 * n_key_heads) * D, H), clustered(H, n_heads * D)
        w = lambda: torch.from_numpy(rng.standard_normal(D) * 0.1 + 1).float().cuda()  # noqa: E731
        freq = 1e4 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
        self.norm = cq.HeadNorm(D, w(), w(), freq=freq.cuda())
        k, v = (torch.zeros((pages, page_size, n_key_heads, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.cache = cq.PagedCache(k, v)
        self.table = torch.full((n_seqs, width), -1, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(n_seqs, dtype=torch.int32, device="cuda")

    def project(self, W, rows, scale=None):
        T = rows.shape[0]
        groups = torch.tensor([0, T], dtype=torch.int32, device="cuda")
        kind = cq.CQ_A_F16 if scale is None else cq.CQ_A_INT8_CODES
        return cq.cq_codebook_grouped_gemm(W, rows, kind, scale, None, groups, T, cq.CQ_EPI_NONE, cq.CQ_OUT_F32)

    def heads(self, x):
        """Queries, keys and values of rows x [T, H] f32, as slices of the projection's rows."""
        rq = cq.cq_rotate_quant(x, self.R, 8)
        rows = self.project(self.w_qkv, rq["Q"], rq["scale"]).view(x.shape[0], -1, self.D)
        return rows.split([self.Hq, self.Hk, self.Hk], dim=1)

    def mix(self, q, k, v, offsets=None):
        """Attention [T, Hq, D] f16 of new tokens, whose keys and values join the cache.  lengths counts them already; offsets: where each
        sequence's tokens begin (None: one token each)."""
        q = cq.cq_cache_append(self.cache, k, v, self.table, self.lengths, offsets, norm=self.norm, q=q)
        if offsets is None:
            return cq.cq_cache_attention(self.cache, q, self.table, self.lengths, out_dtype=torch.float16)["out"]
        # a prompt: every token is a sequence of its own that ends with it
        new = (offsets[1:] - offsets[:-1]).long()
        seq = torch.repeat_interleave(torch.arange(len(new), device="cuda"), new)
        behind = offsets.long()[seq + 1] - torch.arange(len(seq), device="cuda") - 1      # tokens of the prompt behind this one
        lengths = (self.lengths.long()[seq] - behind).to(torch.int32)
        return cq.cq_cache_attention(self.cache, q, self.table[seq], lengths, out_dtype=torch.float16)["out"]

    def __call__(self, x, offsets=None):
        o = self.mix(*self.heads(x), offsets)
        return self.project(self.w_out, o.reshape(x.shape[0], -1))


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


def attend_and_serve(inputs, block, lengths, request_adapter, g, page_size=16, steps=4):
    """A whole block, attention and layer, over the prompts and then token by token."""
    H, S = inputs.cfg.H, len(lengths)
    rnd = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    width = max(lengths) // page_size + 1
    attention = Attention(H, 4, 2, 64, S * width, page_size, width, S, torch.from_numpy(inputs.R).cuda())
    attention.table.copy_(torch.arange(S * width, dtype=torch.int32).view(S, width))
    before, between = cq.BlockNorm(w_pre=torch.ones(H, device="cuda")), cq.BlockNorm(w_pre=torch.ones(H, device="cuda"))
    for step in range(steps + 1):
        new = lengths if step == 0 else [1] * S
        offsets = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda() if step == 0 else None
        ids = torch.cat([torch.full((n,), a, dtype=torch.int32) for n, a in zip(new, request_adapter)]).cuda()
        h, gate = rnd(sum(new), H).bfloat16(), rnd(sum(new))
        attention.lengths += torch.tensor(new, dtype=torch.int32).cuda()
        a = attention(cq.cq_block_norm(before, h)["x"], offsets)
        mid = cq.cq_block_norm(between, h, a)
        out, _ = block(mid["h"], mid["x"], gate, ids)
        print(f"whole block, {'prompts' if step == 0 else f'token {step}'}: stream norm {out.float().norm().item():.3f}, "
              f"cached {attention.lengths.tolist()}")
    return attention


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
    attend_and_serve(inputs, blocks[0], lengths, request_adapter, g)
    # a router that prefers the first experts
    h = torch.randn((512, cfg.H), generator=g, device="cuda") + 0.5
    Wr = torch.from_numpy(inputs.Wr).cuda()
    R = torch.from_numpy(inputs.R).cuda()
    Wr[0] += 0.5 * (torch.ones(cfg.H, device="cuda") @ R) / cfg.H ** 0.5
    losses, counts = train_router(h, Wr, R, torch.ones(cfg.H, device="cuda"), cfg.top_k)
    print(f"balance loss {losses[0]:.4f} -> {losses[-1]:.4f} (1 is even), counts {counts.tolist()}")


if __name__ == "__main__":
    main()

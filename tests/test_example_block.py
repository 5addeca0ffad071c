"""The example program's block (norm, layer beside adapters, gate, residual sum, next norm) against the oracles, and its training of
router and norm."""
import os
import sys

import numpy as np
import pytest

from oracle import around_oracle as A
from oracle import cq_oracle as O
from tests import helpers as Hp

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_block_matches_the_oracles():
    """One block on tokens whose router logits have a margin.  The layer is held to 2e-3 of a token's row; what follows adds a norm
    of it to the stream (branch_scale 0.5), which is stored in bf16 (2^-8 / 2 of a value)."""
    import torch
    import moe_block as M
    from paper_2604_10496_amd import binding as cq
    inputs, first, blocks = M.make_model(n_blocks=1)
    c = inputs.cfg
    rng = np.random.default_rng(3)
    w_first = first.w_pre.double().cpu().numpy()
    T = 24
    h = torch.from_numpy(rng.standard_normal((4 * T, c.H))).bfloat16()
    # tokens whose selected experts no rounding changes
    x64 = A.block_norm(h.double().numpy(), None, None, w_first, None, 1e-6, 1, 1, False)[0]["x"]
    top = -np.sort(-O.router_logits(O.rotate(x64, inputs.R), inputs.Wr, inputs.bias), axis=1)[:, :c.top_k + 1]
    keep = np.nonzero((top[:, :-1] - top[:, 1:]).min(axis=1) > 1e-2)[0][:T]
    assert len(keep) == T
    h, x64 = h[keep].contiguous(), x64[keep]
    gate = torch.from_numpy(rng.standard_normal(T)).float()
    ids = torch.from_numpy(rng.integers(-1, 4, T).astype(np.int32))
    got_h, got_x = M.serve(first, blocks, h.cuda(), gate.cuda(), ids.cuda())
    x32 = cq.cq_block_norm(first, h.cuda())["x"].cpu().numpy()     # (the layer's oracle takes the very input that the layer had)
    y = O.moe_forward(x32, inputs.R, inputs.Wr, inputs.bias, inputs.experts, c.E, c.top_k, c.act_bits)["Y"]
    b = blocks[0]
    y, _ = A.adapter_apply(x32.astype(np.float64), ids.numpy(), b.adapters.A.double().cpu().numpy(), b.adapters.B.double().cpu().numpy(),
                           b.adapters.scale.double().cpu().numpy(), None, y)
    ref, _ = A.block_norm(h.double().numpy(), y, gate.double().numpy(), b.norm.w_pre.double().cpu().numpy(),
                          b.norm.w_post.double().cpu().numpy(), 1e-6, 1.0, 0.5, True)
    # an activation code at a rounding tie differs by one step of 1/127 of its row's maximum in one of 256 values: such rows are
    # held to twice the layer's bar
    assert Hp.row_rel_l2(got_h.double().cpu().numpy(), ref["h"]).max() <= 2 * 2e-3 + 2.0 ** -9
    assert Hp.row_rel_l2(got_x.double().cpu().numpy(), ref["x"]).max() <= 2 * 2e-3


def test_router_and_norm_learn_to_spread_the_load():
    import torch
    import moe_block as M
    inputs, _, _ = M.make_model(n_blocks=1)
    c = inputs.cfg
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.randn((512, c.H), generator=g, device="cuda") + 0.5
    R, Wr = torch.from_numpy(inputs.R).cuda(), torch.from_numpy(inputs.Wr).cuda()
    Wr[0] += 0.5 * (torch.ones(c.H, device="cuda") @ R) / c.H ** 0.5
    off = torch.tensor([0, 100, 100, 512], dtype=torch.int32, device="cuda")
    losses, counts = M.train_router(h, Wr, R, torch.ones(c.H, device="cuda"), c.top_k, seq_offsets=off)
    print("losses", [round(v, 4) for v in losses], "counts", counts.tolist(), flush=True)
    assert counts.sum().item() == 512 * c.top_k and counts[1].sum().item() == 0
    assert losses[0] > 1.2                                  # the loaded expert
    assert losses[-1] < losses[0] - 0.5 * (losses[0] - 1.0)  # at least half of what is above an even load is gone


def test_the_example_runs(capsys):
    import moe_block as M
    M.main()
    out = capsys.readouterr().out
    assert "prompts: 64 tokens" in out and "decode step 3" in out and "balance loss" in out

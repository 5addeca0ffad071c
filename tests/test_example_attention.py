"""The example program's attention half: projection rows -> heads, cache, attention, for prompts and then token by token, against the
oracle on the very rows that its projection gave."""
import os
import sys

import numpy as np
import pytest

from oracle import heads_oracle as O

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_attention_half_matches_the_oracle():
    """Keys and values are rounded to bf16 (half a step: 2^-8 of a value) where they are stored, results to f16; the oracle takes the cache
    as it stands, so that the attention is held to 2^-11 of its values and 2^-10 of sum p |v| (scores of queries in fp32: 2 dz with
    dz = (D + 16) 2^-24 sum |q| |k| scale < 2^-14 here, two parts of P: 2^-16)."""
    import torch
    import moe_block as M
    from paper_2604_10496_amd import synth
    cfg = synth.CONFIGS["tiny"]
    inputs = synth.make_layer(cfg)
    g = torch.Generator(device="cuda").manual_seed(3)
    lengths, page, width = [20, 1, 33], 16, 3
    R = torch.from_numpy(inputs.R).cuda()
    a = M.Attention(cfg.H, 4, 2, 64, 9, page, width, 3, R)
    a.table.copy_(torch.randperm(9, device="cuda", generator=g).to(torch.int32).view(3, width))
    table = a.table.cpu().numpy()
    keys, have = {}, [0, 0, 0]
    for step in range(4):
        new = lengths if step == 0 else [1, 1, 1]
        off = np.concatenate([[0], np.cumsum(new)])
        a.lengths += torch.tensor(new, dtype=torch.int32).cuda()
        x = torch.randn((sum(new), cfg.H), generator=g, device="cuda")
        q, k, v = a.heads(x)
        out = a.mix(q, k, v, torch.tensor(off, dtype=torch.int32).cuda() if step == 0 else None)
        pos = np.concatenate([np.arange(h, h + n) for h, n in zip(have, new)])
        freq = a.norm.freq.cpu().numpy()
        d = lambda t: t.double().cpu().numpy()  # noqa: E731
        q_ref, _ = O.head_norm(d(q), d(a.norm.w_q), a.norm.eps, freq, False, 1.0, pos)
        k_ref, k_mag = O.head_norm(d(k), d(a.norm.w_k), a.norm.eps, freq, False, 1.0, pos)
        kc, vc = d(a.cache.k), d(a.cache.v)
        seq = np.repeat(np.arange(3), new)
        for t, s in enumerate(seq):                        # what was stored, and where
            p = pos[t]
            row = table[s, p // page], p % page
            assert (np.abs(kc[row] - k_ref[t]) <= 2.0 ** -8 * np.abs(k_ref[t]) + 2.0 ** -18 * k_mag[t]).all()
            assert (vc[row] == d(v[t].bfloat16())).all()
            keys[s, p] = kc[row].copy()
        assert all((kc[table[s, p // page], p % page] == row).all() for (s, p), row in keys.items())   # and is left as it was
        ref, _, mag, _, _ = O.attention(q_ref, kc, vc, table[seq], pos + 1, 64 ** -0.5)
        err = np.abs(d(out) - ref)
        assert (err <= 2.0 ** -11 * np.abs(ref) + 2.0 ** -10 * mag + 2.0 ** -25).all()
        have = [h + n for h, n in zip(have, new)]
        assert a.lengths.tolist() == have
        assert torch.isfinite(a.project(a.w_out, out.reshape(sum(new), -1))).all()


def test_the_whole_block_runs(capsys):
    import moe_block as M
    M.main()
    out = capsys.readouterr().out
    assert "whole block, prompts" in out and "whole block, token 4" in out and "cached [24, 37, 15]" in out

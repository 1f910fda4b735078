"""The weights' quantiser of the example (CPU)."""
import os
import runpy

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_blocks_of_zeros():
    """Scale 1 and codes 0, as everywhere else: no NaN out of 0 / 0."""
    quantise_blocks = runpy.run_path(os.path.join(ROOT, "examples", "moe_layer.py"), run_name="moe_layer")["quantise_blocks"]
    w = torch.randn((256, 384), generator=torch.Generator().manual_seed(1))
    w[:128, 128:256] = 0
    code, scale = quantise_blocks(w)
    assert scale[0, 1] == 1 and (code[:128, 128:256].float() == 0).all()
    wide = code.float() * scale.repeat_interleave(128, 0).repeat_interleave(128, 1)
    assert ((wide - w).abs() <= scale.repeat_interleave(128, 0).repeat_interleave(128, 1) * 16.0).all()

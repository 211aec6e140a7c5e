"""Refusals of the residual block's Python side that need no device."""
import pytest
import torch


def test_operand_types_of_an_expert_block():
    from paper_2207_02849_b200.expert_block import ExpertBlock
    for dtype in (torch.float32, torch.int8):
        with pytest.raises(ValueError, match="bf16 or fp16"):
            ExpertBlock(2, 64, 64, 8, dtype=dtype)


def test_a_gate_of_no_rows_is_left_to_the_library():
    """rows_per_gate 0 is an argument error of the call, not a division by zero before it."""
    import paper_2207_02849_b200 as bt
    cfg = bt.BlockNorm(64, gate=bt.GATE_LINEAR, rows_per_gate=0)
    assert cfg._gate(None, 4, torch.bfloat16, "gate") == (None, 0)
    from paper_2207_02849_b200 import build
    build.build()
    with pytest.raises(bt.BettyError) as e:
        bt.betty_block_norm_workspace_size(cfg, 4)
    assert e.value.status == bt.BETTY_ERR_INVALID_ARG

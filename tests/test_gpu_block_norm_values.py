"""Block norm at the ends of its ranges: calls without rows, rows of very large and very small values, gates where they saturate."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, HF, F = torch.bfloat16, torch.float16, torch.float32


def test_no_rows_and_no_gate_rows():
    """A call without rows has gates without rows, whatever addresses come with them: none is read, and the parameter gradients
    are zeros."""
    import paper_2207_02849_b200 as bt
    cfg = bt.BlockNorm(256, gate=bt.GATE_SIGMOID, rows_per_gate=4)
    params, dparams = torch.ones(3, 256, device="cuda"), torch.full((3, 256), float("nan"), device="cuda")
    y = torch.ones(1, 256, dtype=BF, device="cuda")                  # an address for the block's output; its gate has none
    ws = bt.Workspace.of_bytes(bt.betty_block_norm_workspace_size(cfg, 0))
    args = [y.data_ptr(), 256, None, 0] + [y.data_ptr(), 256] * 4 + [None, 0]
    status = bt.lib().betty_block_norm_backward(cfg._ref(BF, BF), params.data_ptr(), 0, y.data_ptr(), 256, *args, dparams.data_ptr(), ws.ptr, ws.nbytes,
                                                torch.cuda.current_stream().cuda_stream)
    assert status == bt.BETTY_OK and bt.betty_poll_status(ws)[0] == bt.BETTY_OK
    assert float(dparams.abs().max()) == 0.0 and float((y - 1).abs().max()) == 0.0

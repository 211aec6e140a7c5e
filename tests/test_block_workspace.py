"""Workspace sizes of the block norm's backward pass (host arithmetic: no device is needed)."""
import pytest


@pytest.fixture(scope="module")
def bt():
    from paper_2207_02849_b200 import build
    build.build()
    import paper_2207_02849_b200 as bt
    return bt


@pytest.mark.parametrize("d", [1, 100, 200, 300, 515, 1000, 2048, 4095, 4096, 8192, 16384])
@pytest.mark.parametrize("act,per_gate", [("NONE", 1), ("LINEAR", 1), ("SIGMOID", 3), ("LINEAR", 200)])
@pytest.mark.parametrize("bias", [False, True])
def test_a_workspace_serves_fewer_rows(bt, d, act, per_gate, bias):
    """The size for some rows holds for any fewer: a few rows are laid out otherwise than many, in more blocks."""
    cfg = bt.BlockNorm(d, gate=getattr(bt, "GATE_" + act), rows_per_gate=per_gate, bias=bias)
    rows = [0, 1, 7, 60, 147, 148, 149, 295, 296, 591, 592, 593, 1183, 1184, 1500, 2367, 2368, 4735, 4736, 5000, 9471, 9472, 20000, 100000]
    sizes = [bt.betty_block_norm_workspace_size(cfg, r) for r in rows]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("per_gate", [2, 7, 100])
@pytest.mark.parametrize("rows,d", [(16384, 4096), (100000, 512), (5000, 1001)])
def test_gates_of_few_rows_need_no_more_than_a_copy_of_a_matrix(bt, rows, d, per_gate):
    """Beside the parameters' sums, which a gate does not change: a gradient row for each pair of a walker and a gate, at most one for
    each row of the matrices; of contiguous rows that start on 16-byte boundaries at most two for each walker, of whom there are no
    more than eight in each of two blocks on every SM, or eight blocks."""
    plain = bt.BlockNorm(d, gate=bt.GATE_LINEAR, rows_per_gate=1)
    gated = bt.BlockNorm(d, gate=bt.GATE_LINEAR, rows_per_gate=per_gate)
    none = bt.BlockNorm(d)
    base = max(bt.betty_block_norm_workspace_size(c, rows) for c in (plain, none))
    slack = 1 << 16
    assert bt.betty_block_norm_workspace_size(gated, rows) <= base + (rows + 8) * d * 4 + slack
    assert bt.betty_block_norm_workspace_size(gated, rows, False) <= bt.betty_block_norm_workspace_size(gated, rows)
    if d % 8 == 0:
        assert bt.betty_block_norm_workspace_size(gated, rows, False) <= base + 2 * 16 * 148 * d * 4 + slack

"""Matrices whose rows start anywhere, copied to 16-byte boundaries, give the bits of the same matrix read in place: all starts of a row, and
widths around the accesses of a lane, a warp and a block's share."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _held(t, ld, start):
    """t [..., rows, cols] with the leading dimension ld, beginning `start` values behind a 16-byte boundary, NaN around it."""
    rows, cols = t.shape[-2:]
    flat = torch.full((t.numel() // cols * ld + 16,), float("nan"), dtype=t.dtype, device="cuda")
    v = flat[start:].as_strided(t.shape, (rows * ld, ld, 1)[-t.dim():])
    v.copy_(t)
    return v


WIDTHS = [1, 2, 3, 7, 8, 9, 15, 16, 17, 31, 130, 255, 256, 257, 511, 516, 769, 1021, 1030, 1088, 1089, 1196, 1281, 1285, 1537, 2051, 2310]


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("vocab", [60, 2500])
def test_the_matrix_of_a_vocabulary(d, vocab):
    import paper_2207_02849_b200 as bt
    g = torch.Generator().manual_seed(d)
    w, x = (torch.randn(vocab, d, generator=g) / d ** 0.5).to(BF), torch.randn(9, d, generator=g).to(BF).cuda()
    target = torch.randint(vocab, (9,), generator=g).cuda()
    cfg = bt.VocabLoss(vocab, d)
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, 9, any_layout=True))

    def losses(m):
        out = torch.full((2, 9), float("nan"), device="cuda")
        bt.betty_vocab_ce(cfg, x, m, target, out[0], out[1], ws)
        return out

    whole = -(-d // 8) * 8
    want = losses(_held(w, whole, 0))
    assert bool(want.isfinite().all())
    for ld in {d, d + 1, whole + 2, whole + 4, whole + 8}:
        for start in range(8):
            assert torch.equal(losses(_held(w, ld, start)), want), (ld, start)


@pytest.mark.parametrize("d", WIDTHS)
def test_the_operands_of_expert_products(d):
    import paper_2207_02849_b200 as bt
    g = torch.Generator().manual_seed(d)
    n, n_out, rows = 3, 40, 77
    w, x = (torch.randn(n, n_out, d, generator=g) / d ** 0.5).to(BF), torch.randn(rows, d, generator=g).to(BF)
    offsets = torch.tensor([0, 30, 30, rows], dtype=torch.int32, device="cuda")
    cfg = bt.Grouped(n, d, n_out)
    ws = bt.Workspace.of_bytes(bt.betty_grouped_workspace_size(cfg, rows, True))

    def product(a, b):
        y = torch.full((rows, n_out), float("nan"), dtype=torch.float32, device="cuda")
        bt.betty_grouped_forward(cfg, offsets, a, b, y, ws)
        return y

    whole = -(-d // 8) * 8
    want = product(_held(x, whole, 0), _held(w, whole, 0))
    assert bool(want.isfinite().all())
    for ld in {d, whole + 2, whole + 4}:
        for start in range(8):
            assert torch.equal(product(_held(x, ld, start), _held(w, whole + 1, 7 - start)), want), (ld, start)

"""Products grouped by expert with offsets that are out of order or range, in all three directions."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("bad", [[0, 50, 20, 100], [0, 50, 400, 100], [-7, 10, 20, 100], [0, -5, 60, 1 << 30], [3, 10, 20, 100]])
@pytest.mark.parametrize("n_in,n_out", [(128, 192), (65, 33)])
def test_results_are_those_of_the_clamped_offsets(bad, n_in, n_out):
    """The offsets count as the running maximum of their values within [0, rows], the first as 0: results equal those of offsets that
    are so from the start, the status says that they were not, and nothing beside the results is written."""
    import paper_2207_02849_b200 as bt
    rows, top, good = 100, 0, []
    for v in bad:
        top = max(top, min(max(v, 0), rows))
        good.append(top)
    good[0] = 0
    g = torch.Generator().manual_seed(5)
    x, w, dy = (torch.randn(*s, generator=g).to(BF).cuda() for s in ((rows, n_in), (3, n_out, n_in), (rows, n_out)))
    cfg = bt.Grouped(3, n_in, n_out)
    ws = bt.Workspace.of_bytes(bt.betty_grouped_workspace_size(cfg, rows))
    runs = []
    for offsets in (bad, good):
        o = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        guards = [torch.full((rows + 2, n_out), 7.0, dtype=BF, device="cuda"), torch.full((rows + 2, n_in), 7.0, dtype=BF, device="cuda"),
                  torch.full((5, n_out, n_in), 7.0, dtype=BF, device="cuda")]
        inner = [t[1:-1] for t in guards]
        for call in (lambda: bt.betty_grouped_forward(cfg, o, x, w, inner[0], ws), lambda: bt.betty_grouped_backward_data(cfg, o, dy, w, inner[1], ws),
                     lambda: bt.betty_grouped_backward_weight(cfg, o, dy, x, inner[2], ws)):
            call()
            want = bt.BETTY_ERR_INVALID_ARG if offsets is bad else bt.BETTY_OK
            assert bt.betty_poll_status(ws, raise_on_error=False)[0] == want
            bt.betty_reset_status(ws)
        for t in guards:
            assert bool((t[0] == 7).all()) and bool((t[-1] == 7).all())
        runs.append(inner)
    for a, b in zip(*runs):
        assert torch.equal(a, b)

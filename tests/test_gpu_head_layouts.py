"""A language head's matrix as the callers hold it: slices of wider and of longer buffers."""
import pytest
import torch

pytestmark = pytest.mark.gpu
VOCAB, D, ROWS = 777, 136, 150


def _matrix(w, kind):
    if kind == "wide":                 # leading dimension not a multiple of 8
        v = torch.full((VOCAB, D + 3), float("nan"), dtype=w.dtype, device="cuda")[:, :D]
    elif kind == "late":               # begins between two 16-byte boundaries
        v = torch.empty(VOCAB * D + 1, dtype=w.dtype, device="cuda")[1:].view(VOCAB, D)
    else:
        return w
    v.copy_(w)
    return v


def _data(dtype):
    g = torch.Generator().manual_seed(2)
    r = lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).cuda()  # noqa: E731
    return (r(VOCAB, D, scale=2 * D ** -0.5).to(dtype), r(ROWS, D).to(dtype), torch.randint(VOCAB, (ROWS,), generator=g).cuda(),
            torch.randint(VOCAB, (ROWS, 6), generator=g).cuda(), r(ROWS, 6, scale=3.0), torch.rand(ROWS, generator=g).cuda())


def _both(head, w, u, target, ids, logits, weights):
    out = []
    for loss, kept in (head.forward(w, u, target), head.forward_teacher(w, u, ids, logits)):
        out += [loss, *head.backward(w, kept, weights).values()]
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kind", ["wide", "late"])
@pytest.mark.parametrize("rows", [ROWS, 20])
def test_any_layout_gives_the_results_of_a_contiguous_matrix(dtype, kind, rows):
    from paper_2207_02849_b200.language_head import LanguageHead
    w, *rest = _data(dtype)
    rest = [t[:rows] for t in rest]
    head = LanguageHead(VOCAB, D, ROWS, 6, dtype)
    want = [t.clone() for t in _both(head, w, *rest)]
    assert all(torch.equal(a, b) for a, b in zip(want, _both(head, _matrix(w, kind), *rest)))


@pytest.mark.parametrize("kind", ["wide", "late"])
def test_without_room_forward_and_backward_refuse_alike(kind):
    from paper_2207_02849_b200.language_head import LanguageHead
    w, u, target, ids, logits, weights = _data(torch.bfloat16)
    head, odd = LanguageHead(VOCAB, D, ROWS, 6, any_layout=False), _matrix(w, kind)
    assert head.ws.nbytes + VOCAB * D * 2 <= LanguageHead(VOCAB, D, ROWS, 6).ws.nbytes
    _, kept = head.forward(w, u, target)
    _, kept_teacher = head.forward_teacher(w, u, ids, logits)
    for call in (lambda: head.forward(odd, u, target), lambda: head.forward_teacher(odd, u, ids, logits), lambda: head.backward(odd, kept, weights),
                 lambda: head.backward(odd, kept_teacher, weights, wants=("u",))):
        with pytest.raises(ValueError, match="any_layout"):
            call()
    assert sorted(head.backward(w, kept, weights)) == ["u", "w"]

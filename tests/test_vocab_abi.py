"""The losses over a vocabulary: descriptor against the header, workspace sizes, and the refusals that are made before anything touches a
device."""
import ctypes as C
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20          # an aligned address that no refused call reads


@pytest.fixture(scope="module")
def bt():
    from paper_2207_02849_b200 import build
    build.build()
    import paper_2207_02849_b200 as bt
    return bt


def test_struct_layout_matches_the_header():
    from paper_2207_02849_b200 import binding
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "betty.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} betty_vocab_cfg;", header).group(1)
    types = {"int32_t": C.c_int32, "int64_t": C.c_int64, "float": C.c_float}
    want = [(n.strip(), types[d.split()[0]]) for d in body.split(";") if d.strip() for n in d.split(None, 1)[1].split(",")]
    assert want == binding._VocabCfg._fields_


def _cfg(**change):
    from paper_2207_02849_b200 import binding
    f = dict(vocab=300, d=64, dtype=binding.BETTY_BF16, temperature=1.0, smoothing=0.0, z_loss=0.0)
    f.update(change)
    return binding._VocabCfg(*f.values())


def _ce(bt, c, rows=4, x=P, ldx=64, w=P, ldw=64, target=P, tt=4, loss=P, lse=P, ws=P, nb=1 << 30):
    return bt.lib().betty_vocab_ce(c, rows, x, ldx, w, ldw, target, tt, loss, lse, ws, nb, None)


def _ce_back(bt, c, rows=4, x=P, ldx=64, w=P, ldw=64, target=P, tt=4, lse=P, dloss=P, dx=P, lddx=64, dxt=1, dw=P, lddw=64, dwt=1, ws=P, nb=1 << 30):
    return bt.lib().betty_vocab_ce_backward(c, rows, x, ldx, w, ldw, target, tt, lse, dloss, dx, lddx, dxt, dw, lddw, dwt, ws, nb, None)


def _kd(bt, c, rows=4, x=P, ldx=64, w=P, ldw=64, top=5, ids=P, ldi=5, it=4, t=P, ldt=5, tt=0, loss=P, lse=P, ws=P, nb=1 << 30):
    return bt.lib().betty_vocab_distill(c, rows, x, ldx, w, ldw, top, ids, ldi, it, t, ldt, tt, loss, lse, ws, nb, None)


def _kd_back(bt, c, rows=4, x=P, ldx=64, w=P, ldw=64, top=5, ids=P, ldi=5, it=4, t=P, ldt=5, tt=0, lse=P, dloss=P, dx=P, lddx=64, dxt=1, dw=P, lddw=64, dwt=1, ws=P,
             nb=1 << 30):
    return bt.lib().betty_vocab_distill_backward(c, rows, x, ldx, w, ldw, top, ids, ldi, it, t, ldt, tt, lse, dloss, dx, lddx, dxt, dw, lddw, dwt, ws, nb, None)


ALL = (_ce, _ce_back, _kd, _kd_back)


@pytest.mark.parametrize("change,status", [
    ({"vocab": 0}, "SHAPE"), ({"d": 0}, "SHAPE"), ({"vocab": 1 << 22}, "UNSUPPORTED"), ({"d": (1 << 16) + 1}, "UNSUPPORTED"), ({"dtype": 0}, "DTYPE"),
    ({"dtype": 2}, "DTYPE"), ({"temperature": 0.0}, "INVALID_ARG"), ({"temperature": -1.0}, "INVALID_ARG"), ({"temperature": float("nan")}, "INVALID_ARG"),
    ({"temperature": float("inf")}, "INVALID_ARG"), ({"smoothing": -0.1}, "INVALID_ARG"), ({"smoothing": 1.5}, "INVALID_ARG"),
    ({"smoothing": float("nan")}, "INVALID_ARG"), ({"z_loss": -1.0}, "INVALID_ARG"), ({"z_loss": float("inf")}, "INVALID_ARG")])
def test_descriptor_refusals(bt, change, status):
    c, n, want = _cfg(**change), C.c_size_t(0), getattr(bt, "BETTY_ERR_" + status)
    assert all(f(bt, C.byref(c)) == want for f in ALL)
    assert bt.lib().betty_vocab_workspace_size(C.byref(c), 4, 5, 0, C.byref(n)) == want


def test_pointer_refusals(bt):
    c = C.byref(_cfg())
    for f in ALL:
        assert f(bt, None) == bt.BETTY_ERR_INVALID_ARG and f(bt, c, rows=-1) == bt.BETTY_ERR_INVALID_ARG
        assert f(bt, c, rows=(1 << 22) + 1) == bt.BETTY_ERR_UNSUPPORTED
        assert f(bt, c, x=None) == bt.BETTY_ERR_INVALID_ARG and f(bt, c, w=None) == bt.BETTY_ERR_INVALID_ARG and f(bt, c, lse=None) == bt.BETTY_ERR_INVALID_ARG
        assert f(bt, c, ldx=63) == bt.BETTY_ERR_SHAPE and f(bt, c, ldw=63) == bt.BETTY_ERR_SHAPE and f(bt, c, ldw=1 << 33) == bt.BETTY_ERR_UNSUPPORTED
        assert f(bt, c, x=P + 1) == bt.BETTY_ERR_ALIGNMENT and f(bt, c, w=P + 1) == bt.BETTY_ERR_ALIGNMENT and f(bt, c, lse=P + 2) == bt.BETTY_ERR_ALIGNMENT
        assert f(bt, c, ws=None) == bt.BETTY_ERR_WORKSPACE and f(bt, c, ws=P + 8) == bt.BETTY_ERR_WORKSPACE and f(bt, c, nb=100) == bt.BETTY_ERR_WORKSPACE
        assert f(bt, c, nb=5000) == bt.BETTY_ERR_WORKSPACE                # too small for its arrays
    for f in (_ce, _ce_back):
        assert f(bt, c, target=None) == bt.BETTY_ERR_INVALID_ARG and f(bt, c, tt=0) == bt.BETTY_ERR_DTYPE and f(bt, c, target=P + 4) == bt.BETTY_ERR_ALIGNMENT
    for f in (_kd, _kd_back):
        assert f(bt, c, top=0) == bt.BETTY_ERR_SHAPE and f(bt, c, top=1025, ldi=1025, ldt=1025) == bt.BETTY_ERR_UNSUPPORTED and f(bt, c, top=-1) == bt.BETTY_ERR_SHAPE
        assert f(bt, c, ids=None) == bt.BETTY_ERR_INVALID_ARG and f(bt, c, t=None) == bt.BETTY_ERR_INVALID_ARG
        assert f(bt, c, ldi=4) == bt.BETTY_ERR_SHAPE and f(bt, c, ldt=4) == bt.BETTY_ERR_SHAPE
        assert f(bt, c, it=0) == bt.BETTY_ERR_DTYPE and f(bt, c, tt=2) == bt.BETTY_ERR_DTYPE and f(bt, c, tt=-1) == bt.BETTY_ERR_DTYPE and f(bt, c, t=P + 2) == bt.BETTY_ERR_ALIGNMENT
        for k in ({"smoothing": 0.1}, {"z_loss": 1e-4}):
            assert f(bt, C.byref(_cfg(**k))) == bt.BETTY_ERR_UNSUPPORTED
    for f in (_ce, _kd):
        assert f(bt, c, loss=None) == bt.BETTY_ERR_INVALID_ARG and f(bt, c, rows=0, x=None, w=None) == bt.BETTY_OK
    for f in (_ce_back, _kd_back):
        assert f(bt, c, dx=None, dw=None) == bt.BETTY_ERR_INVALID_ARG and f(bt, c, dloss=None) == bt.BETTY_ERR_INVALID_ARG
        assert f(bt, c, dxt=3) == bt.BETTY_ERR_DTYPE and f(bt, c, dwt=3) == bt.BETTY_ERR_DTYPE
        assert f(bt, c, lddx=63) == bt.BETTY_ERR_SHAPE and f(bt, c, lddw=63) == bt.BETTY_ERR_SHAPE
        assert f(bt, c, dxt=0, dx=P + 2) == bt.BETTY_ERR_ALIGNMENT and f(bt, c, dw=P + 1) == bt.BETTY_ERR_ALIGNMENT
        assert f(bt, c, rows=0, x=None, w=None, dw=None) == bt.BETTY_OK


@pytest.mark.parametrize("vocab,d", [(1, 1), (300, 64), (5000, 515), (65536, 4096), (250000, 1024)])
@pytest.mark.parametrize("top", [0, 1, 7, 64])
def test_a_workspace_serves_fewer_rows(bt, vocab, d, top):
    """The size for some rows holds for any fewer, and grows by no more than the rows' own arrays and a piece of the vocabulary."""
    cfg = bt.VocabLoss(vocab, d, bt.BETTY_F16)
    rows = [0, 1, 7, 127, 128, 129, 255, 256, 257, 500, 1000, 2000, 5000, 16384, 20000, 100000]
    sizes = [bt.betty_vocab_workspace_size(cfg, r, top) for r in rows]
    assert sizes == sorted(sizes)
    for r, n in zip(rows, sizes):
        padded, wide = r + 256, d + 64
        # x twice, dX's sums (two rounds of tiles of 256 x 256 or 128 x 128 for 148 SMs beside one sum), a piece of 2^27 coefficients or 1024
        # columns, or two statistics for each 16 columns and row
        piece = max((1 << 27) + padded * 256, padded * 1024) * 2
        assert n <= 4 * padded * wide * 2 + 4 * wide * 256 + 80 * 2 ** 20 + max(min(piece, padded * (vocab + 256) * 2), padded * (vocab / 16 + 2) * 8) + padded * (64 + 24 * max(top, 1)) + (1 << 14)
    assert bt.betty_vocab_workspace_size(cfg, 100, top, True) >= bt.betty_vocab_workspace_size(cfg, 100, top, False) + vocab * d * 2


def test_python_refusals(bt):
    from paper_2207_02849_b200.language_head import LanguageHead
    for dtype in (torch.float32, torch.int8):
        with pytest.raises(ValueError, match="bf16 or fp16"):
            LanguageHead(100, 64, 8, dtype=dtype)
    cfg = bt.VocabLoss(100, 64)
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(100, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA tensor"):
        cfg._operands(x, w)
    with pytest.raises(ValueError, match="bf16 or fp16"):
        bt.VocabLoss(100, 64, bt.BETTY_F32)._operands(x, w)
    with pytest.raises(ValueError, match="int32 or int64"):
        cfg._entries(x, x, 4)
    with pytest.raises(bt.BettyError) as e:
        bt.betty_vocab_workspace_size(bt.VocabLoss(100, 64, temperature=-1.0), 4)
    assert e.value.status == bt.BETTY_ERR_INVALID_ARG

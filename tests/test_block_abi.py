"""Descriptors of the residual block's operators against the header, and the refusals that are made before anything touches a
device."""
import ctypes as C
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def bt():
    from paper_2207_02849_b200 import build
    build.build()
    import paper_2207_02849_b200 as bt
    return bt


@pytest.mark.parametrize("struct,mirror", [("betty_block_norm_cfg", "_BlockNormCfg"), ("betty_act8_cfg", "_Act8Cfg"), ("betty_grouped_cfg", "_GroupedCfg")])
def test_struct_layouts_match_the_header(struct, mirror):
    from paper_2207_02849_b200 import binding
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "betty.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % struct, header).group(1)
    types = {"int32_t": C.c_int32, "int64_t": C.c_int64, "float": C.c_float}
    want = [types[d.split()[0]] for d in body.split(";") if d.strip() for _ in d.split(",")]
    assert want == [f[1] for f in getattr(binding, mirror)._fields_]


P = 1 << 20          # an aligned address that no refused call reads


def _norm(bt, **change):
    from paper_2207_02849_b200 import binding
    f = dict(d=64, x_dtype=bt.BETTY_BF16, y_dtype=bt.BETTY_BF16, pre=bt.NORM_RMS, post=bt.NORM_RMS, gate=bt.GATE_NONE, bias=0, rows_per_gate=1, eps=1e-6)
    f.update(change)
    return binding._BlockNormCfg(*f.values())


@pytest.mark.parametrize("change,status", [
    ({"d": 0}, "SHAPE"), ({"d": 16385}, "UNSUPPORTED"), ({"pre": 3}, "INVALID_ARG"), ({"post": -1}, "INVALID_ARG"), ({"gate": 9}, "INVALID_ARG"),
    ({"rows_per_gate": 0}, "INVALID_ARG"), ({"eps": -1.0}, "INVALID_ARG"), ({"eps": float("nan")}, "INVALID_ARG"), ({"x_dtype": 2}, "DTYPE"),
    ({"x_dtype": 3}, "DTYPE"), ({"y_dtype": 0}, "DTYPE")])
def test_block_norm_refusals(bt, change, status):
    L, c = bt.lib(), _norm(bt, **change)
    want = getattr(bt, "BETTY_ERR_" + status)
    n = C.c_size_t(0)
    assert L.betty_block_norm(C.byref(c), P, 4, P, 64, P, 64, None, 0, P, 64, P, 64, None) == want
    assert L.betty_block_norm_workspace_size(C.byref(c), 4, C.byref(n)) == want
    assert L.betty_block_norm_backward(C.byref(c), P, 4, P, 64, P, 64, None, 0, P, 64, P, 64, P, 64, P, 64, None, 0, P, P, 1 << 30, None) == want


def test_block_norm_pointer_refusals(bt):
    L, c = bt.lib(), _norm(bt)
    f = lambda params=P, rows=4, x=P, ldx=64, y=P, xo=P, u=P: L.betty_block_norm(C.byref(c), params, rows, x, ldx, y, 64, None, 0, xo, 64, u, 64, None)  # noqa: E731
    assert L.betty_block_norm(None, P, 4, P, 64, P, 64, None, 0, P, 64, P, 64, None) == bt.BETTY_ERR_INVALID_ARG
    assert f(params=None) == bt.BETTY_ERR_INVALID_ARG and f(x=None) == bt.BETTY_ERR_INVALID_ARG and f(xo=None) == bt.BETTY_ERR_INVALID_ARG
    assert f(y=None, u=None) == bt.BETTY_ERR_INVALID_ARG and f(rows=-1) == bt.BETTY_ERR_INVALID_ARG
    assert f(ldx=63) == bt.BETTY_ERR_SHAPE and f(x=P + 1) == bt.BETTY_ERR_ALIGNMENT and f(params=P + 4) == bt.BETTY_ERR_ALIGNMENT
    assert f(rows=1 << 31) == bt.BETTY_ERR_UNSUPPORTED and f(ldx=1 << 30) == bt.BETTY_ERR_UNSUPPORTED
    assert f(rows=0, x=None) == bt.BETTY_OK
    g = _norm(bt, gate=bt.GATE_LINEAR)
    assert L.betty_block_norm(C.byref(g), P, 4, P, 64, P, 64, None, 0, P, 64, P, 64, None) == bt.BETTY_ERR_INVALID_ARG


@pytest.mark.parametrize("cols,dtype,act,status", [(0, 1, 0, "SHAPE"), (8, 2, 0, "DTYPE"), (8, 1, 3, "INVALID_ARG"), (8, 1, -1, "INVALID_ARG"),
                                                   (1 << 29, 1, 0, "UNSUPPORTED")])
def test_act8_refusals(bt, cols, dtype, act, status):
    from paper_2207_02849_b200 import binding
    L, c = bt.lib(), binding._Act8Cfg(cols, dtype, act, 0)
    want = getattr(bt, "BETTY_ERR_" + status)
    assert L.betty_act8_store(C.byref(c), 4, P, cols, P, cols, P, cols, P, 8, None) == want
    assert L.betty_act8_restore(C.byref(c), 4, P, cols, P, 8, P, cols, None) == want
    assert L.betty_act8_backward(C.byref(c), 4, P, cols, P, 8, P, cols, P, cols, P, cols, None) == want


def test_act8_pointer_refusals(bt):
    from paper_2207_02849_b200 import binding
    L, c = bt.lib(), binding._Act8Cfg(256, 1, 1, 1)
    f = lambda z=P, ldz=512, q=P, sc=P, lds=4: L.betty_act8_store(C.byref(c), 4, z, ldz, P, 256, q, 512, sc, lds, None)  # noqa: E731
    assert f(z=None) == bt.BETTY_ERR_INVALID_ARG and f(q=None) == bt.BETTY_ERR_INVALID_ARG and f(sc=None) == bt.BETTY_ERR_INVALID_ARG
    assert f(ldz=511) == bt.BETTY_ERR_SHAPE and f(lds=3) == bt.BETTY_ERR_SHAPE
    assert f(z=P + 1) == bt.BETTY_ERR_ALIGNMENT and f(sc=P + 2) == bt.BETTY_ERR_ALIGNMENT
    assert L.betty_act8_backward(C.byref(c), 4, P, 512, P, 4, P, 256, None, 0, None, 0, None) == bt.BETTY_ERR_INVALID_ARG
    assert L.betty_act8_backward(C.byref(c), 4, P, 512, P, 4, None, 0, P, 512, None, 0, None) == bt.BETTY_ERR_INVALID_ARG


@pytest.mark.parametrize("groups,dtype,n_in,n_out,status", [(0, 1, 8, 8, "SHAPE"), (2, 0, 8, 8, "DTYPE"), (2, 1, 0, 8, "SHAPE"), (2, 1, 8, 0, "SHAPE"),
                                                            (1025, 1, 8, 8, "UNSUPPORTED"), (2, 1, 1 << 25, 8, "UNSUPPORTED")])
def test_grouped_refusals(bt, groups, dtype, n_in, n_out, status):
    from paper_2207_02849_b200 import binding
    L, c = bt.lib(), binding._GroupedCfg(groups, dtype, n_in, n_out)
    want = getattr(bt, "BETTY_ERR_" + status)
    n = C.c_size_t(0)
    assert L.betty_grouped_workspace_size(C.byref(c), 4, 0, C.byref(n)) == want
    for f in (L.betty_grouped_forward, L.betty_grouped_backward_data):
        assert f(C.byref(c), 4, P, P, n_in, P, n_in, n_in * n_out, P, n_out, 1, P, 1 << 30, None) == want
    assert L.betty_grouped_backward_weight(C.byref(c), 4, P, P, n_out, P, n_in, P, n_in, n_in * n_out, 1, P, 1 << 30, None) == want


def test_grouped_pointer_refusals(bt):
    from paper_2207_02849_b200 import binding
    L, c = bt.lib(), binding._GroupedCfg(2, 1, 64, 32)

    def f(rows=4, off=P, x=P, ldx=64, w=P, ldw=64, gs=2048, y=P, ldy=32, dt=1, ws=P, nb=1 << 20):
        return L.betty_grouped_forward(C.byref(c), rows, off, x, ldx, w, ldw, gs, y, ldy, dt, ws, nb, None)

    for k in ("off", "x", "w", "y"):
        assert f(**{k: None}) == bt.BETTY_ERR_INVALID_ARG
    assert f(rows=-1) == bt.BETTY_ERR_INVALID_ARG and f(rows=(1 << 30) + 1) == bt.BETTY_ERR_UNSUPPORTED
    assert f(ldx=63) == bt.BETTY_ERR_SHAPE and f(ldw=63) == bt.BETTY_ERR_SHAPE and f(gs=2047) == bt.BETTY_ERR_SHAPE and f(ldy=31) == bt.BETTY_ERR_SHAPE
    assert f(dt=3) == bt.BETTY_ERR_DTYPE and f(x=P + 1) == bt.BETTY_ERR_ALIGNMENT and f(off=P + 2) == bt.BETTY_ERR_ALIGNMENT
    assert f(ws=None) == bt.BETTY_ERR_WORKSPACE and f(ws=P + 8) == bt.BETTY_ERR_WORKSPACE and f(nb=16) == bt.BETTY_ERR_WORKSPACE
    assert f(rows=0) == bt.BETTY_OK


def test_workspace_sizes_grow_with_the_rows(bt):
    cfg = bt.BlockNorm(520, gate=bt.GATE_LINEAR, rows_per_gate=9, bias=True)
    sizes = [bt.betty_block_norm_workspace_size(cfg, r) for r in (0, 1, 100, 10000)]
    assert sizes == sorted(sizes) and sizes[0] > 256
    g = bt.Grouped(3, 64, 72)
    assert bt.betty_grouped_workspace_size(g, 50) < bt.betty_grouped_workspace_size(g, 50, True)
    assert bt.betty_grouped_workspace_size(bt.Grouped(3, 65, 72), 50) > bt.betty_grouped_workspace_size(g, 50)


def test_levels_refuse_the_activation_they_do_not_have(bt):
    """A level's hidden layers know ReLU and GELU; SiLU belongs to the 8-bit checkpoint calls."""
    from paper_2207_02849_b200 import binding as b
    widths = (C.c_int64 * 3)(8, 8, 4)
    s = b._Level()
    s.loss, s.param_kind, s.params, s.n_params = bt.LOSS_MLP_CE_REWEIGHT, bt.PARAM_MLP, P, 8 * 8 + 8 + 4 * 8 + 4
    s.X, s.x_dtype, s.n, s.d, s.y, s.n_layers, s.widths = P, bt.BETTY_BF16, 4, 8, P, 2, widths
    n = C.c_size_t(0)
    arr = (C.POINTER(b._Level) * 1)(C.pointer(s))
    assert bt.lib().betty_workspace_size(arr, 1, C.byref(n)) == bt.BETTY_OK
    s.activation = bt.ACT_SILU
    assert bt.lib().betty_lower_step(C.byref(s), 1, P, n.value, None) == bt.BETTY_ERR_UNSUPPORTED

"""What the calls of 8-bit layers with a scale for each token, of the selection over large vocabularies and of the reordering
of states refuse: before any launch, so without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2206_07882_amd import qrnnt

OK, NULL, SHAPE, ALIGN, RANGE, WORKSPACE, LAYOUT, UNSUPPORTED = 0, 1, 2, 3, 4, 5, 6, 7


@pytest.fixture(scope="module")
def lib():
    return qrnnt.load()


def test_quantize_tokens(lib):
    f = lambda x=0x1000, dt=0, rows=4, cols=20, ld=20, q=0x20000, ld_q=32, s=0x30000: lib.qrnnt_quantize_tokens(x, dt, rows, cols, ld, q, ld_q, s, None)
    assert f(x=None) == NULL and f(q=None) == NULL and f(s=None) == NULL
    assert f(dt=3) == RANGE and f(dt=-1) == RANGE
    assert f(rows=-1) == SHAPE and f(cols=0) == SHAPE and f(ld=19) == SHAPE and f(ld_q=16) == SHAPE and f(ld_q=40) == SHAPE
    assert f(rows=1 << 31) == UNSUPPORTED and f(cols=(1 << 30) + 1, ld=1 << 31, ld_q=(1 << 30) + 16) == UNSUPPORTED and f(ld=1 << 59) == UNSUPPORTED
    assert f(x=0x1002) == ALIGN and f(q=0x20008) == ALIGN and f(s=0x30002) == ALIGN and f(x=0x1001, dt=2) == ALIGN
    assert f(rows=0) == OK and f(rows=0, x=None) == OK


def test_rms_norm_quant(lib):
    def f(x=0x10000, res=0x20000, w=0x30000, dt=0, rows=4, cols=20, ld=20, ld_r=20, eps=1e-5, out=0x40000, ld_s=20, q=0x50000, ld_q=32, s=0x60000):
        return lib.qrnnt_rms_norm_quant(x, res, w, dt, rows, cols, ld, ld_r, eps, out, ld_s, q, ld_q, s, None)
    assert f(x=None) == NULL and f(out=None) == NULL and f(q=None) == NULL and f(s=None) == NULL
    assert f(dt=9) == RANGE and f(eps=-1.0) == RANGE and f(eps=float("nan")) == RANGE and f(eps=float("inf")) == RANGE
    assert f(cols=-2) == SHAPE and f(ld=3) == SHAPE and f(ld_r=3) == SHAPE and f(ld_s=3) == SHAPE and f(ld_q=24) == SHAPE
    assert f(x=0x10001) == ALIGN and f(res=0x20002) == ALIGN and f(w=0x30001) == ALIGN and f(out=0x40003) == ALIGN and f(q=0x50001) == ALIGN
    # the sum may take the place of an input, not overlap it otherwise
    assert f(out=0x10004) == RANGE and f(out=0x20000 - 4) == RANGE and f(out=0x10000, ld_s=24) == RANGE and f(out=0x20000 + 79 * 4) == RANGE
    assert f(ld_r=1 << 60) == UNSUPPORTED and f(ld_s=1 << 60) == UNSUPPORTED and f(ld_r=1 << 60, res=None, x=None) == NULL
    assert f(rows=0) == OK


def _mat(rows=64, cols=100, bits=8, layout=qrnnt.LAYOUT_TILED, packed=0x1000):
    return qrnnt.CQMat(packed, 0x2000, rows, cols, layout, bits)


def test_linear_tokens(lib):
    def f(m=None, bias=None, a=0x10000, ld_a=112, sa=0x3000, M=5, y=0x40000, dt=0, ld_y=64, ws=None, n=0):
        return lib.qrnnt_linear_tokens(C.byref(m or _mat()), bias, a, ld_a, sa, M, y, dt, ld_y, ws, n, None)
    assert lib.qrnnt_linear_tokens(None, None, 0x10000, 112, 0x3000, 5, 0x40000, 0, 64, None, 0, None) == NULL
    assert f(a=None) == NULL and f(sa=None) == NULL and f(y=None) == NULL and f(_mat(packed=None)) == NULL
    assert f(_mat(layout=2)) == LAYOUT and f(_mat(bits=4)) == UNSUPPORTED and f(_mat(bits=5)) == RANGE and f(_mat(cols=131072), ld_a=131072) == UNSUPPORTED
    assert f(dt=3) == RANGE
    assert f(M=-1) == SHAPE and f(ld_a=96) == SHAPE and f(ld_a=120) == SHAPE and f(ld_y=63) == SHAPE and f(_mat(rows=0)) == SHAPE
    assert f(a=0x10008) == ALIGN and f(y=0x40002) == ALIGN and f(y=0x40001, dt=1) == ALIGN and f(bias=0x5001) == ALIGN and f(sa=0x3002) == ALIGN
    assert f(M=(1 << 30) + 1) == UNSUPPORTED and f(_mat(rows=(1 << 30) + 1), ld_y=1 << 31) == UNSUPPORTED and f(ld_y=1 << 60) == UNSUPPORTED
    assert f(M=(1 << 28) + 1) == UNSUPPORTED and f(_mat(rows=(1 << 28) + 1), ld_y=1 << 31) == UNSUPPORTED
    assert f(_mat(rows=1 << 20), M=1 << 20, ld_y=1 << 20) == UNSUPPORTED   # more tiles than a grid has
    assert f(M=0) == OK and f(M=0, a=None, y=None) == OK
    assert lib.qrnnt_linear_tokens_workspace(None, 4) == 0 and lib.qrnnt_linear_tokens_workspace(C.byref(_mat()), 0) == 0
    for rows, cols, M in ((64, 131071, 33), (64, 8192, 16), (100, 4096, 200), (8192, 8192, 8192)):
        m = _mat(rows, cols)
        need = lib.qrnnt_linear_tokens_workspace(C.byref(m), M)
        ld_a = (cols + 15) // 16 * 16
        if need:
            assert f(m, ld_a=ld_a, M=M, ld_y=rows) == NULL
            assert f(m, ld_a=ld_a, M=M, ld_y=rows, ws=0x100000, n=need - 1) == WORKSPACE
            assert f(m, ld_a=ld_a, M=M, ld_y=rows, ws=0x100010, n=need) == ALIGN


def test_beam_select(lib):
    def f(score=0x1000, logits=0x10000, dt=0, ld=100, fin=None, end=-1, B=2, W=4, V=100, n=4, par=0x2000, tok=0x3000, val=0x4000, done=None, ws=0x100000, size=1 << 30):
        return lib.qrnnt_beam_select(score, logits, dt, ld, 1, fin, end, B, W, V, n, par, tok, val, done, ws, size, None)
    for name in ("score", "logits", "par", "tok", "val", "ws"):
        assert f(**{name: None}) == NULL
    assert f(dt=3) == RANGE and f(fin=0x5000) == RANGE and f(fin=0x5000, end=100) == RANGE
    assert f(B=-1) == SHAPE and f(W=0) == SHAPE and f(V=0) == SHAPE and f(n=0) == SHAPE and f(ld=99) == SHAPE
    assert f(W=65) == UNSUPPORTED and f(n=65) == UNSUPPORTED and f(W=64, V=1 << 25, ld=1 << 25) == UNSUPPORTED and f(B=1 << 30, W=4) == UNSUPPORTED
    assert f(W=1, V=(1 << 30) + 1, ld=1 << 31) == UNSUPPORTED and f(ld=1 << 60) == UNSUPPORTED
    assert f(B=(1 << 21) + 1, W=1) == UNSUPPORTED and qrnnt.beam_select_workspace((1 << 21) + 1, 1, 100, 1) == 0
    assert f(score=0x1002) == ALIGN and f(logits=0x10001, dt=1) == ALIGN and f(par=0x2001) == ALIGN and f(ws=0x100008) == ALIGN
    need = qrnnt.beam_select_workspace(2, 4, 100, 4)
    assert need > 0 and f(size=need - 1) == WORKSPACE
    assert f(B=0) == OK and f(B=0, score=None, ws=None) == OK
    assert qrnnt.beam_select_workspace(1, 65, 10, 1) == 0 and qrnnt.beam_select_workspace(1, 4, 10, 65) == 0 and qrnnt.beam_select_workspace(-1, 4, 10, 5) == 0


def test_reorder_states(lib):
    S = qrnnt.CStateRows
    def f(states, parent=0x900000, B=2, W=4, W_out=4, n=None):
        arr = (S * max(1, len(states)))(*states)
        return lib.qrnnt_reorder_states(arr, len(states) if n is None else n, parent, B, W, W_out, None)
    good = S(0x10000, 0x20000, 64, 64, 64)
    assert lib.qrnnt_reorder_states(None, 1, 0x900000, 2, 4, 4, None) == NULL
    assert f([good], parent=None) == NULL and f([S(None, 0x20000, 64, 64, 64)]) == NULL and f([S(0x10000, None, 64, 64, 64)]) == NULL
    assert f([], n=0) == RANGE and f([good] * 33) == RANGE
    assert f([good], B=-1) == SHAPE and f([good], W=0) == SHAPE and f([good], W_out=0) == SHAPE and f([good], W=65) == UNSUPPORTED and f([good], W_out=65) == UNSUPPORTED
    assert f([S(0x10000, 0x20000, 0, 64, 64)]) == SHAPE and f([S(0x10000, 0x20000, 64, 63, 64)]) == SHAPE and f([S(0x10000, 0x20000, 64, 64, 63)]) == SHAPE
    assert f([good], parent=0x900002) == ALIGN and f([S(0x10000, 0x20000, 64, 1 << 60, 64)]) == UNSUPPORTED and f([S(0x10000, 0x20000, 64, 64, 1 << 60)]) == UNSUPPORTED
    assert f([good], B=1 << 30, W=1, W_out=1, parent=0x9000000000) == RANGE
    # overlaps: a destination with another row of its source, with another array, with the parents; the same rows at another beam
    assert f([S(0x10000, 0x10040, 64, 64, 64)]) == RANGE and f([S(0x10000, 0x10000, 64, 64, 128)]) == RANGE
    assert f([S(0x10000, 0x10000, 64, 64, 64)], W_out=3) == RANGE
    assert f([good, S(0x30000, 0x20040, 64, 64, 64)]) == RANGE and f([good, S(0x20000, 0x30000, 64, 64, 64)]) == RANGE
    assert f([S(0x10000, 0x10000, 40, 64, 64), S(0x10020, 0x10020, 32, 64, 64)]) == RANGE
    assert f([good], parent=0x20020) == RANGE
    assert f([S(1 << 44, 1 << 45, 15, 15, 15)], B=1 << 29, W=1, W_out=1, parent=1 << 46) == UNSUPPORTED   # 15 single bytes a row
    assert f([good], B=0) == OK


def test_wrappers_refuse_counts_that_do_not_fit_32_bits():
    x = torch.zeros(1, dtype=torch.int8)
    for rows, cols, pitch in ((1, 1 << 31, 1 << 31), (1 << 31, 1, 1), (2, 16, 1 << 31)):
        with pytest.raises(ValueError):
            qrnnt._matrix(torch.empty_strided((rows, cols), (pitch, 1), dtype=torch.int8, device="meta"), torch.int8, rows, cols)
    with pytest.raises(ValueError):
        qrnnt.StateGroup([x], 1 << 32, 1)
    with pytest.raises(RuntimeError):
        qrnnt._check(UNSUPPORTED, "qrnnt_beam_select")


def test_wrappers_refuse_tensors_that_are_not_on_the_gpu():
    x = torch.zeros((4, 32))
    for call in (lambda: qrnnt.quantize_tokens(x), lambda: qrnnt.rms_norm_quant(x), lambda: qrnnt.beam_select(x, x),
                 lambda: qrnnt.StateGroup([x], 1, 4)):
        with pytest.raises(ValueError):
            call()
    m = qrnnt.QMat(torch.zeros(2048, dtype=torch.uint8), torch.zeros(16), 16, 32, qrnnt.LAYOUT_TILED, 8)
    with pytest.raises(ValueError):
        qrnnt.linear_tokens(m, torch.zeros((4, 32), dtype=torch.int8), torch.zeros(4))

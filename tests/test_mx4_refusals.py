"""What the calls of microscaled 4-bit floats and of token scores refuse: before any launch, so without a GPU."""
import ctypes as C
import random

import pytest
import torch

from paper_2206_07882_amd import qrnnt

OK, NULL, SHAPE, ALIGN, RANGE, WORKSPACE, LAYOUT, UNSUPPORTED = 0, 1, 2, 3, 4, 5, 6, 7


@pytest.fixture(scope="module")
def lib():
    return qrnnt.load()


def test_pitches(lib):
    assert [qrnnt.mx4_pitch(c) for c in (1, 32, 33, 64, 1283, 1 << 30)] == [16, 16, 32, 32, 41 * 16, 1 << 29]
    assert [qrnnt.mx4_scale_pitch(c) for c in (1, 256, 257, 1283, 1 << 30)] == [8, 8, 16, 48, 1 << 25]
    for bad in (0, -1, (1 << 30) + 1):
        assert qrnnt.mx4_pitch(bad) == 0 and qrnnt.mx4_scale_pitch(bad) == 0
    with pytest.raises(ValueError):
        qrnnt.mx4_pitch(1 << 32)


@pytest.mark.parametrize("back", [False, True])
def test_quantizer_and_values(lib, back):
    def f(x=0x1000, dt=0, rows=4, cols=40, ld=40, q=0x20000, ld_q=32, s=0x30000, ld_s=8):
        if back:
            return lib.qrnnt_dequantize_mx4(q, ld_q, s, ld_s, rows, cols, x, dt, ld, None)
        return lib.qrnnt_quantize_mx4(x, dt, rows, cols, ld, q, ld_q, s, ld_s, None)
    assert f(x=None) == NULL and f(q=None) == NULL and f(s=None) == NULL
    assert f(dt=3) == RANGE and f(dt=-1) == RANGE
    assert f(rows=-1) == SHAPE and f(cols=0) == SHAPE and f(ld=39) == SHAPE and f(ld_q=16) == SHAPE and f(ld_q=40) == SHAPE and f(ld_s=0) == SHAPE and f(ld_s=12) == SHAPE
    assert f(cols=300, ld=300, ld_q=160) == SHAPE   # two times eight scales
    assert f(rows=1 << 31) == UNSUPPORTED and f(cols=(1 << 30) + 1, ld=1 << 31, ld_q=1 << 30) == UNSUPPORTED and f(ld=1 << 59) == UNSUPPORTED
    assert f(x=0x1002) == ALIGN and f(q=0x20008) == ALIGN and f(s=0x30004) == ALIGN and f(x=0x1001, dt=2) == ALIGN
    assert f(rows=0) == OK and f(rows=0, x=None, q=None, s=None) == OK


def test_pack(lib):
    f = lambda q=0x1000, ld_q=32, s=0x2001, ld_s=2, rows=5, cols=40, out=0x10000: lib.qrnnt_pack_mx4(q, ld_q, s, ld_s, rows, cols, out, None)
    assert f(q=None) == NULL and f(s=None) == NULL and f(out=None) == NULL
    assert f(rows=0) == SHAPE and f(cols=-1) == SHAPE and f(ld_q=16) == SHAPE and f(ld_q=40) == SHAPE and f(ld_s=1) == SHAPE
    assert f(q=0x1008) == ALIGN and f(out=0x10008) == ALIGN
    assert f(cols=(1 << 20) + 1, ld_q=1 << 20, ld_s=1 << 20) == UNSUPPORTED and f(rows=(1 << 28) + 1) == UNSUPPORTED and f(rows=1 << 28, cols=512, ld_q=256, ld_s=16) == UNSUPPORTED
    assert lib.qrnnt_pack_mx4_bytes(5, 40) == 2048 + 128 and lib.qrnnt_pack_mx4_bytes(17, 257) == 4 * 2176
    for bad in ((0, 4), (4, 0), (-1, 4), (4, (1 << 20) + 1), ((1 << 28) + 1, 4)):
        assert lib.qrnnt_pack_mx4_bytes(*bad) == 0


def _mat(rows=64, cols=100, packed=0x1000):
    return qrnnt.CMx4(packed, rows, cols)


def test_linear(lib):
    def f(m=None, bias=None, a=0x10000, ld_a=64, s=0x3000, ld_s=8, M=5, y=0x40000, dt=0, ld_y=64, ws=None, n=0):
        return lib.qrnnt_linear_mx4(C.byref(m or _mat()), bias, a, ld_a, s, ld_s, M, y, dt, ld_y, ws, n, None)
    assert lib.qrnnt_linear_mx4(None, None, 0x10000, 64, 0x3000, 8, 5, 0x40000, 0, 64, None, 0, None) == NULL
    assert f(a=None) == NULL and f(s=None) == NULL and f(y=None) == NULL and f(_mat(packed=None)) == NULL
    assert f(_mat(rows=0)) == SHAPE and f(_mat(cols=0)) == SHAPE and f(M=-1) == SHAPE and f(ld_a=48) == SHAPE and f(ld_a=72) == SHAPE and f(ld_s=4) == SHAPE and f(ld_y=63) == SHAPE
    assert f(dt=3) == RANGE
    assert f(a=0x10008) == ALIGN and f(y=0x40002) == ALIGN and f(y=0x40001, dt=1) == ALIGN and f(bias=0x5001) == ALIGN and f(s=0x3004) == ALIGN and f(_mat(packed=0x1008)) == ALIGN
    assert f(M=(1 << 28) + 1) == UNSUPPORTED and f(_mat(rows=(1 << 28) + 1), ld_y=1 << 31) == UNSUPPORTED and f(ld_y=1 << 60) == UNSUPPORTED
    assert f(_mat(cols=(1 << 20) + 1), ld_a=1 << 20, ld_s=1 << 16) == UNSUPPORTED
    assert f(_mat(rows=1 << 20), M=1 << 20, ld_y=1 << 20) == UNSUPPORTED   # more tiles than a grid has
    assert f(M=0) == OK and f(M=0, a=None, y=None) == OK
    assert lib.qrnnt_linear_mx4_workspace(None, 4) == 0 and lib.qrnnt_linear_mx4_workspace(C.byref(_mat()), 0) == 0
    some = 0
    for rows, cols, M in ((64, 1 << 20, 33), (64, 8192, 16), (100, 9000, 200), (8192, 8192, 8192)):
        m = _mat(rows, cols)
        need = lib.qrnnt_linear_mx4_workspace(C.byref(m), M)
        more = dict(ld_a=qrnnt.mx4_pitch(cols), ld_s=qrnnt.mx4_scale_pitch(cols), M=M, ld_y=rows)
        if need:
            some += 1
            assert f(m, **more) == NULL
            assert f(m, ws=0x100000, n=need - 1, **more) == WORKSPACE
            assert f(m, ws=0x100010, n=need, **more) == ALIGN
    assert some >= 2


def test_workspaces_do_not_fall_as_a_call_grows(lib):
    rising = lambda sizes: all(a <= b for a, b in zip(sizes, sizes[1:]))
    rng = random.Random(3)
    for _ in range(1000):
        rows, cols, M = int(16 * 2000 ** rng.random()), int(40 * 2000 ** rng.random()), int(1 + 17 * 2000 ** rng.random())
        m = _mat(rows, cols)
        assert rising([lib.qrnnt_linear_mx4_workspace(C.byref(m), max(1, int(M * f))) for f in (0.1, 0.3, 0.5, 0.9, 0.99, 1, 1.01, 1.1, 2, 10)])
    largest = (1 << 25, 1 << 30, 64)
    for _ in range(1000):
        sizes = [rng.choice([1, 2, 15, 16, 255, 256, 257, 4000]), rng.choice([1, 2048, 8193, 16384, 16385, 32000, 131072, 300000, 1 << 20]), rng.randint(0, 64)]
        at = rng.randrange(3)
        got = []
        for v in sorted({min(largest[at], max(1, int(sizes[at] * f))) for f in (0.5, 0.9, 0.999, 1, 1.001, 1.1, 2, 7)}):
            sizes[at] = v
            got.append(qrnnt.token_scores_workspace(*sizes))
        assert all(got) and rising(got)


def test_token_scores(lib):
    def f(x=0x10000, dt=0, ld=100, t=0x1000, rows=3, V=100, n=4, lp=0x2000, ent=0x3000, tok=0x4000, val=0x5000, ws=0x100000, size=1 << 30):
        return lib.qrnnt_token_scores(x, dt, ld, t, rows, V, n, lp, ent, tok, val, ws, size, None)
    for name in ("x", "t", "tok", "val", "ws"):
        assert f(**{name: None}) == NULL
    assert f(dt=3) == RANGE
    assert f(rows=-1) == SHAPE and f(V=0) == SHAPE and f(n=-1) == SHAPE and f(ld=99) == SHAPE
    assert f(n=65) == UNSUPPORTED and f(rows=(1 << 25) + 1) == UNSUPPORTED and f(V=(1 << 30) + 1, ld=1 << 31) == UNSUPPORTED and f(ld=1 << 60) == UNSUPPORTED
    assert f(x=0x10002) == ALIGN and f(x=0x10001, dt=1) == ALIGN and f(t=0x1001) == ALIGN and f(lp=0x2002) == ALIGN and f(ent=0x3001) == ALIGN and f(tok=0x4002) == ALIGN
    assert f(val=0x5002) == ALIGN and f(ws=0x100040) == ALIGN
    need = qrnnt.token_scores_workspace(3, 100, 4)
    assert need > 0 and f(size=need - 1) == WORKSPACE
    assert f(rows=0) == OK and f(rows=0, x=None, ws=None) == OK
    for bad in ((-1, 10, 1), (1, 0, 1), (1, 10, 65), (1, 10, -1), ((1 << 25) + 1, 10, 0)):
        assert qrnnt.token_scores_workspace(*bad) == 0
    for at in range(3):
        sizes = [2, 100, 4]
        sizes[at] += 1 << 32
        with pytest.raises(ValueError):
            qrnnt.token_scores_workspace(*sizes)


def test_wrappers_refuse_tensors_that_are_not_on_the_gpu():
    x, codes, scale = torch.zeros((4, 32)), torch.zeros((4, 16), dtype=torch.uint8), torch.zeros((4, 8), dtype=torch.uint8)
    m = qrnnt.Mx4Mat(torch.zeros(2176, dtype=torch.uint8), 16, 32)
    for call in (lambda: qrnnt.quantize_mx4(x), lambda: qrnnt.dequantize_mx4(codes, scale, 32), lambda: qrnnt.pack_mx4(codes, scale, 32),
                 lambda: qrnnt.linear_mx4(m, codes, scale), lambda: qrnnt.token_scores(x)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        qrnnt.linear_mx4_workspace(m, 1 << 32)


def test_wrappers_refuse_codes_of_other_shapes_and_types():
    u8 = lambda *shape: torch.zeros(shape, dtype=torch.uint8)
    ok = qrnnt._mx4(u8(4, 32), u8(4, 8), 4, 40)
    assert ok[1] == 32 and ok[3] == 8
    assert qrnnt._mx4(u8(1, 32), u8(1, 8), 1, 40)[1::2] == (32, 8) and qrnnt._mx4(u8(0, 32), u8(0, 8), 0, 40)[1::2] == (32, 8)
    assert qrnnt._mx4(u8(4, 64)[:, :32], u8(4, 24)[:, :8], 4, 40)[1::2] == (64, 24)
    assert qrnnt._mx4(u8(2, 3, 64)[:1, 0], u8(3, 24)[1:2, :8], 1, 40)[1::2] == (32, 8)
    for codes, scale in ((u8(4, 31), u8(4, 8)), (u8(4, 32), u8(4, 7)), (u8(3, 32), u8(4, 8)), (u8(4, 32), u8(5, 8)), (u8(4, 64)[:, ::2], u8(4, 8)),
                         (u8(4, 32), u8(4, 16)[:, ::2]), (u8(32, 4).t(), u8(4, 8)), (u8(1, 32).expand(4, 32), u8(4, 8)), (u8(1, 64)[:, ::2], u8(1, 8))):
        with pytest.raises(ValueError):
            qrnnt._mx4(codes, scale, codes.shape[0] if codes.shape[0] == 1 else 4, 40)
    for codes, scale in ((u8(4, 32).to(torch.int8), u8(4, 8)), (u8(4, 32), u8(4, 8).to(torch.int8))):
        with pytest.raises(TypeError):
            qrnnt._mx4(codes, scale, 4, 40)
    far = lambda rows, cols, pitch: torch.empty_strided((rows, cols), (pitch, 1), dtype=torch.uint8, device="meta")
    for codes, scale, rows in ((far(2, 32, 1 << 31), far(2, 8, 8), 2), (far(2, 32, 32), far(2, 8, 1 << 31), 2), (far(1 << 31, 32, 32), far(1 << 31, 8, 8), 1 << 31)):
        with pytest.raises(ValueError):
            qrnnt._mx4(codes, scale, rows, 40)

"""4-bit experts without a GPU: the oracle's own format, the sizes the library
reports, and every refusal of the calls (nothing is enqueued by any of them)."""
import ctypes

import numpy as np
import pytest

from oracle import mx
from paper_2609_36222_amd import binding as bd
from test_abi import (ALIGN, BUDGET, DTYPE, FAKE, NULL, OK, SHAPE, WS,  # noqa: F401
                      decode, layer, lib)

MXL = dict(w_layout=4)


def test_oracle_rounds_to_the_nearest_code_and_even_on_ties():
    grid = np.concatenate([-mx.E2M1[::-1], mx.E2M1])
    t = np.linspace(-7.99, 7.99, 3197)
    v = np.zeros((len(t), 32))
    v[:, 0], v[:, 1] = 6.0, t          # 6 (or t itself, below 8) fixes the scale at 2^0
    codes, scales = mx.quantize(v)
    assert (scales == 127).all()
    got = mx.dequantize(codes, scales)[:, 1]
    best = np.abs(grid[None] - np.clip(t, -6, 6)[:, None]).min(1)
    assert np.allclose(np.abs(got - np.clip(t, -6, 6)), best, atol=1e-12)
    ties = {0.25: 0.0, 0.75: 1.0, 1.25: 1.0, 1.75: 2.0, 2.5: 2.0, 3.5: 4.0, 5.0: 4.0}
    for a, b in ties.items():
        v = np.zeros((2, 32))
        v[:, 0], v[0, 1], v[1, 1] = 4.0, a, -a
        assert mx.dequantize(*mx.quantize(v))[:, 1].tolist() == [b, -b]


def test_oracle_special_blocks():
    v = np.zeros((5, 32))
    v[1, 3], v[2, 5], v[3, 0], v[4, 1] = np.nan, -np.inf, 2.0 ** -140, 3.0e38
    codes, scales = mx.quantize(v)
    assert scales.ravel().tolist() == [0, 255, 255, 0, 127 + 127 - 2]
    assert (codes[:3] == 0).all() and np.isnan(mx.dequantize(codes, scales)[1:3]).all()


@pytest.mark.parametrize("E,d,I", [(1, 256, 64), (3, 512, 192), (60, 2048, 1408), (8, 4096, 14336)])
def test_bytes(lib, E, d, I):
    L = layer(E=E, K=1, d=d, I=I)
    per = lambda rows, K: rows // 16 * (-(-K // 512) * 256 + -(-K // 128) * 1024)  # noqa: E731
    assert lib.base_mx_w13_bytes(ctypes.byref(L)) == E * per(2 * I, d)
    assert lib.base_mx_w2_bytes(ctypes.byref(L)) == E * per(d, I)


@pytest.mark.parametrize("kw", [dict(E=0), dict(E=257), dict(d=128), dict(d=300), dict(d=16640),
                                dict(I=0), dict(I=100), dict(I=32832)])
def test_bytes_of_a_bad_shape(lib, kw):
    assert lib.base_mx_w13_bytes(ctypes.byref(layer(**kw))) == 0
    assert lib.base_mx_w2_bytes(ctypes.byref(layer(**kw))) == 0


def test_bytes_null(lib):
    assert lib.base_mx_w13_bytes(None) == 0 and lib.base_mx_w2_bytes(None) == 0


def test_layer_layout(lib):
    assert decode(lib, layer(dtype=0, **MXL), nbytes=1 << 40) == DTYPE
    L = layer(**MXL)
    n = lib.base_workspace_bytes(ctypes.byref(L), 16, 4)
    assert n > 0
    assert decode(lib, L, nbytes=n - 1) == WS
    assert decode(lib, layer(w13=0, **MXL)) == NULL
    assert decode(lib, layer(w2=FAKE + 8, **MXL)) == ALIGN
    assert decode(lib, L, budget=0, nbytes=n) == BUDGET
    assert lib.base_pack_experts(ctypes.byref(L), FAKE, FAKE, None) == SHAPE
    for w in (2, 3, 5):
        assert decode(lib, layer(w_layout=w), nbytes=1 << 40) == SHAPE


@pytest.mark.parametrize("B", [1, 64, 65, 1024])
def test_workspace_covers_smaller_budgets(lib, B):
    """Sized for one budget it holds every smaller one."""
    L = layer(E=256, K=8, n_shared=3, w13_shared=FAKE, w2_shared=FAKE, **MXL)
    n = [lib.base_workspace_bytes(ctypes.byref(L), B, b) for b in (1, 2, 7, 64, 65, 255, 256, 999)]
    assert n == sorted(n) and n[-1] == n[-2] and n[0] > 0


@pytest.mark.parametrize("kw", [dict(), dict(d=256, E=4, K=2, I=64), dict(E=8, K=1, I=14336, n_shared=2,
                                                                          w13_shared=FAKE, w2_shared=FAKE)])
def test_workspace_covers_smaller_batches(lib, kw):
    """A serving program sizes its workspace for its largest batch."""
    L = layer(**kw, **MXL)
    for budget in (1, 4, 200):
        n = [lib.base_workspace_bytes(ctypes.byref(L), B, budget)
             for B in (1, 2, 4, 5, 8, 9, 16, 17, 31, 32, 33, 48, 63, 64, 65, 66, 100, 128, 500, 1024)]
        assert n == sorted(n) and n[0] > 0


def test_stages(lib):
    """The launches of a 4-bit layer: the plan of few tokens makes their routes, down's
    launch their combine (while their slots are few)."""
    def launched(B, budget, **kw):
        return bd.layer_stages(layer(**kw, **MXL), B, budget)
    assert launched(1, 10) == ("scores", "select", "ffn_gateup", "ffn_down")
    assert launched(4, 128) == ("scores", "select", "ffn_gateup", "ffn_down")
    assert launched(16, 10) == ("scores", "select", "ffn_gateup", "ffn_down", "combine")
    assert launched(16, 4) == ("scores", "select", "ffn_gateup", "ffn_down")
    assert launched(17, 4) == ("scores", "tail", "select", "ffn_gateup", "ffn_down", "combine")
    assert launched(65, 4) == ("scores", "tail", "select", "compact", "ffn_gateup", "ffn_down", "combine")


@pytest.mark.parametrize("d,E,K,I,B,budget,joined", [
    # one to four tokens: few workgroups, long ones
    (256, 64, 8, 768, 1, 8, True), (256, 32, 8, 768, 4, 32, False), (256, 32, 8, 7168, 1, 8, False),
    (256, 32, 8, 14336, 4, 32, False), (512, 64, 8, 4096, 4, 8, True), (512, 64, 8, 4608, 4, 8, False),
    (1024, 64, 8, 512, 2, 16, False), (1024, 16, 2, 14336, 2, 2, True), (1024, 64, 8, 7168, 4, 16, False),
    (2048, 128, 8, 768, 4, 32, True), (2048, 64, 8, 4096, 1, 8, True), (2048, 32, 8, 6144, 1, 8, False),
    (2048, 8, 2, 14336, 4, 8, False), (3584, 32, 8, 6144, 4, 12, True), (3584, 32, 8, 6144, 4, 16, False),
    (4096, 8, 2, 14336, 4, 8, True), (4096, 64, 8, 1024, 4, 32, True), (4608, 64, 8, 1408, 1, 2, True),
    (4608, 64, 8, 1408, 1, 4, False), (16384, 16, 4, 4096, 4, 4, False),
    # five to eight, nine to sixteen
    (2048, 64, 8, 2048, 8, 10, True), (2048, 64, 8, 2048, 8, 12, False), (2048, 16, 4, 6144, 8, 6, False),
    (2048, 64, 8, 2048, 16, 4, True), (2048, 64, 8, 2048, 16, 5, False), (2048, 16, 4, 6144, 16, 2, False)])
def test_where_downs_launch_combines(lib, d, E, K, I, B, budget, joined):
    """The side of its line that is faster, for both sides of each term."""
    s = bd.layer_stages(layer(d=d, E=E, K=K, I=I, **MXL), B, budget)
    assert ("combine" not in s) == joined, s


def test_quantize_refusals(lib):
    def q(dtype=1, src=FAKE, rows=4, cols=64, ld=64, codes=FAKE, scales=FAKE):
        return lib.base_mx_quantize(dtype, src, rows, cols, ld, codes, scales, None)
    assert q(dtype=2) == DTYPE
    for kw in (dict(rows=0), dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=48),
               dict(cols=-32), dict(cols=(1 << 24) + 32, ld=1 << 25), dict(ld=63), dict(ld=0),
               dict(ld=-64), dict(ld=(1 << 40) + 1)):
        assert q(**kw) == SHAPE, kw
    assert q(src=0) == NULL and q(codes=0) == NULL and q(scales=0) == NULL
    assert q(src=FAKE + 1) == ALIGN and q(src=FAKE + 2, dtype=0) == ALIGN
    assert q(codes=FAKE + 8) == ALIGN


def test_dequantize_refusals(lib):
    def q(dtype=1, dst=FAKE, rows=4, cols=64, ld=64, codes=FAKE, scales=FAKE):
        return lib.base_mx_dequantize(codes, scales, rows, cols, dtype, dst, ld, None)
    assert q(dtype=-1) == DTYPE
    for kw in (dict(rows=0), dict(cols=31), dict(ld=32)):
        assert q(**kw) == SHAPE, kw
    assert q(dst=0) == NULL and q(codes=0) == NULL and q(scales=0) == NULL
    assert q(dst=FAKE + 1) == ALIGN and q(dst=FAKE + 2, dtype=0) == ALIGN


def test_pack_refusals(lib):
    def p(L, *ptr):
        return lib.base_mx_pack_experts(ctypes.byref(L), *(ptr or [FAKE] * 6), None)
    ok = [FAKE] * 6
    for i in range(6):
        assert p(layer(), *[0 if j == i else v for j, v in enumerate(ok)]) == NULL
    for i in (0, 2, 4, 5):
        assert p(layer(), *[v + 8 if j == i else v for j, v in enumerate(ok)]) == ALIGN
    assert p(layer(w_layout=1)) == SHAPE and p(layer(**MXL)) == SHAPE
    assert p(layer(I=96)) == SHAPE and p(layer(d=128)) == SHAPE and p(layer(dtype=3)) == DTYPE
    assert lib.base_mx_pack_experts(None, *ok, None) == NULL


def test_quantize_experts_refusals(lib):
    def p(L, a=FAKE, b=FAKE):
        return lib.base_mx_quantize_experts(ctypes.byref(L), a, b, None)
    assert p(layer(), a=0) == NULL and p(layer(), b=FAKE + 4) == ALIGN
    assert p(layer(w13=0)) == NULL and p(layer(w2=FAKE + 4)) == ALIGN
    assert p(layer(w_layout=1)) == SHAPE and p(layer(**MXL)) == SHAPE
    assert lib.base_mx_quantize_experts(None, FAKE, FAKE, None) == NULL


def test_calibration_takes_the_layout(lib):
    L = layer(**MXL)
    n = lib.base_calib_ws_bytes(ctypes.byref(L), 300)
    assert n > 0
    assert lib.base_calib_accumulate(ctypes.byref(L), FAKE, 300, FAKE, FAKE, n - 1, None) == WS


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        bd.mx_quantize(torch.zeros(2, 64))
    with pytest.raises(ValueError):
        bd.mx_quantize(torch.zeros(2, 64, dtype=torch.float16))
    with pytest.raises(ValueError):
        bd.mx_dequantize(torch.zeros(2, 32, dtype=torch.uint8), torch.zeros(2, 3, dtype=torch.uint8))


def packed(n, d, I):
    torch = pytest.importorskip("torch")
    L = layer(E=n, K=1, d=d, I=I)
    return [torch.zeros(f(ctypes.byref(L)), dtype=torch.uint8)
            for f in (bd.load().base_mx_w13_bytes, bd.load().base_mx_w2_bytes)]


def test_binding_compares_packed_experts_with_the_router():
    """The packed bytes carry no shape, and the kernels read as far as the layer's."""
    torch = pytest.importorskip("torch")
    def make(E=4, d=512, w=(4, 512, 192), I=192, shared=None, **kw):
        return bd.Layer.mxfp4(torch.zeros(E, d), None, None, None, *packed(*w), I, shared=shared, **kw)
    lay = make(shared=(*packed(2, 512, 192), torch.zeros(512), 2))
    assert (lay.E, lay.d, lay.I, lay.desc(2).n_shared) == (4, 512, 192, 2)
    assert make(shared=(None, None, None, 0)).desc(2).n_shared == 0
    for kw in (dict(E=5), dict(E=3), dict(d=768), dict(I=256), dict(I=128),
               dict(shared=(*packed(1, 512, 192), None, 2)),              # fewer than said
               dict(shared=(*packed(1, 512, 768), None, 1)),              # a wider one in one piece
               dict(shared=(*packed(1, 256, 192), None, 1)),
               dict(shared=(*packed(1, 512, 192), torch.zeros(256), 1)),
               dict(shared=(*packed(1, 512, 192), torch.zeros(512).bfloat16(), 1))):
        with pytest.raises(ValueError):
            make(**kw)
    for bad in (lambda t: t[:-1], lambda t: t.view(torch.int8), lambda t: torch.cat((t, t))[::2]):
        a, b = packed(4, 512, 192)
        for pair in ((bad(a), b), (a, bad(b))):
            with pytest.raises(ValueError):
                bd.Layer.mxfp4(torch.zeros(4, 512), None, None, None, *pair, 192)
    with pytest.raises(bd.BaseError):
        make(I=100)


def test_binding_compares_experts_with_the_router():
    """... of as many bytes, too: half the experts of twice the width."""
    torch = pytest.importorskip("torch")
    z = torch.zeros
    def rowmajor(E, d, n, dw, I, Is=None, ds=None):
        shared = None if Is is None else (z(1, 2 * Is, ds), z(1, ds, Is), None)
        return bd.Layer(z(E, d), None, None, None, z(n, 2 * I, dw), z(n, dw, I), shared=shared)
    for a in ((4, 256, 2, 512, 64), (4, 512, 3, 512, 64), (4, 256, 4, 512, 64), (4, 256, 4, 256, 64, 128, 256),
              (4, 256, 4, 256, 64, 64, 512)):
        with pytest.raises(ValueError, match="w13, w2: "):
            bd.mx_layer(rowmajor(*a))
    u8 = dict(dtype=torch.uint8)
    def pair(n, rows, cols):
        return z(n, rows, cols // 2, **u8), z(n, rows, cols // 32, **u8)
    def codes(E, d, n, dw, I, Is=None, ds=None):
        shared = None if Is is None else (pair(1, 2 * Is, ds), pair(1, ds, Is), None)
        return bd.mx_layer_from_codes(z(E, d), None, None, None, pair(n, 2 * I, dw), pair(n, dw, I), shared=shared)
    for a in ((4, 256, 2, 512, 64), (4, 512, 3, 512, 64), (4, 256, 4, 512, 64), (4, 256, 4, 256, 64, 128, 256),
              (4, 256, 4, 256, 64, 64, 512)):
        with pytest.raises(ValueError, match="w13, w2: "):
            codes(*a)

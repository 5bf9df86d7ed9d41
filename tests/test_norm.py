"""Refusals of the norm calls, without a GPU (nothing is enqueued)."""
import ctypes

import pytest

from paper_2609_36222_amd import binding as bd
from test_abi import ALIGN, BUDGET, DTYPE, FAKE, FLAGS, NULL, SHAPE, WS, layer, lib  # noqa: F401

INF, NAN = float("inf"), float("nan")


def norms(**kw):
    v = dict(d=2048, dtype=1, eps=1e-6, res_scale=1.0, post_gain=FAKE, gate=FAKE, gate_ld=0, pre_gain=FAKE)
    v.update(kw)
    return bd.base_norms(*(v[f] for f, _ in bd.base_norms._fields_))


def call(lib, N, rows=4, y=FAKE, yl=2048, h=FAKE << 1, hl=2048, ho=FAKE << 2, hol=2048, xo=FAKE << 3, xol=2048):
    return lib.base_norm_residual(ctypes.byref(N) if N else None, rows, y, yl, h, hl, ho, hol, xo, xol, None)


@pytest.mark.parametrize("kw,expect", [
    (dict(d=0), SHAPE), (dict(d=-1), SHAPE), (dict(d=16385), SHAPE), (dict(dtype=2), DTYPE),
    (dict(dtype=-1), DTYPE), (dict(eps=-1e-6), SHAPE), (dict(eps=NAN), SHAPE), (dict(eps=INF), SHAPE),
    (dict(res_scale=INF), SHAPE), (dict(res_scale=NAN), SHAPE), (dict(gate_ld=2047), SHAPE),
    (dict(gate_ld=-1), SHAPE), (dict(gate_ld=(1 << 40) + 1), SHAPE), (dict(pre_gain=0), NULL),
    (dict(post_gain=FAKE + 2), ALIGN), (dict(gate=FAKE + 1), ALIGN), (dict(pre_gain=FAKE + 2), ALIGN)])
def test_parameters(lib, kw, expect):
    assert call(lib, norms(**kw)) == expect


def test_rows_and_pointers(lib):
    N = norms()
    assert call(lib, None) == NULL and call(lib, N, h=0) == NULL
    assert call(lib, N, ho=0, xo=0) == NULL
    for rows in (0, -5, 1 << 31):
        assert call(lib, N, rows=rows) == SHAPE
    for f in ("yl", "hl", "hol", "xol"):
        assert call(lib, N, **{f: 2047}) == SHAPE and call(lib, N, **{f: (1 << 40) + 1}) == SHAPE
    for f in ("y", "h", "ho", "xo"):
        assert call(lib, N, **{f: FAKE + 1}) == ALIGN
        assert call(lib, norms(dtype=0), **{f: FAKE + 2}) == ALIGN
    assert call(lib, N, y=0) == FLAGS                       # nothing to add to h
    assert call(lib, N, ho=FAKE << 3) == FLAGS              # both outputs in one place
    assert call(lib, N, ho=FAKE << 1, hol=4096) == FLAGS    # in place, another stride
    assert call(lib, N, xo=FAKE, xol=4096) == FLAGS
    assert call(lib, N, ho=0, xo=FAKE << 1, xol=4096) == FLAGS
    assert call(lib, N, ho=FAKE, hol=4096) == FLAGS


def test_block_refusals(lib):
    def blk(L=None, N=None, B=4, budget=4, flags=0, x=FAKE, h=FAKE, ho=FAKE << 2, xo=FAKE << 3, ws=FAKE, n=None):
        L, N = L or layer(), N or norms()
        n = lib.base_workspace_bytes(ctypes.byref(L), 4, 4) if n is None else n
        return lib.base_decode_block(ctypes.byref(L), ctypes.byref(N), x, B, budget, flags, h, ho, xo, None, ws, n, None)
    assert blk(B=0) == SHAPE and blk(budget=0) == BUDGET and blk(flags=4) == FLAGS
    assert blk(x=0) == NULL and blk(h=0) == NULL and blk(ho=0, xo=0) == NULL and blk(ws=0) == NULL
    assert blk(N=norms(d=1024)) == SHAPE and blk(N=norms(dtype=0)) == DTYPE
    assert blk(N=norms(eps=-1.0)) == SHAPE and blk(N=norms(pre_gain=0)) == NULL
    for f in ("h", "ho", "xo"):
        assert blk(**{f: FAKE + 8}) == ALIGN
    for f in ("post_gain", "gate", "pre_gain"):
        assert blk(N=norms(**{f: FAKE + 4})) == ALIGN
    assert blk(N=norms(gate_ld=2050)) == ALIGN
    assert blk(ho=FAKE << 3) == FLAGS
    n = lib.base_workspace_bytes(ctypes.byref(layer()), 4, 4)
    assert blk(n=n - 1) == WS
    assert lib.base_decode_block(ctypes.byref(layer()), None, FAKE, 4, 4, 0, FAKE, FAKE, 0, None, FAKE, n, None) == NULL


def test_binding_refusals():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        bd.Norms(64, torch.float16)
    with pytest.raises(ValueError):
        bd.Norms(64, torch.bfloat16, post_gain=torch.ones(64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        bd.Norms(64, torch.bfloat16, pre_gain=torch.ones(63))
    with pytest.raises(ValueError):
        bd.Norms(64, torch.bfloat16, post_gain=torch.ones(4, 64))
    n = bd.Norms(64, torch.bfloat16)
    h = torch.zeros(4, 64, dtype=torch.bfloat16)
    for bad in (torch.zeros(4, 32, dtype=torch.bfloat16), torch.zeros(3, 64, dtype=torch.bfloat16),
                torch.zeros(4, 64), h):          # the last: on the host
        with pytest.raises(ValueError):
            bd.base_norm_residual(n, bad, h)

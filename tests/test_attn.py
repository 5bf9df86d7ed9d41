"""Refusals of the calls on heads, the paged cache and its attention, without a GPU (nothing
is enqueued), and the frequencies' helper."""
import ctypes

import pytest

from paper_2609_36222_amd import binding as bd
from test_abi import ALIGN, DTYPE, FAKE, FLAGS, NULL, SHAPE, WS, lib  # noqa: F401

INF, NAN = float("inf"), float("nan")
BIG = (1 << 40) + 8


def make(cls, base, kw):
    v = dict(base)
    v.update(kw)
    return cls(*(v[f] for f, _ in cls._fields_))


def rope(**kw):
    return make(bd.base_rope, dict(D=128, rot=128, dtype=1, layout=0, eps=1e-6, rot_scale=1.0, inv_freq=FAKE,
                                   q_gain=FAKE, k_gain=FAKE), kw)


def heads(p=FAKE, row=4096, head=128):
    return p, row, head


def cache(**kw):
    return make(bd.base_kv_cache, dict(Hk=4, D=128, dtype=1, page_size=16, n_pages=100, k=FAKE, v=FAKE << 1,
                                       k_page=8192, k_slot=128, k_head=2048, v_page=8192, v_slot=128,
                                       v_head=2048), kw)


def batch(**kw):
    return make(bd.base_kv_batch, dict(n_seq=3, max_pages=20, table_ld=20, max_q=2, table=FAKE, q_start=FAKE,
                                       kv_len=FAKE), kw)


def ref(x):
    return None if x is None else ctypes.byref(x)


def turn(lib, R=rope(), rows=4, pos=FAKE, Hq=32, q=heads(), qo=heads(FAKE << 1), Hk=4, k=heads(FAKE << 2),
         ko=heads(FAKE << 3)):
    return lib.base_head_rope(ref(R), rows, pos, Hq, *q, *qo, Hk, *k, *ko, None)


def append(lib, R=rope(), C=cache(), S=batch(), rows=4, pos=None, Hq=32, q=heads(), qo=heads(FAKE << 1),
           k=heads(FAKE << 2), v=heads(FAKE << 3)):
    return lib.base_kv_append(ref(R), ref(C), ref(S), rows, pos, Hq, *q, *qo, *k, *v, None)


def attend(lib, C=cache(), S=batch(), rows=4, Hq=32, q=heads(), out=heads(FAKE << 1), lse=None, scale=0.1, window=0,
           ws=FAKE, n=1 << 40):
    return lib.base_paged_attention(ref(C), ref(S), rows, Hq, *q, *out, lse, scale, window, ws, n, None)


BAD_ROPE = [(dict(D=4), SHAPE), (dict(D=264), SHAPE), (dict(D=124), SHAPE), (dict(rot=-2), SHAPE),
            (dict(rot=130), SHAPE), (dict(rot=63), SHAPE), (dict(dtype=2), DTYPE), (dict(layout=2), FLAGS),
            (dict(eps=-1.0), SHAPE), (dict(eps=NAN), SHAPE), (dict(rot_scale=INF), SHAPE), (dict(inv_freq=0), NULL),
            (dict(inv_freq=FAKE + 2), ALIGN), (dict(q_gain=FAKE + 1), ALIGN), (dict(k_gain=FAKE + 2), ALIGN)]


@pytest.mark.parametrize("kw,expect", BAD_ROPE)
def test_rope(lib, kw, expect):
    assert turn(lib, rope(**kw)) == expect
    assert append(lib, rope(**kw)) == expect


def test_head_rope_arguments(lib):
    assert turn(lib, None) == NULL and turn(lib, pos=None) == NULL and turn(lib, pos=FAKE + 2) == ALIGN
    for rows in (0, -1, 1 << 31):
        assert turn(lib, rows=rows) == SHAPE
    assert turn(lib, Hq=0, Hk=0) == SHAPE and turn(lib, Hq=-1) == SHAPE and turn(lib, Hk=1025) == SHAPE
    for f in ("q", "qo", "k", "ko"):
        assert turn(lib, **{f: heads(0)}) == NULL
        assert turn(lib, **{f: heads(FAKE + 1)}) == ALIGN
        assert turn(lib, rope(dtype=0), **{f: heads(FAKE + 2)}) == ALIGN
        for bad in (heads(row=-1), heads(head=-8), heads(row=BIG), heads(head=BIG)):
            assert turn(lib, **{f: bad}) == SHAPE
    assert turn(lib, qo=heads(row=4104)) == FLAGS                 # in place, another stride
    assert turn(lib, ko=heads(FAKE << 2, head=136)) == FLAGS


BAD_CACHE = [(dict(Hk=0), SHAPE), (dict(Hk=1025), SHAPE), (dict(D=4), SHAPE), (dict(D=260), SHAPE),
             (dict(dtype=-1), DTYPE), (dict(page_size=8), SHAPE), (dict(page_size=48), SHAPE),
             (dict(page_size=131072), SHAPE), (dict(n_pages=0), SHAPE), (dict(k=0), NULL), (dict(v=0), NULL),
             (dict(k=FAKE + 8), ALIGN), (dict(v=FAKE + 2), ALIGN), (dict(k_page=-8), SHAPE), (dict(k_slot=BIG), SHAPE), (dict(v_slot=(1 << 25) + 8), SHAPE),
             (dict(k_head=4), ALIGN), (dict(v_page=BIG), SHAPE), (dict(v_slot=132), ALIGN), (dict(v_head=-1), SHAPE)]
BAD_BATCH = [(dict(n_seq=0), SHAPE), (dict(n_seq=65537), SHAPE), (dict(max_pages=0), SHAPE),
             (dict(max_pages=(1 << 26) + 1), SHAPE), (dict(table_ld=19), SHAPE), (dict(table_ld=BIG), SHAPE),
             (dict(max_q=0), SHAPE), (dict(table=0), NULL), (dict(q_start=0), NULL), (dict(kv_len=0), NULL),
             (dict(table=FAKE + 1), ALIGN), (dict(q_start=FAKE + 2), ALIGN), (dict(kv_len=FAKE + 3), ALIGN)]


@pytest.mark.parametrize("kw,expect", BAD_CACHE)
def test_cache(lib, kw, expect):
    assert append(lib, C=cache(**kw)) == expect and attend(lib, C=cache(**kw)) == expect


@pytest.mark.parametrize("kw,expect", BAD_BATCH)
def test_batch(lib, kw, expect):
    assert append(lib, S=batch(**kw)) == expect and attend(lib, S=batch(**kw)) == expect


def test_append_arguments(lib):
    assert append(lib, None) == NULL and append(lib, C=None) == NULL and append(lib, S=None) == NULL
    assert append(lib, rope(D=64, rot=64)) == SHAPE and append(lib, rope(dtype=0)) == DTYPE
    assert append(lib, rows=0) == SHAPE and append(lib, Hq=0) == SHAPE and append(lib, Hq=1025) == SHAPE
    assert append(lib, pos=FAKE + 2) == ALIGN
    for f in ("q", "qo", "k", "v"):
        assert append(lib, **{f: heads(0)}) == NULL and append(lib, **{f: heads(FAKE + 1)}) == ALIGN
        assert append(lib, **{f: heads(row=BIG)}) == SHAPE
    assert append(lib, qo=heads(row=4104)) == FLAGS


def test_attention_arguments(lib):
    assert attend(lib, None) == NULL and attend(lib, S=None) == NULL
    for rows in (0, 1 << 31):
        assert attend(lib, rows=rows) == SHAPE
    for Hq in (0, 3, 30, 1028):
        assert attend(lib, Hq=Hq) == SHAPE
    assert attend(lib, S=batch(max_q=1 << 30)) == SHAPE            # packed rows past 32 bits
    assert attend(lib, rows=(1 << 28) + 1) == SHAPE                # rows * Hq past 2^33
    assert attend(lib, scale=NAN) == SHAPE and attend(lib, scale=INF) == SHAPE and attend(lib, window=-1) == SHAPE
    for f in ("q", "out"):
        assert attend(lib, **{f: heads(0)}) == NULL and attend(lib, **{f: heads(FAKE + 1)}) == ALIGN
        assert attend(lib, **{f: heads(head=-1)}) == SHAPE
    assert attend(lib, out=heads(head=136)) == FLAGS and attend(lib, lse=FAKE + 2) == ALIGN
    assert attend(lib, ws=None) == NULL and attend(lib, ws=FAKE + 128) == ALIGN


@pytest.mark.parametrize("kw", [dict(), dict(D=64), dict(D=256), dict(dtype=0)])
def test_workspace(lib, kw):
    C = cache(**kw)
    for S in (batch(), batch(max_q=700), batch(max_pages=1), batch(max_pages=1 << 20, table_ld=1 << 20, n_seq=65536)):
        n = lib.base_attention_workspace_bytes(ref(C), ref(S), 4, 32)
        assert n > 0 and n % 256 == 0 and n < 2 << 30
        assert attend(lib, C, S, n=n - 1) == WS
    # a max_q far beyond what the rows can hold, at the largest batches
    S = batch(max_q=1 << 26, max_pages=1 << 20, table_ld=1 << 20, n_seq=65536)
    assert 0 < lib.base_attention_workspace_bytes(ref(C), ref(S), 1 << 27, 32) < 2 << 30
    assert lib.base_attention_workspace_bytes(ref(cache(D=4)), ref(batch()), 4, 32) == 0
    assert lib.base_attention_workspace_bytes(ref(cache()), ref(batch()), 0, 32) == 0
    assert lib.base_attention_workspace_bytes(None, None, 4, 32) == 0


def test_binding_refusals():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        bd.Rope(64, torch.float16)
    with pytest.raises(ValueError):
        bd.Rope(64, torch.bfloat16, inv_freq=torch.ones(32))       # not on the GPU
    with pytest.raises(ValueError):
        bd.KVCache(torch.zeros(4, 16, 2, 64), torch.zeros(4, 16, 2, 64))
    with pytest.raises(ValueError):
        bd.KVBatch(torch.zeros(3, 4, dtype=torch.int32), torch.zeros(4, dtype=torch.int32),
                   torch.zeros(3, dtype=torch.int32), 1)
    for bad in (dict(rot=7), dict(rot=8, base=0.0), dict(rot=8, factor=0.5), dict(rot=8, factor=2, trained=0),
                dict(rot=8, factor=2, trained=100, fast=1, slow=1)):
        with pytest.raises(ValueError):
            bd.rope_frequencies(**bad)
    assert bd.rope_frequencies(0)[0].numel() == 0


def test_frequencies_by_parts():
    np = pytest.importorskip("numpy")
    inv, s = bd.rope_frequencies(128, 1e6, 4.0, trained=32768)
    plain = 1e6 ** (-2.0 * np.arange(64) / 128)
    turns = 32768 * plain / (2 * np.pi)
    ratio = inv.numpy() / plain
    assert abs(s - (0.1 * np.log(4) + 1)) < 1e-12
    assert np.allclose(ratio[turns > 40], 1) and np.allclose(ratio[turns < 0.8], 0.25)
    assert (np.diff(ratio) <= 1e-6).all() and ((ratio > 0.26) & (ratio < 0.99)).any()


@pytest.mark.parametrize("rot,base,factor,trained,fast,slow", [
    (128, 1e4, 4.0, 131072, 32.0, 1.0),        # the last pair turns 2.4 times: between the two
    (64, 1e4, 8.0, 200000, 32.0, 1.0), (128, 500.0, 2.0, 65536, 32.0, 1.0),
    (128, 1e6, 4.0, 32768, 32.0, 1.0), (64, 1e4, 40.0, 4096, 32.0, 1.0), (8, 10.0, 4.0, 3000, 32.0, 1.0),
    (128, 1e4, 4.0, 100, 32.0, 1.0), (64, 1e4, 4.0, 5, 32.0, 1.0), (2, 1e4, 4.0, 100, 32.0, 1.0)])
def test_frequencies_of_any_trained_length(rot, base, factor, trained, fast, slow):
    """Pairs that turn more than `fast` times keep their angle, those that turn less than
    `slow` times have it divided, also where no pair, or every one, is beyond a border; the
    mixture between is linear in the pair's number and ends where `slow` turns are, whether
    or not a pair is there."""
    np = pytest.importorskip("numpy")
    got = bd.rope_frequencies(rot, base, factor, trained, fast, slow)[0].double().numpy()
    plain = base ** (-2.0 * np.arange(rot // 2) / rot)
    turns = trained * plain / (2 * np.pi)
    # the pair's number at which n turns are: base^(-2 i / rot) trained / 2 pi = n
    at = [rot / 2 * np.log(trained / (2 * np.pi * n)) / np.log(base) for n in (fast, slow)]
    lo, hi = max(np.floor(at[0]), 0), min(np.ceil(at[1]), rot - 1)
    far = np.where(turns < slow, 1, np.clip((np.arange(rot // 2) - lo) / max(hi - lo, 1e-3), 0, 1))
    assert np.allclose(got, plain * (1 - far) + plain / factor * far, rtol=2.0 ** -22, atol=0)
    assert np.allclose(got[turns < slow], plain[turns < slow] / factor, rtol=2.0 ** -22, atol=0)
    assert np.allclose(got[turns > fast], plain[turns > fast], rtol=2.0 ** -22, atol=0)


def test_handles_of_another_gpu():
    """A rotation, cache or batch whose tensors lie on another GPU than the current one is
    refused before anything is enqueued: the kernels would read that GPU's addresses here."""
    torch = pytest.importorskip("torch")

    def made(cls, dev):
        m = cls.__new__(cls)
        m.dev, m.D, m.Hk, m.torch_dtype, m.desc = dev, 64, 2, torch.bfloat16, None
        return m
    here = torch.cuda.current_device() if torch.cuda.is_initialized() else 0
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    kinds = (bd.Rope, bd.KVCache, bd.KVBatch)
    for other in kinds:
        r, c, b = (made(k, here + (k is other)) for k in kinds)
        said = f"{other.__name__}: made on GPU {here + 1}, the current one is {here}"
        with pytest.raises(ValueError, match=said):
            bd.base_kv_append(r, c, b, x, x, x, x)
        if other is bd.Rope:
            with pytest.raises(ValueError, match=said):
                bd.base_head_rope(r, None, x, None, x, None)
        else:
            with pytest.raises(ValueError, match=said):
                bd.base_paged_attention(c, b, x, x, x)

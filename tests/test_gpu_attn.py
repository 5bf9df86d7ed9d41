"""Attention over a paged cache on the GPU against 64-bit arithmetic: every head size's
kernel, head layouts, lengths, page sizes, windows, rows that see nothing, garbage around
what is seen.  Tolerances: see attn_util.attend."""
import numpy as np
import pytest

import attn_util as U

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
BF, F32 = U.BF, U.F32


@pytest.fixture(scope="module")
def bd(gpu):
    return gpu


def check(bd, b, Hq, scale=None, window=0, max_q=None, q=None, pad_rows=0):
    q = b.queries(Hq) if q is None else q
    cache, batch = b.device(bd, max_q)
    rows = b.rows + pad_rows
    qd = torch.full((rows, Hq, b.D), float("nan"), dtype=b.dtype, device="cuda")
    qd[:b.rows] = q.cuda()
    out = torch.full((rows, Hq, b.D), 7.0, dtype=b.dtype, device="cuda")
    lse = torch.full((rows, Hq), 7.0, device="cuda")
    n = bd.attention_workspace_bytes(cache, batch, rows, Hq)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    bd.base_paged_attention(cache, batch, qd, out, ws, scale, window, lse)
    torch.cuda.synchronize()
    want, bound, wl, lb = U.attend(b, q, b.D ** -0.5 if scale is None else scale, window)
    U.near(out[:b.rows], want, bound, b.dtype, "out")
    got = lse[:b.rows].double().cpu().numpy()
    assert np.array_equal(np.isinf(got), np.isinf(wl))
    fine = np.isfinite(wl)
    assert (np.abs(got - wl)[fine] <= lb[fine]).all(), np.abs(got - wl)[fine].max()
    assert (out[b.rows:] == 7).all() and (lse[b.rows:] == 7).all()
    return out, lse


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [8, 40, 64, 72, 96, 128, 136, 200, 256])
def test_head_sizes(bd, dtype, D):
    b = U.Batch([(1, 300), (3, 33), (1, 1)], 2, D, 16, dtype, seed=D)
    b.fill()
    check(bd, b, 6)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (3, 3), (8, 1), (12, 4), (32, 1), (40, 2), (66, 2)])
def test_head_layouts(bd, dtype, Hq, Hk):
    b = U.Batch([(1, 700), (2, 70), (1, 129)], Hk, 64, 32, dtype, seed=Hq)
    b.fill()
    check(bd, b, Hq)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kv", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 4097])
def test_lengths(bd, dtype, kv):
    b = U.Batch([(1, kv)], 2, 128, 16, dtype, seed=kv)
    b.fill()
    check(bd, b, 8)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("ps,heads_first", [(16, True), (16, False), (64, False), (128, True), (1024, True)])
def test_pages(bd, dtype, ps, heads_first):
    b = U.Batch([(1, 1000), (5, 517), (2, 48)], 3, 128, ps, dtype, seed=ps, heads_first=heads_first)
    b.fill()
    check(bd, b, 6)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,kv", [(2, 2), (5, 5), (17, 100), (33, 33), (64, 64), (65, 300), (130, 130), (257, 700)])
def test_chunks(bd, dtype, D, n, kv):
    b = U.Batch([(n, kv)], 2, D, 16, dtype, seed=n)
    b.fill()
    check(bd, b, 8)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("window", [1, 2, 16, 31, 64, 100, 1000])
def test_windows(bd, dtype, window):
    """The keys that a window leaves behind may hold anything, their pages may be gone."""
    lens = [(1, 900), (7, 300), (130, 401), (3, 3)]
    b = U.Batch(lens, 2, 64, 16, dtype, seed=window)
    lowest = [max(0, kv - n + 1 - window) for n, kv in lens]
    b.fill(lowest)
    for s, lo in enumerate(lowest):
        b.table[s, :lo // 16] = -1
    check(bd, b, 8, window=window)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_mixed_and_empty(bd, dtype):
    """Single tokens, chunks, places without a sequence, more new tokens than tokens, rows
    behind the last sequence."""
    lens = [(1, 77), (0, 0), (150, 150), (0, 40), (1, 1), (40, 1200), (9, 4), (2, 0), (1, 2000), (0, 0)]
    b = U.Batch(lens, 2, 128, 16, dtype, seed=5)
    b.fill()
    check(bd, b, 8, pad_rows=5)
    check(bd, b, 8, pad_rows=5, max_q=1000)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_sequences(bd, dtype):
    g = np.random.default_rng(3)
    lens = [(int(g.integers(0, 3)), int(g.integers(2, 90))) for _ in range(211)]
    b = U.Batch(lens, 1, 64, 16, dtype, seed=6)
    b.fill()
    check(bd, b, 4)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [1.0, -0.3, 0.0, 30.0])
def test_scales(bd, dtype, scale):
    b = U.Batch([(1, 600), (40, 111)], 2, 64, 16, dtype, seed=9)
    b.fill()
    check(bd, b, 4, scale=scale)


def test_every_key_counts(bd):
    """With equal products lse is the log of the number of keys, and a mean of ones and
    zeros counts them."""
    for dtype in (BF, F32):
        for n, kv, window in ((1, 5000, 0), (100, 1000, 0), (100, 1000, 37), (3, 120, 0)):
            b = U.Batch([(n, kv)], 1, 64, 16, dtype, seed=kv)
            b.fill()
            q = torch.zeros(b.rows, 4, 64, dtype=dtype)
            _, lse = check(bd, b, 4, window=window, q=q)
            seen = np.minimum(kv - n + 1 + np.arange(n), window or kv)
            assert (np.round(np.exp(lse.double().cpu().numpy())) == seen[:, None]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strides_and_in_place(bd, dtype):
    """q and out inside wider rows at odd offsets; out in q's place."""
    b = U.Batch([(1, 333), (50, 222)], 2, 64, 16, dtype, seed=11)
    b.fill()
    Hq, D = 6, 64
    q = b.queries(Hq)
    cache, batch = b.device(bd)
    want, bound, *_ = U.attend(b, q, D ** -0.5)
    ws = torch.empty(bd.attention_workspace_bytes(cache, batch, b.rows, Hq), dtype=torch.uint8, device="cuda")

    def wide(fill):
        buf = torch.full((b.rows * (Hq * (D + 3) + 5) + 1,), fill, dtype=dtype, device="cuda")
        return buf, buf[1:].view(b.rows, Hq * (D + 3) + 5)[:, 5:].unflatten(1, (Hq, D + 3))[..., 3:]
    qb, qv = wide(3.0)
    qv.copy_(q)
    ob, ov = wide(9.0)
    bd.base_paged_attention(cache, batch, qv, ov, ws)
    U.near(ov, want, bound, dtype)
    before = ob.clone()
    ov.fill_(9.0)
    assert (ob == 9).all() and (before != 9).any()
    bd.base_paged_attention(cache, batch, qv, qv, ws)
    U.near(qv, want, bound, dtype)
    qv.fill_(3.0)
    assert (qb == 3).all()


def test_long_context_far_offsets(bd):
    """Pages past 2^32 elements and bytes from the cache's start, and a long context."""
    ps, Hk, D, kv = 256, 1, 128, 70001
    b = U.Batch([(1, kv)], Hk, D, ps, BF, seed=12)
    n = 280
    stride = 1 << 24                       # elements from page to page: the last at 280 2^24 > 2^32
    base = torch.zeros(1, dtype=BF, device="cuda")
    need = (n - 1) * stride + ps * D
    buf = torch.empty(need * 2, dtype=BF, device="cuda")     # 18.8 GB
    k = buf[:need].as_strided((n, ps, Hk, D), (stride, D, D, 1))
    v = buf[need:].as_strided((n, ps, Hk, D), (stride, D, D, 1))
    order = np.random.default_rng(1).permutation(n)[:b.width]
    b.table[0, :] = -1
    b.table[0, :len(order)] = order[:b.width]
    page, slot = b.slots(0, 0, kv)
    k[page.cuda(), slot.cuda()], v[page.cuda(), slot.cuda()] = b.k[0].cuda(), b.v[0].cuda()
    q = b.queries(8)
    put = lambda t: torch.from_numpy(t).cuda()  # noqa: E731
    batch = bd.KVBatch(put(b.table), put(b.starts), put(np.array([kv], np.int32)), 1)
    out = bd.paged_attention(q.cuda(), bd.KVCache(k, v), batch)
    want, bound, *_ = U.attend(b, q, D ** -0.5)
    U.near(out, want, bound, BF)
    del base


def test_repeat_and_graph(bd):
    """The same bits every time, with any workspace, eagerly and replayed from a graph whose
    lengths and tables change between replays."""
    lens = [(1, 3000), (1, 40), (1, 700), (1, 1)]
    b = U.Batch(lens, 2, 128, 16, BF, seed=13)
    b.fill()
    q = b.queries(16).cuda()
    cache, batch = b.device(bd)
    n = bd.attention_workspace_bytes(cache, batch, b.rows, 16)
    ws = torch.full((n,), 0x7F, dtype=torch.uint8, device="cuda")
    first = torch.empty_like(q)
    bd.base_paged_attention(cache, batch, q, first, ws)
    for fill in (0, 0xFF):
        ws.fill_(fill)
        again = torch.empty_like(q)
        bd.base_paged_attention(cache, batch, q, again, ws)
        assert torch.equal(again, first)
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            bd.base_paged_attention(cache, batch, q, out, ws)
    torch.cuda.synchronize()
    full = batch.tensors[2].clone()
    for cut in (0, 17, 700, 0, 2999):
        batch.tensors[2].copy_((full - cut).clamp_min(0))
        eager = torch.empty_like(q)
        ws2 = torch.empty_like(ws)
        bd.base_paged_attention(cache, batch, q, eager, ws2)
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        if cut == 0:
            assert torch.equal(out, first)


def test_other_stream(bd):
    b = U.Batch([(1, 900), (64, 300)], 2, 64, 16, BF, seed=14)
    b.fill()
    q = b.queries(8).cuda()
    cache, batch = b.device(bd)
    want = bd.paged_attention(q, cache, batch)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got, lse = bd.paged_attention(q, cache, batch, return_lse=True, stream=s)
    s.synchronize()
    assert torch.equal(got, want) and lse.isfinite().all()


def test_bad_device_data_stays_in_bounds(bd):
    """Page numbers outside the cache, starts and lengths beyond everything: no fault (the
    kernels bound each access), and sequences with sound data keep their results."""
    lens = [(1, 500), (2, 200), (1, 300)]
    b = U.Batch(lens, 2, 64, 16, BF, seed=15, fill=0.0)
    b.fill()
    q = b.queries(4)
    want, bound, *_ = U.attend(b, q, 0.125)
    b.table[1, :] = [b.n_pages, -7, 1 << 30, -(1 << 31)] * (b.width // 4) + [5] * (b.width % 4)
    cache, batch = b.device(bd)
    out = bd.paged_attention(q.cuda(), cache, batch)
    U.near(out[:1], want[:1], bound[:1], BF)
    U.near(out[3:], want[3:], bound[3:], BF)
    batch.tensors[2].copy_(torch.tensor([500, 2 ** 31 - 1, -5], dtype=torch.int32))
    out = bd.paged_attention(q.cuda(), cache, batch)
    U.near(out[:1], want[:1], bound[:1], BF)
    assert (out[3:] == 0).all()             # a length below zero: no key
    batch.tensors[1].copy_(torch.tensor([0, 1, -3, 2 ** 31 - 1], dtype=torch.int32))
    bd.paged_attention(q.cuda(), cache, batch)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("q", [1, 6])
def test_several_units_a_workgroup(bd, dtype, D, q):
    """More work than workgroups: each goes through parts and wholes of several units."""
    g = np.random.default_rng(D + q)
    lens = [(int(g.integers(1, q + 1)), int(g.integers(q, 400))) for _ in range(90)]
    b = U.Batch(lens, 9, D, 16, dtype, seed=D)
    b.fill()
    check(bd, b, 36)


# A table wide enough that a call counts as a large one (the host knows the table's width, not
# the lengths): these go through the kernels of many rows, with short sequences.
def wide(lens, Hk, D, ps, Hq, **kw):
    rows = sum(n for n, _ in lens)
    shape = 64 if D <= 64 else 128 if D <= 128 else 256
    return U.Batch(lens, Hk, D, ps, BF, extra=int(3.2e9 / (4 * shape * Hq * rows * ps)) + 1, **kw)


@pytest.mark.parametrize("D", [8, 40, 64, 96, 128, 136, 160, 256])
@pytest.mark.parametrize("n,kv", [(17, 17), (33, 100), (64, 64), (65, 300), (130, 130), (257, 700)])
def test_wide_chunks(bd, D, n, kv):
    b = wide([(n, kv)], 2, D, 16, 6, seed=D + n)
    b.fill()
    check(bd, b, 6)


@pytest.mark.parametrize("Hq,Hk", [(1, 1), (3, 3), (12, 4), (32, 1), (66, 2)])
def test_wide_head_layouts(bd, Hq, Hk):
    b = wide([(1, 700), (40, 70), (35, 129)], Hk, 128, 32, Hq, seed=Hq, heads_first=False)
    b.fill()
    check(bd, b, Hq)


@pytest.mark.parametrize("D", [64, 80, 128, 192])
def test_wide_mixed_and_empty(bd, D):
    lens = [(1, 77), (0, 0), (150, 150), (0, 40), (1, 1), (40, 1200), (9, 4), (2, 0), (200, 130), (1, 2000), (0, 0)]
    b = wide(lens, 2, D, 64, 8, seed=D)
    b.fill()
    check(bd, b, 8, pad_rows=5)
    check(bd, b, 8, pad_rows=5, max_q=1000)


@pytest.mark.parametrize("scale", [1.0, -0.3, 0.0, 30.0])
def test_wide_scales(bd, scale):
    b = wide([(1, 600), (40, 111), (70, 333)], 2, 64, 16, 4, seed=9)
    b.fill()
    check(bd, b, 4, scale=scale)


@pytest.mark.parametrize("D,window", [(64, 1), (64, 31), (128, 64), (128, 100), (128, 1000), (96, 37), (256, 50)])
def test_large_windows(bd, D, window):
    """Calls that are large by their rows; what a window leaves behind may hold anything."""
    lens = [(1, 900), (7, 300), (730, 1401), (450, 450), (3, 3)]
    b = U.Batch(lens, 1, D, 16, BF, seed=window)
    lowest = [max(0, kv - n + 1 - window) for n, kv in lens]
    b.fill(lowest)
    for s, lo in enumerate(lowest):
        b.table[s, :lo // 16] = -1
    Hq = 16
    shape = 64 if D <= 64 else 128 if D <= 128 else 256
    assert 4 * shape * Hq * b.rows * (window + 730) > 3e9
    check(bd, b, Hq, window=window)


@pytest.mark.parametrize("lens,Hq", [([(1200, 1200), (3, 50), (700, 701)], 1), ([(2100, 2100)], 1), ([(90, 95)] * 70, 2)])
def test_many_tiles(bd, lens, Hq):
    """Sequences of more tiles than a lane counts by itself, of more than 64 tiles; more than
    64 sequences of several."""
    for dtype in (BF, F32):
        b = U.Batch(lens, 1, 8, 16, dtype, seed=len(lens))
        b.fill()
        check(bd, b, Hq)
    b = wide(lens, 1, 8, 16, Hq, seed=len(lens))
    b.fill()
    check(bd, b, Hq)


def test_wide_many_tiles(bd):
    for lens, Hq in (([(1030, 1040), (1, 9)], 16), ([(40, 60), (300, 300)] * 40, 4)):
        b = wide(lens, 1, 16, 16, Hq, seed=3)
        b.fill()
        check(bd, b, Hq)


def test_wide_every_key_counts(bd):
    for n, kv in ((100, 1000), (300, 300)):
        b = wide([(n, kv), (1, 5000)], 1, 64, 16, 4, seed=kv)
        b.fill()
        _, lse = check(bd, b, 4, q=torch.zeros(b.rows, 4, 64, dtype=BF))
        seen = np.concatenate([kv - n + 1 + np.arange(n), [5000]])
        assert (np.round(np.exp(lse.double().cpu().numpy())) == seen[:, None]).all()


def test_wide_repeat_graphs_and_streams(bd):
    """The same bits every time, with any workspace; two graphs of one workspace replayed in
    turn, two calls at once with a workspace each, lengths that change between replays."""
    lens = [(1, 3000), (90, 340), (64, 700), (1, 1), (130, 130)]
    b = wide(lens, 2, 128, 16, 8, seed=13)
    b.fill()
    q = b.queries(8).cuda()
    cache, batch = b.device(bd)
    n = bd.attention_workspace_bytes(cache, batch, b.rows, 8)
    ws = torch.full((n,), 0x7F, dtype=torch.uint8, device="cuda")

    def call(w, window=0):
        out = torch.full_like(q, 5.0)
        bd.base_paged_attention(cache, batch, q, out, w, None, window)
        return out
    first = call(ws)
    for fill in (0, 0xFF):
        ws.fill_(fill)
        assert torch.equal(call(ws), first)
    outs, graphs = [torch.empty_like(q) for _ in range(2)], [torch.cuda.CUDAGraph() for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for i, window in enumerate((0, 100)):
            with torch.cuda.graph(graphs[i], stream=side):
                bd.base_paged_attention(cache, batch, q, outs[i], ws, None, window)
    torch.cuda.synchronize()
    full = batch.tensors[2].clone()
    for cut in (0, 17, 250, 0, 2999):
        batch.tensors[2].copy_((full - cut).clamp_min(0))
        for o in outs:
            o.fill_(5.0)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        other = torch.empty_like(ws)
        assert torch.equal(outs[0], call(other)) and torch.equal(outs[1], call(other, 100))
        assert cut or torch.equal(outs[0], first)
    batch.tensors[2].copy_(full)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    works = [torch.empty_like(ws) for _ in range(2)]
    got = [[torch.empty_like(q) for _ in range(4)] for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for i in range(4):
        for s, w, o in zip(streams, works, got):
            bd.base_paged_attention(cache, batch, q, o[i], w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for os in got for o in os)


def test_wide_bad_device_data_stays_in_bounds(bd):
    lens = [(60, 500), (70, 200), (1, 300)]
    b = wide(lens, 2, 96, 16, 4, seed=15, fill=0.0)
    b.fill()
    q = b.queries(4)
    want, bound, *_ = U.attend(b, q, 96 ** -0.5)
    b.table[1, :] = np.resize(np.array([b.n_pages, -7, 1 << 30, -(1 << 31)], np.int64), b.width).astype(np.int32)
    cache, batch = b.device(bd)
    out = bd.paged_attention(q.cuda(), cache, batch)
    U.near(out[:60], want[:60], bound[:60], BF)
    U.near(out[130:], want[130:], bound[130:], BF)
    batch.tensors[2].copy_(torch.tensor([500, 2 ** 31 - 1, -5], dtype=torch.int32))
    out = bd.paged_attention(q.cuda(), cache, batch)
    U.near(out[:60], want[:60], bound[:60], BF)
    assert (out[130:] == 0).all()
    batch.tensors[1].copy_(torch.tensor([0, 60, -3, 2 ** 31 - 1], dtype=torch.int32))
    bd.paged_attention(q.cuda(), cache, batch)
    torch.cuda.synchronize()


@pytest.mark.parametrize("D,Hq", [(256, 64), (128, 128)])
def test_large_calls_of_short_contexts(bd, D, Hq):
    """Tables of two blocks of keys: a workgroup a unit in the kernel of few rows, no parts."""
    lens = [(100, 100), (2, 60), (128, 128), (1, 1), (0, 0), (110, 128), (1, 128), (100, 128)]
    b = U.Batch(lens, 32, D, 16, BF, seed=D, extra=0)
    b.fill()
    assert 4 * D * Hq * b.rows * b.width * 16 > 3e9 and b.width <= 8
    check(bd, b, Hq)


def test_starts_that_fall_and_rise(bd):
    """Starts that make more work than the rows can be: the call ends (what it writes is
    nobody's), the next one with sound starts is right."""
    lens = [(40, 60)] * 70
    for b in (U.Batch(lens, 1, 64, 16, BF, seed=8, fill=0.0), wide(lens, 1, 64, 16, 4, seed=8, fill=0.0)):
        b.fill()
        q = b.queries(4)
        cache, batch = b.device(bd, max_q=b.rows)
        sound = batch.tensors[1].clone()
        bad = torch.zeros_like(sound)
        bad[1::2] = b.rows
        batch.tensors[1].copy_(bad)
        bd.paged_attention(q.cuda(), cache, batch)
        torch.cuda.synchronize()
        batch.tensors[1].copy_(sound)
        out = bd.paged_attention(q.cuda(), cache, batch)
        want, bound, *_ = U.attend(b, q, 0.125)
        U.near(out, want, bound, BF)


def call(bd, b, q, cache, batch, window=0):
    out, lse = bd.paged_attention(q, cache, batch, window=window, return_lse=True)
    return out, lse


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 100, 2 ** 30])
def test_windows_wider_than_any_table(bd, dtype, window):
    """A window that no sequence can fill is none: the same bits, small calls and large ones,
    with more new tokens than tokens among them."""
    lens = [(9, 4), (200, 130), (1, 77), (40, 900), (2, 0)]
    for b in [U.Batch(lens, 2, 64, 16, dtype, seed=17)] + ([wide(lens, 2, 128, 16, 8, seed=17)] if dtype is BF else []):
        b.fill()
        q = b.queries(8)
        check(bd, b, 8, window=window, q=q)
        cache, batch = b.device(bd)
        for got, want in zip(call(bd, b, q.cuda(), cache, batch, window), call(bd, b, q.cuda(), cache, batch)):
            assert torch.equal(got, want)


def test_a_wide_window_takes_a_large_calls_kernel(bd):
    """The kernel of a large call does not hang on how no window is said."""
    b = U.Batch([(600, 700)], 2, 128, 16, BF, seed=18)
    b.fill()
    q = b.queries(16).cuda()
    assert 4 * 128 * 16 * 600 * 700 > 2e9
    cache, batch = b.device(bd)
    for got, want in zip(call(bd, b, q, cache, batch, 2 ** 31 - 1), call(bd, b, q, cache, batch)):
        assert torch.equal(got, want)


def paths(dtype):
    """Batches whose units are done whole, in parts, and (16 bits) in the kernel of chunks."""
    lens = [(1, 20), (3, 45), (1, 33)]
    yield U.Batch(lens, 2, 64, 16, dtype, seed=21)
    yield U.Batch([(1, 3000), (4, 1500), (1, 1)], 2, 64, 16, dtype, seed=22)
    if dtype is BF:
        yield wide([(70, 300), (64, 64), (1, 700)], 2, 64, 16, 8, seed=23)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("what", ["q", "k", "v", "q inf", "k inf"])
def test_nan_and_infinity_where_tokens_see_them(bd, dtype, what):
    """A row whose softmax is NaN says so in out and lse (-infinity is a row without keys); the
    other rows keep their results (to the bit where no score changes: when a tile's maxima
    are raised hangs on all its rows)."""
    bad = float("inf") if "inf" in what else float("nan")
    for b in paths(dtype):
        b.fill()
        q = b.queries(8)
        cache, batch = b.device(bd)
        clean, clean_lse = call(bd, b, q.cuda(), cache, batch)
        want, bound, wl, lb = U.attend(b, q, 0.125)
        n = b.lens[1][0]
        hit = torch.zeros(b.rows, 8, dtype=torch.bool)        # rows and heads that see it
        if what[0] == "q":
            q[2, 5, 7] = bad
            hit[2, 5] = True
        else:
            # the second sequence's first token, of the second key head
            page, slot = b.slots(1, 0, 1)
            t = cache.tensors["kv".index(what[0])]
            t[page.cuda(), slot.cuda(), 1, 7] = bad
            hit[b.starts[1]:b.starts[1] + n, 4:] = True
        out, lse = call(bd, b, q.cuda(), cache, batch)
        hit = hit.cuda()
        keep = (~hit).cpu().numpy()
        U.near(out[~hit], want[keep], bound[keep], dtype)
        assert (np.abs(lse[~hit].double().cpu().numpy() - wl[keep]) <= lb[keep]).all()
        if what == "v":
            assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit])
            assert out[hit][:, 7].isnan().all() and torch.equal(lse[hit], clean_lse[hit])
            assert torch.equal(out[hit][:, :7], clean[hit][:, :7]) and torch.equal(out[hit][:, 8:], clean[hit][:, 8:])
        elif what == "q" or what == "k":
            assert out[hit].isnan().all() and lse[hit].isnan().all()
        else:
            # an infinity's products are +inf (NaN) or -inf (no weight, or where all are, no keys)
            assert torch.equal(out[hit].isnan().any(1), lse[hit].isnan())
            assert lse[hit].isnan().any() and not (lse[hit] == float("inf")).any()


@pytest.mark.parametrize("lens,D,window", [([(1, 300), (3, 500), (1, 17)], 64, 0), ([(1, 2000), (4, 1000)], 128, 100),
                                           ([(2, 40), (1, 25)], 256, 0)])
def test_few_rows_keep_their_exponentials_in_two_parts(bd, lens, D, window):
    """bf16 calls of few rows hold an exponential as a bf16 and the bf16 of what that leaves:
    off by 2^-16 of itself, so out by 2^-16 of the largest |v| in place of 2^-8 of their mean.
    (With one part, worked out on the CPU, 221, 606 and 831 values here are beyond the bound.)"""
    b = U.Batch(lens, 2, D, 16, BF, seed=D)
    b.fill()
    q = b.queries(8, 0.5)
    cache, batch = b.device(bd)
    out = bd.paged_attention(q.cuda(), cache, batch, window=window)
    b.dtype = F32                       # the bound without the rounding to one bf16
    want, bound, *_ = U.attend(b, q, D ** -0.5, window)
    b.dtype = BF
    U.near(out, want, bound + 2.0 ** -16 * max(float(v.abs().max()) for v in b.v), BF)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_largest_table(bd, dtype):
    """A table of 2^30 tokens a sequence: the units' costs are counted in several blocks."""
    ps, width = 65536, 1 << 14
    g = np.random.default_rng(31)
    lens = [(int(g.integers(0, 4)), int(g.integers(4, 700))) for _ in range(30)] + [(60, 5000), (1, 3333), (300, 300)]
    b = U.Batch(lens, 4, 8, ps, dtype, seed=31, extra=width - 1)
    assert b.width == width and len(lens) * 4 * (1 << 30) // 64 > 10 ** 9
    b.fill()
    check(bd, b, 8)


@pytest.mark.parametrize("width", [2, 40])
def test_the_most_sequences(bd, width):
    """65536 sequences, of one or no new token."""
    n = 65536
    lens = [(int(i % 3 != 1), 1 + i % 17) for i in range(n)]
    b = U.Batch(lens, 1, 8, 16, BF, seed=32, extra=width - 2)
    b.fill()
    check(bd, b, 1)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout", ["pages", "tokens", "heads"])
def test_views_of_one_cache_and_of_a_wider_table(bd, dtype, layout):
    """Keys and values side by side in one tensor (page by page, token by token, head by head),
    the table a view of a wider one's first entries."""
    b = U.Batch([(1, 700), (40, 130), (3, 33)], 2, 72, 32, dtype, seed=33)
    b.fill()
    q = b.queries(6)
    at = {"pages": 1, "tokens": 2, "heads": 3}[layout]
    both = torch.stack([b.kc, b.vc], at).contiguous().cuda()
    k, v = both.unbind(at)
    put = lambda t: torch.from_numpy(t).cuda()  # noqa: E731
    table = np.full((3, 500), -1, np.int32)
    table[:, :b.width] = b.table
    batch = bd.KVBatch(put(table)[:, :b.width], put(b.starts), put(np.array([kv for _, kv in b.lens], np.int32)), 40)
    out = bd.paged_attention(q.cuda(), bd.KVCache(k, v), batch)
    want, bound, *_ = U.attend(b, q, 72 ** -0.5)
    U.near(out, want, bound, dtype)

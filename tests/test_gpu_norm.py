"""The norms around a block on the GPU against 64-bit arithmetic, in place, with
strides, for rows of every kernel's range; the block call against its parts bit
for bit.

Tolerance, from the arithmetic: a sum of d squares over threads of at most 16
elements, 6 tree levels and 16 partial sums is off by less than 40 2^-24 of itself,
so r = 1 / sqrt(.) by 20 2^-24 and two roundings; the products and the fused
multiply-add add at most 5 2^-24: 64 2^-24 =: u covers each term.  With t the
block's term, dh = u (|a h| + |t|) is the error of h' before its rounding, and
x' = w h' r moves by |w| r dh, by u |x'| and, through r, by |x'| |dh| / |h'| (2-norms
of the row).  Then each output's rounding: finfo.eps / 2 of it."""
import numpy as np
import pytest

import workloads as W

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def gu(gpu):
    import gpu_util
    return gpu_util


@pytest.fixture(scope="module")
def bd(gpu):
    return gpu


def reference(h, y, post, gate, pre, scale, eps):
    """(h', bound, x', bound) in float64, before the outputs' rounding."""
    u = 64 * 2.0 ** -24
    def rstd(v):
        m = np.mean(v * v, 1, keepdims=True) + eps
        with np.errstate(divide="ignore"):
            return np.where(m > 0, 1 / np.sqrt(m), np.where(m == 0, 0.0, m))
    dh = np.zeros_like(h)
    if y is not None:
        t = y if post is None else y * rstd(y) * post
        t = t if gate is None else t * gate
        dh = u * (np.abs(scale * h) + np.abs(t))
        h = scale * h + t
    if pre is None:
        return h, dh, None, None
    r = rstd(h)
    x = h * r * pre
    n = np.linalg.norm(h, axis=1, keepdims=True)
    rel = np.linalg.norm(dh, axis=1, keepdims=True) / np.where(n > 0, n, 1)
    return h, dh, x, np.abs(pre) * r * dh + (u + rel) * np.abs(x)


def place(a, dtype, pad, off, fill=7.0):
    """a's rows inside rows `pad` longer, the first element `off` past an aligned one."""
    rows, d = a.shape
    buf = torch.full((rows * (d + pad) + off,), fill, dtype=dtype, device="cuda")
    v = buf[off:].view(rows, d + pad)[:, :d]
    v.copy_(torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(dtype))
    return buf, v


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def run(bd, rows, d, dtype, post=True, gate="channel", pre=True, block=True, pad=0, off=0, scale=0.75, eps=1e-6,
        inplace="", edit=None, seed=0):
    g = np.random.default_rng(seed + d + rows)
    vals = [3 * g.standard_normal((rows, d)), 0.4 * g.standard_normal((rows, d))]
    if edit:
        edit(*vals)
    hb, h = place(vals[0], dtype, pad, off)
    yb, y = place(vals[1], dtype, pad, off) if block else (None, None)
    f32 = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
    wpost, wpre = (1 + 0.1 * f32(d)) if post else None, (1 + 0.1 * f32(d)) if pre else None
    gt = {"none": None, "channel": f32(d), "token": f32(rows, d + 3)[:, :d]}[gate] if block else None
    h64, y64 = f64(h), f64(y) if block else None
    n64 = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    want_h, bh, want_x, bx = reference(h64, y64, n64(wpost), n64(gt), n64(wpre), scale, eps)
    ho = xo = hob = xob = None
    if block:
        hob, ho = (hb, h) if "h" in inplace else place(np.zeros((rows, d)), dtype, pad, off)
    if pre:
        xob, xo = (yb, y) if "y" in inplace else place(np.zeros((rows, d)), dtype, pad, off)
    bd.norm_residual(h, y, wpost, gt, wpre, scale, eps, ho, xo)
    half = torch.finfo(dtype).eps / 2
    for got, want, b in ((ho, want_h, bh), (xo, want_x, bx)):
        if got is None:
            continue
        v = f64(got)
        fine = np.isfinite(want)
        assert np.array_equal(np.isnan(v), np.isnan(want))
        err = np.abs(v - want)[fine]
        lim = (b + half * (np.abs(want) + b) + 1e-37)[fine]
        assert (err <= lim).all(), float((err / lim).max())
    for buf, view in ((hob, ho), (xob, xo)):
        if buf is not None and pad:
            rest = torch.ones_like(buf, dtype=torch.bool)
            rest[off:].view(rows, d + pad)[:, :d] = False
            assert bool((buf[rest] == 7.0).all())
    return ho, xo


DTYPES = [torch.bfloat16, torch.float32]
LENGTHS = [1, 2, 7, 8, 63, 64, 65, 500, 512, 513, 1000, 1024, 1025, 2047, 2048, 2056, 4096, 4100, 5001, 8192, 8200,
           16383, 16384]


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("d", LENGTHS)
def test_lengths(bd, dtype, d):
    run(bd, 3, d, dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 2, 4, 5, 255, 1023, 5000])
@pytest.mark.parametrize("d", [96, 2048])
def test_row_counts(bd, dtype, rows, d):
    run(bd, rows, d, dtype, gate="token")


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("pre", [True, False])
def test_forms(bd, dtype, post, gate, pre):
    for d in (768, 1536):
        run(bd, 6, d, dtype, post=post, gate=gate, pre=pre)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [40, 640, 3000])
def test_norm_before_the_first_block(bd, dtype, d):
    run(bd, 5, d, dtype, block=False, post=False)


def test_without_a_block_its_parameters_are_not_read(bd):
    """One Norms for a step: its norm before the first block, where the residual scale,
    the gate and the post gain have no part, whatever they hold."""
    import ctypes
    h, pre = torch.randn(5, 96, device="cuda").bfloat16(), torch.randn(96, device="cuda")
    want, x = torch.empty_like(h), torch.empty_like(h)
    bd.base_norm_residual(bd.Norms(96, h.dtype, pre_gain=pre), None, h, None, want)
    n = bd.Norms(96, h.dtype, torch.ones(96, device="cuda"), torch.ones(7, 96, device="cuda"), pre)
    bd.base_norm_residual(n, None, h, None, x)               # a gate for another batch
    assert torch.equal(x, want)
    for kw in (dict(res_scale=float("nan")), dict(res_scale=float("inf")), dict(gate_ld=-1), dict(gate_ld=1 << 50),
               dict(post_gain=2), dict(gate=1)):
        v = dict(d=96, dtype=1, eps=1e-6, res_scale=1.0, post_gain=0, gate=pre.data_ptr(), gate_ld=0,
                 pre_gain=pre.data_ptr())
        v.update(kw)
        x.fill_(3.0)
        N = bd.base_norms(*(v[f] for f, _ in bd.base_norms._fields_))
        assert bd.load().base_norm_residual(ctypes.byref(N), 5, None, 0, h.data_ptr(), 96, None, 0, x.data_ptr(), 96,
                                            bd._stream(None)) == 0, kw
        assert torch.equal(x, want), kw


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("d,pad,off", [(512, 8, 0), (512, 4, 0), (512, 3, 0), (512, 0, 1), (2048, 64, 0),
                                       (2048, 1, 3), (5001, 7, 1)])
def test_strides_and_alignment(bd, dtype, d, pad, off):
    run(bd, 7, d, dtype, pad=pad, off=off)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("d,rows", [(3, 40), (5, 7), (9, 33), (87, 515), (126, 3), (128, 21), (129, 301), (200, 3), (255, 1001),
                                    (256, 9), (257, 65), (511, 6), (1023, 700), (1029, 801), (1501, 600), (5003, 300),
                                    (8191, 5), (8193, 5)])
@pytest.mark.parametrize("post", [True, False])
def test_rows_that_share_wavefronts_or_overlap_their_pieces(bd, dtype, d, rows, post):
    """Lengths on both sides of each line and off the pieces' size, apart and in place,
    with row counts that leave a wavefront's last rows empty."""
    for inplace in ("", "h", "y", "hy"):
        run(bd, rows, d, dtype, post=post, gate="token", inplace=inplace)


@pytest.mark.parametrize("inplace", ["h", "y", "hy"])
@pytest.mark.parametrize("d,pad", [(512, 0), (2048, 16), (4099, 0)])
def test_in_place(bd, inplace, d, pad):
    run(bd, 9, d, torch.bfloat16, pad=pad, inplace=inplace)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 2048])
def test_rows_of_zeros_without_eps(bd, dtype, d):
    """n(0) is 0 where eps is 0 too; the other rows are as ever."""
    def edit(h, y):
        h[1], y[1] = 0.0, 0.0
        y[3] = 0.0
    ho, xo = run(bd, 5, d, dtype, eps=0.0, edit=edit)
    assert not xo[1].any() and not ho[1].any()


@pytest.mark.parametrize("d", [128, 2048])
def test_nan_and_infinity_stay_in_their_rows(bd, d):
    def edit(h, y):
        h[1, 5] = np.nan
        y[2, 0] = np.nan
    ho, xo = run(bd, 6, d, torch.bfloat16, edit=edit)
    assert torch.isnan(xo[1]).all() and torch.isnan(ho[2]).all() and torch.isfinite(xo[[0, 3, 4, 5]]).all()


@pytest.mark.parametrize("bits", [0xFFFFFFFF, 0x7FFFFFFF, 0x7F800001], ids=hex)
@pytest.mark.parametrize("d", [87, 128, 513, 2048, 5001])
def test_every_nan_of_a_gate_or_gain_reaches_bf16_rows(bd, d, bits):
    """NaNs whose bits are all ones (memory filled with 0xFF), where an integer
    rounding carries into a zero: h' and x' are NaN where the formula is."""
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    h, y = r(5, d).bfloat16(), r(5, d).bfloat16()
    bad = torch.tensor([bits], dtype=torch.int64).to(torch.int32).view(torch.float32).cuda()
    def call(which, at):
        w = dict(post_gain=1 + 0.1 * r(d), gate=r(5, d), pre_gain=1 + 0.1 * r(d))
        w[which].view(-1, d)[-1, at] = bad[0]
        assert torch.isnan(w[which]).any()
        return bd.norm_residual(h, y, **w)
    for at in (0, d - 1):
        ho, xo = call("gate", at)            # the last row's gate
        assert torch.isnan(ho[4, at]) and int(torch.isnan(ho).sum()) == 1
        assert torch.isnan(xo[4]).all() and int(torch.isnan(xo).sum()) == d
        ho, xo = call("post_gain", at)
        assert torch.isnan(ho[:, at]).all() and int(torch.isnan(ho).sum()) == 5 and torch.isnan(xo).all()
        ho, xo = call("pre_gain", at)
        assert torch.isfinite(ho).all() and torch.isnan(xo[:, at]).all() and int(torch.isnan(xo).sum()) == 5


def test_small_and_large_values(bd):
    """Squares near both ends of fp32."""
    for f in (1e-15, 1e15):
        def edit(h, y, f=f):
            h *= f
            y *= f
        run(bd, 4, 1024, torch.float32, eps=0.0, edit=edit)


def test_another_stream_and_a_graph(bd):
    d, rows = 2048, 33
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    hs, ys = [r(rows, d).bfloat16() for _ in range(3)], [r(rows, d).bfloat16() for _ in range(3)]
    post, pre, gate = r(d), r(d), r(rows, d)
    n = bd.Norms(d, torch.bfloat16, post, gate, pre, 0.5)
    want = []
    for h, y in zip(hs, ys):
        ho, xo = torch.empty_like(h), torch.empty_like(h)
        bd.base_norm_residual(n, y, h, ho, xo)
        want.append((ho, xo))
    torch.cuda.synchronize()
    h, y, ho, xo = hs[0].clone(), ys[0].clone(), torch.empty_like(hs[0]), torch.empty_like(hs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        bd.base_norm_residual(n, y, h, ho, xo)
    for i in (1, 0, 2, 2, 1):
        h.copy_(hs[i])
        y.copy_(ys[i])
        ho.zero_()
        xo.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ho, want[i][0]) and torch.equal(xo, want[i][1])


# ------------------------------------------------------------------- block --
def block_norms(bd, d, dtype, B, per_token, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    gate = torch.sigmoid(r(B, d) if per_token else r(d))
    return bd.Norms(d, dtype, 1 + 0.1 * r(d), gate, 1 + 0.1 * r(d), 0.9)


@pytest.mark.parametrize("bf16,kind,d,B", [(True, "mx", 256, 1), (True, "mx", 512, 7), (True, "packed", 256, 40),
                                           (True, "mx", 256, 100), (False, "rowmajor", 256, 9),
                                           (True, "packed", 4096, 3), (True, "mx", 8192, 5),
                                           (True, "packed", 16384, 2), (False, "rowmajor", 16384, 2),
                                           (False, "rowmajor", 512, 64), (False, "rowmajor", 1024, 64),
                                           (False, "rowmajor", 2048, 64), (False, "rowmajor", 4096, 64),
                                           (False, "rowmajor", 8192, 64)])
def test_block_is_its_parts(gu, bd, bf16, kind, d, B):
    """base_decode_block against base_decode_layer and base_norm_residual, bit for
    bit, with shared experts, dropped routes (rows of nothing) and in place."""
    ns = 1 if bf16 else 0
    inp = W.custom_layer(d, 8, 3, 64, B, bf16=bf16, seed=d + B, n_shared=ns, shared_gate=bool(ns))
    gl = gu.GpuLayer(inp, packed=kind == "packed")
    if kind == "mx":
        gl.layer = bd.mx_layer(gl.layer)
        gl.desc = gl.layer.desc(gl.K)
    x = gl.x(inp["x"])
    n = block_norms(bd, d, x.dtype, B, B % 2 == 1)
    h = torch.randn(B, d, device="cuda").to(x.dtype)
    for flags in (0, 2):
        ws, y = gl.workspace(B, 4), gl.y_like(B)
        bd.base_decode_layer(gl.desc, x, B, 4, flags, None, y, ws)
        want = torch.empty_like(h), torch.empty_like(h)
        bd.base_norm_residual(n, y, h, *want)
        got = torch.empty_like(h), torch.empty_like(h)
        bd.base_decode_block(gl.desc, n, x, B, 4, flags, h, ws, *got)
        h2, x2 = h.clone(), x.clone()
        bd.base_decode_block(gl.desc, n, x2, B, 4, flags, h2, ws, h2, x2)
        for a, b, c in zip(want, got, (h2, x2)):
            assert torch.equal(a, b) and torch.equal(a, c)
        only = torch.empty_like(h)
        bd.base_decode_block(gl.desc, n, x, B, 4, flags, h, ws, None, only)
        assert torch.equal(only, want[1])


@pytest.mark.parametrize("B", [1, 12, 90])
def test_a_step_through_4bit_layers(gu, bd, B):
    """A decode step as a program runs it: the first norm, then a block per layer, on
    one workspace, captured once and replayed, against the separate calls; and
    against 64 bits layer by layer."""
    from test_gpu_mx import MxCase
    d, L = 512, 4
    cases = [MxCase(gu, bd, d, 16, 4, 192, B, 1, True, seed=20 + i) for i in range(L)]
    norms = [block_norms(bd, d, torch.bfloat16, B, False, 50 + i) for i in range(L)]
    first = bd.Norms(d, torch.bfloat16, pre_gain=torch.ones(d, device="cuda"))
    need = max(bd.base_workspace_bytes(c.gl.desc, B, 9) for c in cases)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    h0 = torch.randn(B, d, device="cuda").bfloat16()

    def parts(h):
        seen = []
        x = torch.empty_like(h)
        bd.base_norm_residual(first, None, h, None, x)
        for c, n in zip(cases, norms):
            y, ho, xo = torch.empty_like(h), torch.empty_like(h), torch.empty_like(h)
            w = c.gl.workspace(B, 9)
            plan = bd.base_decode_layer(c.gl.desc, x, B, 9, 0, None, y, w)
            bd.base_norm_residual(n, y, h, ho, xo)
            seen.append((c, x, gu.plan_arrays(plan, w, B, 4, 16, 9, True, 1), y))
            h, x = ho, xo
        return h, x, seen

    h, x = h0.clone(), torch.empty_like(h0)

    def step():
        bd.base_norm_residual(first, None, h, None, x)
        for c, n in zip(cases, norms):
            bd.base_decode_block(c.gl.desc, n, x, B, 9, 0, h, ws, h, x)

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        step()
    for f in (1.0, -2.0, 0.25):
        start = (h0 * f).contiguous()
        want_h, want_x, seen = parts(start)
        h.copy_(start)
        ws.fill_(0x5A)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, want_h) and torch.equal(x, want_x)
    for c, xin, plan, y in seen:
        c.inp["x"] = f64(xin).astype(np.float32)
        want, bound = c.outputs64(plan, None)
        assert (np.abs(f64(y) - want) <= bound).all()

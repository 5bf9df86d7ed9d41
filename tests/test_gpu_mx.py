"""4-bit experts on the GPU: codes and scales bit for bit against the oracle, the
packed layout byte for byte, and the layer against 64-bit products of the
weights' values (the plan bit for bit, as for every layer).

Tolerance of the layer's output, from the arithmetic: the activation and the
output are each rounded to bf16 (at most 2^-8 of the value), the fp32 sums of n
products are off by at most n 2^-24 of the sum of magnitudes; so with A = sum over
the executed pairs of |gate| |W_d| |h| and P the same with |W_g| |x|, |W_u| |x| for
h's own sums, |y - y64| <= 2^-8 |y| + 2^-8 A + (d + I + 64) 2^-23 (A + A').  A' bounds
what the sums' error in g and u does to the output through |silu'| <= 1.1.  Up to 32
tokens the activation has a second part of E5M2, whose rounding is off by at most
2^-3 of it, so 2^-3 2^-8 of h where it is in range and nothing more below (2^-16 / 2 /
2^9 = 2^-26): there 2^-11 A + 2^-26 A0 in the place of 2^-8 A, A0 = sum |gate| |W_d|."""
import numpy as np
import pytest

import workloads as W
from oracle import method, mx

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def gu(gpu):
    import gpu_util
    return gpu_util


@pytest.fixture(scope="module")
def bd(gpu):
    return gpu


def rounded(a, dtype):
    return a.astype(np.float32) if dtype == "f32" else W.bf16_bits_to_f32(W.f32_to_bf16_bits(a))


def to_dev(a, dtype):
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()
    return t if dtype == "f32" else t.bfloat16()


def special_rows(cols, dtype, seed):
    g = np.random.default_rng(seed)
    v = g.standard_normal((12, cols))
    v[1] *= 1e-30
    v[2] *= 2.0 ** -130          # below the smallest normal
    v[3] *= 1e37
    v[4] = 0.0
    v[5] = -0.0
    v[6] = g.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.9375], cols) * g.choice([-1, 1], cols)
    v[7] = rounded(v[7], dtype)
    v[8, ::32] = 3.3e38          # an outlier in every block
    v[9] = 2.0 ** g.integers(-126, 127, cols)
    v = rounded(v, dtype)
    v[10, 7] = np.nan
    v[11, cols - 1] = -np.inf
    return v


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad,off", [(12, 32, 0, 0), (12, 2048, 0, 0), (12, 4128, 0, 0),
                                               (12, 96, 3, 1), (12, 2080, 8, 0), (12, 64, 1, 0)])
def test_quantize(bd, dtype, rows, cols, pad, off):
    """off: the first element lies that many elements past an aligned address."""
    v = special_rows(cols, dtype, cols + pad)
    ld = cols + pad
    buf = torch.zeros(rows * ld + off, dtype=torch.float32 if dtype == "f32" else torch.bfloat16,
                      device="cuda")
    src = buf[off:].view(rows, ld)[:, :cols]
    src.copy_(to_dev(v, dtype))
    codes, scales = bd.mx_quantize(src)
    want_c, want_s = mx.quantize(v.astype(np.float64))
    assert np.array_equal(scales.cpu().numpy(), want_s)
    assert np.array_equal(codes.cpu().numpy(), want_c)
    out = torch.full((rows * ld + off,), 9.0, dtype=buf.dtype, device="cuda")
    dst = out[off:].view(rows, ld)[:, :cols]
    bd.mx_dequantize(codes, scales, out=dst)
    got = dst.float().cpu().numpy().astype(np.float64)
    want = mx.dequantize(want_c, want_s)
    assert np.array_equal(got, want, equal_nan=True)
    rest = torch.ones_like(out, dtype=torch.bool)
    rest[off:].view(rows, ld)[:, :cols] = False
    assert bool((out[rest] == 9.0).all())      # between the rows: untouched


@pytest.mark.parametrize("rows", [1, 3, 5, 1023, 4097])
def test_quantize_row_counts(bd, rows):
    g = np.random.default_rng(rows)
    v = rounded(g.standard_normal((rows, 160)), "bf16")
    codes, scales = bd.mx_quantize(to_dev(v, "bf16"))
    want_c, want_s = mx.quantize(v.astype(np.float64))
    assert np.array_equal(scales.cpu().numpy(), want_s) and np.array_equal(codes.cpu().numpy(), want_c)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_code_with_every_scale(bd, dtype):
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 16, 1)
    v = bd.mx_dequantize(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), dtype)
    with np.errstate(over="ignore"):
        want = mx.dequantize(codes, scales).astype(np.float32)
    assert np.array_equal(v.float().cpu().numpy(), want, equal_nan=True)


def quantised_experts(n, d, I, seed, spread=True):
    """(w13, w2) as row-major bf16 bits, and their (codes, scales) pairs."""
    g = np.random.default_rng(seed)
    w13 = g.standard_normal((n * 2 * I, d)) / np.sqrt(d)
    w2 = g.standard_normal((n * d, I)) / np.sqrt(I)
    if spread:
        w13 *= np.exp(0.5 * g.standard_normal((n * 2 * I, 1)))
    w13, w2 = rounded(w13, "bf16"), rounded(w2, "bf16")
    return w13, w2, mx.quantize(w13), mx.quantize(w2)


@pytest.mark.parametrize("E,d,I", [(1, 256, 64), (2, 512, 192), (1, 768, 704), (3, 256, 576)])
def test_packed_layout(bd, E, d, I):
    w13, w2, q13, q2 = quantised_experts(E, d, I, 5)
    def cut(q, rows, u):
        return q[0].reshape(E, rows, -1)[u], q[1].reshape(E, rows, -1)[u]
    want13 = np.concatenate([mx.pack(*cut(q13, 2 * I, u), mx.w13_tiles(I)) for u in range(E)])
    want2 = np.concatenate([mx.pack(*cut(q2, d, u), mx.w2_tiles(d)) for u in range(E)])
    dev = lambda q, *s: (torch.from_numpy(q[0]).cuda().view(*s, -1), torch.from_numpy(q[1]).cuda().view(*s, -1))  # noqa: E731
    p13, p2 = bd.mx_pack_experts(dev(q13, E, 2 * I), dev(q2, E, d))
    assert np.array_equal(p13.cpu().numpy(), want13) and np.array_equal(p2.cpu().numpy(), want2)
    for dt in ("bf16", "f32"):
        r13, r2 = bd.mx_quantize_experts(to_dev(w13, dt).view(E, 2 * I, d), to_dev(w2, dt).view(E, d, I))
        assert torch.equal(r13, p13) and torch.equal(r2, p2)


class MxCase:
    """A layer whose experts are 4-bit, its oracle inputs the weights' values."""

    def __init__(self, gu, bd, d, E, K, I, B, ns=0, gate=False, norm_topk=1, rule=0, seed=0):
        inp = W.custom_layer(d, E, K, I, B, seed=seed, n_shared=ns, shared_gate=gate)
        self.sh, self.ns, self.norm_topk, self.rule = inp["shape"], ns, norm_topk, rule
        if ns:
            gu_in = dict(inp)
        src = gu.GpuLayer(inp if not ns else gu_in, norm_topk=norm_topk, score_rule=rule)
        self.gl = src
        src.layer = bd.mx_layer(src.layer)
        src.desc = src.layer.desc(K)
        def values(bits, rows, cols):
            q = mx.quantize(W.bf16_bits_to_f32(bits).reshape(rows, cols).astype(np.float64))
            return W.f32_to_bf16_bits(mx.dequantize(*q).astype(np.float32)).reshape(bits.shape)
        inp["w13"] = values(inp["w13"], E * 2 * I, d)
        inp["w2"] = values(inp["w2"], E * d, I)
        if ns:
            inp["w13_shared"] = values(inp["w13_shared"], ns * 2 * I, d)
            inp["w2_shared"] = values(inp["w2_shared"], ns * d, I)
        self.inp = inp

    def oracle(self, budget, flags, residual):
        inp = self.inp
        shared = None
        if self.ns:
            shared = dict(experts=method.Experts(inp["w13_shared"], inp["w2_shared"], True),
                          gate=inp["shared_gate"])
        return method.decode_layer_c(inp["x"], inp["w_router"], inp["b_router"], inp["pred_a"],
                                     inp["pred_b"], self.sh.K, budget, None, self.norm_topk, flags,
                                     residual, self.rule, shared)

    def outputs64(self, ref, residual):
        """(y, bound) in 64 bits from the plan's own gates."""
        inp, sh = self.inp, self.sh
        x = inp["x"].astype(np.float64)
        B, d, I = x.shape[0], sh.d, sh.I
        y = np.zeros_like(x) if residual is None else residual.astype(np.float64).copy()
        A, A2, A0 = np.zeros_like(x), np.zeros_like(x), np.zeros_like(x)

        def add(t, g, b13, b2):
            w13 = W.bf16_bits_to_f32(b13).astype(np.float64)
            w2 = W.bf16_bits_to_f32(b2).astype(np.float64)
            gg, uu = x[t] @ w13[:I].T, x[t] @ w13[I:].T
            s = gg / (1 + np.exp(-gg))
            h = s * uu
            ag, au = np.abs(x[t]) @ np.abs(w13[:I]).T, np.abs(x[t]) @ np.abs(w13[I:]).T
            y[t] += g[:, None] * (h @ w2.T)
            A[t] += np.abs(g)[:, None] * (np.abs(h) @ np.abs(w2).T)
            A0[t] += np.abs(g)[:, None] * np.abs(w2).sum(1)[None]
            A2[t] += np.abs(g)[:, None] * ((1.1 * ag * np.abs(uu) + np.abs(s) * au) @ np.abs(w2).T)

        for u in range(sh.E):
            t, j = np.nonzero(ref["exec_ids"] == u)
            for rank in np.unique(j):
                m = j == rank
                add(t[m], ref["exec_gates"][t[m], j[m]].astype(np.float64), inp["w13"][u], inp["w2"][u])
        if self.ns:
            g = np.ones(B)
            if inp["shared_gate"] is not None:
                g = method.shared_gate64(inp["x"], inp["shared_gate"])
            for i in range(self.ns):
                add(np.arange(B), np.asarray(g, np.float64).reshape(B), inp["w13_shared"][i], inp["w2_shared"][i])
        h_err = 2.0 ** -11 * A + 2.0 ** -26 * A0 if B <= 32 else 2.0 ** -8 * A
        bound = 2.0 ** -8 * np.abs(y) + h_err + (d + I + 64) * 2.0 ** -23 * (A + A2) + 1e-30
        return y, bound

    def check(self, gu, bd, budget, flags=0, with_residual=False, seed=1):
        sh, gl = self.sh, self.gl
        B, K, E = self.inp["x"].shape[0], sh.K, sh.E
        print(f"4-bit layer d={sh.d} E={E} K={K} I={sh.I} B={B} budget={budget} flags={flags} ns={self.ns}",
              flush=True)
        residual = None
        if with_residual:
            residual = rounded(np.random.default_rng(seed).standard_normal((B, sh.d)), "bf16")
        ref = self.oracle(budget, flags, residual)
        x, res = gl.x(self.inp["x"]), None if residual is None else gl.x(residual)
        ws = gl.workspace(B, budget)
        ws.fill_(0xAB)
        y = torch.full((B + 3, sh.d), 5.0, dtype=torch.bfloat16, device="cuda")
        plan = bd.base_decode_layer(gl.desc, x, B, budget, flags, res, y, ws)
        torch.cuda.synchronize()
        assert bool((y[B:] == 5.0).all())      # rows behind the batch
        got = gu.plan_arrays(plan, ws, B, K, E, budget, True, self.ns)
        for f in ("topk_ids", "sel_ids", "slot_of_expert", "exec_ids", "exec_gates", "offsets", "pair_tok",
                  "pair_gate", "pair_of"):
            assert np.array_equal(got[f], ref[f]), f
        want, bound = self.outputs64(ref, residual)
        yv = gu.to_np_f32(y[:B]).astype(np.float64)
        over = np.abs(yv - want) - bound
        assert (over <= 0).all(), (float(over.max()), int((over > 0).sum()))
        # far below the worst case: independent roundings of h (past 32 tokens) and y, each
        # 2^-8 / sqrt 3 of the value at most in the mean
        most = 2.0 ** -8 * np.sqrt((1 if B <= 32 else 2) / 3) * 1.1
        assert np.linalg.norm(yv - want) <= most * np.linalg.norm(want) + 1e-20
        # staged calls: the same bits
        logits, ids, w = gl.route(x, B)
        cost = gl.predict(x, B, ids, w)
        _, _, sel, nsel, slot = gl.select(B, ids, cost, budget)
        ws2, y2 = gl.workspace(B, budget), gl.y_like(B)
        bd.base_moe_forward(gl.desc, x, B, logits, ids, sel, nsel, slot, budget, flags, res, y2, ws2)
        assert torch.equal(y2.view(torch.int16), y[:B].view(torch.int16))
        return yv


SHAPES = [
    # d, E, K, I, B, budget, flags, ns, gate, norm_topk, residual
    (256, 4, 2, 64, 1, 3, 0, 0, False, 1, False),       # half a step of down, one token
    (256, 1, 1, 64, 2, 1, 0, 0, False, 1, True),        # one expert
    (512, 8, 3, 192, 3, 5, 0, 0, False, 0, True),       # a step and a half
    (768, 16, 4, 320, 16, 6, 1, 0, False, 1, False),
    (256, 16, 4, 128, 17, 4, 2, 0, False, 1, True),     # dropped routes: rows of nothing
    (512, 16, 4, 576, 33, 9, 0, 2, True, 0, True),      # shared experts, gated
    (256, 8, 2, 704, 48, 8, 3, 1, False, 0, False),
    (1024, 8, 8, 256, 64, 8, 0, 0, False, 1, False),    # every slot full
    (256, 8, 2, 128, 65, 3, 0, 0, False, 1, True),      # parts from here on
    (512, 8, 4, 192, 200, 8, 1, 3, True, 0, True),
    (256, 32, 8, 64, 257, 20, 2, 0, False, 1, False),
    (256, 4, 1, 64, 1024, 2, 2, 0, False, 1, True),     # slots of many parts, most rows empty
    (256, 16, 16, 64, 500, 16, 0, 8, False, 1, False),  # every expert by every token
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(int(v)) for v in s))
def test_layer(gu, bd, shape):
    d, E, K, I, B, budget, flags, ns, gate, norm_topk, res = shape
    MxCase(gu, bd, d, E, K, I, B, ns, gate, norm_topk, seed=B).check(gu, bd, budget, flags, res)


# with SHAPES, every kernel instance of a 4-bit layer (test_mx_instances.py asks the
# library's own rules which ones these are)
INSTANCES = [
    # the plans, by experts (64, 128, more), tokens a wavefront and the way they rank the
    # kept experts
    (256, 128, 4, 64, 1, 3, 0, 0, False, 1, False),
    (256, 128, 8, 64, 16, 60, 0, 0, False, 0, True),
    (256, 128, 8, 64, 48, 20, 0, 1, True, 1, False),
    (256, 128, 8, 64, 40, 100, 1, 0, False, 0, True),
    (512, 200, 4, 64, 9, 30, 0, 0, False, 1, False),
    (256, 256, 16, 64, 16, 200, 1, 0, False, 1, False),
    (256, 200, 8, 64, 40, 150, 0, 0, False, 1, True),
    (256, 200, 8, 64, 33, 12, 1, 0, False, 0, False),
    (256, 64, 8, 64, 40, 60, 0, 0, False, 1, False),
    (256, 64, 16, 64, 16, 64, 1, 0, False, 1, False),
    (256, 128, 2, 64, 16, 24, 0, 0, False, 1, True),
    (256, 200, 8, 64, 10, 40, 0, 0, False, 0, False),
    (256, 64, 1, 64, 12, 9, 0, 0, False, 1, False),
    (256, 64, 2, 64, 40, 30, 1, 0, False, 1, False),
    (256, 128, 3, 64, 33, 40, 0, 0, False, 0, True),
    # gate/up of eight wavefronts side by side, its last row group half there, slots of
    # one to four token tiles
    (256, 64, 4, 832, 72, 64, 0, 0, False, 1, False),
    (256, 24, 4, 1856, 200, 24, 0, 2, True, 0, True),
    (256, 24, 8, 2112, 120, 24, 2, 0, False, 1, False),
    # down with the combine, two and four loads of four rows a step
    (512, 16, 4, 576, 7, 4, 0, 1, True, 1, True),
    (512, 16, 4, 576, 13, 3, 0, 0, False, 0, False),
    # down in shares, one, two and four token tiles
    (256, 4, 4, 4352, 12, 4, 0, 0, False, 1, True),
    (256, 2, 1, 4096, 17, 2, 0, 0, False, 1, False),
    (256, 3, 2, 4160, 40, 3, 0, 0, False, 0, True),
]


@pytest.mark.parametrize("shape", INSTANCES, ids=lambda s: "-".join(str(int(v)) for v in s))
def test_layer_instances(gu, bd, shape):
    d, E, K, I, B, budget, flags, ns, gate, norm_topk, res = shape
    MxCase(gu, bd, d, E, K, I, B, ns, gate, norm_topk, seed=B + E).check(gu, bd, budget, flags, res)


@pytest.mark.parametrize("E,K,B,budget,flags,rule,norm_topk", [
    (16, 6, 1, 4, 2, 0, 1), (16, 6, 9, 5, 3, 0, 0), (100, 8, 16, 7, 2, 2, 1), (200, 5, 12, 9, 3, 0, 0), (40, 4, 16, 40, 0, 0, 1),
    (128, 16, 16, 30, 1, 2, 0), (256, 16, 5, 64, 2, 1, 1), (24, 6, 33, 5, 0, 2, 1), (200, 8, 64, 90, 1, 0, 0),
    (128, 8, 80, 20, 3, 3, 1)])
def test_ties_and_dropped_routes(gu, bd, E, K, B, budget, flags, rule, norm_topk):
    """Groups of experts with one logit each (+0 and -0 among them), identical tokens
    and so tied batch scores, a token of zeros; the whole plan, the routes' weights and
    the scores against the staged calls too."""
    c = MxCase(gu, bd, 256, E, K, 64, B, rule=rule, norm_topk=norm_topk, seed=E + B)
    inp, gl = c.inp, c.gl
    wr, br = inp["w_router"].copy(), inp["b_router"].copy()
    for experts, bias in ((range(3, 8), 1.5), (range(9, E, 4), -0.0), (range(10, E, 4), 0.0)):
        for e in experts:
            wr[e], br[e] = 0.0, bias
    inp["w_router"], inp["b_router"] = wr, br
    inp["pred_a"] = np.repeat(inp["pred_a"][::2], 2, 0)[:E].copy()
    inp["pred_b"] = np.repeat(inp["pred_b"][::2], 2)[:E].copy()
    inp["x"] = inp["x"].copy()
    inp["x"][B // 2:] = inp["x"][B // 2]
    if B > 1:
        inp["x"][0] = 0.0
    for t, a in zip(gl.layer.tensors[:4], (wr, br, inp["pred_a"], inp["pred_b"])):
        t.copy_(torch.from_numpy(a))
    c.check(gu, bd, budget, flags, True)
    x = gl.x(inp["x"])
    logits, ids, w = gl.route(x, B)
    cost = gl.predict(x, B, ids, w)
    scores, counts, sel, nsel, _ = gl.select(B, ids, cost, budget)
    ws, y = gl.workspace(B, budget), gl.y_like(B)
    got = gu.plan_arrays(bd.base_decode_layer(gl.desc, x, B, budget, flags, None, y, ws), ws, B, K, E, budget, True)
    for name, t in dict(logits=logits, topk_ids=ids, topk_w=w, cost=cost, scores=scores, counts=counts,
                        sel_ids=sel).items():
        assert np.array_equal(got[name], t.cpu().numpy()), name
    assert got["n_sel"] == int(nsel[0])
    routes = logits.gather(1, ids.long())
    assert B == 1 or bool((routes[:, 1:] == routes[:, :-1]).any())      # ties did decide


@pytest.mark.parametrize("rule", [1, 2, 3, 4])
def test_rules(gu, bd, rule):
    MxCase(gu, bd, 256, 16, 4, 64, 9, rule=rule, seed=3).check(gu, bd, 5)


def test_staged_and_fused_take_the_same_sums(gu, bd):
    """A budget far above the slots a few tokens can fill: the fused layer knows that
    the slots are few, the staged call does not, and the bits agree all the same."""
    c = MxCase(gu, bd, 512, 64, 1, 2048, 4, seed=31)
    gl = c.gl
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    for _ in range(40):
        x = torch.randn(4, 512, generator=g, device="cuda").bfloat16()
        ws, y, z = gl.workspace(4, 64), gl.y_like(4), gl.y_like(4)
        bd.base_decode_layer(gl.desc, x, 4, 64, 0, None, y, ws)
        logits, ids, w = gl.route(x, 4)
        _, _, sel, nsel, slot = gl.select(4, ids, gl.predict(x, 4, ids, w), 64)
        bd.base_moe_forward(gl.desc, x, 4, logits, ids, sel, nsel, slot, 64, 0, None, z, ws)
        assert torch.equal(y.view(torch.int16), z.view(torch.int16))


@pytest.mark.parametrize("E,K,I,B,budget,ns", [(1, 1, 512, 1, 1, 0), (2, 2, 1088, 2, 2, 0), (4, 2, 2112, 3, 1, 2),
                                               (16, 16, 576, 16, 1, 0), (256, 16, 64, 16, 256, 8),
                                               (64, 16, 192, 16, 64, 0)])
def test_few_tokens(gu, bd, E, K, I, B, budget, ns):
    """Down's launch that combines: one slot shared by many wavefronts, more slots than
    wavefronts, a chunk of one step and shares that end inside the contraction."""
    MxCase(gu, bd, 256, E, K, I, B, ns, ns == 2, seed=E + I).check(gu, bd, budget, 0, True)


@pytest.mark.parametrize("d,E,K,I,B,budget,ns", [(2048, 32, 8, 64, 4, 32, 0), (2048, 16, 8, 64, 3, 16, 2),
                                                 (2304, 4, 2, 4288, 4, 4, 0), (4608, 4, 2, 320, 2, 4, 1),
                                                 (256, 8, 8, 4608, 2, 8, 0), (256, 32, 8, 768, 4, 32, 0),
                                                 (4608, 8, 2, 320, 3, 6, 3), (512, 16, 8, 2048, 8, 11, 0)])
def test_few_tokens_on_both_sides_of_the_line(gu, bd, d, E, K, I, B, budget, ns):
    """More slots than a workgroup's wavefronts, many chunks a wavefront, and the shapes
    next to these that take down and the combine in two launches."""
    MxCase(gu, bd, d, E, K, I, B, ns, bool(ns), seed=d + B).check(gu, bd, budget, 0, True)


def test_long_contraction(gu, bd):
    """Many chunks in both products."""
    MxCase(gu, bd, 4096, 3, 2, 4160, 7, seed=2).check(gu, bd, 2)


@pytest.mark.parametrize("E,K,I,B,budget,ns", [(2, 1, 4096, 17, 2, 0), (3, 2, 4160, 40, 3, 0), (2, 2, 4416, 70, 2, 1),
                                               (1, 1, 4096, 300, 1, 0), (16, 8, 3968, 12, 16, 0),
                                               (16, 8, 4096, 12, 16, 0)])
def test_contraction_in_shares(gu, bd, E, K, I, B, budget, ns):
    """Few slots of long contractions: down's workgroups share one, with a last share
    that ends inside a chunk; the shapes on both sides of the line."""
    c = MxCase(gu, bd, 256, E, K, I, B, ns, seed=60 + B)
    c.check(gu, bd, budget, 0, True)
    gl, x = c.gl, c.gl.x(c.inp["x"])
    n = bd.Norms(256, torch.bfloat16, torch.ones(256, device="cuda"), None, torch.ones(256, device="cuda"), 0.5)
    ws, y, h = gl.workspace(B, budget), gl.y_like(B), torch.randn(B, 256, device="cuda").bfloat16()
    bd.base_decode_layer(gl.desc, x, B, budget, 0, None, y, ws)
    want, got = (torch.empty_like(h), torch.empty_like(h)), (torch.empty_like(h), torch.empty_like(h))
    bd.base_norm_residual(n, y, h, *want)
    bd.base_decode_block(gl.desc, n, x, B, budget, 0, h, ws, *got)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("B", [4, 40, 100])
def test_an_expert_twice_among_a_tokens_routes(gu, bd, B):
    """Routes the router never makes: a slot then has more pairs than tokens."""
    c = MxCase(gu, bd, 256, 4, 4, 64, B, seed=8)
    gl, x = c.gl, c.gl.x(c.inp["x"])
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    logits = torch.zeros(B, 4, device="cuda")
    ids = i32([[2, 2, 2, 1]] * B)
    sel, nsel, slot = i32([2, 1, -1]), i32([2]), i32([-1, 1, 0, -1])
    ws, y = gl.workspace(B, 3), gl.y_like(B)
    plan = bd.base_moe_forward(gl.desc, x, B, logits, ids, sel, nsel, slot, 3, 2, None, y, ws)
    got = gu.plan_arrays(plan, ws, B, 4, 4, 3, False)
    assert (got["exec_ids"] == [2, 2, 2, 1]).all()
    want, bound = c.outputs64(got, None)
    assert (np.abs(gu.to_np_f32(y).astype(np.float64) - want) <= bound).all()


@pytest.mark.parametrize("B,budget", [(5, 6), (64, 12), (130, 12)])
def test_noalloc_is_the_same(gu, bd, B, budget):
    c = MxCase(gu, bd, 512, 16, 4, 192, B, 1, True, seed=4)
    x = c.gl.x(c.inp["x"])
    ws, y, z = c.gl.workspace(B, budget), c.gl.y_like(B), c.gl.y_like(B)
    bd.base_decode_layer(c.gl.desc, x, B, budget, 0, None, y, ws)
    bd.base_decode_layer_noalloc(c.gl.desc, x, B, budget, 0, None, z)
    assert torch.equal(y.view(torch.int16), z.view(torch.int16))


@pytest.mark.parametrize("B", [3, 30, 90])
def test_rows_beyond_a_slots_are_not_read(gu, bd, B):
    """Garbage, NaN among it, in every place of the workspace and of y before the call,
    and twice in a row on one workspace with a smaller batch between."""
    c = MxCase(gu, bd, 512, 12, 3, 320, B, 1, True, seed=40)
    gl, x = c.gl, c.gl.x(c.inp["x"])
    out = []
    for fill in (0x00, 0xFF, 0x7F):
        ws, y = gl.workspace(B, 7), gl.y_like(B)
        ws.fill_(fill)
        bd.base_decode_layer(gl.desc, x, B, 7, 0, None, y, ws)
        small = gl.y_like(2)
        bd.base_decode_layer(gl.desc, x[:2].contiguous(), 2, 3, 2, None, small, ws)
        again = gl.y_like(B)
        bd.base_decode_layer(gl.desc, x, B, 7, 0, None, again, ws)
        assert torch.equal(y.view(torch.int16), again.view(torch.int16))
        out.append(y)
    assert all(torch.equal(out[0].view(torch.int16), o.view(torch.int16)) for o in out[1:])


def test_fp32_master_weights(gu, bd):
    """An fp32 layer's experts quantised: its activations are bf16 from then on."""
    inp = W.custom_layer(256, 4, 2, 128, 6, bf16=False, seed=3)
    src = gu.GpuLayer(inp)
    lay = bd.mx_layer(src.layer)
    assert lay.torch_dtype == torch.bfloat16
    c = MxCase.__new__(MxCase)
    q = lambda a: W.f32_to_bf16_bits(mx.dequantize(*mx.quantize(a.reshape(-1, a.shape[-1]).astype(np.float64)))  # noqa: E731
                                     .astype(np.float32)).reshape(a.shape)
    x = rounded(inp["x"], "bf16")
    c.inp = dict(inp, x=x, w13=q(inp["w13"]), w2=q(inp["w2"]))
    c.sh, c.ns = inp["shape"], 0
    desc = lay.desc(2)
    ws = torch.empty(bd.base_workspace_bytes(desc, 6, 4), dtype=torch.uint8, device="cuda")
    y = torch.empty(6, 256, dtype=torch.bfloat16, device="cuda")
    plan = bd.base_decode_layer(desc, to_dev(x, "bf16"), 6, 4, 0, None, y, ws)
    want, bound = c.outputs64(gu.plan_arrays(plan, ws, 6, 2, 4, 4, True), None)
    assert (np.abs(gu.to_np_f32(y).astype(np.float64) - want) <= bound).all()


@pytest.mark.parametrize("scale", [1e-6, 1e4, 1e18])
@pytest.mark.parametrize("B", [5, 40])
def test_small_and_large_activations(gu, bd, B, scale):
    """Activations below and above the second part's range, to 1e36: nothing is lost
    but precision, nothing overflows that the values do not."""
    c = MxCase(gu, bd, 256, 4, 2, 192, B, seed=50)
    c.inp["x"] = rounded(c.inp["x"] * scale, "bf16")
    gl, x = c.gl, c.gl.x(c.inp["x"])
    logits = torch.randn(B, 4, device="cuda")
    ids = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :2].int().contiguous()
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    ws, y = gl.workspace(B, 4), gl.y_like(B)
    plan = bd.base_moe_forward(gl.desc, x, B, logits, ids, i32([0, 1, 2, 3]), i32([4]), i32([0, 1, 2, 3]), 4, 0,
                               None, y, ws)
    with np.errstate(over="ignore"):
        want, bound = c.outputs64(gu.plan_arrays(plan, ws, B, 2, 4, 4, False), None)
    got = gu.to_np_f32(y).astype(np.float64)
    assert np.isfinite(got).all() and (np.abs(got - want) <= bound).all()


@pytest.mark.parametrize("B,budget", [(1, 4), (48, 12), (200, 10)])
def test_captured_and_replayed(gu, bd, B, budget):
    """A graph replayed between eager calls with other inputs, on a stream of its own."""
    c = MxCase(gu, bd, 512, 16, 4, 192, B, 1, False, seed=6)
    x0 = c.gl.x(c.inp["x"])
    xs = [x0, x0.flip(0).contiguous(), (x0 * 0.5).contiguous()]
    want = []
    for x in xs:
        y, ws = c.gl.y_like(B), c.gl.workspace(B, budget)
        bd.base_decode_layer(c.gl.desc, x, B, budget, 0, x, y, ws)
        want.append(y)
    side = torch.cuda.Stream()
    x, y, ws = x0.clone(), c.gl.y_like(B), c.gl.workspace(B, budget)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        bd.base_decode_layer(c.gl.desc, x, B, budget, 0, x, y, ws)
    for i in (0, 1, 2, 1, 0):
        x.copy_(xs[i])
        y.fill_(3.0)
        ws.fill_(0xCD)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y.view(torch.int16), want[i].view(torch.int16)), i


def test_calibration_statistics(gu, bd):
    """The statistics of a 4-bit layer against those of the bf16 layer whose weights
    have the same values: targets log ||E(z)||^2 of outputs that differ by the
    roundings of h (2^-8 in norm, so 2 log(1 + 2^-8) < 2^-6 in the target)."""
    c = MxCase(gu, bd, 256, 8, 3, 192, 150, seed=9)
    ref = gu.GpuLayer(c.inp, packed=True)
    out = []
    for gl in (ref, c.gl):
        stats = bd.calib_stats(gl.desc)
        for _ in range(2):
            bd.calib_accumulate(gl.desc, gl.x(c.inp["x"]), 150, stats)
        torch.cuda.synchronize()
        out.append(stats.cpu().numpy())
    head = [s[:8 * 32].view(np.float64).reshape(8, 4) for s in out]
    n = head[0][:, 0]
    assert np.array_equal(n, head[1][:, 0]) and n.sum() == 2 * 150 * 3
    assert (np.abs(head[0][:, 1] - head[1][:, 1]) <= 2.0 ** -6 * n).all()
    up = lambda v: -(-v // 256) * 256  # noqa: E731
    o = up(8 * 32)
    assert np.array_equal(out[0][o:o + 8 * 256 * 8], out[1][o:o + 8 * 256 * 8])   # sum of z_bar: no expert output


def test_a_scale_of_nan_and_extreme_scales(gu, bd):
    """NaN blocks make the rows that meet them NaN and no others; scales at both ends
    of the format are exact."""
    d, I, E, B = 256, 64, 2, 3
    g = np.random.default_rng(0)
    w13 = rounded(g.standard_normal((E * 2 * I, d)) / 16, "bf16")
    w2 = rounded(g.standard_normal((E * d, I)) / 8, "bf16")
    c13, s13 = mx.quantize(w13)
    c2, s2 = mx.quantize(w2)
    s2[5, 1] = 255                       # expert 0, output row 5
    s2[d + 9] = 0                        # expert 1, output row 9: 2^-127
    t = lambda a, *s: torch.from_numpy(a).cuda().view(*s, -1)  # noqa: E731
    wr = torch.zeros(E, d, device="cuda")
    lay = bd.mx_layer_from_codes(wr, torch.tensor([1.0, 0.0]).cuda(), None, None, (t(c13, E, 2 * I), t(s13, E, 2 * I)),
                                 (t(c2, E, d), t(s2, E, d)), score_rule=2)
    desc = lay.desc(1)
    x = torch.randn(B, d, device="cuda").bfloat16()
    ys = []
    for bias in (1.0, -1.0):             # every token to expert 0, then to expert 1
        lay.tensors[1][0] = bias
        ws = torch.empty(bd.base_workspace_bytes(desc, B, 1), dtype=torch.uint8, device="cuda")
        y = torch.empty(B, d, dtype=torch.bfloat16, device="cuda")
        bd.base_decode_layer(desc, x, B, 1, 0, None, y, ws)
        ys.append(y.float().cpu())
    assert torch.isnan(ys[0][:, 5]).all() and int(torch.isnan(ys[0]).sum()) == B
    assert torch.isfinite(ys[1]).all() and (ys[1][:, 9].abs() < 1e-30).all()


def test_nan_and_infinity_in_one_token_stay_in_its_row(gu, bd):
    """The scoring leaves such a batch's plan unspecified, so the routes are given."""
    c = MxCase(gu, bd, 256, 4, 2, 192, 20, seed=12)
    x = c.gl.x(c.inp["x"])
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    logits = torch.randn(20, 4, device="cuda")
    ids = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :2].int().contiguous()
    args = (i32([0, 1, 2, 3]), i32([4]), i32([0, 1, 2, 3]), 4, 0)
    ys = []
    for bad in (False, True):
        xb = x.clone()
        if bad:
            xb[7, 3], xb[11] = float("nan"), float("inf")
        y, ws = c.gl.y_like(20), c.gl.workspace(20, 4)
        bd.base_moe_forward(c.gl.desc, xb, 20, logits, ids, *args, None, y, ws)
        ys.append(y)
    keep = [t for t in range(20) if t not in (7, 11)]
    assert torch.equal(ys[0][keep].view(torch.int16), ys[1][keep].view(torch.int16))
    assert not torch.isfinite(ys[1][[7, 11]]).any()


def pool_of(t):
    """The stream in whose memory a tensor lies."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not the allocator's")


def test_new_tensors_lie_in_the_memory_of_the_stream_that_writes_them(gu, bd):
    """A block freed on the current stream may still be in use there, so a kernel on
    another stream must not get it."""
    cur, side = torch.cuda.current_stream(), torch.cuda.Stream()
    src, gain = torch.randn(8, 256, device="cuda").bfloat16(), torch.ones(256, device="cuda")
    inp = W.custom_layer(256, 4, 2, 64, 5, seed=3, n_shared=1, shared_gate=True)
    gl = gu.GpuLayer(inp)
    torch.cuda.synchronize()
    for stream, where in ((side, side.cuda_stream), (None, cur.cuda_stream)):
        codes, scales = bd.mx_quantize(src, stream=stream)
        new = [codes, scales, bd.mx_dequantize(codes, scales, stream=stream)]
        new += bd.norm_residual(src, src, pre_gain=gain, stream=stream)
        for lay in (bd.mx_layer(gl.layer, stream), bd.packed_layer(gl.layer, 2, stream)):
            new += [*lay.tensors[4:6], *lay.shared[:2]]
        torch.cuda.synchronize()
        assert all(pool_of(t) == where for t in new)
    want = bd.mx_quantize(src)
    torch.cuda.synchronize()
    for stream in (side, None):
        got = bd.mx_quantize(src, stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))

"""Norms of heads with the rotation by position, and the same into a paged cache, on the
GPU against 64-bit arithmetic (tolerance: attn_util.rotate); a run of the calls together."""
import numpy as np
import pytest

import attn_util as U

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
BF, F32 = U.BF, U.F32


@pytest.fixture(scope="module")
def bd(gpu):
    return gpu


def cuda(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def make(g, rows, H, D, dtype, std=2.0):
    return torch.from_numpy(g.standard_normal((rows, H, D), np.float32) * np.float32(std)).to(dtype)


def gains(g, D, norm):
    return [1 + 0.2 * g.standard_normal(D).astype(np.float32) if norm else None for _ in range(2)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(8, 8), (8, 2), (16, 16), (40, 40), (64, 64), (64, 0), (72, 70), (80, 32), (96, 48),
                                   (128, 128), (128, 64), (128, 34), (136, 136), (192, 64), (256, 256), (256, 16)])
def test_rotation(bd, dtype, interleaved, D, rot):
    g = np.random.default_rng(D * 1000 + rot)
    rows, Hq, Hk = 37, 5, 2
    for norm in (False, True):
        q, k = make(g, rows, Hq, D, dtype), make(g, rows, Hk, D, dtype)
        inv, scale = U.frequencies(rot), 1.0 if norm else 1.25
        pos = g.integers(-5, 200000, rows).astype(np.int32)
        gq, gk = gains(g, D, norm)
        r = bd.Rope(D, dtype, cuda(inv) if rot else None, interleaved, scale, cuda(gq), cuda(gk), 1e-6)
        qo, ko = bd.head_rope(r, cuda(pos) if rot else None, q.cuda(), k.cuda())
        for x, gain, got in ((q, gq, qo), (k, gk, ko)):
            want, bound = U.rotate(x.double().numpy(), gain, pos, inv, scale, interleaved, 1e-6)
            U.near(got, want, bound, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(16, 8), (24, 16), (24, 18), (32, 18), (40, 24), (72, 64), (80, 50), (88, 72), (120, 120),
                                   (128, 18), (128, 110), (128, 120), (232, 96), (248, 248), (256, 18), (256, 250)])
def test_rotation_of_a_part(bd, dtype, interleaved, D, rot):
    """Parts that are no whole runs: in place and out of place, norms with them."""
    g = np.random.default_rng(D * 1000 + rot)
    rows, Hq, Hk = 21, 19, 3
    q, k = make(g, rows, Hq, D, dtype), make(g, rows, Hk, D, dtype)
    inv, pos = U.frequencies(rot), g.integers(0, 200000, rows).astype(np.int32)
    gq, gk = gains(g, D, True)
    r = bd.Rope(D, dtype, cuda(inv), interleaved, 1.0, cuda(gq), cuda(gk), 1e-6)
    qo, ko = bd.head_rope(r, cuda(pos), q.cuda(), k.cuda())
    for x, gain, got in ((q, gq, qo), (k, gk, ko)):
        want, bound = U.rotate(x.double().numpy(), gain, pos, inv, 1.0, interleaved, 1e-6)
        U.near(got, want, bound, dtype)
    qi, ki = q.cuda(), k.cuda()
    bd.base_head_rope(r, cuda(pos), qi, ki, qi, ki)
    assert torch.equal(qi, qo) and torch.equal(ki, ko)


@pytest.mark.parametrize("rows", [1, 2, 3, 65, 1000, 20000])
@pytest.mark.parametrize("Hq,Hk", [(1, 0), (0, 3), (32, 4), (13, 13)])
def test_rows_and_heads(bd, rows, Hq, Hk):
    g = np.random.default_rng(rows)
    D, inv = 64, U.frequencies(64)
    pos = g.integers(0, 1 << 21, rows).astype(np.int32)
    gq, gk = gains(g, D, True)
    r = bd.Rope(D, BF, cuda(inv), False, 1.0, cuda(gq), cuda(gk), 1e-5)
    q, k = (make(g, rows, H, D, BF) if H else None for H in (Hq, Hk))
    outs = [None if t is None else torch.empty_like(t, device="cuda") for t in (q, k)]
    bd.base_head_rope(r, cuda(pos), *(None if t is None else t.cuda() for t in (q, k)), *outs)
    for x, gain, got in ((q, gq, outs[0]), (k, gk, outs[1])):
        if x is not None:
            want, bound = U.rotate(x.double().numpy(), gain, pos, inv, 1.0, False, 1e-5)
            U.near(got, want, bound, BF)


def test_far_positions_and_extremes(bd):
    """The largest positions, a row of zeros, an eps of 0, NaN and infinities in one head."""
    g = np.random.default_rng(2)
    D, rows = 128, 6
    inv = U.frequencies(D)
    pos = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 16777217], np.int32)
    x = make(g, rows, 3, D, F32)
    gq = gains(g, D, True)[0]
    r = bd.Rope(D, F32, cuda(inv), False, 1.0, cuda(gq), None, 0.0)
    x[0, 0] = 0
    x[1, 1, 5], x[2, 1, 7] = float("nan"), float("inf")
    out = bd.head_rope(r, cuda(pos), x.cuda())[0].cpu()
    assert (out[0, 0] == 0).all()
    clean = x.clone()
    clean[0, 0] = clean[1, 1] = clean[2, 1] = 1
    want, bound = U.rotate(clean.double().numpy(), gq, pos, inv, 1.0, False, 0.0)
    # 2^31 positions times 2^-53 of a turn: the fraction is off by 2^-24 at most
    bound = bound + 2.0 ** -21 * np.abs(want).max(2, keepdims=True)
    keep = np.ones((rows, 3), bool)
    keep[0, 0] = keep[1, 1] = keep[2, 1] = False
    U.near(out[torch.from_numpy(keep)], want[keep], bound[keep], F32)
    assert out[1, 1].isnan().any() and not out[2, 1].isfinite().all()
    plain = bd.Rope(D, F32, cuda(inv))
    out = bd.head_rope(plain, cuda(pos), x.cuda())[0].cpu()
    assert int(out[1, 1].isnan().sum()) == 2          # only the pair


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,rot", [(64, 64), (128, 48), (80, 30)])
def test_strides_and_in_place(bd, dtype, D, rot):
    g = np.random.default_rng(D)
    rows, H = 19, 5
    inv = U.frequencies(rot)
    pos = g.integers(0, 5000, rows).astype(np.int32)
    x = make(g, rows, H, D, dtype)
    want, bound = U.rotate(x.double().numpy(), None, pos, inv, 1.0, False, 1e-6)
    r = bd.Rope(D, dtype, cuda(inv))
    buf = torch.full((rows * (H * (D + 1) + 3) + 1,), 7.0, dtype=dtype, device="cuda")
    v = buf[1:].view(rows, H * (D + 1) + 3)[:, 3:].unflatten(1, (H, D + 1))[..., 1:]
    v.copy_(x)
    out = torch.empty(H, rows, D, dtype=dtype, device="cuda").transpose(0, 1)   # heads outermost
    bd.base_head_rope(r, cuda(pos), v, None, out, None)
    U.near(out, want, bound, dtype)
    bd.base_head_rope(r, cuda(pos), v, None, v, None)
    U.near(v, want, bound, dtype)
    v.fill_(7.0)
    assert (buf == 7).all()


def append(bd, b, Hq, rot, interleaved, norm, positions=None, extra_rows=0, inplace=False, seed=0):
    """The new tokens of b into its cache; checks q, the cache and what lies around."""
    g = np.random.default_rng(seed)
    D, rows = b.D, b.rows + extra_rows
    inv = U.frequencies(rot)
    gq, gk = gains(g, D, norm)
    qkv = torch.from_numpy(g.standard_normal((rows, Hq + 2 * b.Hk, D), np.float32)).to(b.dtype).cuda()
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + b.Hk], qkv[:, Hq + b.Hk:]
    kept = qkv.clone()
    cache, batch = b.device(bd)
    old = [t.clone() for t in cache.tensors]
    r = bd.Rope(D, b.dtype, cuda(inv) if rot else None, interleaved, 1.0, cuda(gq), cuda(gk))
    out = q if inplace else torch.full((rows, Hq, D), 7.0, dtype=b.dtype, device="cuda")
    bd.base_kv_append(r, cache, batch, q, k, v, out, cuda(positions))
    torch.cuda.synchronize()
    own = np.concatenate([kv - n + np.arange(n) for n, kv in b.lens]).astype(np.int64)
    pos = own if positions is None else positions[:b.rows]
    want, bound = U.rotate(kept[:b.rows, :Hq].double().cpu().numpy(), gq, pos, inv, 1.0, interleaved, 1e-6)
    U.near(out[:b.rows], want, bound, b.dtype, "q")
    if not inplace:
        assert (out[b.rows:] == 7).all() and torch.equal(qkv, kept)
    kw, kb = U.rotate(kept[:b.rows, Hq:Hq + b.Hk].double().cpu().numpy(), gk, pos, inv, 1.0, interleaved, 1e-6)
    touched = torch.zeros(old[0].shape[:2], dtype=torch.bool)
    for s, (n, kv) in enumerate(b.lens):
        lo = max(kv - n, 0)
        if lo >= kv or not n:
            continue
        page, slot = b.slots(s, lo, kv)
        t = slice(b.starts[s] + n - (kv - lo), b.starts[s] + n)
        U.near(cache.tensors[0][page.cuda(), slot.cuda()], kw[t], kb[t], b.dtype, "k")
        assert torch.equal(cache.tensors[1][page.cuda(), slot.cuda()], kept[t, Hq + b.Hk:])
        touched[page, slot] = True
    for now, was in zip(cache.tensors, old):
        assert torch.equal(now[~touched.cuda()], was[~touched.cuda()])
    return cache, batch, out


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,rot,interleaved", [(128, 128, False), (64, 32, True), (80, 20, False), (256, 256, True),
                                               (24, 0, False)])
@pytest.mark.parametrize("ps,heads_first", [(16, True), (64, False)])
def test_append(bd, dtype, D, rot, interleaved, ps, heads_first):
    lens = [(1, 1), (3, 40), (0, 9), (70, 70), (1, 129), (0, 0), (5, 64), (4, 2), (2, 300)]
    b = U.Batch(lens, 3, D, ps, dtype, seed=D, heads_first=heads_first, fill=3.0)
    append(bd, b, 7, rot, interleaved, D != 64, extra_rows=4, inplace=D == 80)


@pytest.mark.parametrize("n_seq", [1, 63, 64, 65, 200, 4097])
def test_append_many_sequences(bd, n_seq):
    g = np.random.default_rng(n_seq)
    lens = [(int(g.integers(0, 3)), int(g.integers(2, 40))) for _ in range(n_seq)]
    lens[-1] = (1, 7)
    append(bd, U.Batch(lens, 1, 16, 16, BF, seed=n_seq, fill=3.0), 2, 16, False, True)


def test_append_positions(bd):
    """Given positions turn the heads; the slots stay the tokens' own."""
    b = U.Batch([(3, 10), (1, 500)], 2, 64, 16, BF, seed=1, fill=3.0)
    append(bd, b, 4, 64, False, True, positions=np.array([7, -2, 1 << 20, 123456], np.int32))


def test_append_bad_pages(bd):
    """Tokens whose page is not in the cache, or past the table, are left out of it."""
    b = U.Batch([(2, 20), (3, 35)], 1, 16, 16, BF, seed=4, fill=3.0, extra=0)
    b.table[0, 1] = b.n_pages
    b.table[1, 2] = -1
    cache, batch = b.device(bd)
    batch.tensors[2][1] = 50                      # past the table's three pages
    g = np.random.default_rng(1)
    q, k, v = (make(g, b.rows, h, 16, BF).cuda() for h in (2, 1, 1))
    out = torch.empty_like(q)
    bd.base_kv_append(bd.Rope(16, BF), cache, batch, q, k, v, out)
    assert torch.equal(out, q) and all((t == 3).all() for t in cache.tensors)
    batch.tensors[1].copy_(torch.tensor([3, -1, 2 ** 31 - 1], dtype=torch.int32))
    bd.base_kv_append(bd.Rope(16, BF), cache, batch, q, k, v, out)
    torch.cuda.synchronize()


def test_scaled_frequencies(bd):
    inv, s = bd.rope_frequencies(64, 10000.0)
    assert s == 1.0 and np.allclose(inv.numpy(), U.frequencies(64), rtol=2e-7)
    inv4, s4 = bd.rope_frequencies(64, 10000.0, 4.0)
    assert s4 == 1.0 and np.allclose(4 * inv4.numpy(), inv.numpy(), rtol=2e-7)
    part, sp = bd.rope_frequencies(64, 10000.0, 4.0, trained=4096)
    assert abs(sp - (0.1 * np.log(4.0) + 1)) < 1e-12
    turns = 4096 * U.frequencies(64).astype(np.float64) / (2 * np.pi)
    ratio = part.numpy() / inv.numpy()
    assert np.allclose(ratio[turns > 40], 1) and np.allclose(ratio[turns < 0.75], 0.25)
    assert (np.diff(ratio) <= 1e-6).all()


def test_whole_block(bd):
    """A decode step of one block as a program runs it -- norm, projection, append, attention,
    projection, norm and experts -- against the same in 64 bits, for a prompt and then
    single tokens on its cache."""
    import workloads as W
    from oracle import method
    d, Hq, Hk, D, ps, dt = 512, 8, 2, 64, 16, BF
    inp = W.custom_layer(d, 32, 4, 128, 48, bf16=True, seed=11)
    g = np.random.default_rng(0)
    wqkv = torch.from_numpy(g.standard_normal((Hq + 2 * Hk) * D * d).astype(np.float32).reshape(-1, d) * d ** -0.5).to(dt)
    wo = torch.from_numpy(g.standard_normal((d, Hq * D)).astype(np.float32) * (Hq * D) ** -0.5).to(dt)
    gq, gk = gains(g, D, True)
    pre = 1 + 0.1 * g.standard_normal(d).astype(np.float32)
    inv, eps = U.frequencies(D), 1e-6
    f32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()  # noqa: E731
    bits = lambda a: torch.from_numpy(a.view(np.int16)).cuda().view(dt)  # noqa: E731
    layer = bd.Layer(f32(inp["w_router"]), f32(inp["b_router"]), f32(inp["pred_a"]), f32(inp["pred_b"]),
                     bits(inp["w13"]), bits(inp["w2"]))
    desc = layer.desc(inp["shape"].K)
    rope = bd.Rope(D, dt, cuda(inv), False, 1.0, cuda(gq), cuda(gk), eps)
    n_seq, pages = 3, 12
    kc, vc = (torch.full((pages, Hk, ps, D), float("nan"), dtype=dt, device="cuda").transpose(1, 2) for _ in range(2))
    cache = bd.KVCache(kc, vc)
    table = torch.from_numpy(g.permutation(pages).astype(np.int32).reshape(n_seq, 4)).cuda()
    norms = bd.Norms(d, dt, pre_gain=f32(pre), eps=eps)
    stream = [torch.zeros(0, d, dtype=torch.float64) for _ in range(n_seq)]     # normed inputs in 64 bits
    lens = np.zeros(n_seq, np.int64)
    budget = 6
    for new in ([20, 1, 9], [1, 1, 1], [1, 0, 1], [2, 5, 1]):
        rows = sum(new)
        lens += new
        h = torch.from_numpy(g.standard_normal((rows, d)).astype(np.float32)).to(dt).cuda()
        starts = torch.tensor([0, *np.cumsum(new)], dtype=torch.int32).cuda()
        batch = bd.KVBatch(table, starts, torch.from_numpy(lens.astype(np.int32)).cuda(), max(new))
        _, x = bd.norm_residual(h, pre_gain=f32(pre), eps=eps)
        qkv = (x.float() @ wqkv.cuda().float().T).to(dt).unflatten(1, (-1, D))
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
        bd.base_kv_append(rope, cache, batch, q, k, v, q)
        o = bd.paged_attention(q, cache, batch)
        y = (o.flatten(1).float() @ wo.cuda().float().T).to(dt)
        h1, x1 = bd.norm_residual(h, y, pre_gain=f32(pre), eps=eps)
        h2, x2 = torch.empty_like(h), torch.empty_like(h)
        ws = torch.empty(bd.base_workspace_bytes(desc, rows, budget), dtype=torch.uint8, device="cuda")
        bd.base_decode_block(desc, norms, x1, rows, budget, 0, h1, ws, h2, x2)
        # the attention half again from the normed rows the GPU used, in 64 bits
        xs = x.double().cpu()
        at, want = 0, []
        for s in range(n_seq):
            stream[s] = torch.cat([stream[s], xs[at:at + new[s]]])
            at += new[s]
            z = (stream[s] @ wqkv.double().T).view(-1, Hq + 2 * Hk, D).numpy()
            pos = np.arange(len(z))
            qs, ks = (U.rotate(z[:, a:b], gn, pos, inv, 1.0, False, eps)[0]
                      for a, b, gn in ((0, Hq, gq), (Hq, Hq + Hk, gk)))
            out = np.zeros((new[s], Hq, D))
            for i in range(new[s]):
                p = len(z) - new[s] + i
                for hh in range(Hq):
                    e = ks[:p + 1, hh // 4] @ qs[p, hh] * D ** -0.5
                    e = np.exp(e - e.max())
                    out[i, hh] = e @ z[:p + 1, Hq + Hk + hh // 4] / e.sum()
            want.append(out.reshape(new[s], Hq * D))
        want = np.concatenate(want)
        got = o.flatten(1).double().cpu().numpy()
        # q, k, v, the exponentials and the output each rounded to bf16 (half a step 2^-8;
        # scores of normed heads reach |gain|^2 sqrt(D) and move by 4 roundings' share of that)
        tol = 2.0 ** -8 * (4 + 4 * 1.5 * D ** 0.5) * np.abs(want).max()
        assert np.abs(got - want).max() <= tol
        assert np.linalg.norm(got - want) <= 2.0 ** -8 * 4 * np.linalg.norm(want)
        # and the experts' half from what it was given
        ref = method.decode_layer_c(x1.float().cpu().numpy(), inp["w_router"], inp["b_router"], inp["pred_a"],
                                    inp["pred_b"], inp["shape"].K, budget,
                                    method.Experts(inp["w13"], inp["w2"], True))
        step = h1.float().cpu().numpy() + ref["y"]
        assert np.abs(h2.float().cpu().numpy() - step).max() <= 2e-2 + 2.0 ** -8 * np.abs(step).max()


@pytest.mark.parametrize("starts,lens,width", [
    ([0, 5], [10], 2),                       # the last start beyond the rows (a padded batch)
    ([-3, 2, 9], [6, 40], 3),                # and the first before them
    ([0, 1, 4], [9, 50], 3),                 # a length beyond the table's row
    ([0, 2, 4], [-4, 2 ** 31 - 1], 2), ([0, 2, 2 ** 31 - 1], [7, 2 ** 31 - 1], 2)])
def test_starts_and_lengths_are_taken_within_their_bounds(bd, starts, lens, width):
    """Append and attention take the same starts and lengths, those of 0 .. rows and 0 .. the
    table's row: the calls give what they give with these written out."""
    g = np.random.default_rng(5)
    rows, D, ps = 4, 32, 16
    n_seq = len(lens)
    table = cuda(np.arange(n_seq * width, dtype=np.int32).reshape(n_seq, width))
    r = bd.Rope(D, BF, cuda(U.frequencies(D)))
    qkv = make(g, rows, 6, D, BF).cuda()
    old = make(g, n_seq * width * 2 * ps, 1, D, BF).view(2, n_seq * width, ps, 1, D).cuda()
    within = np.clip(starts, 0, rows)
    got = []
    for q_start, kv_len in ((starts, lens), (within, np.clip(lens, 0, width * ps))):
        k, v = old.clone()
        cache = bd.KVCache(k, v)
        batch = bd.KVBatch(table, *(cuda(np.array(t, np.int64).astype(np.int32)) for t in (q_start, kv_len)), rows)
        q = torch.full((rows, 4, D), 7.0, dtype=BF, device="cuda")
        bd.base_kv_append(r, cache, batch, qkv[:, :4], qkv[:, 4:5], qkv[:, 5:], q)
        out, lse = bd.paged_attention(q, cache, batch, return_lse=True)
        got.append((q, k, v, out, lse))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    # and these are the tokens' places: the last of the sequence's new rows in its last slot
    for s in range(n_seq):
        kv, n = int(np.clip(lens[s], 0, width * ps)), int(within[s + 1] - within[s])
        for i in range(max(n - kv, 0), n):
            at = kv - n + i
            assert torch.equal(got[0][2][s * width + at // ps, at % ps, 0], qkv[within[s] + i, 5])


MANY = (1 << 26) + 5      # a wavefront a row: more than one launch can have


def test_more_rows_than_a_launch_has(bd):
    """The rows of one call against the same in parts that a launch holds."""
    inv = cuda(U.frequencies(8))
    r = bd.Rope(8, BF, inv)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    q = torch.randn(MANY, 1, 8, generator=gen, dtype=BF, device="cuda")
    pos = torch.arange(MANY, dtype=torch.int32, device="cuda")
    got = torch.zeros_like(q)
    bd.base_head_rope(r, pos, q, None, got, None)
    step = 1 << 24
    for at in range(0, MANY, step):
        part = slice(at, min(at + step, MANY))
        want = bd.head_rope(r, pos[part], q[part])[0]
        assert torch.equal(got[part], want), at
    want, bound = U.rotate(q[-7:].double().cpu().numpy(), None, pos[-7:].cpu().numpy(), U.frequencies(8), 1.0, False, 1e-6)
    # (a turn's fraction of 2^26 positions: fp64, as near as any)
    U.near(got[-7:], want, bound, BF)


def test_append_of_more_rows_than_a_launch_has(bd):
    """Three sequences, the second over the launches' border; most of its tokens have negative
    numbers and stay out of the cache.  Rows of no sequence are left."""
    r = bd.Rope(8, BF, cuda(U.frequencies(8)))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    qkv = torch.randn(MANY, 3, 8, generator=gen, dtype=BF, device="cuda")
    q, k, v = qkv[:, :1], qkv[:, 1:2], qkv[:, 2:]
    starts, lens = [5, 8, (1 << 26) + 1, MANY - 1], [3, 100, 50]
    kc, vc = (torch.full((3 * 7, 16, 1, 8), 3.0, dtype=BF, device="cuda") for _ in range(2))
    table = torch.arange(21, dtype=torch.int32, device="cuda").view(3, 7)
    batch = bd.KVBatch(table, cuda(np.array(starts, np.int32)), cuda(np.array(lens, np.int32)), 1 << 26)
    got = torch.full((MANY, 1, 8), 7.0, dtype=BF, device="cuda")
    bd.base_kv_append(r, bd.KVCache(kc, vc), batch, q, k, v, got)
    assert (got[:5] == 7).all() and (got[-1] == 7).all()
    pos = torch.cat([torch.arange(n - (b - a), n, dtype=torch.int32) for a, b, n in zip(starts, starts[1:], lens)]).cuda()
    step = 1 << 24
    for at in range(5, MANY - 1, step):
        part = slice(at, min(at + step, MANY - 1))
        assert torch.equal(got[part], bd.head_rope(r, pos[at - 5:part.stop - 5], q[part])[0]), at
    for s, (stop, n) in enumerate(zip(starts[1:], lens)):
        rows = slice(max(stop - n, starts[s]), stop)
        new = rows.stop - rows.start
        turned = bd.head_rope(r, pos[rows.start - 5:rows.stop - 5], k[rows])[0]
        for c, want in ((kc, turned), (vc, v[rows])):
            have = c.view(3, 112, 1, 8)[s]
            assert torch.equal(have[n - new:n], want)
            assert (have[:n - new] == 3).all() and (have[n:] == 3).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_captured_step(bd, dtype):
    """Append and attention captured together and replayed token by token, the program writing
    the next token's heads and the lengths between the replays, with eager work of its own."""
    g = np.random.default_rng(41)
    D, Hq, Hk, ps, n_seq, steps = 64, 8, 2, 16, 5, 20
    r = bd.Rope(D, dtype, cuda(U.frequencies(D)), True, 1.0, *(cuda(t) for t in gains(g, D, True)))
    start = np.array([0, 15, 16, 47, 130], np.int32)
    pages = n_seq * 10
    table = cuda(g.permutation(pages).astype(np.int32).reshape(n_seq, 10))
    first = torch.randn(2, pages, ps, Hk, D, dtype=dtype, device="cuda")
    runs = []
    for captured in (False, True):
        k, v = first.clone()
        cache = bd.KVCache(k, v)
        kv_len = cuda(start + 1)
        batch = bd.KVBatch(table, torch.arange(n_seq + 1, dtype=torch.int32, device="cuda"), kv_len, 1)
        qkv = torch.empty(n_seq, Hq + 2 * Hk, D, dtype=dtype, device="cuda")
        q, out = (torch.empty(n_seq, Hq, D, dtype=dtype, device="cuda") for _ in range(2))
        ws = torch.empty(bd.attention_workspace_bytes(cache, batch, n_seq, Hq), dtype=torch.uint8, device="cuda")

        def step():
            bd.base_kv_append(r, cache, batch, qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:], q)
            bd.base_paged_attention(cache, batch, q, out, ws)
        if captured:
            qkv.zero_()
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
                step()
            torch.cuda.synchronize()
        h = np.random.default_rng(42)
        got = []
        for i in range(steps):
            qkv.copy_(make(h, n_seq, Hq + 2 * Hk, D, dtype).cuda())
            graph.replay() if captured else step()
            got.append((out.clone(), q.clone()))
            kv_len += 1
            if i % 5 == 4:
                torch.cuda.synchronize()
        runs.append((got, k, v))
    (eager, ke, ve), (replayed, kr, vr) = runs
    for a, b in zip(eager, replayed):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(ke, kr) and torch.equal(ve, vr)

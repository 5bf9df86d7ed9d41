"""The library's operators on 4-bit experts and on the residual stream, measured on one MI355X.

Two families.  Microscaled 4-bit floating point (blocks of 32 elements along the contraction, E2M1 codes with
one E8M0 scale): rows quantised and read back (`base_mx_quantize`, `base_mx_dequantize`), the experts' grouped
SwiGLU products with such weights on a given routing (`base_moe_forward` on a BASE_W_MXFP4 layer), and the whole
decode layer for a few tokens (`base_decode_layer`).  The norms around a block, with its gate and the residual
scale (`base_norm_residual`).

With `own` false every operator is computed from elementary torch operations instead, in 32 bits (routing
scores, which decide whole numbers, in 64).  Shapes are those of the models in `workloads` or generic ones;
hidden states, routers and experts follow its recipe, drawn on the GPU.
"""
import math

import torch

own = False

FFN = dict(kind="ffn", norm_topk=1, flags=0, residual=False, n_shared=0, shared_gate=False)
LAYER = dict(kind="layer", norm_topk=1, flags=0, residual=False, n_shared=0, shared_gate=False)
QWEN3 = dict(d=2048, E=128, K=8, I=768)
# norm: post (normalise the block's output), gate ("none", "channel", "token"), pre (write the next block's input)
NORM = dict(kind="norm", dtype="bf16", post=True, gate="channel", pre=True, block=True, pad=0)


def listed():
    return [
        # one expert's projection requantised: a launch's latency
        dict(kind="quant", name="quant_expert", dtype="bf16", rows=1536, cols=2048, pad=0),
        # load time: all gate/up projections of a layer
        dict(kind="quant", name="quant_layer", dtype="bf16", rows=128 * 1536, cols=2048, pad=0),
        # the method's own operating point: batch 16 with ten kept experts
        dict(FFN, **QWEN3, name="ffn_b16", B=16, budget=10),
        # a ragged batch with raw softmax weights, gated shared experts, renormalised gates
        dict(FFN, name="ffn_b61_shared", d=2048, E=60, K=4, I=1408, B=61, budget=16, norm_topk=0, flags=1,
             n_shared=4, shared_gate=True),
        # the headline batch
        dict(FFN, **QWEN3, name="ffn_b256", B=256, budget=32, residual=True),
        # the largest batch with every expert kept
        dict(FFN, **QWEN3, name="ffn_b1024_all", B=1024, budget=128),
        # few, large experts
        dict(FFN, name="ffn_wide_b128", d=4096, E=8, K=2, I=14336, B=128, budget=4),
        # one sequence being served, the whole layer
        dict(LAYER, **QWEN3, name="layer_b1", B=1, budget=10, residual=True),
        # a few sequences
        dict(LAYER, name="layer_b5", d=2048, E=64, K=8, I=1024, B=5, budget=24),
        # the norms of one token between two blocks
        dict(NORM, name="norm_b1", rows=1, d=2048),
        # a decode batch with gates of its own per token, rows inside wider ones
        dict(NORM, name="norm_b255_token_gate", rows=255, d=4096, gate="token", pad=64),
        # a prompt's rows in fp32, odd length, no norm behind the block
        dict(NORM, name="norm_prompt_fp32", rows=8191, d=5001, dtype="f32", post=False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# bounds that keep a drawn case below the largest listed ones: weights of all experts, of the kept ones, and
# pairs times the expert's size
_ALL, _KEPT, _PAIRS = 1.4e9, 7.0e8, 3.8e10


def draw(rng):
    kind = rng.choice(["quant", "ffn", "ffn", "ffn", "ffn", "layer", "layer", "norm", "norm"])
    if kind == "quant":
        cols = 32 * _log_int(rng, 1, 448)
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), cols=cols,
                    rows=_log_int(rng, 1, max(2, int(1.5e8 / cols))), pad=rng.choice([0, 0, 8, 3]))
    if kind == "norm":
        d = _log_int(rng, 64, 16384)
        case = dict(NORM, d=d, rows=_log_int(rng, 1, max(2, int(4e7 / d))), dtype=rng.choice(["bf16", "bf16", "f32"]),
                    post=rng.random() < 0.6, gate=rng.choice(["none", "channel", "token"]), pre=rng.random() < 0.8,
                    pad=rng.choice([0, 0, 0, 16, 5]))
        # the norm in front of the first block has no block's output to add
        return case if rng.random() < 0.8 else dict(case, block=False, post=False, gate="none", pre=True)
    few = kind == "layer"
    E, d = _log_int(rng, 8, 256), 256 * _log_int(rng, 2, 16)
    K, B, budget = rng.randint(1, min(10, E)), _log_int(rng, 1, 16 if few else 1024), _log_int(rng, 1, E)
    ns = rng.choice([0, 0, 0, 1, 2, 4])
    I = 64 * _log_int(rng, 1, 224)
    most = min(_ALL / (3 * d * (E + ns)), _KEPT / (3 * d * (min(budget, E) + ns)), _PAIRS / (3 * d * B * (K + ns)))
    return dict(LAYER if few else FFN, d=d, E=E, K=K, B=B, budget=budget, I=max(64, min(I, int(most) // 64 * 64)),
                n_shared=ns, shared_gate=bool(ns) and rng.random() < 0.5, residual=rng.random() < 0.5,
                norm_topk=rng.randint(0, 1), flags=rng.choice([0, 0, 0, 1, 2]))


# ------------------------------------------------------------------ inputs --
def _normal(seed, stream, shape, std=1.0, dtype=torch.float32):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 64 + stream)
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype).mul_(std)


def _rand_rank(seed, stream, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 64 + stream)
    return torch.randperm(n, generator=g, device="cuda")


def _padded(t, pad):
    """The same rows inside rows that are `pad` elements longer."""
    if not pad:
        return t
    wide = torch.full((t.shape[0], t.shape[1] + pad), 7.0, dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _dt(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _hidden(seed, stream, B, d):
    z = _normal(seed, stream, (B, d))
    return (z / (z.square().mean(1, keepdim=True) + 1e-6).sqrt()).to(torch.bfloat16)


def _quantised(seed, stream, n, rows, cols):
    """n matrices of std 1/sqrt(cols) as codes [n, rows, cols / 2] and scales [n, rows, cols / 32]."""
    w = _normal(seed, stream, (n * rows, cols), cols ** -0.5, torch.bfloat16)
    codes, scales = quantize(w)
    return codes.view(n, rows, cols // 2), scales.view(n, rows, cols // 32)


def _router(case, seed):
    E = case["E"]
    p = (_rand_rank(seed, 2, E).double() + 1.0) ** -1.1
    return _normal(seed, 1, (E, case["d"]), 0.075), (p / p.sum()).log().float()


def _predictor(case, seed):
    E, d = case["E"], case["d"]
    return _normal(seed, 3, (E, d), 0.3), math.log(0.18 * d) + _normal(seed, 4, (E,), 0.25)


def _experts(case, seed, n, stream):
    d, I = case["d"], case["I"]
    return _quantised(seed, stream, n, 2 * I, d), _quantised(seed, stream + 1, n, d, I)


def _routing(case, logits):
    """What a schedule hands to the experts: the routes, and the most routed experts as the kept set."""
    E, K, bc = case["E"], case["K"], min(case["budget"], case["E"])
    ids = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :K]
    counts = torch.bincount(ids.flatten(), minlength=E)
    order = torch.sort(counts, descending=True, stable=True).indices[:bc]
    used = counts[order] > 0
    sel = torch.where(used, order, -1).int()
    slot = torch.full((E,), -1, dtype=torch.int32, device="cuda")
    slot[order[used]] = torch.arange(int(used.sum()), dtype=torch.int32, device="cuda")
    return ids.int().contiguous(), sel, used.sum().int().view(1), slot


def prepare(case, seed):
    st = dict(case=case)
    if case["kind"] == "quant":
        w = _normal(seed, 0, (case["rows"], case["cols"]), case["cols"] ** -0.5)
        w *= torch.exp(0.5 * _normal(seed, 1, (case["rows"], 1)))     # rows of different strength
        st["w"] = _padded(w.to(_dt(case)), case["pad"])
        return st
    if case["kind"] == "norm":
        n, d, dt, pad = case["rows"], case["d"], _dt(case), case["pad"]
        st["h"] = _padded(_normal(seed, 0, (n, d), 3.0).to(dt), pad)
        st["y"] = _padded(_normal(seed, 1, (n, d), 0.4).to(dt), pad) if case["block"] else None
        st["post"] = 1.0 + _normal(seed, 2, (d,), 0.1) if case["post"] else None
        gate = {"none": None, "channel": (d,), "token": (n, d)}[case["gate"]]
        st["gate"] = None if gate is None else torch.sigmoid(_normal(seed, 3, gate))
        st["pre"] = 1.0 + _normal(seed, 4, (d,), 0.1) if case["pre"] else None
        st["scale"], st["eps"] = 0.875, 1e-6
        blank = torch.zeros(n, d, dtype=dt, device="cuda")
        st["h_out"] = _padded(blank, pad) if case["block"] else None
        st["x_out"] = _padded(blank.clone(), pad) if case["pre"] else None
        return st
    B, d, E, ns = case["B"], case["d"], case["E"], case["n_shared"]
    st["x"] = _hidden(seed, 0, B, d)
    st["residual"] = _hidden(seed, 5, B, d) if case["residual"] else None
    st["wr"], st["br"] = _router(case, seed)
    w13, w2 = _experts(case, seed, E, 8)
    shared = None
    if ns:
        gate = _normal(seed, 6, (d,), d ** -0.5) if case["shared_gate"] else None
        shared = (*_experts(case, seed, ns, 12), gate)
    if case["kind"] == "ffn":
        st["logits"] = (st["x"].float() @ st["wr"].T + st["br"]).contiguous()
        st["ids"], st["sel"], st["n_sel"], st["slot"] = _routing(case, st["logits"])
        st["pa"] = st["pb"] = None
    else:
        st["pa"], st["pb"] = _predictor(case, seed)
    if own:
        # the experts in the layout the products read, laid out once as a serving program does at load time
        from paper_2609_36222_amd import binding as bd
        st["layer"] = bd.mx_layer_from_codes(st["wr"], st["br"], st["pa"], st["pb"], w13, w2, case["norm_topk"],
                                             shared=shared)
        st["desc"] = st["layer"].desc(case["K"])
        st["ws"] = torch.empty(bd.base_workspace_bytes(st["desc"], B, case["budget"]), dtype=torch.uint8,
                               device="cuda")
        st["y"] = torch.empty(B, d, dtype=torch.bfloat16, device="cuda")
    else:
        st.update(w13=w13, w2=w2, shared=shared)
    return st


# ------------------------------------------------------------- plain forms --
def quantize(w):
    """codes [rows, cols / 2] (low half byte: the even element) and E8M0 scales [rows, cols / 32]."""
    b = w.float().unflatten(1, (-1, 32))
    top = (b.abs().amax(2).view(torch.int32) >> 23)            # the largest magnitude's biased exponent
    byte = torch.where(top == 255, 255, (top - 2).clamp_min(0))
    inv = ((254 - byte).clamp_min(1) << 23).view(torch.float32)   # 2^(127 - byte)
    v = b.abs() * inv[..., None]
    code = (v > 0.25).to(torch.uint8)
    code += v >= 0.75
    code += v > 1.25
    code += v >= 1.75
    code += v > 2.5
    code += v >= 3.5
    code += v > 5.0
    code += torch.signbit(b).to(torch.uint8) << 3
    code = torch.where((byte == 255)[..., None], torch.zeros_like(code), code).flatten(1)
    return code[:, 0::2] | (code[:, 1::2] << 4), byte.to(torch.uint8)


def dequantize(codes, scales):
    """The values [..., cols] in 32 bits."""
    lut = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    lut = torch.cat([lut, -lut])
    both = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()
    s = scales.int()
    step = torch.where(s == 0, 1 << 22, s << 23).view(torch.float32)   # 2^(s - 127)
    step = torch.where(s == 255, math.nan, step)
    return (lut[both].unflatten(-1, (-1, 32)) * step[..., None]).flatten(-2)


def _pick(w, index):
    return dequantize(w[0][index], w[1][index])


def _gates(case, logits, kept):
    """The gate of every (token, expert) pair that is executed, 0 elsewhere: [B, E] in 64 bits."""
    K = case["K"]
    l = logits.double()
    top, order = torch.sort(l, dim=1, descending=True, stable=True)
    num = (top - top[:, :1]).exp()
    den = (num[:, :K] if case["norm_topk"] else num).sum(1, keepdim=True)
    cand = kept[order]
    if case["flags"] & 2:
        cand = cand & (torch.arange(case["E"], device=l.device) < K)
    take = cand & (cand.cumsum(1) <= K)
    g = num * take
    if case["flags"] & 1:
        den = g.sum(1, keepdim=True)
    g = torch.where(take, g / den, torch.zeros_like(g))
    return torch.zeros_like(l).scatter_(1, order, g)


def _ffn(x, w13, w2, gate):
    """sum over experts of gate [n, B] times expert, in 32 bits: w13 [n, 2I, d], w2 [n, d, I]."""
    n, I = w13.shape[0], w2.shape[2]
    a = (w13.flatten(0, 1) @ x.T).view(n, 2 * I, -1)
    g, u = a[:, :I], a[:, I:]
    h = g / (1.0 + torch.exp(-g)) * u * gate[:, None]
    return torch.bmm(w2, h).sum(0).T


def _experts_plain(st, logits, sel, kept):
    case, x = st["case"], st["x"].float()
    used = sel.clamp_min(0).long()
    gate = torch.where(sel[:, None] >= 0, _gates(case, logits, kept).T[used], 0.0).float()
    y = _ffn(x, _pick(st["w13"], used), _pick(st["w2"], used), gate)
    if st["shared"] is not None:
        w13, w2, sg = st["shared"]
        one = torch.ones(x.shape[0], device=x.device) if sg is None else torch.sigmoid(x @ sg)
        y = y + _ffn(x, dequantize(*w13), dequantize(*w2), one.expand(case["n_shared"], -1))
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return y.to(torch.bfloat16)


def _layer_plain(st):
    case, K, E = st["case"], st["case"]["K"], st["case"]["E"]
    x = st["x"].double()
    l = x @ st["wr"].double().T + st["br"].double()
    top, order = torch.sort(l, dim=1, descending=True, stable=True)
    num, ids = (top - top[:, :1]).exp(), order[:, :K]
    w = num[:, :K] / (num[:, :K] if case["norm_topk"] else num).sum(1, keepdim=True)
    s = ((x / x.norm(dim=1, keepdim=True)) @ st["pa"].double().T + st["pb"].double()).gather(1, ids)
    cost = w * w * s.exp()
    score = torch.full((E,), -1.0, dtype=torch.float64, device=x.device)
    routed = torch.zeros(E, dtype=torch.float64, device=x.device).index_add_(0, ids.flatten(),
                                                                           torch.ones_like(cost).flatten()) > 0
    total = torch.zeros_like(score).index_add_(0, ids.flatten(), cost.flatten())
    order = torch.sort(torch.where(routed, total, score), descending=True, stable=True).indices
    sel = order[:min(case["budget"], E)]
    sel = torch.where(routed[sel], sel, -1)
    kept = torch.zeros(E + 1, dtype=torch.bool, device=x.device)
    kept[sel] = True                      # -1 marks the last entry, which is dropped
    return _experts_plain(st, l, sel, kept[:E])


def _rms(v, eps):
    return v / (v.square().mean(1, keepdim=True) + eps).sqrt()


def _norm_plain(st):
    h = st["h"].float()
    if st["y"] is not None:
        y = st["y"].float()
        if st["post"] is not None:
            y = _rms(y, st["eps"]) * st["post"]
        if st["gate"] is not None:
            y = y * st["gate"]
        h = st["scale"] * h + y
    out = dict(h=h.to(st["h"].dtype)) if st["y"] is not None else {}
    if st["pre"] is not None:
        out["x"] = (_rms(h, st["eps"]) * st["pre"]).to(st["h"].dtype)
    return out


def run(st):
    case = st["case"]
    if own:
        from paper_2609_36222_amd import binding as bd
    if case["kind"] == "quant":
        if own:
            codes, scales = bd.mx_quantize(st["w"])
            return dict(values=bd.mx_dequantize(codes, scales, st["w"].dtype))
        return dict(values=dequantize(*quantize(st["w"])).to(st["w"].dtype))
    if case["kind"] == "norm":
        if not own:
            return _norm_plain(st)
        bd.norm_residual(st["h"], st["y"], post_gain=st["post"], gate=st["gate"], pre_gain=st["pre"],
                         res_scale=st["scale"], eps=st["eps"], h_out=st["h_out"], x_out=st["x_out"])
        return {k: v for k, v in (("h", st["h_out"]), ("x", st["x_out"])) if v is not None}
    if case["kind"] == "layer":
        if not own:
            return dict(y=_layer_plain(st))
        bd.base_decode_layer(st["desc"], st["x"], case["B"], case["budget"], case["flags"], st["residual"],
                             st["y"], st["ws"])
        return dict(y=st["y"])
    if not own:
        return dict(y=_experts_plain(st, st["logits"], st["sel"], st["slot"] >= 0))
    bd.base_moe_forward(st["desc"], st["x"], case["B"], st["logits"], st["ids"], st["sel"], st["n_sel"], st["slot"],
                        case["budget"], case["flags"], st["residual"], st["y"], st["ws"])
    return dict(y=st["y"])


def work(case):
    if case["kind"] == "quant":
        n, size = case["rows"] * case["cols"], 4 if case["dtype"] == "f32" else 2
        return {"bytes": n * (2 * size + 2 * 17 / 32), "flops": 0}
    if case["kind"] == "norm":
        n, size = case["rows"] * case["d"], 4 if case["dtype"] == "f32" else 2
        moved = size * (1 + (2 if case["block"] else 0) + (1 if case["pre"] else 0))
        return {"bytes": n * (moved + (4 if case["gate"] == "token" else 0)), "flops": 0}
    d, I, E, K, B, ns = (case[k] for k in ("d", "I", "E", "K", "B", "n_shared"))
    kept = min(case["budget"], E, B * K)
    each = min(K, kept) if not case["flags"] & 2 else min(K, max(1, K * kept // E))
    rows = B * d * 2 * (3 if case["residual"] else 2)
    scores = 2 * E * d * 4 if case["kind"] == "layer" else B * E * 4
    return {"bytes": (kept + ns) * 3 * d * I * 17 / 32 + rows + scores,
            "flops": 2 * B * (each + ns) * 3 * d * I}


# ----------------------------------------------------- the same in 64 bits --
_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _values64(codes, scales):
    mag = torch.tensor(_E2M1, dtype=torch.float64, device=codes.device)
    out = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.float64, device=codes.device)
    for odd in (0, 1):
        c = (codes >> (4 * odd)).long() & 15
        out[..., odd::2] = mag[c & 7] * torch.where(c >= 8, -1.0, 1.0).double()
    return out * torch.pow(2.0, scales.double() - 127.0).repeat_interleave(32, -1)


def _expert64(x, w13, w2, u):
    a = x @ _values64(w13[0][u], w13[1][u]).T
    I = a.shape[1] // 2
    return (torch.nn.functional.silu(a[:, :I]) * a[:, I:]) @ _values64(w2[0][u], w2[1][u]).T


def _quant64(w):
    v = w.double().unflatten(1, (-1, 32))
    most = v.abs().amax(2, keepdim=True)
    _, e = torch.frexp(most)                        # most = m 2^e, m in [0.5, 1)
    step = torch.pow(2.0, torch.where(most > 0, e.double() - 3.0, -127.0).clamp_min(-127.0))
    grid = torch.tensor(_E2M1, dtype=torch.float64, device=w.device)
    mid = (grid[1:] + grid[:-1]) / 2
    t = (v.abs() / step).contiguous()
    lo, hi = torch.searchsorted(mid, t, right=False), torch.searchsorted(mid, t, right=True)
    near = torch.where(lo % 2 == 0, lo, hi)          # between two codes: the even one
    return (grid[near] * step * torch.sign(v)).flatten(1)


def _norm64(case, seed):
    st = prepare(case, seed)
    h = st["h"].double()
    unit = lambda v: v * torch.rsqrt(v.pow(2).sum(1, keepdim=True) / case["d"] + st["eps"])  # noqa: E731
    out = {}
    if st["y"] is not None:
        y = st["y"].double()
        y = unit(y) * st["post"].double() if case["post"] else y
        h = st["scale"] * h + (y * st["gate"].double() if case["gate"] != "none" else y)
        out["h"] = h
    if case["pre"]:
        out["x"] = unit(h) * st["pre"].double()
    return out


def exact(case, seed):
    if case["kind"] == "quant":
        return dict(values=_quant64(prepare(case, seed)["w"])) if case["rows"] * case["cols"] < 4e7 else None
    if case["kind"] == "norm":
        return _norm64(case, seed)
    B, d, E, K, ns = (case[k] for k in ("B", "d", "E", "K", "n_shared"))
    x = _hidden(seed, 0, B, d).double()
    wr, br = _router(case, seed)
    if case["kind"] == "ffn":
        l32 = (x.float() @ wr.T + br).contiguous()
        l = l32.double()
        kept = _routing(case, l32)[3] >= 0
    else:
        l = x @ wr.double().T + br.double()
    order = torch.argsort(l, dim=1, descending=True, stable=True)
    p = torch.exp(l - l.gather(1, order[:, :1]))
    routed = torch.zeros(B, E, dtype=torch.bool, device="cuda").scatter_(1, order[:, :K], True)
    den = (p * routed if case["norm_topk"] else p).sum(1)
    if case["kind"] == "layer":
        pa, pb = _predictor(case, seed)
        s = torch.nn.functional.normalize(x, dim=1) @ pa.double().T + pb.double()
        cost = ((p / den[:, None]).square() * s.exp() * routed).sum(0)
        key = torch.where(routed.any(0), cost, -1.0)
        best = torch.argsort(key, descending=True, stable=True)[:min(case["budget"], E)]
        kept = torch.zeros(E, dtype=torch.bool, device="cuda")
        kept[best[key[best] >= 0]] = True
    ran = torch.zeros_like(routed)
    for t in range(B):
        mine = order[t][kept[order[t]]] if not case["flags"] & 2 else order[t, :K][kept[order[t, :K]]]
        ran[t, mine[:K]] = True
    g = p * ran
    g = g / (g.sum(1) if case["flags"] & 1 else den)[:, None].clamp_min(1e-300)
    y = _hidden(seed, 5, B, d).double() if case["residual"] else torch.zeros_like(x)
    w13, w2 = _experts(case, seed, E, 8)
    for u in kept.nonzero().flatten().tolist():
        t = ran[:, u].nonzero().flatten()
        if len(t):
            y[t] += g[t, u, None] * _expert64(x[t], w13, w2, u)
    if ns:
        w13, w2 = _experts(case, seed, ns, 12)
        sg = torch.sigmoid(x @ _normal(seed, 6, (d,), d ** -0.5).double()) if case["shared_gate"] else torch.ones(B).cuda()
        for u in range(ns):
            y += sg[:, None] * _expert64(x, w13, w2, u)
    return dict(y=y)

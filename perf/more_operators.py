"""The attention half of a decode step, measured on one MI355X: what stands between the norm in front of a block
and the experts.

Three calls.  The norms of query and key heads with the rotation by position (`base_head_rope`); the same on the
way into a paged cache, the values beside them (`base_kv_append`); and the attention of each sequence's new tokens,
one or a chunk, over that cache (`base_paged_attention`).  A "step" is the last two as a serving program makes them.

With `own` false every operator is computed from elementary torch operations instead, in 32 bits (angles in 64).
Head counts and lengths are generic; hidden sizes do not enter.
"""
import math
import random

import torch

own = False

ROPE = dict(kind="rope", dtype="bf16", D=128, rot=128, interleaved=False, norm=True, factor=1.0, far=40000)
# S sequences with up to q new tokens each and up to kv tokens behind and with them; lens: "even" (all the
# largest), "ragged", "mixed" (one chunk among single tokens).  heads_first: a page holds its tokens head by head
PAGED = dict(dtype="bf16", Hq=32, Hk=4, D=128, ps=16, lens="even", heads_first=True)
APPEND = dict(PAGED, kind="append", rot=128, interleaved=False, norm=True, factor=1.0)
ATTN = dict(PAGED, kind="attn", window=0, lse=False)
STEP = dict(APPEND, kind="step", window=0)


def listed():
    return [
        # one token's heads: a launch's latency
        dict(ROPE, name="rope_b1", rows=1, Hq=32, Hk=4),
        # a prompt in fp32, half of each head rotated, positions of a scaled long context
        dict(ROPE, name="rope_prompt_fp32", dtype="f32", rows=8191, Hq=16, Hk=16, rot=64, interleaved=True,
             norm=False, factor=8.0, far=1000000),
        # a decode batch's new tokens into the cache
        dict(APPEND, name="append_b64", S=64, q=1, kv=4096, lens="ragged"),
        # prompts of several sequences
        dict(APPEND, name="append_prompts", S=5, q=2301, kv=6000, lens="ragged", Hq=64, Hk=8, ps=64),
        # one sequence, a short context: latency
        dict(ATTN, name="attn_b1", S=1, q=1, kv=517),
        # one sequence, a long context
        dict(ATTN, name="attn_b1_long", S=1, q=1, kv=131071, ps=64),
        # a decode batch of sequences of all lengths
        dict(ATTN, name="attn_b64_ragged", S=64, q=1, kv=8192, lens="ragged"),
        # a large batch, every query head with keys of its own, pages token by token
        dict(ATTN, name="attn_b256_mha", S=256, q=1, kv=1000, Hq=16, Hk=16, heads_first=False, lse=True),
        # a chunk of a prompt behind its first part
        dict(ATTN, name="attn_chunk", S=1, q=2048, kv=8191, ps=64),
        # a chunk joins a decode batch, all with a window
        dict(ATTN, name="attn_mixed_window", S=17, q=509, kv=3001, Hq=24, Hk=8, lens="mixed", window=1024),
        # fp32 heads of a small experiment
        dict(ATTN, name="attn_fp32", dtype="f32", S=3, q=61, kv=777, Hq=8, Hk=2, D=64, lens="ragged", lse=True),
        # a step of drafted tokens, four a sequence: cache and attention
        dict(STEP, name="step_b32_q4", S=32, q=4, kv=2050, Hq=32, Hk=8, D=64, rot=64),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# bounds that keep a drawn case below the largest listed ones: elements of the heads, of the cache's read part (also
# padded to the longest sequence), and of the scores
_HEADS, _CACHE, _SCORES = 3.0e7, 4.0e8, 4.0e8


def draw(rng):
    kind = rng.choice(["rope", "append", "append", "attn", "attn", "attn", "attn", "attn", "step"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    D = rng.choice([64, 128, 128, 128, 256, 96, 80, 8 * rng.randint(1, 32)])
    Hk, G = _log_int(rng, 1, 16), rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 8, 12, 16])
    rot = D if rng.random() < 0.6 else 2 * rng.randint(1, D // 2)
    angle = dict(rot=rot, interleaved=rng.random() < 0.4, norm=rng.random() < 0.6, factor=rng.choice([1.0, 1.0, 4.0]))
    if kind == "rope":
        return dict(kind=kind, dtype=dtype, D=D, **angle, far=_log_int(rng, 1, 2000000), Hq=Hk * G, Hk=Hk,
                    rows=_log_int(rng, 1, max(2, int(_HEADS / (D * Hk * (G + 1))))))
    case = dict(kind=kind, dtype=dtype, Hq=Hk * G, Hk=Hk, D=D, ps=rng.choice([16, 16, 32, 64, 256]),
                lens=rng.choice(["even", "ragged", "ragged", "mixed"]), heads_first=rng.random() < 0.6)
    S = _log_int(rng, 1, 256)
    few = rng.random() < (0.0 if kind == "append" else 0.6)
    q = rng.randint(1, 5) if few else _log_int(rng, 1, 4096)
    most = _CACHE / (S * Hk * D * (2 if dtype == "f32" else 1))
    if kind != "append":
        most = min(most, _SCORES / (S * Hk * G * min(q, 64)))
        if dtype == "f32":
            most = min(most, 4.0e7 / (Hk * G * min(q, 64)))
    most = max(2, min(131072, int(most)))
    kv = _log_int(rng, 1 if rng.random() < 0.15 else min(100, most), most)
    q = min(q, kv)
    if kind != "append":
        q = max(1, min(q, int(min(_SCORES if dtype == "bf16" else 1.0e8, 6.0e10 / D) / (S * Hk * G * kv))))
    q = max(1, min(q, int(_HEADS / (S * D * Hk * (G + 2)))))
    case.update(S=S, q=q, kv=kv)
    if kind != "append":
        case["window"] = rng.choice([0, 0, 0, _log_int(rng, 1, 4096)])
    if kind == "attn":
        return dict(case, lse=rng.random() < 0.3)
    return dict(case, **angle)


def _lens(case):
    """(new tokens, all tokens) of each sequence."""
    S, q, kv = case["S"], case["q"], case["kv"]
    if case["lens"] == "even":
        return [(q, kv)] * S
    rng, got = random.Random(S * 1000003 + q * 10007 + kv), [(q, kv)]
    for _ in range(S - 1):
        n = _log_int(rng, max(1, kv // 64), kv)
        new = 1 if case["lens"] == "mixed" else rng.randint(1, q)
        # now and then a place of the batch that no sequence has
        got.append((0, 0) if rng.random() < 0.04 else (min(new, n), n))
    return got


# ------------------------------------------------------------------ inputs --
def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 64 + stream)
    return g


def _normal(seed, stream, shape, std=1.0, dtype=torch.float32):
    return torch.randn(shape, generator=_gen(seed, stream), device="cuda", dtype=dtype).mul_(std)


def _dt(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _ints(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def _frequencies(case):
    """The angle of each pair per position (a context `factor` times the trained one: positions closer together)
    and the factor of cosine and sine."""
    i = torch.arange(case["rot"] // 2, dtype=torch.float64)
    inv = 10000.0 ** (-2.0 * i / case["rot"]) / case["factor"]
    return inv.float().cuda(), 1.0 if case["factor"] == 1.0 else 0.1 * math.log(case["factor"]) + 1.0


def _gains(case, seed):
    if not case["norm"]:
        return None, None
    return tuple(1.0 + _normal(seed, s, (case["D"],), 0.1) for s in (20, 21))


def _heads(case, seed, rows):
    """q, k and v as a projection leaves them: parts of one row."""
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    std = 3.0 if case.get("norm") else 1.0
    qkv = _normal(seed, 0, (rows, Hq + 2 * Hk, D), std, _dt(case))
    return qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]


def _cache(case, seed, lens):
    """k and v [pages, ps, Hk, D] with every page filled, and each sequence's pages in an order of chance."""
    S, ps, Hk, D = case["S"], case["ps"], case["Hk"], case["D"]
    need = [-(-kv // ps) for _, kv in lens]
    pages = sum(need) + 3
    shape = (pages, Hk, ps, D) if case["heads_first"] else (pages, ps, Hk, D)
    k, v = (_normal(seed, s, shape, 1.0, _dt(case)) for s in (1, 2))
    if case["heads_first"]:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    order = torch.randperm(pages, generator=_gen(seed, 3), device="cuda").int().cpu()
    table = torch.full((S, max(need)), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return k, v, table.cuda()


def prepare(case, seed):
    st = dict(case=case)
    if case["kind"] == "rope":
        rows, dt = case["rows"], _dt(case)
        st["q"], st["k"], _ = _heads(case, seed, rows)
        st["positions"] = torch.randint(0, case["far"], (rows,), generator=_gen(seed, 4), device="cuda").int()
        st["inv"], st["rot_scale"] = _frequencies(case)
        st["gains"] = _gains(case, seed)
        st["q_out"], st["k_out"] = (torch.empty(rows, case[h], case["D"], dtype=dt, device="cuda") for h in ("Hq", "Hk"))
    else:
        lens = _lens(case)
        rows = sum(n for n, _ in lens)
        starts = [0]
        for n, _ in lens:
            starts.append(starts[-1] + n)
        st["rows"], st["starts"], st["kv_len"] = rows, _ints(starts), _ints([kv for _, kv in lens])
        st["kc"], st["vc"], st["table"] = _cache(case, seed, lens)
        if case["kind"] == "attn":
            st["q"] = _normal(seed, 0, (rows, case["Hq"], case["D"]), 1.5, _dt(case))
        else:
            st["q"], st["k"], st["v"] = _heads(case, seed, rows)
            st["inv"], st["rot_scale"] = _frequencies(case)
            st["gains"] = _gains(case, seed)
            st["q_out"] = torch.empty(rows, case["Hq"], case["D"], dtype=_dt(case), device="cuda")
        if case["kind"] != "append":
            st["out"] = torch.empty(rows, case["Hq"], case["D"], dtype=_dt(case), device="cuda")
            st["lse"] = torch.empty(rows, case["Hq"], device="cuda") if case.get("lse") else None
    if own:
        # descriptors and the workspace, as a serving program keeps them
        from paper_2609_36222_amd import binding as bd
        if case["kind"] != "attn":
            st["rope"] = bd.Rope(case["D"], _dt(case), st["inv"], case["interleaved"], st["rot_scale"], *st["gains"],
                                 eps=1e-6)
        if case["kind"] != "rope":
            st["cache"] = bd.KVCache(st["kc"], st["vc"])
            st["batch"] = bd.KVBatch(st["table"], st["starts"], st["kv_len"], case["q"])
        if case["kind"] in ("attn", "step"):
            n = bd.attention_workspace_bytes(st["cache"], st["batch"], rows, case["Hq"])
            st["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------- plain forms --
def _rows_of(st):
    """Each row's sequence and position."""
    rows = torch.arange(st["rows"], device="cuda")
    starts = st["starts"].long()
    seq = torch.searchsorted(starts, rows, right=True) - 1
    return seq, st["kv_len"].long()[seq] - starts[seq + 1] + rows


def _rotate(case, x, gain, cos, sin):
    """x [rows, H, D] in 32 bits, normalised and rotated; cos and sin [rows, 1, rot / 2]."""
    x = x.float()
    if gain is not None:
        x = x / (x.square().mean(2, keepdim=True) + 1e-6).sqrt() * gain
    rot = case["rot"]
    t = x[..., :rot]
    a, b = (t[..., 0::2], t[..., 1::2]) if case["interleaved"] else (t[..., :rot // 2], t[..., rot // 2:])
    a, b = a * cos - b * sin, a * sin + b * cos
    t = torch.stack([a, b], -1).flatten(2) if case["interleaved"] else torch.cat([a, b], 2)
    return torch.cat([t, x[..., rot:]], 2)


def _heads_plain(st, positions):
    case = st["case"]
    angle = positions.double()[:, None] * st["inv"].double()
    cos, sin = ((f(angle) * st["rot_scale"]).float()[:, None] for f in (torch.cos, torch.sin))
    return (_rotate(case, st["q"], st["gains"][0], cos, sin).to(_dt(case)),
            _rotate(case, st["k"], st["gains"][1], cos, sin).to(_dt(case)))


def _append_plain(st):
    case, (seq, at) = st["case"], _rows_of(st)
    q, k = _heads_plain(st, at)
    page = st["table"].long()[seq, at // case["ps"]]
    st["kc"][page, at % case["ps"]] = k
    st["vc"][page, at % case["ps"]] = st["v"]
    return q


def _attention_plain(st, q):
    case = st["case"]
    S, Q, Hq, Hk, D = (case[k] for k in ("S", "q", "Hq", "Hk", "D"))
    seq, at = _rows_of(st)
    table = st["table"].long().clamp_min(0)
    k, v = (c[table].flatten(1, 2).float().permute(0, 2, 1, 3) for c in (st["kc"], st["vc"]))   # [S, Hk, keys, D]
    within = torch.arange(st["rows"], device="cuda") - st["starts"].long()[seq]
    padded = torch.zeros(S, Q, Hq, D, device="cuda")
    padded[seq, within] = q.float()
    where = torch.full((S, Q), -1, device="cuda", dtype=torch.long)
    where[seq, within] = at
    padded = padded.view(S, Q, Hk, Hq // Hk, D).permute(0, 2, 3, 1, 4).flatten(2, 3)              # [S, Hk, heads x Q, D]
    s = padded @ k.transpose(2, 3) * D ** -0.5
    key = torch.arange(k.shape[2], device="cuda")
    seen = key <= where[..., None]
    if case["window"]:
        seen &= key > where[..., None] - case["window"]
    seen = seen[:, None, None].expand(S, Hk, Hq // Hk, Q, -1).flatten(2, 3)
    s = torch.where(seen, s, -math.inf)
    top = s.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(s - top)
    total = p.sum(3, keepdim=True)
    o = p @ v / torch.where(total == 0, 1.0, total)
    lse = torch.log(total) + top
    both = [t.view(S, Hk, Hq // Hk, Q, -1).permute(0, 3, 1, 2, 4).flatten(2, 3)[seq, within] for t in (o, lse)]
    return both[0].to(_dt(case)), both[1][..., 0]


def run(st):
    case = st["case"]
    if own:
        from paper_2609_36222_amd import binding as bd
    if case["kind"] == "rope":
        if not own:
            q, k = _heads_plain(st, st["positions"])
            return dict(q=q, k=k)
        bd.base_head_rope(st["rope"], st["positions"], st["q"], st["k"], st["q_out"], st["k_out"])
        return dict(q=st["q_out"], k=st["k_out"])
    if case["kind"] != "attn":
        if own:
            bd.base_kv_append(st["rope"], st["cache"], st["batch"], st["q"], st["k"], st["v"], st["q_out"])
            q = st["q_out"]
        else:
            q = _append_plain(st)
        if case["kind"] == "append":
            return dict(q=q, k=st["kc"], v=st["vc"])
    else:
        q = st["q"]
    if own:
        bd.base_paged_attention(st["cache"], st["batch"], q, st["out"], st["ws"], window=case["window"], lse=st["lse"])
        out, lse = st["out"], st["lse"]
    else:
        out, lse = _attention_plain(st, q)
    if case["kind"] == "step":
        return dict(out=out, k=st["kc"], v=st["vc"])
    return dict(out=out, lse=lse) if case["lse"] else dict(out=out)


def work(case):
    size, Hq, Hk, D = 4 if case["dtype"] == "f32" else 2, case["Hq"], case["Hk"], case["D"]
    if case["kind"] == "rope":
        return {"bytes": case["rows"] * (2 * (Hq + Hk) * D * size + 4), "flops": 0}
    keys = pairs = rows = 0
    for n, kv in _lens(case):
        rows += n
        lowest = max(0, kv - n + 1 - case["window"]) if case.get("window") else 0
        keys += kv - lowest if n else 0
        for r in range(kv - n, kv):
            pairs += min(r + 1, case["window"]) if case.get("window") else r + 1
    cached = rows * 2 * Hk * D * size
    if case["kind"] == "append":
        return {"bytes": 2 * (rows * Hq * D * size + cached), "flops": 0}
    read = keys * 2 * Hk * D * size + 2 * rows * Hq * D * size + (rows * Hq * 4 if case.get("lse") else 0)
    if case["kind"] == "step":
        read += cached
    return {"bytes": read, "flops": 4 * pairs * Hq * D}


# ----------------------------------------------------- the same in 64 bits --
def _turn64(x, gain, position, inv, scale, interleaved):
    """One [rows, H, D] in 64 bits, pair by pair as complex numbers."""
    x = x.double()
    if gain is not None:
        x = x * torch.rsqrt(x.pow(2).sum(2, keepdim=True) / x.shape[2] + 1e-6) * gain.double()
    n = inv.numel()
    w = torch.polar(torch.full((len(position), n), scale, dtype=torch.float64, device="cuda"),
                    torch.outer(position.double(), inv.double()))[:, None]
    out = x.clone()
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * w
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _attend64(q, k, v, position, window):
    """q [n, Hq, D] at the positions given over k, v [kv, Hk, D]: the output and the log of the sum."""
    n, Hq, D = q.shape
    G = Hq // k.shape[1]
    j = torch.arange(k.shape[0], device="cuda")
    hidden = j[None] > position[:, None]
    if window:
        hidden = hidden | (j[None] <= position[:, None] - window)
    out, lse = torch.empty_like(q), torch.empty(n, Hq, dtype=torch.float64, device="cuda")
    for h in range(Hq):
        s = (q[:, h] @ k[:, h // G].T / math.sqrt(D)).masked_fill(hidden, -math.inf)
        out[:, h], lse[:, h] = torch.softmax(s, 1) @ v[:, h // G], torch.logsumexp(s, 1)
    return out, lse


def exact(case, seed):
    if work(case)["flops"] > 1.5e12:
        return None
    st = prepare(case, seed)
    if case["kind"] == "rope":
        turn = (st["positions"], st["inv"], st["rot_scale"], case["interleaved"])
        return dict(q=_turn64(st["q"], st["gains"][0], *turn), k=_turn64(st["k"], st["gains"][1], *turn))
    kc, vc = st["kc"].double(), st["vc"].double()
    if case["kind"] == "attn":
        q = st["q"].double()
    else:
        position = torch.cat([torch.arange(kv - n, kv) for n, kv in _lens(case)]).cuda()
        turn = (position, st["inv"], st["rot_scale"], case["interleaved"])
        q, k = _turn64(st["q"], st["gains"][0], *turn), _turn64(st["k"], st["gains"][1], *turn)
    table, ps = st["table"].long(), case["ps"]
    out, lse = torch.zeros_like(q), torch.zeros(len(q), case["Hq"], dtype=torch.float64, device="cuda")
    at = 0
    for s, (n, kv) in enumerate(_lens(case)):
        if not n:
            continue
        slot = torch.arange(kv, device="cuda")
        page, slot = table[s, slot // ps], slot % ps
        if case["kind"] != "attn":
            kc[page[kv - n:], slot[kv - n:]] = k[at:at + n]
            vc[page[kv - n:], slot[kv - n:]] = st["v"][at:at + n].double()
        if case["kind"] != "append":
            # the cache and the queries are held in the inputs' type between the two calls
            near = (lambda t: t.to(_dt(case)).double()) if case["kind"] == "step" else (lambda t: t)
            out[at:at + n], lse[at:at + n] = _attend64(near(q[at:at + n]), near(kc[page, slot]), vc[page, slot],
                                                       torch.arange(kv - n, kv, device="cuda"), case["window"])
        at += n
    if case["kind"] == "append":
        return dict(q=q, k=kc, v=vc)
    if case["kind"] == "step":
        return dict(out=out, k=kc, v=vc)
    return dict(out=out, lse=lse) if case["lse"] else dict(out=out)

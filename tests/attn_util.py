"""Batches, caches and 64-bit references for the tests of the rotation, the paged cache and
its attention (NumPy and torch on the CPU)."""
import numpy as np
import torch

BF, F32 = torch.bfloat16, torch.float32


def frequencies(rot, base=10000.0):
    return (base ** (-2.0 * np.arange(rot // 2) / max(rot, 1))).astype(np.float32)


def rotate(x, gain, pos, inv, scale, interleaved, eps):
    """(value, bound of the fp32 error) of x [rows, H, D] in 64 bits.

    The bound: a sum of D squares in chains of 16 and a tree, the mean and the root are
    off by less than 32 2^-24 of the norm, and the two products by 2 2^-24; a turn's
    fraction is rounded to 2^-25 and its sine and cosine, with the angle's 2 pi, the
    series and rot_scale, are off by less than 8 2^-24; the two products and their sum
    by 2 2^-24 of their sizes.  So 64 2^-24 of |a| + |b| covers an element."""
    x = x.astype(np.float64)
    u = 64 * 2.0 ** -24
    if gain is not None:
        m = np.mean(x * x, 2, keepdims=True) + eps
        with np.errstate(divide="ignore"):
            x = x * np.where(m > 0, 1 / np.sqrt(np.where(m > 0, m, 1)), 0) * gain.astype(np.float64)
    n = len(inv)
    w = pos.astype(np.float64)[:, None] * inv.astype(np.float64)
    c, s = (scale * f(w)[:, None] for f in (np.cos, np.sin))
    i, j = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if interleaved else (np.arange(n), np.arange(n, 2 * n))
    y, b = x.copy(), u * np.abs(x)
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., i] * s + x[..., j] * c
    b[..., i] = b[..., j] = u * abs(scale) * (np.abs(x[..., i]) + np.abs(x[..., j]))
    return y, b


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def near(got, want, bound, dtype, what=""):
    """Within `bound` before the rounding to dtype, and half a step of it."""
    got = got.double().cpu().numpy()
    h = half_step(dtype)
    most = bound + h * (np.abs(want) + bound) + 1e-38
    bad = ~(np.abs(got - want) <= most)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], most[bad][:3])


class Batch:
    """Sequences [(new tokens, all tokens)] with their pages in a cache filled with `fill`."""

    def __init__(self, lens, Hk, D, ps, dtype, seed=0, heads_first=True, fill=float("nan"), extra=2, unused=-1):
        g = np.random.default_rng(seed)
        self.lens, self.Hk, self.D, self.ps, self.dtype = lens, Hk, D, ps, dtype
        need = [-(-kv // ps) for _, kv in lens]
        self.width = max(max(need), 1) + extra
        n = sum(need) + 3
        order = g.permutation(n)
        self.table = np.full((len(lens), self.width), unused, np.int32)
        at = 0
        for s, k in enumerate(need):
            self.table[s, :k] = order[at:at + k]
            at += k
        self.n_pages = n
        shape = (n, Hk, ps, D) if heads_first else (n, ps, Hk, D)
        self.kc, self.vc = (torch.full(shape, fill, dtype=dtype) for _ in range(2))
        if heads_first:
            self.kc, self.vc = self.kc.transpose(1, 2), self.vc.transpose(1, 2)
        self.k = [torch.from_numpy(g.standard_normal((kv, Hk, D), np.float32)).to(dtype) for _, kv in lens]
        self.v = [torch.from_numpy(g.standard_normal((kv, Hk, D), np.float32)).to(dtype) for _, kv in lens]
        self.starts = np.concatenate([[0], np.cumsum([q for q, _ in lens])]).astype(np.int32)
        self.rows = int(self.starts[-1])
        self.g = g

    def slots(self, s, lo, hi):
        j = np.arange(lo, hi)
        return torch.from_numpy(self.table[s, j // self.ps].astype(np.int64)), torch.from_numpy(j % self.ps)

    def fill(self, first=0):
        """Every sequence's tokens from `first` on (an int, or one a sequence) into the cache."""
        for s, (_, kv) in enumerate(self.lens):
            lo = first if isinstance(first, int) else first[s]
            if lo < kv:
                page, slot = self.slots(s, lo, kv)
                self.kc[page, slot], self.vc[page, slot] = self.k[s][lo:], self.v[s][lo:]

    def queries(self, Hq, std=1.5):
        q = self.g.standard_normal((self.rows, Hq, self.D), np.float32) * std
        return torch.from_numpy(q).to(self.dtype)

    def device(self, bd, max_q=None):
        put = lambda t: torch.from_numpy(t).cuda()  # noqa: E731
        kc, vc = (t.cuda() for t in (self.kc, self.vc))
        most = max([q for q, _ in self.lens] + [1])
        return (bd.KVCache(kc, vc), bd.KVBatch(put(self.table), put(self.starts),
                                               put(np.array([kv for _, kv in self.lens], np.int32)),
                                               most if max_q is None else max_q))


def attend(b, q, scale, window=0):
    """(out, bound, lse, its bound) in 64 bits.

    The bound.  A product of D elements is summed in fp32 in some order: off by less than
    D 2^-24 sum |q||k|, and scaled by 2 2^-24 of itself more; so an exponential is off by
    e = that plus 2^-21 (the exponent's difference and the function) relative to itself.
    In 16 bits it is rounded to bf16 (2^-8) for the sum with v, not for the sum of its own.
    Sums of L terms, their joins and rescalings add (L + 64) 2^-24.  With A = sum p |v| /
    sum p: out is off by (e + 2^-8 + (L + 64) 2^-24) A + (e + (L + 64) 2^-24) |out|, lse by
    e + (L + 64) 2^-24 + 2 2^-23 |lse|."""
    rows, Hq, D = q.shape
    out, bound = np.zeros((rows, Hq, D)), np.zeros((rows, Hq, D))
    lse, lb = np.full((rows, Hq), -np.inf), np.zeros((rows, Hq))
    G = Hq // b.Hk
    u = 2.0 ** -24
    p_round = 2.0 ** -8 if b.dtype is BF else 0.0
    for s, (n, kv) in enumerate(b.lens):
        t0 = b.starts[s]
        for h in range(Hq):
            k, v = (t[s][:, h // G].double().numpy() for t in (b.k, b.v))
            qq = q[t0:t0 + n, h].double().numpy()
            pos = kv - n + np.arange(n)
            j = np.arange(kv)
            seen = j[None] <= pos[:, None]
            if window:
                seen &= j[None] > pos[:, None] - window
            x = scale * (qq @ k.T)
            size = abs(scale) * (np.abs(qq) @ np.abs(k).T)
            e = (np.where(seen, (D + 4) * u * size, 0).max(1) if kv else np.zeros(n)) + 2.0 ** -21
            some = seen.any(1)
            if not some.any():
                continue
            m = np.where(seen, x, -np.inf).max(1, where=seen, initial=-1e300)
            p = np.where(seen, np.exp(np.where(seen, x - m[:, None], 0)), 0)
            t = p.sum(1)
            tt = np.where(some, t, 1)
            o, A = p @ v / tt[:, None], p @ np.abs(v) / tt[:, None]
            L = (seen.sum(1) + 64) * u
            out[t0:t0 + n, h] = o
            bound[t0:t0 + n, h] = (e + p_round + L)[:, None] * A + (e + L)[:, None] * np.abs(o)
            lse[t0:t0 + n, h] = np.where(some, m + np.log(tt), -np.inf)
            lb[t0:t0 + n, h] = e + L + 2 * 2.0 ** -23 * np.abs(m + np.log(tt))
    return out, bound, lse, lb

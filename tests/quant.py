"""Inputs and 64-bit references for the tests of a quantised cache and of drafted tokens (CPU, numpy)."""
import numpy as np
import torch

from answer import Problem

LEAST, MOST = {"f16": -15, "bf16": -117}, {"f16": 8, "bf16": 120}       # powers of two of a cache


def _values():
    """The numbers that the bytes 0 .. 127 stand for, by the format's definition: four bits of exponent, biased by 7, three of fraction."""
    v = [np.ldexp(c & 7, -9) if c < 8 else np.ldexp(8 + (c & 7), (c >> 3) - 10) for c in range(127)]
    return np.array(v + [np.nan])


VALUES = np.concatenate([_values(), -_values()])


def to_codes(x):
    """The nearest number's byte, ties to the even one; |x| <= 448, NaN to 0x7F."""
    a = np.abs(x)
    hi = np.clip(np.searchsorted(VALUES[:127], a), 0, 126)              # the first number at or above
    lo = np.maximum(hi - 1, 0)
    down, up = a - VALUES[lo], VALUES[hi] - a
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isnan(a), 127, code).astype(np.uint8)
    return np.where(np.signbit(x) & ~np.isnan(x), code | 128, code).astype(np.uint8)


def quantise(x, dtype):
    """x [.., d] in 64 bits: bytes, and the powers' exponents."""
    most = np.ldexp(240.0, MOST[dtype])
    y = np.where(np.isfinite(x), np.clip(x, -most, most), np.nan)
    top = np.nanmax(np.concatenate([np.abs(y), np.zeros(y.shape[:-1] + (1,))], -1), -1)
    e = np.full(top.shape, LEAST[dtype])
    while True:
        low = np.ldexp(448.0, e) < top
        if not low.any():
            break
        e = e + low
    return to_codes(np.ldexp(y, -e[..., None])), e


def values(codes, e):
    return np.ldexp(VALUES[codes], np.asarray(e)[..., None])


class Problem8(Problem):
    """A Problem whose cache is quantised: k and v are what it stands for, and the unused slots hold NaN, or anything, under powers
    of any byte.  scales: the order of the powers' pools."""

    def __init__(self, *args, scales="token", loud=1.0, **kw):
        super().__init__(*args, **kw)
        rng = np.random.default_rng(len(self.own) + self.tokens)
        self.scales, self.codes, self.powers = scales, [], []
        for name in ("k", "v"):
            x = getattr(self, name)
            used = ~np.isnan(x[:, 0, 0])
            codes = rng.integers(0, 256, x.shape).astype(np.uint8)
            codes[:, :, ::3] = 0x7F
            powers = rng.integers(0, 256, x.shape[:2]).astype(np.uint8)
            if used.any():
                # powers of their own for every token and head
                y = x[used] * np.exp2(rng.integers(-3, 4, x[used].shape[:2]) * loud)[..., None]
                y = torch.from_numpy(y).to(self.tdtype).double().numpy()
                codes[used], e = quantise(y, self.dtype)
                powers[used] = e + 127
                x[used] = values(codes[used], e)
            self.codes.append(codes)
            self.powers.append(powers)

    def cache(self, P):
        def pool(x, order):
            t = torch.from_numpy(x).view(-1, self.page, *x.shape[1:])
            return t.transpose(1, 2).contiguous().cuda().transpose(1, 2) if order == "head" else t.cuda()
        k, v = (pool(x, self.major) for x in self.codes)
        ks, vs = (pool(x, self.scales) for x in self.powers)
        return P.KvCache(k, v, ks, vs, dtype=self.tdtype)


def verify(logits, tokens, uniform, q_off, lens, draft=None, scale=1.0):
    """accepted, follows, lens; and whether a decision is nearer to its border than what 64 bits and their order of sums can tell."""
    accepted, follows, out, near = [], [], [], []
    x = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64))
    vocab = x.shape[1]

    def weights(t):
        row, top = x[t], x[t].max()
        if top == -np.inf:
            return np.zeros(vocab)
        if top == np.inf:
            w = (row == np.inf).astype(np.float64)
        else:
            w = np.exp(scale * (row - top))
        return w / w.sum()

    for s in range(len(q_off) - 1):
        t0, n = int(q_off[s]), int(q_off[s + 1] - q_off[s])
        a, close = 0, False
        while a + 1 < n:
            t = t0 + a + 1
            tok = int(tokens[t])
            if not 0 <= tok < vocab:
                break
            if scale == 0:
                if tok != int(np.argmax(x[t - 1])) or x[t - 1].max() == -np.inf:
                    break
            else:
                d = 1.0 if draft is None else max(float(np.nan_to_num(draft[t, tok])), 0.0)
                p = weights(t - 1)[tok]
                close |= float(uniform[t]) * d > 0 and abs(float(uniform[t]) * d - p) < 1e-12 * d
                if not float(uniform[t]) * d < p:
                    break
            a += 1
        accepted.append(a)
        out.append(int(lens[s]) - max(0, n - 1 - a))
        token = -1
        if n and scale == 0:
            row = x[t0 + a]
            token = int(np.argmax(row)) if row.max() > -np.inf else -1
        elif n:
            p = weights(t0 + a)
            w = p
            if a + 1 < n:
                tok = int(tokens[t0 + a + 1])
                if draft is not None:
                    d = draft[t0 + a + 1].astype(np.float64)
                    w = np.maximum(p - np.where(d > 0, d, 0.0), 0.0)
                elif 0 <= tok < vocab:
                    w = p.copy()
                    w[tok] = 0.0
                if not w.sum() > 0:
                    w = p
            if w.sum() > 0:
                run = np.cumsum(w)
                reach = float(uniform[t0]) * run[-1]
                token = int(np.argmax(run > reach)) if (run > reach).any() else int(np.nonzero(w)[0][-1])
                close |= float(uniform[t0]) > 0 and np.abs(run[w > 0] - reach).min() < 1e-11 * run[-1]
        follows.append(token)
        near.append(close)
    return np.array(accepted), np.array(follows), np.array(out), np.array(near)

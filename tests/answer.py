"""Inputs and 64-bit references for the tests of the paged cache, its attention and the beam step (CPU, numpy)."""
import numpy as np
import torch

DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
U = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}       # largest relative error of rounding to nearest


class Problem:
    """A paged cache whose unused slots hold NaN, and a step's sequences: new tokens, own keys (the new ones among
    them) and groups as (sequences, prefix keys); sequences behind the last group have no prefix."""

    def __init__(self, new, own, groups=(), hkv=2, d=64, page=16, own_page=None, prefix_page=None, dtype="bf16", major="token", seed=0,
                 spare=2, fill=True):
        g = torch.Generator().manual_seed(seed)
        self.new, self.own, self.groups, self.hkv, self.d = list(new), list(own), list(groups), hkv, d
        self.page, self.own_page, self.prefix_page = page, own_page or page, prefix_page or page
        self.dtype, self.tdtype = dtype, DT[dtype]
        need = [-(-n // page) for n in self.own]
        pneed = [-(-p // page) for _, p in self.groups]
        total = sum(need) + sum(pneed) + spare
        order = torch.randperm(total, generator=g).tolist()
        per, pper = page // self.own_page, page // self.prefix_page
        # entries that no key uses name nothing
        table = np.full((len(new), max(1, max(need + [0]) * per) + 1), -7, np.int64)
        ptable = np.full((max(1, len(groups)), max(1, max(pneed + [0]) * pper) + 1), 2 ** 31 - 1, np.int64)
        at = 0
        for s, n in enumerate(need):
            for i in range(n * per):
                table[s, i] = order[at + i // per] * per + i % per
            at += n
        for s, n in enumerate(pneed):
            for i in range(n * pper):
                ptable[s, i] = order[at + i // pper] * pper + i % pper
            at += n
        self.table, self.ptable = table, ptable
        self.slots = total * page
        self.q_off = np.concatenate([[0], np.cumsum(self.new)])
        self.tokens = int(self.q_off[-1])
        # [slot, head, d] as float64 of values of the cache's type; NaN where no key lies
        self.k = np.full((self.slots, hkv, d), np.nan)
        self.v = np.full((self.slots, hkv, d), np.nan)
        if fill:
            used = [self.own_slots(s) for s in range(len(new))] + [self.prefix_slots(i) for i in range(len(groups))]
            used = np.concatenate(used) if used else np.zeros(0, np.int64)
            for x in (self.k, self.v):
                x[used] = torch.randn(len(used), hkv, d, generator=g).to(self.tdtype).double().numpy()
        self.major = major
        self.gen = g

    def own_slots(self, s, n=None):
        j = np.arange(self.own[s] if n is None else n)
        return self.table[s, j // self.own_page] * self.own_page + j % self.own_page

    def prefix_slots(self, g):
        j = np.arange(self.groups[g][1])
        return self.ptable[g, j // self.prefix_page] * self.prefix_page + j % self.prefix_page

    def group(self, s):
        for g, (n, _) in enumerate(self.groups):
            if s < n:
                return g
            s -= n
        return -1

    def prefix(self, s):
        g = self.group(s)
        return 0 if g < 0 else self.groups[g][1]

    def rows(self, heads):
        return torch.randn(self.tokens, heads, self.d, generator=self.gen).to(self.tdtype)

    # -- on the GPU -----------------------------------------------------------------------------------
    def pool(self, x):
        t = torch.from_numpy(x).to(self.tdtype).view(-1, self.page, self.hkv, self.d)
        if self.major == "head":
            return t.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        return t.cuda()

    def cache(self, P):
        return P.KvCache(self.pool(self.k), self.pool(self.v))

    def step(self, P, **hints):
        i32 = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()
        kw = {}
        if self.groups:
            kw = dict(group_off=i32(np.concatenate([[0], np.cumsum([n for n, _ in self.groups])])), prefix_lens=i32([p for _, p in self.groups]),
                      prefix_table=i32(self.ptable), prefix_page=self.prefix_page)
        return P.KvStep(i32(self.q_off), i32(self.own), i32(self.table), page=self.own_page, n_tokens=self.tokens, **kw, **hints)

    # -- in 64 bits -----------------------------------------------------------------------------------
    def attend(self, q, scale, window=0, sinks=0):
        """out, lse, and per element the bound of what rounding may do to out."""
        q = q.double().numpy()
        hq = q.shape[1]
        rep = hq // self.hkv
        out, lse, tol = np.zeros(q.shape), np.full(q.shape[:2], -np.inf), np.zeros(q.shape)
        u = U[self.dtype]
        for s in range(len(self.new)):
            slots = self.own_slots(s)
            plen, n, m = self.prefix(s), self.own[s], self.new[s]
            if plen:
                slots = np.concatenate([self.prefix_slots(self.group(s)), slots])
            j = np.arange(plen + n)
            for i in range(m):
                p = plen + n - m + i
                sees = j <= p
                if window:
                    sees &= (p - j < window) | (j < sinks)
                if not sees.any():
                    continue
                t = self.q_off[s] + i
                kk, vv = self.k[slots[sees]], self.v[slots[sees]]
                for h in range(hq):
                    k, v, x = kk[:, h // rep], vv[:, h // rep], q[t, h]
                    sc = scale * (k @ x)
                    w = np.exp(sc - sc.max())
                    z = w.sum()
                    w = w / z
                    out[t, h], lse[t, h] = w @ v, sc.max() + np.log(z)
                    # a score is off by at most (d + 4) roundings of its terms' sum; its weight by that factor. The weights and the result
                    # are rounded once each to the cache's type, weights of f16 below 2^-22 of the largest to 2^-33 of it
                    e = (self.d + 4) * 2.0 ** -24 * scale * (np.abs(k) @ np.abs(x)).max() + 2.0 ** -20
                    tol[t, h] = (2 * u + 2 * e) * (w @ np.abs(v)) + 2.0 ** -24
                    if self.dtype == "f16":
                        tol[t, h] += len(w) * 2.0 ** -31 * np.abs(v).max(0)
        return out, lse, tol


def rotate(x, pos, rotary, rot, interleaved):
    """[tokens, heads, d] in 64 bits; and what 32-bit products and sums may be off by."""
    x = x.double().numpy().copy()
    c, s = rotary[pos, :rot // 2].astype(np.float64)[:, None], rotary[pos, rot // 2:].astype(np.float64)[:, None]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    xa, xb = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = xa * c - xb * s, xb * c + xa * s
    slack = np.zeros(x.shape)
    slack[..., a] = slack[..., b] = 3 * 2.0 ** -24 * (np.abs(xa) * np.abs(c) + np.abs(xb) * np.abs(s) + np.abs(xb) * np.abs(c) + np.abs(xa) * np.abs(s))
    return x, slack


def beam_step(logits, scores, k, done=None, eos=-1):
    """One prompt after the other, in 64 bits: scores, parents, tokens, done."""
    p, b, vocab = logits.shape
    out = np.full((p, k), -np.inf), np.zeros((p, k), np.int64), np.full((p, k), -1, np.int64), np.ones((p, k), bool)
    for i in range(p):
        cand = []
        for r in range(b):
            run = float(scores[i, r])
            if not run > -np.inf:
                continue
            if done is not None and done[i, r]:
                cand.append((-run, r, 0.0, eos))
                continue
            x = logits[i, r].astype(np.float64)
            x[np.isnan(x)] = -np.inf
            top = x.max()
            if top == -np.inf:
                continue
            with np.errstate(invalid="ignore"):
                dx = np.where(x == top, 0.0, x - top)
            z = np.log(np.exp(dx).sum())
            best = np.argsort(-x, kind="stable")[:k]
            cand += [(-(run + dx[t] - z), r, -x[t], int(t)) for t in best if dx[t] > -np.inf]
        cand.sort()
        out[1][i] = i * b
        for n, (sc, r, _, t) in enumerate(cand[:k]):
            out[0][i, n], out[1][i, n], out[2][i, n] = -sc, i * b + r, t
            out[3][i, n] = (done is not None and bool(done[i, r])) or t == eos
    return out

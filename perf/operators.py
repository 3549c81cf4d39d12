"""The operators of answering from retrieved passages, as cases that can be timed and compared.

A case is a dict of plain values; `op` says which entry point it goes through:

  append   `ivf_kv_append`: the new tokens' keys and values, rotated by their positions, into a paged cache; the queries
           are rotated in the same call
  attend   `ivf_attend`: the new tokens against the cache; groups of sequences share a prefix (the passages that were
           retrieved for a micro-batch, the prompt of a beam search); optionally a sliding window with some first tokens
           that stay visible
  select   `ivf_beam_step`: the best continuations over beams and vocabulary, and the rows of the beams' states moved
           to their new places

Lengths run evenly from a lower to an upper bound over the sequences of a group, in an order that the seed chooses, so
that a case has the same work with every seed.
"""
import math
import random

import torch

own = False

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ELEM = {"f32": 4, "f16": 2, "bf16": 2}
EOS = 2


def listed():
    return [
        # one request, one new token: launches and latency are all there is
        dict(name="append_one", op="append", dtype="bf16", seqs=1, q_lo=1, q_hi=1, own_lo=900, own_hi=900, hq=32, hkv=8, d=128,
             page=16, major="token", rot=128, pairs="halves"),
        # a serving step of 200 requests; head-major pages, half of every head is rotated, in interleaved pairs
        dict(name="append_step", op="append", dtype="f16", seqs=200, q_lo=1, q_hi=1, own_lo=0, own_hi=8000, hq=32, hkv=8, d=128,
             page=64, major="head", rot=64, pairs="interleaved"),
        # the passages of six retrievals enter the cache
        dict(name="append_passages", op="append", dtype="bf16", seqs=6, q_lo=700, q_hi=5001, own_lo=0, own_hi=37, hq=64, hkv=8, d=128,
             page=32, major="token", rot=128, pairs="halves"),
        # one request, one token, a short past
        dict(name="attend_one", op="attend", dtype="bf16", groups=1, seqs=1, q_lo=1, q_hi=1, own_lo=700, own_hi=700, prefix=0, hq=32,
             hkv=8, d=128, page=16, own_page=16, major="token", window=0, sinks=0, lse=False),
        # a micro-batch of 48 queries answered from the same passages
        dict(name="attend_shared", op="attend", dtype="bf16", groups=1, seqs=48, q_lo=1, q_hi=1, own_lo=30, own_hi=800, prefix=16000,
             hq=32, hkv=8, d=128, page=16, own_page=16, major="token", window=0, sinks=0, lse=False),
        # beam search: six prompts, eight beams each, whose pasts are named token by token; as many key as query heads
        dict(name="attend_beams", op="attend", dtype="f16", groups=6, seqs=8, q_lo=1, q_hi=1, own_lo=200, own_hi=200, prefix=3001, hq=16,
             hkv=16, d=64, page=64, own_page=1, major="token", window=0, sinks=0, lse=True),
        # 24 requests of very different lengths, the longest 60,000 tokens
        dict(name="attend_ragged", op="attend", dtype="bf16", groups=24, seqs=1, q_lo=1, q_hi=1, own_lo=411, own_hi=60000, prefix=0,
             hq=64, hkv=8, d=128, page=64, own_page=64, major="head", window=0, sinks=0, lse=False, spread=True),
        # 64 long conversations with a window of 4096 tokens and four first tokens kept
        dict(name="attend_window", op="attend", dtype="f16", groups=64, seqs=1, q_lo=1, q_hi=3, own_lo=100, own_hi=20000, prefix=0,
             hq=32, hkv=8, d=128, page=32, own_page=32, major="token", window=4096, sinks=4, lse=False, spread=True),
        # three questions with passages of their own behind shared ones, a few thousand tokens at once
        dict(name="attend_passages", op="attend", dtype="f16", groups=1, seqs=3, q_lo=333, q_hi=2500, own_lo=0, own_hi=0, prefix=6000,
             hq=32, hkv=8, d=64, page=16, own_page=16, major="token", window=0, sinks=0, lse=False),
        # the largest: one prompt of 16,000 tokens
        dict(name="attend_prompt", op="attend", dtype="bf16", groups=1, seqs=1, q_lo=16000, q_hi=16000, own_lo=0, own_hi=0, prefix=0,
             hq=32, hkv=8, d=128, page=64, own_page=64, major="token", window=0, sinks=0, lse=False),
        # three prompts of five beams over an odd vocabulary of 32-bit logits
        dict(name="select_small", op="select", dtype="f32", prompts=3, beams=5, out=5, vocab=50001, table=256, done=0.2),
        # a serving step of 64 prompts with eight beams each
        dict(name="select_step", op="select", dtype="bf16", prompts=64, beams=8, out=8, vocab=131072, table=512, done=0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "select"])
    dtype = rng.choice(["f16", "bf16"])
    if op == "select":
        beams = _log_int(rng, 1, 16)
        vocab = _log_int(rng, 1000, 160000)
        prompts = max(1, min(_log_int(rng, 1, 96), int(6.7e7 / (beams * vocab))))
        return dict(op=op, dtype=rng.choice(["f16", "bf16", "f32"]), prompts=prompts, beams=beams, out=rng.choice([beams, max(1, beams - 1), min(16, beams + 3)]),
                    vocab=vocab, table=_log_int(rng, 1, 600), done=rng.choice([0.0, 0.2]))
    hkv = rng.choice([1, 2, 4, 8, 16])
    hq = hkv * rng.choice([1, 2, 4, 7, 8]) if hkv < 16 else hkv
    d = rng.choice([64, 96, 128, 128, 256])
    page = rng.choice([1, 8, 16, 32, 64, 128])
    major = rng.choice(["token", "head"])
    if op == "append":
        seqs = _log_int(rng, 1, 300)
        q = _log_int(rng, 1, max(1, min(5000, int(1.3e8 / (seqs * d * (hq + 2 * hkv))))))
        rot = rng.choice([d, d // 2])
        return dict(op=op, dtype=dtype, seqs=seqs, q_lo=max(1, q // 3), q_hi=q, own_lo=0, own_hi=_log_int(rng, 1, 2000), hq=hq, hkv=hkv, d=d,
                    page=page, major=major, rot=rot, pairs=rng.choice(["halves", "interleaved"]))
    groups = _log_int(rng, 1, 24)
    seqs = _log_int(rng, 1, 48)
    many = rng.random() < 0.4                     # prompts rather than single tokens
    q = _log_int(rng, 2, 4000) if many else rng.choice([1, 1, 1, 2, 5])
    case = dict(op=op, dtype=dtype, groups=groups, seqs=seqs, q_lo=max(1, q // 3), q_hi=q, own_lo=rng.choice([0, 100]), own_hi=_log_int(rng, 101, 20000),
                prefix=rng.choice([0, _log_int(rng, 1, 16000)]), hq=hq, hkv=hkv, d=d, page=page, own_page=rng.choice([page, page, 1]),
                major=major, window=rng.choice([0, 0, _log_int(rng, 1, 4096)]), sinks=rng.choice([0, 4, 17]), lse=rng.random() < 0.3)
    while True:                                   # a pass costs no more than the largest listed one of its kind
        n = case["prefix"] + case["own_hi"] + case["q_hi"]
        rows = case["groups"] * case["seqs"] * case["q_hi"]
        if rows * hq * n <= 8.0e9 and case["groups"] * case["seqs"] * n * hkv * d <= 1.2e9:
            cost = work(case)
            if cost["flops"] <= 2.0e12 and cost["bytes"] <= 2.9e9:
                return case
        at = max(("own_hi", "prefix", "seqs", "groups", "q_hi"), key=lambda f: case[f] / (200 if f in ("own_hi", "prefix", "q_hi") else 1))
        case[at] = max(1, int(case[at] * 0.6))
        case["own_lo"] = min(case["own_lo"], case["own_hi"])
        case["q_lo"] = min(case["q_lo"], case["q_hi"])


# ---- inputs -----------------------------------------------------------------------------------
def _even(lo, hi, n):
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _lengths(case):
    """(group, new tokens, own keys with the new ones, prefix) of every sequence, before the seed shuffles them."""
    groups, seqs = case.get("groups", 1), case["seqs"]
    across = case.get("spread", False)            # the range is run through by the groups, not inside each
    n = groups if across else seqs
    new, past = _even(case["q_lo"], case["q_hi"], n), _even(case["own_lo"], case["own_hi"], n)
    prefix = _even(case.get("prefix", 0) * 7 // 10, case.get("prefix", 0), groups)
    at = [(g, g if across else j) for g in range(groups) for j in range(seqs)]
    return [(g, new[i], past[i] + new[i], prefix[g]) for g, i in at]


def _shuffled(case, seed):
    rows = _lengths(case)
    rng = random.Random(int(seed) + 17)
    if case.get("spread", False):
        lens = [r[1:3] for r in rows]
        rng.shuffle(lens)
        return [(r[0], *n, r[3]) for r, n in zip(rows, lens)]
    out = []
    for g in range(case.get("groups", 1)):
        part = [r for r in rows if r[0] == g]
        rng.shuffle(part)
        out += part
    return out


def _randn(shape, dtype, gen, factor=1.0):
    """Normal values, drawn in pieces of whole first rows."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // max(1, out[0].numel()))
    for s in range(0, shape[0], step):
        out[s:s + step] = torch.randn(out[s:s + step].shape, generator=gen, device="cuda") * factor
    return out


def _i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def _cache(case, seed):
    """The pools [pages, page, heads, d] and the tables: pages in random order, the own table by entries of own_page tokens."""
    rows = _shuffled(case, seed)
    page, g = case["page"], case.get("own_page", case["page"])
    per = page // g                               # own entries of a page
    need = [-(-n // page) for _, _, n, _ in rows]
    groups = case.get("groups", 1)
    plen = [next(r[3] for r in rows if r[0] == i) for i in range(groups)]
    pneed = [-(-n // page) for n in plen]
    total = sum(need) + sum(pneed) + 3
    cpu = torch.Generator().manual_seed(int(seed))
    order = torch.randperm(total, generator=cpu).to(torch.int32)
    table = torch.zeros(len(rows), max(1, max(need) * per), dtype=torch.int32)
    ptable = torch.zeros(groups, max(1, max(pneed)), dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        entries = (order[at:at + n, None] * per + torch.arange(per, dtype=torch.int32)).reshape(-1)
        table[i, :n * per] = entries
        at += n
    for i, n in enumerate(pneed):
        ptable[i, :n] = order[at:at + n]
        at += n
    gen = torch.Generator(device="cuda").manual_seed(int(seed) + 1)
    shape = (total, page, case["hkv"], case["d"]) if case["major"] == "token" else (total, case["hkv"], page, case["d"])
    k, v = (_randn(shape, TORCH[case["dtype"]], gen) for _ in range(2))
    if case["major"] == "head":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    q_off = [0]
    for r in rows:
        q_off.append(q_off[-1] + r[1])
    count = [sum(r[0] == i for r in rows) for i in range(groups)]
    group_off = [sum(count[:i]) for i in range(groups + 1)]
    st = dict(case=case, k=k, v=v, table=table.cuda(), lens=_i32([r[2] for r in rows]), q_off=_i32(q_off), tokens=q_off[-1],
              max_q=max(r[1] for r in rows), max_len=max(r[2] for r in rows))
    if case.get("prefix", 0):
        st.update(prefix_table=ptable.cuda(), prefix_lens=_i32(plen), group_off=_i32(group_off), max_prefix=max(plen))
    return st, rows, gen


def _rotary(case, most):
    """Cosines and sines [positions, rot], as a program keeps them."""
    half = case["rot"] // 2
    angle = torch.arange(most, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    return torch.cat([angle.cos(), angle.sin()], 1).float().cuda()


def prepare(case, seed):
    if case["op"] == "select":
        gen = torch.Generator(device="cuda").manual_seed(int(seed))
        p, b = case["prompts"], case["beams"]
        logits = _randn((p * b, case["vocab"]), TORCH[case["dtype"]], gen, 3.0).view(p, b, -1)
        scores = -torch.rand(p, b, generator=gen, device="cuda").mul_(1.5).cumsum(1) - 4.0
        done = torch.rand(p, b, generator=gen, device="cuda") < case["done"]
        table = torch.randint(0, 1 << 20, (p * b, case["table"]), generator=gen, device="cuda").int()
        history = torch.randint(0, case["vocab"], (p * b, 200), generator=gen, device="cuda").int()
        return dict(case=case, logits=logits, scores=scores, done=done, table=table, history=history,
                    new_table=torch.zeros(p * case["out"], case["table"], dtype=torch.int32, device="cuda"),
                    new_history=torch.zeros(p * case["out"], 200, dtype=torch.int32, device="cuda"))
    st, rows, gen = _cache(case, seed)
    t, d, dt = st["tokens"], case["d"], TORCH[case["dtype"]]
    if case["op"] == "attend":
        st["q"] = _randn((t, case["hq"], d), dt, gen, 2.0)
        st["out"] = torch.empty_like(st["q"])
        return st
    # the projections' output: queries, keys and values of a token side by side
    qkv = _randn((t, case["hq"] + 2 * case["hkv"], d), dt, gen)
    st["q"], st["new_k"], st["new_v"] = qkv.split([case["hq"], case["hkv"], case["hkv"]], 1)
    st["rotary"] = _rotary(case, st["max_len"] + 1)
    st["q_out"] = torch.empty(t, case["hq"], d, dtype=dt, device="cuda")
    return st


# ---- one pass -----------------------------------------------------------------------------------
def _step(state):
    """What a program keeps through the layers of a step: the tables, and the layer's cache."""
    if "step" not in state:
        import paper_2502_20969_amd as P
        case = state["case"]
        shared = {}
        if "prefix_table" in state:
            shared = dict(group_off=state["group_off"], prefix_lens=state["prefix_lens"], prefix_table=state["prefix_table"],
                          prefix_page=case["page"], max_prefix=state["max_prefix"])
        state["step"] = P.KvStep(state["q_off"], state["lens"], state["table"], page=case.get("own_page", case["page"]), n_tokens=state["tokens"],
                                 max_q=state["max_q"], max_len=state["max_len"], **shared)
        state["cache"] = P.KvCache(state["k"], state["v"])
        state["P"] = P
    return state["P"], state["step"], state["cache"]


def run(state):
    case = state["case"]
    if case["op"] == "append":
        return _append(state)
    if case["op"] == "attend":
        return _attend(state)
    return _select(state)


def _tokens(state):
    """Sequence of every new token, and its place among the sequence's own keys."""
    q_off, lens = state["q_off"].long(), state["lens"].long()
    t = torch.arange(state["tokens"], device="cuda")
    seq = torch.searchsorted(q_off, t, right=True) - 1
    return seq, lens[seq] - q_off[seq + 1] + t


def _slot(entry, off, entry_tokens, page):
    """Page and place inside it of the token `off` behind the start of table entry `entry`."""
    token = entry.long() * entry_tokens + off
    return token // page, token % page


def _rotated(x, c, s, case):
    """x [tokens, heads, d] in 32 bits."""
    half = case["rot"] // 2
    out = x.clone()
    a, b = (slice(0, half), slice(half, 2 * half)) if case["pairs"] == "halves" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    out[..., a] = x[..., a] * c - x[..., b] * s
    out[..., b] = x[..., b] * c + x[..., a] * s
    return out


def _append(state):
    case = state["case"]
    if own:
        P, step, cache = _step(state)
        P.ivf_kv_append(step, cache, state["new_k"], state["new_v"], rotary=state["rotary"], interleaved=case["pairs"] == "interleaved",
                        q=state["q"], q_out=state["q_out"])
        return [state["k"], state["v"], state["q_out"]]
    page = case["page"]
    seq, place = _tokens(state)
    at = _slot(state["table"][seq, place // page], place % page, page, page)
    half = case["rot"] // 2
    c, s = (state["rotary"][place][:, None, i * half:(i + 1) * half] for i in range(2))
    state["k"][at] = _rotated(state["new_k"].float(), c, s, case).to(state["k"].dtype)
    state["v"][at] = state["new_v"]
    state["q_out"].copy_(_rotated(state["q"].float(), c, s, case))
    return [state["k"], state["v"], state["q_out"]]


def _attend(state):
    case = state["case"]
    d, hq, hkv = case["d"], case["hq"], case["hkv"]
    scale = d ** -0.5
    if own:
        P, step, cache = _step(state)
        lse = torch.empty(state["tokens"], hq, dtype=torch.float32, device="cuda") if case["lse"] else None
        P.ivf_attend(step, cache, state["q"], out=state["out"], lse=lse, scale=scale, window=case["window"], sinks=case["sinks"])
        return [state["out"], lse] if case["lse"] else [state["out"]]
    lens, q_off = state["lens"].long(), state["q_off"].long()
    nseq, page, own_page = lens.numel(), case["page"], case["own_page"]
    plen, most = torch.zeros_like(lens), state["max_len"]
    # keys of every sequence, the shared ones first, padded to the longest
    if case["prefix"]:
        group = torch.searchsorted(state["group_off"].long(), torch.arange(nseq, device="cuda"), right=True) - 1
        plen = state["prefix_lens"].long()[group]
        most += state["max_prefix"]
    j = torch.arange(most, device="cuda")[None]
    mine = (j - plen[:, None]).clamp(min=0)
    entry = torch.gather(state["table"], 1, (mine // own_page).clamp(max=state["table"].shape[1] - 1))
    at = torch.stack(_slot(entry, mine % own_page, own_page, page))
    if case["prefix"]:
        first = j.clamp(max=state["max_prefix"] - 1).expand(nseq, -1)
        entry = torch.gather(state["prefix_table"][group], 1, first // page)
        at = torch.where(j < plen[:, None], torch.stack(_slot(entry, first % page, page, page)), at)
    k, v = (x[at[0], at[1]].float().transpose(1, 2).contiguous() for x in (state["k"], state["v"]))       # [seq, hkv, keys, d]
    # queries of every sequence, padded to the most new tokens
    m = q_off[1:] - q_off[:-1]
    i = torch.arange(state["max_q"], device="cuda")[None]
    token = (q_off[:-1, None] + i).clamp(max=state["tokens"] - 1)
    q = state["q"][token].float().view(nseq, -1, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(nseq, hkv, -1, d).contiguous()
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).view(nseq, hkv, hq // hkv, state["max_q"], most)
    pos = (plen + lens - m)[:, None] + i
    hidden = j[:, None] > pos[..., None]
    if case["window"]:
        hidden |= (pos[..., None] - j[:, None] >= case["window"]) & (j[:, None] >= case["sinks"])
    s.masked_fill_(hidden[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp(min=-1e30)
    s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(nseq, hkv, -1, most), v).view(nseq, hkv, hq // hkv, -1, d)
    o = torch.where(total > 0, o / total.clamp(min=1e-30), torch.zeros_like(o)).permute(0, 3, 1, 2, 4).reshape(nseq, -1, hq, d)
    real = i < m[:, None]
    state["out"].copy_(o[real])
    if not case["lse"]:
        return [state["out"]]
    lse = (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(nseq, -1, hq)
    return [state["out"], lse[real]]


def _select(state):
    case = state["case"]
    p, b, n = case["prompts"], case["beams"], case["out"]
    states = [(state["table"], state["new_table"]), (state["history"], state["new_history"])]
    if own:
        import paper_2502_20969_amd as P
        return [*P.ivf_beam_step(state["logits"], state["scores"], n, done=state["done"], eos=EOS, states=states), *(x[1] for x in states)]
    x = state["logits"].float()
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    top = x.amax(-1, keepdim=True)
    logp = (x - top) - (x - top).exp().sum(-1, keepdim=True).log()
    stop = torch.full((case["vocab"],), -math.inf, device="cuda")
    stop[EOS] = 0.0
    logp = torch.where(state["done"][..., None], stop, logp)
    # the best of each beam, equal ones by token, then the best of all, equal ones by beam
    best, token = torch.sort(logp, dim=-1, descending=True, stable=True)
    m = min(n, case["vocab"])
    total = (state["scores"][..., None] + best[..., :m]).view(p, -1)
    total = torch.where(torch.isnan(total), torch.full_like(total, -math.inf), total)
    if total.shape[1] < n:
        total = torch.cat([total, torch.full((p, n - total.shape[1]), -math.inf, device="cuda")], 1)
    score, at = torch.sort(total, dim=-1, descending=True, stable=True)
    score, at = score[:, :n], at[:, :n]
    none = torch.isinf(score)
    beam = torch.where(none, torch.zeros_like(at), at // m)
    token = token[..., :m].reshape(p, -1).gather(1, at.clamp(max=b * m - 1))
    token = torch.where(none, torch.full_like(token, -1), token).int()
    done = none | state["done"].gather(1, beam) | (token == EOS)
    parent = (beam + torch.arange(p, device="cuda")[:, None] * b).int()
    rows = parent.long().view(-1)
    torch.index_select(state["table"], 0, rows, out=state["new_table"])
    torch.index_select(state["history"], 0, rows, out=state["new_history"])
    return [score, parent, token, done, state["new_table"], state["new_history"]]


# ---- what a pass cannot do without ---------------------------------------------------------------
def _visible(case, pos):
    """Keys that a token at position pos sees."""
    w = case["window"]
    if not w or pos < w:
        return pos + 1
    return w + min(case["sinks"], pos + 1 - w)


def work(case):
    if case["op"] == "select":
        rows, to = case["prompts"] * case["beams"], case["prompts"] * case["out"]
        live = rows * (1.0 - case["done"])
        moved = 4.0 * (case["table"] + 200)
        return {"bytes": live * case["vocab"] * ELEM[case["dtype"]] + (rows + to) * moved + 5.0 * rows + 13.0 * to, "flops": 4.0 * live * case["vocab"]}
    lens = _lengths(case)
    e, d, hq, hkv = ELEM[case["dtype"]], case["d"], case["hq"], case["hkv"]
    t = sum(r[1] for r in lens)
    if case["op"] == "append":
        return {"bytes": 2.0 * t * (hq + 2 * hkv) * d * e + 4.0 * t * case["rot"] + 8.0 * t, "flops": 3.0 * t * (hq + hkv) * case["rot"]}
    pairs, keys, first = 0.0, 0.0, {}
    for g, m, n, plen in lens:
        end = plen + n
        pairs += sum(_visible(case, p) for p in range(end - m, end)) if case["window"] else m * (end - m) + m * (m + 1) / 2
        # the keys that any of the m tokens sees: those of the window and the first ones
        low = max(0, end - m + 1 - case["window"]) if case["window"] else 0
        sinks = min(case["sinks"], low)
        keys += end - max(low, plen) + max(0, sinks - plen)
        a, b = first.get(g, (plen, 0))
        first[g] = (min(a, low), max(b, min(sinks, plen)))
    for g, m, n, plen in {r[0]: r for r in lens}.values():
        low, sinks = first[g]
        keys += max(0, plen - low) + min(sinks, low)
    return {"bytes": 2.0 * t * hq * d * e + 2.0 * keys * hkv * d * e + (4.0 * t * hq if case["lse"] else 0.0), "flops": 4.0 * d * hq * pairs}


# ---- the same results in 64 bits ------------------------------------------------------------------
def exact(case, seed):
    if case["op"] == "select":
        st = prepare(case, seed)
        p, b, n = case["prompts"], case["beams"], case["out"]
        score = torch.full((p, n), -math.inf, dtype=torch.float64, device="cuda")
        for i in range(p):
            x = st["logits"][i].double()
            cand = st["scores"][i].double()[:, None] + torch.log_softmax(x, -1)
            for r in range(b):
                if st["done"][i, r]:
                    cand[r] = -math.inf
                    cand[r, EOS] = st["scores"][i, r].double()
            best = cand.view(-1).topk(min(n, cand.numel())).values
            score[i, :best.numel()] = best
        return [score, None, None, None, None, None]
    st = prepare(case, seed)
    rows = _shuffled(case, seed)
    d, hq, hkv, page = case["d"], case["hq"], case["hkv"], case["page"]
    table = st["table"].cpu().long()
    if case["op"] == "append":
        k, v, q = st["k"].double(), st["v"].double(), st["q"].double()
        half = case["rot"] // 2
        at = 0
        for s, (_, m, n, _) in enumerate(rows):
            place = torch.arange(n - m, n)
            pg, off = table[s, place // page].cuda(), (place % page).cuda()
            turn = torch.complex(*(st["rotary"][place.cuda()].double().view(m, 2, 1, half).unbind(1)))
            for x, to in ((st["new_k"][at:at + m].double(), k), (q[at:at + m].clone(), None)):
                part = x[..., :2 * half]
                pair = part.reshape(m, -1, 2, half).transpose(2, 3) if case["pairs"] == "halves" else part.reshape(m, -1, half, 2)
                z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
                x[..., :2 * half] = (z.transpose(2, 3) if case["pairs"] == "halves" else z).reshape(part.shape)
                if to is None:
                    q[at:at + m] = x
                else:
                    to[pg, off] = x
            v[pg, off] = st["new_v"][at:at + m].double()
            at += m
        return [k, v, q]
    if sum(r[1] * (r[2] + r[3]) for r in rows) * hq * d * 4 > 5e13:
        return None
    out = torch.zeros(st["tokens"], hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((st["tokens"], hq), -math.inf, dtype=torch.float64, device="cuda")
    at, per = 0, page // case["own_page"]
    for s, (g, m, n, plen) in enumerate(rows):
        j = torch.arange(n)
        token = table[s, j // case["own_page"]] * case["own_page"] + j % case["own_page"]
        if plen:
            jp = torch.arange(plen)
            token = torch.cat([st["prefix_table"][g].cpu().long()[jp // page] * page + jp % page, token])
        token = token.cuda()
        key = torch.arange(plen + n, device="cuda")
        for h in range(hkv):
            heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            kk, vv = (x[token // page, token % page, h].double() for x in (st["k"], st["v"]))
            step = max(1, (1 << 27) // ((plen + n) * (hq // hkv)))
            for i in range(0, m, step):
                pos = plen + n - m + torch.arange(i, min(m, i + step), device="cuda")
                sees = key[None] <= pos[:, None]
                if case["window"]:
                    sees &= (pos[:, None] - key[None] < case["window"]) | (key[None] < case["sinks"])
                sc = st["q"][at + i:at + i + len(pos), heads].double() @ kk.T / math.sqrt(d)
                sc = torch.where(sees[:, None], sc, torch.full_like(sc, -math.inf))
                lse[at + i:at + i + len(pos), heads] = torch.logsumexp(sc, -1)
                out[at + i:at + i + len(pos), heads] = torch.softmax(sc, -1) @ vv
        at += m
    return [out, lse] if case["lse"] else [out]

"""ivf_attend over quantised caches, against the softmax in 64 bits over what they stand for.  Slots that a token does not see hold
NaN and any bytes, under powers of any byte."""
import numpy as np
import pytest
import torch

import paper_2502_20969_amd as P
from quant import LEAST, MOST, Problem8, VALUES, to_codes, values
from test_gpu_attend import _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (8, 1), (14, 2)])
def test_types_and_heads(dtype, d, hq, hkv):
    _run(Problem8([1, 2, 5], [77, 130, 5], hkv=hkv, d=d, dtype=dtype, seed=d + hq), hq)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("new", [70, 300])
def test_prompts_of_types_and_widths(dtype, d, new):
    _run(Problem8([new, 33], [new + 130, 33], hkv=2, d=d, dtype=dtype, seed=d + new), 4)


@pytest.mark.parametrize("own", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 2049])
@pytest.mark.parametrize("d", [64, 128])
def test_lengths_of_single_tokens(own, d):
    _run(Problem8([1], [own], hkv=1, d=d, seed=own), 4)


@pytest.mark.parametrize("new", [2, 7, 8, 9, 16, 31, 32, 33, 63, 65, 100, 129, 200])
@pytest.mark.parametrize("past", [0, 1, 61])
def test_numbers_of_new_tokens(new, past):
    _run(Problem8([new], [new + past], hkv=1, d=64, dtype="f16", seed=new + past), 2)


@pytest.mark.parametrize("page,own_page", [(1, 1), (2, 2), (16, 1), (16, 4), (32, 32), (128, 128), (512, 64)])
@pytest.mark.parametrize("major,scales", [("token", "token"), ("head", "head"), ("token", "head"), ("head", "token")])
def test_pages(page, own_page, major, scales):
    _run(Problem8([1, 40, 3], [300, 41, 150], groups=[(2, 70)], hkv=2, d=64, page=page, own_page=own_page, prefix_page=max(1, page // 2),
                  major=major, scales=scales, seed=page + own_page), 4)


@pytest.mark.parametrize("page,own_page,d", [(64, 64, 128), (128, 16, 128), (16, 16, 256), (8, 8, 256), (32, 32, 96)])
@pytest.mark.parametrize("scales", ["token", "head"])
def test_pages_of_prompts(page, own_page, d, scales):
    _run(Problem8([150, 40], [400, 41], groups=[(2, 64)], hkv=1, d=d, page=page, own_page=own_page, major="head", scales=scales, seed=page + d), 2)


@pytest.mark.parametrize("plen", [1, 5, 64, 65, 700, 2500])
@pytest.mark.parametrize("seqs,new", [(1, 1), (5, 1), (40, 1), (3, 4), (2, 90)])
def test_shared_prefix(plen, seqs, new):
    own = [new + 7 * i for i in range(seqs)]
    _run(Problem8([new] * seqs, own, groups=[(seqs, plen)], hkv=2, d=64, dtype="f16", seed=plen + seqs), 8)


def test_groups_of_many_kinds():
    """Empty groups, groups without keys, sequences of no group, sequences without tokens, without own keys."""
    new = [1, 1, 0, 3, 2, 1, 1, 50, 1, 0, 1]
    own = [9, 1, 4, 3, 2, 88, 1, 50, 300, 0, 77]
    groups = [(2, 100), (0, 30), (3, 0), (1, 513), (3, 17)]
    _run(Problem8(new, own, groups=groups, hkv=2, d=128, seed=4), 6)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 0), (5, 3), (64, 4), (100, 17), (128, 200), (10 ** 6, 4), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("shape", ["tokens", "prompt", "shared"])
def test_windows(window, sinks, shape):
    pr = {"tokens": Problem8([1, 2, 1], [500, 90, 3], hkv=1, d=64, seed=1),
          "prompt": Problem8([300, 130], [300, 200], hkv=1, d=64, dtype="f16", seed=2),
          "shared": Problem8([1, 1, 2, 1], [3, 120, 60, 1], groups=[(3, 333), (1, 40)], hkv=1, d=64, seed=3)}[shape]
    _run(pr, 2, window, sinks)


@pytest.mark.parametrize("window,sinks,new", [(40, 3, 1), (40, 3, 70), (0, 0, 70), (7, 0, 3)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_what_is_not_seen_never_counts(window, sinks, new, d):
    """One key and value after the other becomes NaN under the largest power: the tokens that do not see it keep their results, those
    that do get NaN."""
    pr = Problem8([new], [new + 150], hkv=1, d=d, dtype="f16", seed=new)
    scale = pr.d ** -0.5
    q = pr.rows(2) * 2
    want, _, tol = pr.attend(q, scale, window, sinks)
    slots = pr.own_slots(0)
    keys = [pr.own[0] - 1, pr.own[0] - new // 2, 100, 4, 0] if new > 3 else [4, 60, 100]
    for key in keys:
        p = np.arange(pr.own[0] - new, pr.own[0])
        sees = key <= p
        if window:
            sees &= (p - key < window) | (key < sinks)
        if sees.all():
            continue
        cache = pr.cache(P)
        for pool, powers in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
            pool.view(-1, 1, d)[int(slots[key])] = 0xFF
            powers.view(-1, 1)[int(slots[key])] = 255
        out = P.ivf_attend(pr.step(P), cache, q.cuda(), scale=scale, window=window, sinks=sinks).double().cpu().numpy()
        assert (np.abs(out - want) <= tol)[~sees].all(), key
        assert np.isnan(out[sees]).all()


@pytest.mark.parametrize("new", [1, 70])
def test_a_value_that_is_no_number_reaches_those_who_see_it(new):
    pr = Problem8([new], [new + 80], hkv=1, d=64, dtype="bf16", seed=8)
    q, key, e = pr.rows(1), 60 + new // 2, 5
    pr.codes[1][int(pr.own_slots(0)[key]), 0, e] = 0x7F
    out = P.ivf_attend(pr.step(P), pr.cache(P), q.cuda()).float().cpu()[:, 0]
    sees = torch.arange(80, 80 + new) >= key
    assert torch.isnan(out[sees, e]).all() and torch.isfinite(out[~sees]).all()
    assert torch.isfinite(out[:, [i for i in range(64) if i != e]]).all()


@pytest.mark.parametrize("new,own,hints", [(1, 40, {}), (1, 5000, dict(max_q=1, max_len=5000)), (90, 300, {}), (3, 900, dict(max_q=3, max_len=900))])
def test_a_query_that_is_no_number(new, own, hints):
    """NaN in every element of its head and in lse, however the keys are cut; the other heads and tokens keep their results."""
    pr = Problem8([new, 1], [own, 30], hkv=2, d=128, seed=own)
    q = pr.rows(4)
    want, wl, tol = pr.attend(q, pr.d ** -0.5)
    q[0, 1, 7] = float("nan")
    lse = torch.zeros(pr.tokens, 4).cuda()
    out = P.ivf_attend(pr.step(P, **hints), pr.cache(P), q.cuda(), lse=lse).double().cpu().numpy()
    assert np.isnan(out[0, 1]).all() and bool(torch.isnan(lse[0, 1]))
    rest = np.ones(out.shape[:2], bool)
    rest[0, 1] = False
    assert (np.abs(out - want) <= tol)[rest].all()


def test_what_the_cache_holds_is_what_is_read():
    """Attention over a quantised cache, and over a 16-bit one that holds what ivf_kv_read brings back: of the same numbers, within both's roundings."""
    for new in (1, 80):
        pr = Problem8([new, 2], [new + 400, 90], hkv=2, d=64, page=32, dtype="f16", seed=new)
        q, cache, step = pr.rows(4).cuda(), pr.cache(P), pr.step(P)
        n = [new + 400, 90]
        rows = [torch.zeros(sum(n), 2, 64, dtype=torch.float16, device="cuda") for _ in range(2)]
        P.ivf_kv_read(step, cache, torch.tensor([0, n[0], sum(n)], dtype=torch.int32).cuda(), *rows)
        flat = P.KvCache(*(x.view(-1, 1, 2, 64) for x in rows))
        table = torch.zeros(2, n[0], dtype=torch.int32)
        table[0], table[1, :90] = torch.arange(n[0]), n[0] + torch.arange(90)
        plain = P.KvStep(step._keep[0], step._keep[1], table.cuda(), page=1, n_tokens=pr.tokens)
        a, b = (P.ivf_attend(s, c, q).double().cpu().numpy() for s, c in ((step, cache), (plain, flat)))
        _, _, tol = pr.attend(q.cpu(), 64 ** -0.5)
        assert (np.abs(a - b) <= 2 * tol).all()


def test_rows_that_see_nothing():
    """Fewer own keys than new tokens, and none at all: zeros and -inf."""
    pr = Problem8([3, 40, 2, 1], [3, 40, 2, 5], hkv=1, d=64, seed=6)
    pr.own = [1, 10, 0, 5]
    _run(pr, 2)
    _run(pr, 2, window=3, sinks=1)


def test_extreme_scores():
    pr = Problem8([1, 60], [400, 300], hkv=1, d=64, dtype="bf16", seed=7)
    _run(pr, 2, q=pr.rows(2) * 300)
    _run(pr, 2, q=pr.rows(2) * 0)
    _run(pr, 2, scale=1e-6)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new", [1, 70])
def test_powers_far_apart(dtype, new):
    """Tokens whose powers of two differ by up to 2^18 (f16) or 2^42: each has its own."""
    pr = Problem8([new, 1], [new + 200, 90], hkv=2, d=128, dtype=dtype, loud=3.0 if dtype == "f16" else 7.0, seed=new)
    _run(pr, 4, scale=2.0 ** (-12 if dtype == "f16" else -26), hints=dict(max_q=new, max_len=new + 200))


def _at_the_ends(dtype, d, new, n, x, codes, powers):
    """new tokens of one head, alike, over n keys of which key j has score x[j] (nearly base 2) against each; codes and powers [n, d] and [n] of
    the values.  Compared with the sums in 64 bits; no absolute tolerance but f16's own, for what is tiny here counts."""
    t, u = {"f16": (torch.float16, 2.0 ** -11), "bf16": (torch.bfloat16, 2.0 ** -8)}[dtype]
    page = 32
    pages = -(-n // page)
    flat = lambda a, fill: np.concatenate([a, np.full((pages * page - n,) + a.shape[1:], fill, np.uint8)]).reshape(pages, page, 1, *a.shape[1:])
    k = np.zeros((n, d), np.uint8)
    k[:, 0] = to_codes(x)
    assert np.array_equal(VALUES[k[:, 0]], x)
    q = torch.zeros(new, 1, d, dtype=t)
    q[:, 0, 0] = 1.0
    scale = float(np.float32(np.log(2.0) * (1 - 2.0 ** -12)))
    cache = P.KvCache(*(torch.from_numpy(a).cuda() for a in (flat(k, 0x7F), flat(codes, 0x7F), flat(np.full(n, 127, np.uint8), 255), flat(powers, 255))), dtype=t)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32).cuda()
    step = P.KvStep(i32([0, new]), i32([n]), i32([list(range(pages))]), page=page, n_tokens=new)
    out = P.ivf_attend(step, cache, q.cuda(), scale=scale).double().cpu().numpy()[:, 0]
    v = values(codes, powers.astype(int) - 127)
    for i in range(new):
        w = np.exp(scale * (x[:n - new + 1 + i] - x[:n - new + 1 + i].max()))
        want = w @ v[:len(w)] / w.sum()
        # weights and result are rounded once each; a score of at most 12 is off by 2 roundings of 32 bits, its power of 2 by as much, sums of
        # 600 terms by 600 at most.  Half a step of the type's numbers near zero: 2^-25 (f16), 2^-134 (bf16); f16: weights to 2^-33 of the largest
        tol = (2 * u + 640 * 2.0 ** -24) * (w @ np.abs(v[:len(w)]) / w.sum())
        tol += 2.0 ** -134 if dtype == "bf16" else len(w) * 2.0 ** -31 * np.abs(v[:len(w)]).max(0) + 2.0 ** -25
        bad = ~(np.abs(out[i] - want) <= tol)
        assert not bad.any(), (i, np.flatnonzero(bad)[:4], out[i][bad][:4], want[bad][:4])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("new", [1, 5, 70])
@pytest.mark.parametrize("ends", ["high", "low", "both"])
def test_powers_at_their_ends(dtype, d, new, ends):
    """Values under the largest and the least power that the rows' type allows, of keys whose weights are up to 2^8 above those of the keys before
    them, or far below the largest."""
    n, least, most = 600, 127 + LEAST[dtype], 127 + MOST[dtype]
    rng = np.random.default_rng(d + new)
    # small numbers, zeros among them, of one sign.  Sums are 32 bits wide: 2 * 2^-9 * 2^120 times the weight 2^8 of 90 keys, and 1 of the others, is below 2^127
    codes = np.where(rng.random((n, d)) < 0.5, 0, rng.integers(1, 3, (n, d))).astype(np.uint8)
    codes[:, ::5] = 0
    x, powers = np.zeros(n), np.full(n, most)
    if ends == "high":
        x[64::6] = 8.0
    else:
        # one key before the others, without a value; their weights are no powers of two
        x[0], x[1:] = 12.0, rng.integers(0, 16, n - 1) / 16
        codes[0] = 0
        codes[1:, 1::5] = 0x38 + rng.integers(0, 8, (n - 1, len(range(1, d, 5))))
        powers[:] = least
        if ends == "both":
            # under the largest power too, of which some elements have nothing but zeros
            powers[3::7] = most
            codes[3::7, 1::5] = 0
    _at_the_ends(dtype, d, new, n, x, codes, powers.astype(np.uint8))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 3)])
@pytest.mark.parametrize("first", [0, 1, 5])
def test_zeros_under_the_largest_power(dtype, d, window, sinks, first):
    """Values of zero under the largest power there is, from the `first`th page on every seventh: in prefixes, windows, pieces and tiles at the edges."""
    pr = Problem8([1, 2, 1, 1, 3], [300, 90, 1, 1500, 40], groups=[(3, 700), (1, 33)], hkv=2, d=d, dtype=dtype, seed=d + first)
    for s in range(len(pr.new)):
        for slots in (pr.own_slots(s), pr.prefix_slots(pr.group(s)) if pr.prefix(s) else pr.own_slots(s)[:0]):
            at = slots[first * pr.page::7]
            pr.v[at], pr.codes[1][at], pr.powers[1][at] = 0.0, 0, 255
    _run(pr, 4, window, sinks, hints=dict(max_q=3, max_len=1500, max_prefix=700))


def test_strides_streams_and_hints():
    pr = Problem8([1, 90, 2], [700, 300, 60], groups=[(2, 600)], hkv=2, d=128, page=32, major="head", scales="head", seed=12)
    _run(pr, 8, strided=True, stream=torch.cuda.Stream())
    _run(pr, 8, hints=dict(max_q=1, max_len=5, max_prefix=2))
    _run(pr, 8, hints=dict(max_q=90, max_len=700, max_prefix=600), window=100, sinks=7)


@pytest.mark.parametrize("seqs,own,hkv,d", [(3, 9000, 1, 128), (30, 700, 4, 64), (70, 90, 8, 256), (2, 20000, 1, 64)])
def test_many_keys(seqs, own, hkv, d):
    """Keys that are cut into pieces and joined, workgroups of one wavefront and of two."""
    _run(Problem8([1] * seqs, [own - i for i in range(seqs)], hkv=hkv, d=d, seed=own), 2 * hkv, hints=dict(max_q=1, max_len=own))


def test_prompts_beside_single_tokens():
    _run(Problem8([1, 260, 1, 5], [900, 300, 40, 3000], hkv=2, d=64, dtype="f16", seed=21), 8)
    _run(Problem8([1, 260, 1, 5], [900, 300, 40, 3000], groups=[(4, 1000)], hkv=2, d=128, seed=22), 8, hints=dict(max_q=260, max_len=3000, max_prefix=1000))


def test_slots_beyond_2_31_bytes():
    """Pages of a cache of more than 4 GB: the offsets of codes and powers are 64 bits wide."""
    pages, page, hkv, d = 34000, 64, 8, 256
    k, v = (torch.zeros(pages, page, hkv, d, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((pages, page, hkv), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
    v[pages - 1, :, 3] = 0x38                     # 1.0
    vs[pages - 1, :, 3] = 130                     # times 8
    v[5, :, 3] = 0x40                             # 2.0
    table = torch.tensor([[5, pages - 1]], dtype=torch.int32).cuda()
    step = lambda new: P.KvStep(torch.tensor([0, new], dtype=torch.int32).cuda(), torch.tensor([128], dtype=torch.int32).cuda(), table, page=page, n_tokens=new)
    for new in (1, 50):
        q = torch.zeros(new, hkv, d, dtype=torch.bfloat16, device="cuda")
        out = P.ivf_attend(step(new), P.KvCache(k, v, ks, vs, dtype=torch.bfloat16), q).float().cpu()
        pos = torch.arange(128 - new, 128)
        want = (2.0 * 64 + 8.0 * (pos - 63)) / (pos + 1)
        assert ((out[:, 3] - want[:, None]).abs() <= want[:, None] * 2.0 ** -7).all() and not out[:, [0, 1, 2, 4, 5, 6, 7]].any()

"""ivf_attend against the softmax in 64 bits.  Slots that a token does not see hold NaN wherever a test can arrange
it, and table entries that no key needs name nothing."""
import numpy as np
import pytest
import torch

import paper_2502_20969_amd as P
from answer import Problem

pytestmark = pytest.mark.gpu


def _run(pr, hq, window=0, sinks=0, scale=None, stream=None, hints=None, q=None, strided=False, cache=None):
    scale = pr.d ** -0.5 if scale is None else scale
    q = pr.rows(hq) * 2 if q is None else q
    want, wl, tol = pr.attend(q, scale, window, sinks)
    cache = pr.cache(P) if cache is None else cache
    step = pr.step(P, **(hints or {}))
    if strided:                         # heads before tokens, and room between them
        wide = torch.full((hq, pr.tokens + 3, pr.d + 8), 7.0, dtype=pr.tdtype).cuda()
        qd = wide[:, :pr.tokens, :pr.d].transpose(0, 1)
        qd.copy_(q)
        out = torch.full_like(wide, 7.0)[:, :pr.tokens, :pr.d].transpose(0, 1)
    else:
        qd, out = q.cuda(), torch.full((pr.tokens, hq, pr.d), 7.0, dtype=pr.tdtype).cuda()
    lse = torch.full((pr.tokens, hq), 7.0).cuda()
    need = P.ivf_attend_workspace(step, cache, hq, window, sinks)
    ws = torch.full((need + 16,), 255, dtype=torch.uint8).cuda()        # NaN in whatever is read before it is written
    torch.cuda.synchronize()
    P.ivf_attend(step, cache, qd, out=out, lse=lse, scale=scale, window=window, sinks=sinks, workspace=ws[:need] if need else None, stream=stream)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 255).all()), "the workspace was overrun"
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4], tol[bad][:4])
    none = np.isinf(wl)
    assert np.array_equal(np.isneginf(gl), none)
    # the scores' own error and the roundings of the sum and the logarithm
    np.testing.assert_allclose(gl[~none], wl[~none], rtol=2e-6, atol=1e-4)
    if strided:
        assert bool((out._base[:, pr.tokens:] == 7).all()) and bool((out._base[:, :, pr.d:] == 7).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (8, 1), (14, 2)])
def test_types_and_heads(dtype, d, hq, hkv):
    _run(Problem([1, 2, 5], [77, 130, 5], hkv=hkv, d=d, dtype=dtype, seed=d + hq), hq)


@pytest.mark.parametrize("own", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 2049])
def test_lengths_of_single_tokens(own):
    _run(Problem([1], [own], hkv=1, d=64, seed=own), 4)


@pytest.mark.parametrize("new", [2, 7, 8, 9, 16, 31, 32, 33, 63, 65, 100, 129, 200])
@pytest.mark.parametrize("past", [0, 1, 61])
def test_numbers_of_new_tokens(new, past):
    _run(Problem([new], [new + past], hkv=1, d=64, dtype="f16", seed=new + past), 2)


@pytest.mark.parametrize("page,own_page", [(1, 1), (2, 2), (16, 1), (16, 4), (32, 32), (128, 128), (512, 64)])
@pytest.mark.parametrize("major", ["token", "head"])
def test_pages(page, own_page, major):
    _run(Problem([1, 40, 3], [300, 41, 150], groups=[(2, 70)], hkv=2, d=64, page=page, own_page=own_page, prefix_page=max(1, page // 2),
                 major=major, seed=page + own_page), 4)


@pytest.mark.parametrize("plen", [1, 5, 64, 65, 700, 2500])
@pytest.mark.parametrize("seqs,new", [(1, 1), (5, 1), (40, 1), (3, 4), (2, 90)])
def test_shared_prefix(plen, seqs, new):
    own = [new + 7 * i for i in range(seqs)]
    _run(Problem([new] * seqs, own, groups=[(seqs, plen)], hkv=2, d=64, dtype="f16", seed=plen + seqs), 8)


def test_groups_of_many_kinds():
    """Empty groups, groups without keys, sequences of no group, sequences without tokens, without own keys."""
    new = [1, 1, 0, 3, 2, 1, 1, 50, 1, 0, 1]
    own = [9, 1, 4, 3, 2, 88, 1, 50, 300, 0, 77]
    groups = [(2, 100), (0, 30), (3, 0), (1, 513), (3, 17)]       # sequences 9 and 10 are in none
    _run(Problem(new, own, groups=groups, hkv=2, d=128, seed=4), 6)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 0), (5, 3), (64, 4), (100, 17), (128, 200), (10 ** 6, 4), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("shape", ["tokens", "prompt", "shared"])
def test_windows(window, sinks, shape):
    pr = {"tokens": Problem([1, 2, 1], [500, 90, 3], hkv=1, d=64, seed=1),
          "prompt": Problem([300, 130], [300, 200], hkv=1, d=64, dtype="f16", seed=2),
          "shared": Problem([1, 1, 2, 1], [3, 120, 60, 1], groups=[(3, 333), (1, 40)], hkv=1, d=64, seed=3)}[shape]
    _run(pr, 2, window, sinks)


@pytest.mark.parametrize("window,sinks,new", [(40, 3, 1), (40, 3, 70), (0, 0, 70), (7, 0, 3)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_seen_never_counts(window, sinks, new, value):
    """One key and value after the other of those that some token does not see: the tokens that do not see it keep their
    results; infinities in keys and values both."""
    pr = Problem([new], [new + 150], hkv=1, d=64, dtype="f16", seed=new)
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
        for pool in (cache.k, cache.v):
            pool.view(-1, 1, 64)[int(slots[key])] = value
        out = P.ivf_attend(pr.step(P), cache, q.cuda(), scale=scale, window=window, sinks=sinks).double().cpu().numpy()
        assert (np.abs(out - want) <= tol)[~sees].all(), key
        # and those that see it get what the formula says: nothing finite
        assert not np.isfinite(out[sees]).all() or not sees.any()


def test_a_value_that_is_not_finite_reaches_those_who_see_it():
    """An infinite value and finite keys: the result is infinite in that element, finite in the others."""
    pr = Problem([70], [150], hkv=1, d=64, dtype="bf16", seed=8)
    q = pr.rows(1)
    slot, key, e = None, 120, 5
    slot = int(pr.own_slots(0)[key])
    pr.v[slot, 0, e] = np.inf
    cache = pr.cache(P)
    out = P.ivf_attend(pr.step(P), cache, q.cuda()).float().cpu()[:, 0]
    sees = torch.arange(80, 150) >= key
    assert torch.isposinf(out[sees, e]).all() and torch.isfinite(out[~sees]).all()
    keep = [i for i in range(64) if i != e]
    assert torch.isfinite(out[:, keep]).all()


def test_rows_that_see_nothing():
    """Fewer own keys than new tokens, and none at all: zeros and -inf."""
    pr = Problem([3, 40, 2, 1], [3, 40, 2, 5], hkv=1, d=64, seed=6)
    pr.own = [1, 10, 0, 5]
    _run(pr, 2)
    _run(pr, 2, window=3, sinks=1)


def test_extreme_scores():
    """Scores in the thousands, and equal ones: the largest decide, nothing overflows."""
    pr = Problem([1, 60], [400, 300], hkv=1, d=64, dtype="bf16", seed=7)
    _run(pr, 2, q=pr.rows(2) * 300)
    _run(pr, 2, q=pr.rows(2) * 0)
    _run(pr, 2, scale=1e-6)


def test_rising_scores():
    """The maximum rises with every key, by little and by much, so that whatever was summed is scaled again and again."""
    for rise in (0.05, 0.5, 3.0):
        pr = Problem([1, 33], [700, 700], hkv=1, d=64, dtype="f16", seed=3)
        for s in range(2):
            slots = pr.own_slots(s)
            pr.k[slots] = 0
            pr.k[slots, 0, 0] = torch.from_numpy(np.arange(700) * rise / 8).half().double().numpy()
        q = torch.zeros(34, 1, 64, dtype=torch.float16)
        q[..., 0] = 8.0
        _run(pr, 1, q=q, scale=1.0)


def test_long_tail_of_small_weights():
    """One key above 30,000 others that weigh 2^-16 of it each: together a third of the sum."""
    n = 30000
    pr = Problem([1], [n], hkv=1, d=64, page=64, dtype="f16", seed=3)
    slots = pr.own_slots(0)
    pr.k[slots] = 0
    pr.k[slots[17], 0, 0] = 11.09375
    pr.v[slots] = 1.0
    pr.v[slots[17]] = 0.0
    q = torch.zeros(1, 1, 64, dtype=torch.float16)
    q[..., 0] = 1.0
    _run(pr, 1, q=q, scale=1.0)


@pytest.mark.parametrize("hints", [dict(max_q=1, max_len=1, max_prefix=1), dict(max_q=10 ** 6, max_len=10 ** 6, max_prefix=10 ** 6), dict(max_q=90, max_len=400, max_prefix=900)])
def test_hints_do_not_change_results(hints):
    _run(Problem([1, 90, 3, 1], [400, 91, 5, 1], groups=[(2, 900), (2, 33)], hkv=2, d=64, seed=12), 4, hints=hints)


@pytest.mark.parametrize("dtype,new,own,groups", [("f16", [1, 2], [90, 200], [(2, 300)]), ("bf16", [150], [150], [])])
def test_strides(dtype, new, own, groups):
    _run(Problem(new, own, groups=groups, hkv=2, d=64, dtype=dtype, seed=13), 4, strided=True)


def test_on_another_stream():
    _run(Problem([1, 60], [90, 200], groups=[(2, 300)], hkv=2, d=64, seed=14), 4, stream=torch.cuda.Stream())


def test_many_sequences():
    n = 600
    _run(Problem([1] * n, [1 + (i * 37) % 90 for i in range(n)], groups=[(200, 64), (300, 5)], hkv=1, d=64, seed=15), 2)


def test_one_long_sequence_among_short_ones():
    own = [3, 9000, 1, 20]
    _run(Problem([1] * 4, own, hkv=1, d=64, page=64, seed=16), 4, hints=dict(max_q=1, max_len=9000))


def test_offsets_beyond_32_bits():
    pages, page, hkv, d = 2 ** 14 + 3, 128, 8, 256           # 2^32 elements and some
    k = torch.zeros(pages, page, hkv, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    last, mid = pages - 1, 2 ** 13 + 1
    for pg in (last, mid):
        k[pg] = torch.randn(page, hkv, d).bfloat16()
        v[pg] = torch.randn(page, hkv, d).bfloat16()
    i32 = lambda a: torch.tensor(a, dtype=torch.int32).cuda()
    for new in (1, 100):
        step = P.KvStep(i32([0, new]), i32([200]), i32([[mid, last]]), page=page, n_tokens=new)
        q = torch.randn(new, 8, d).bfloat16()
        out = P.ivf_attend(step, P.KvCache(k, v), q.cuda()).double().cpu()
        kk, vv = (torch.cat([x[mid], x[last]])[:200].double().cpu() for x in (k, v))
        for h in (0, 7):
            sc = q[:, h].double() @ kk[:, h].T / 16.0
            sc = sc.masked_fill(torch.arange(200)[None] > 200 - new + torch.arange(new)[:, None], -float("inf"))
            w = torch.softmax(sc, 1)
            assert bool(((out[:, h] - w @ vv[:, h]).abs() <= (2 * 2.0 ** -8 + 1e-4) * (w @ vv[:, h].abs()) + 1e-6).all())


def test_the_same_twice():
    """Nothing depends on the order in which workgroups end."""
    pr = Problem([1] * 20, [50 + 40 * i for i in range(20)], groups=[(20, 5000)], hkv=2, d=128, seed=17)
    cache, step, q = pr.cache(P), pr.step(P), pr.rows(8).cuda()
    first = P.ivf_attend(step, cache, q)
    for _ in range(5):
        assert torch.equal(P.ivf_attend(step, cache, q).view(torch.int16), first.view(torch.int16))


@pytest.mark.parametrize("new", [1, 40])
def test_in_a_graph(new):
    """Replays follow the lengths that the arrays hold by then, eager calls in between."""
    pr = Problem([new] * 3, [500, 300, 200], groups=[(3, 400)], hkv=2, d=64, page=16, seed=18)
    cache, step, q = pr.cache(P), pr.step(P), pr.rows(4).cuda()
    lens = step._keep[1]
    out = torch.empty_like(q)
    need = P.ivf_attend_workspace(step, cache, 4)
    ws = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")
    P.ivf_attend(step, cache, q, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.ivf_attend(step, cache, q, out=out, workspace=ws)
    for i in range(4):
        lens.copy_(torch.tensor([500 - 100 * i, 300 - 7 * i, 41 + i]))
        q.copy_(torch.randn(q.shape))
        want = P.ivf_attend(step, cache, q)
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("dtype,d", [("f16", 64), ("bf16", 128), ("f16", 256)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 17), (900, 0)])
@pytest.mark.parametrize("new", [[1] * 9, [3, 1, 0, 2, 1, 1, 5, 1, 1], [40, 1, 1, 1, 60, 1, 1, 1, 1]])
def test_long_prefixes_of_several_sequences(dtype, d, window, sinks, new):
    """Prefixes that are read for their whole group at once, beside one without keys and a sequence in no group."""
    own = [n + 13 * i for i, n in enumerate(new)]
    _run(Problem(new, own, groups=[(4, 601), (2, 0), (2, 1500)], hkv=2, d=d, dtype=dtype, seed=d + window), 8, window, sinks)


@pytest.mark.parametrize("page,own_page,prefix_page", [(1, 1, 1), (16, 1, 16), (64, 64, 8)])
def test_long_prefixes_in_pages(page, own_page, prefix_page):
    _run(Problem([1] * 40, [5 + i for i in range(40)], groups=[(30, 1000), (10, 999)], hkv=1, d=128, page=page, own_page=own_page,
                 prefix_page=prefix_page, seed=page), 8)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite_count_where_they_are_seen(value):
    """A prompt long enough for several wavefronts: tokens before the value keep theirs, others take it."""
    pr = Problem([200], [330], hkv=1, d=128, page=16, seed=21)
    key = 230
    pr.v[pr.own_slots(0)[key], 0, 5] = value
    step, cache = pr.step(P), pr.cache(P)
    q = pr.rows(2)
    got = P.ivf_attend(step, cache, q.cuda(), scale=pr.d ** -0.5).double().cpu().numpy()
    sees = np.arange(130, 330) >= key
    assert np.isfinite(got[~sees]).all() and np.isfinite(np.delete(got, 5, axis=2)).all()
    assert (np.isnan(got[sees][:, :, 5]) if value != value else got[sees][:, :, 5] == value).all()


@pytest.mark.parametrize("dtype,d", [("f16", 96), ("bf16", 128), ("f16", 256)])
@pytest.mark.parametrize("window,sinks,groups", [(0, 0, []), (9, 4, [(300, 40)]), (0, 0, [(40, 0), (4, 600)])])
def test_many_short_sequences(dtype, d, window, sinks, groups):
    n = 520
    _run(Problem([1 + i % 3 // 2 for i in range(n)], [2 + (i * 37) % 70 for i in range(n)], groups=groups, hkv=1, d=d, dtype=dtype, seed=17), 2, window, sinks)


def test_many_long_pieces_of_wide_heads():
    _run(Problem([1] * 64, [900 + i for i in range(64)], groups=[(16, 700)] * 4, hkv=8, d=256, page=64, seed=18), 8)


@pytest.mark.parametrize("hints", [dict(), dict(max_q=260, max_len=400)])
def test_prompts_among_single_tokens(hints):
    """Sequences of very different numbers of tokens, some with none, more of them than a wavefront has lanes."""
    new = [(260 if i % 50 == 3 else 129 if i % 70 == 66 else i % 3) for i in range(150)]
    _run(Problem(new, [n + i for i, n in enumerate(new)], groups=[(60, 33)], hkv=1, d=64, dtype="f16", seed=19), 2, hints=hints)


def test_new_tensors_do_not_meet_pending_work():
    """The calls' own tensors on another stream are not memory that the current stream still writes."""
    pr = Problem([1] * 8, [40] * 8, hkv=2, d=64, dtype="f16", seed=20)
    q = pr.rows(8)
    want, _, tol = pr.attend(q, 0.125)
    step, cache, qd, other = pr.step(P), pr.cache(P), q.cuda(), torch.cuda.Stream()
    logits, scores = torch.randn(4, 2, 500).cuda(), torch.zeros(4, 2).cuda()
    plain = P.ivf_beam_step(logits, scores)
    torch.cuda.synchronize()
    blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (qd.nbytes, 96, 8, 4096, 16384)]
    torch.cuda._sleep(100_000_000)
    for b in blocks:
        b.fill_(123)
    del blocks, b
    out = P.ivf_attend(step, cache, qd, scale=0.125, stream=other)
    beams = P.ivf_beam_step(logits, scores, stream=other)
    torch.cuda.synchronize()
    assert (abs(out.double().cpu().numpy() - want) <= tol).all()
    assert all(torch.equal(x, y) for x, y in zip(beams, plain))


@pytest.mark.parametrize("new,own,groups", [([2], [30], []), ([1], [3000], []), ([1] * 3, [700, 5, 90], [(2, 40)]), ([150], [150], []), ([130], [5000], []),
                                            ([1] * 4, [9, 300, 1, 40], [(4, 700)]), ([40] * 3, [40, 90, 41], [(2, 1500)]), ([200, 1, 1], [200, 3000, 900], [])])
@pytest.mark.parametrize("dtype,d", [("f16", 64), ("bf16", 128), ("bf16", 256)])
def test_queries_that_are_not_numbers(new, own, groups, dtype, d):
    """Not a number for the rows whose query is none, in one piece or many; the other rows keep theirs."""
    pr = Problem(new, own, groups=groups, hkv=2, d=d, dtype=dtype, seed=22)
    q = pr.rows(4) * 2
    want, wl, tol = pr.attend(q, pr.d ** -0.5)
    bad = np.zeros((pr.tokens, 4), bool)
    bad[0, 1] = bad[-1, 3] = bad[pr.tokens // 2, 0] = True
    q[torch.from_numpy(bad)] = float("nan")
    q[0, 1] = 1.0
    q[0, 1, 7] = float("nan")                               # one element is enough
    step, cache = pr.step(P), pr.cache(P)
    lse = torch.empty(pr.tokens, 4).cuda()
    got = P.ivf_attend(step, cache, q.cuda(), lse=lse).double().cpu().numpy()
    lse = lse.cpu().numpy()
    assert np.isnan(got[bad]).all() and np.isnan(lse[bad]).all()
    assert (np.abs(got - want) <= tol)[~bad].all()
    np.testing.assert_allclose(lse[~bad], wl[~bad], rtol=2e-6, atol=1e-4)


@pytest.mark.parametrize("new,own,key", [(1, 40, 39), (1, 3000, 2100), (70, 200, 150), (130, 5000, 4700)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_nothing_is_finite_where_a_key_that_is_not_finite_is_seen(new, own, key, value):
    """All elements of a key that is not finite: scores of both signs of infinity, or NaN, and so NaN in every element."""
    pr = Problem([new], [own], hkv=1, d=64, dtype="f16", seed=23)
    q = pr.rows(2) * 2
    want, _, tol = pr.attend(q, pr.d ** -0.5)
    cache = pr.cache(P)
    cache.k.view(-1, 1, 64)[int(pr.own_slots(0)[key])] = value
    got = P.ivf_attend(pr.step(P), cache, q.cuda()).double().cpu().numpy()
    sees = np.arange(own - new, own) >= key
    assert np.isnan(got[sees]).all()
    assert (np.abs(got - want) <= tol)[~sees].all()


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 40, 2 ** 30])
@pytest.mark.parametrize("sinks", [0, 1, 2 ** 31 - 1])
def test_windows_beyond_all_keys_where_rows_see_nothing(window, sinks):
    """Tokens at positions below zero beside others that see keys, under windows that reach beyond every key."""
    pr = Problem([3, 40, 2, 1, 70], [3, 40, 2, 5, 70], hkv=1, d=64, seed=6)
    pr.own = [1, 10, 0, 5, 33]
    _run(pr, 2, window, sinks)
    pr = Problem([3, 4, 40], [3, 4, 40], groups=[(2, 600)], hkv=1, d=64, seed=7)
    pr.own = [1, 2, 9]
    _run(pr, 2, window, sinks)


def test_as_many_keys_as_positions_count():
    """A prefix and own keys that together pass the largest position: of both the first keys count, and a window finds the last."""
    page, d = 1 << 14, 64
    k = torch.zeros(1, page, 1, d, dtype=torch.bfloat16, device="cuda")
    v = torch.ones_like(k)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32).cuda()
    table = torch.zeros(1, 1 << 16, dtype=torch.int32, device="cuda")
    step = P.KvStep(i32([0, 2]), i32([2 ** 31 - 1]), table, page=page, n_tokens=2, group_off=i32([0, 1]), prefix_lens=i32([2 ** 31 - 1]), prefix_table=table)
    lse = torch.empty(2, 1, device="cuda")
    out = P.ivf_attend(step, P.KvCache(k, v), torch.zeros(2, 1, d, dtype=torch.bfloat16, device="cuda"), lse=lse, window=100, sinks=3)
    assert bool((out == 1).all())
    np.testing.assert_allclose(lse.cpu().numpy(), np.log(103.0), rtol=1e-6)


@pytest.mark.parametrize("dtype,d", [("f16", 64), ("bf16", 96), ("bf16", 128), ("f16", 256)])
@pytest.mark.parametrize("new,own,groups", [([300, 1, 0, 2, 1, 8], [300, 3000, 9, 5, 1400, 700], []), ([150, 1, 9, 8, 1], [2500, 3000, 2000, 2000, 40], []),
                                            ([150, 1, 9, 8, 1, 1], [180, 3000, 2000, 2000, 40, 0], [(2, 1300), (2, 0), (1, 40)]),
                                            ([60, 1, 1, 0, 2], [2500, 1, 2500, 0, 90], [(4, 2600)])])
@pytest.mark.parametrize("hints", [False, True])
def test_prompts_beside_long_single_tokens(dtype, d, new, own, groups, hints):
    """Few rows whose keys are cut into pieces beside many whose keys are not, or are too; with and without a shared prefix."""
    pr = Problem(new, own, groups=groups, hkv=2, d=d, dtype=dtype, seed=24)
    _run(pr, 8, hints=dict(max_q=max(new), max_len=max(own), max_prefix=max([p for _, p in groups] + [0])) if hints else {})


@pytest.mark.parametrize("groups", [[], [(300, 700), (200, 0)]])
def test_many_single_tokens_beside_prompts(groups):
    """More places of few rows than wavefronts that join."""
    n = 1100
    new = [40 if i % 100 == 7 else i % 4 for i in range(n)]
    _run(Problem(new, [m + (1500 if i % 97 == 5 else i % 30) for i, m in enumerate(new)], groups=groups, hkv=1, d=64, dtype="f16", seed=25), 8, hints=dict(max_q=40, max_len=1503))

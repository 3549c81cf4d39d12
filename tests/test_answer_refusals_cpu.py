"""What the calls of the paged cache, its attention and the beam step refuse, before any work is enqueued (no GPU)."""
import ctypes as C

import pytest

import paper_2502_20969_amd as P
from paper_2502_20969_amd.binding import BeamStateArg, KvCacheArg, KvStepArg, RowsArg

OK = 1 << 20            # an aligned address that no test lets a kernel see


def _cache(**kw):
    a = KvCacheArg(OK, OK, 10, 16 * 2 * 64, 2 * 64, 64, 16, 2, 64, P.IVF_BF16)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _step(**kw):
    a = KvStepArg(OK, OK, OK, 4)
    a.n_seq, a.n_tokens, a.page = 2, 3, 16
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _rows(data=OK, t=128, h=64):
    return RowsArg(data, t, h)


BAD_CACHE = [dict(k=None), dict(v=None), dict(k=OK + 8), dict(v=OK + 2), dict(n_pages=0), dict(n_heads=0), dict(d=0), dict(page=0), dict(page=12),
             dict(page=-16), dict(page_stride=2044), dict(token_stride=4), dict(head_stride=7), dict(dtype=P.IVF_F32), dict(dtype=9)]
BAD_STEP = [dict(q_off=None), dict(len=None), dict(table=None), dict(table_stride=0), dict(n_seq=0), dict(n_tokens=0), dict(page=3), dict(page=32),
            dict(page=0), dict(max_q=-1), dict(max_len=-1), dict(max_prefix=-1), dict(n_groups=-1), dict(n_groups=1), dict(n_groups=1, group_off=OK, prefix_len=OK),
            dict(n_groups=1, group_off=OK, prefix_len=OK, prefix_table=OK, prefix_stride=4, prefix_page=0),
            dict(n_groups=1, group_off=OK, prefix_len=OK, prefix_table=OK, prefix_stride=0, prefix_page=16)]


def _append(step=None, cache=None, k=None, v=None, rotary=OK, n_pos=10, rot=64, q=None, q_out=None, hq=0):
    return P.load().ivf_kv_append(step or _step(), cache or _cache(), k or _rows(), v or _rows(), rotary, n_pos, rot, 0, None, q, q_out, hq, None)


def _attend(step=None, cache=None, q=None, out=None, hq=4, scale=0.125, window=0, sinks=0, ws=OK, nbytes=1 << 40):
    return P.load().ivf_attend(step or _step(), cache or _cache(), q or _rows(), hq, out or _rows(), None, scale, window, sinks, ws, nbytes, None)


@pytest.mark.parametrize("kw", BAD_CACHE)
def test_caches(kw):
    n = C.c_size_t()
    assert _append(cache=_cache(**kw)) == -1
    assert _attend(cache=_cache(**kw)) == -1
    assert P.load().ivf_attend_workspace(_step(), _cache(**kw), 4, 0, 0, C.byref(n)) == -1


@pytest.mark.parametrize("kw", BAD_STEP)
def test_steps(kw):
    n = C.c_size_t()
    assert _append(step=_step(**kw)) == -1
    assert _attend(step=_step(**kw)) == -1
    assert P.load().ivf_attend_workspace(_step(**kw), _cache(), 4, 0, 0, C.byref(n)) == -1


@pytest.mark.parametrize("rows", [RowsArg(None, 128, 64), RowsArg(OK + 4, 128, 64), RowsArg(OK, 132, 64), RowsArg(OK, 128, 60)])
def test_rows(rows):
    assert _append(k=rows) == -1 and _append(v=rows) == -1
    assert _append(q=rows, q_out=_rows(), hq=2) == -1 and _append(q=_rows(), q_out=rows, hq=2) == -1
    assert _attend(q=rows) == -1 and _attend(out=rows) == -1


def test_appends():
    L = P.load()
    assert _append(q=_rows(), hq=2) == -1 and _append(hq=2) == -1 and _append(q=_rows(), q_out=_rows(), hq=0) == -1 and _append(hq=-1) == -1
    assert _append(rot=24) == -1 and _append(rot=80) == -1 and _append(rot=-16) == -1 and _append(rot=0) == -1
    assert _append(rotary=None) == -1 and _append(n_pos=0) == -1
    assert _append(cache=_cache(d=72)) == -1
    assert _append(cache=_cache(d=1040), rot=0, rotary=None) == -5
    assert L.ivf_kv_append(None, _cache(), _rows(), _rows(), None, 0, 0, 0, None, None, None, 0, None) == -1
    assert L.ivf_kv_append(_step(), None, _rows(), _rows(), None, 0, 0, 0, None, None, None, 0, None) == -1
    assert L.ivf_kv_append(_step(), _cache(), None, _rows(), None, 0, 0, 0, None, None, None, 0, None) == -1
    assert b"k is NULL" in L.ivf_last_error()


def test_attention():
    L = P.load()
    n = C.c_size_t()
    for d in (32, 80, 112, 512):
        assert _attend(cache=_cache(d=d)) == -5
    assert _attend(hq=3) == -1 and _attend(hq=0) == -1 and _attend(window=-1) == -1 and _attend(sinks=-1) == -1
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert _attend(scale=scale) == -1
    assert _attend(ws=OK + 4) == -1
    assert L.ivf_attend_workspace(_step(), _cache(), 4, 0, 0, None) == -1
    assert L.ivf_attend(None, _cache(), _rows(), 4, _rows(), None, 1.0, 0, 0, OK, 1 << 40, None) == -1
    assert L.ivf_attend(_step(), None, _rows(), 4, _rows(), None, 1.0, 0, 0, OK, 1 << 40, None) == -1
    assert L.ivf_attend(_step(), _cache(), None, 4, _rows(), None, 1.0, 0, 0, OK, 1 << 40, None) == -1
    assert L.ivf_attend_workspace(_step(), _cache(), 4, 0, 0, C.byref(n)) == 0
    if n.value:
        assert _attend(nbytes=n.value - 1) == -1 and _attend(ws=None) == -1
        assert b"workspace" in L.ivf_last_error()


def test_beam_steps():
    L = P.load()
    n = C.c_size_t()
    for sizes in ((0, 2, 10, 2), (1, 0, 10, 2), (1, 2, 0, 2), (1, 2, 10, 0)):
        assert L.ivf_beam_workspace(*sizes, C.byref(n)) == -1
    assert L.ivf_beam_workspace(1, 65, 10, 2, C.byref(n)) == -5 and L.ivf_beam_workspace(1, 2, 10, 65, C.byref(n)) == -5
    assert L.ivf_beam_workspace(2 ** 30, 64, 10, 2, C.byref(n)) == -5
    assert L.ivf_beam_workspace(1, 2, 10, 2, None) == -1
    assert L.ivf_beam_workspace(3, 2, 10, 2, C.byref(n)) == 0

    def call(logits=OK, stride=10, dtype=0, p=3, scores=OK, out=OK, parent=OK, token=OK, fin=OK, states=None, n_states=0, ws=OK, nbytes=n.value):
        return L.ivf_beam_step(logits, stride, dtype, p, 2, 10, scores, None, 2, 2, out, parent, token, fin, states, n_states, ws, nbytes, None)

    for kw in (dict(logits=None), dict(scores=None), dict(out=None), dict(parent=None), dict(token=None), dict(fin=None), dict(stride=9), dict(dtype=3),
               dict(dtype=-1), dict(logits=OK + 2), dict(logits=OK + 1, dtype=1), dict(n_states=-1), dict(n_states=1), dict(ws=None), dict(ws=OK + 8),
               dict(nbytes=n.value - 1), dict(p=0)):
        assert call(**kw) == -1, kw
    states = (BeamStateArg * 9)(*[BeamStateArg(OK, OK, 8, 8, 8)] * 9)
    assert call(states=states, n_states=9) == -5
    for bad in (BeamStateArg(None, OK, 8, 8, 8), BeamStateArg(OK, None, 8, 8, 8), BeamStateArg(OK, OK, 0, 8, 8), BeamStateArg(OK, OK, 8, -8, 8), BeamStateArg(OK, OK, 8, 8, 4)):
        assert call(states=(BeamStateArg * 1)(bad), n_states=1) == -1


@pytest.mark.parametrize("kw", [dict(page_stride=1 << 30), dict(token_stride=1 << 31), dict(n_pages=1 << 40)])
def test_caches_beyond_the_limits(kw):
    cache = _cache(**kw)
    assert _append(cache=cache) == -5 and _attend(cache=cache) == -5


def _need(n_seq, n_tokens, hq, hkv, d, keys, page=64, groups=0, prefix=0, hints=(0, 0, 0)):
    """Workspace of steps whose tables have room for `keys` own and `prefix` shared keys."""
    n = C.c_size_t()
    step = _step(n_seq=n_seq, n_tokens=n_tokens, page=page, table_stride=-(-keys // page), max_q=hints[0], max_len=hints[1])
    if groups:
        step.n_groups, step.group_off, step.prefix_len, step.prefix_table = groups, OK, OK, OK
        step.prefix_stride, step.prefix_page, step.max_prefix = -(-prefix // page), page, hints[2]
    cache = _cache(page=page, n_heads=hkv, d=d, n_pages=1 << 20, page_stride=page * hkv * d, token_stride=hkv * d, head_stride=d)
    assert P.load().ivf_attend_workspace(step, cache, hq, 0, 0, C.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("sizes", [dict(n_seq=3, n_tokens=16002, hq=32, hkv=8, d=128, keys=60000, hints=(16000, 60000, 0)),
                                   dict(n_seq=8, n_tokens=32007, hq=64, hkv=8, d=128, keys=100000, hints=(32000, 100000, 0)),
                                   dict(n_seq=3, n_tokens=15000, hq=32, hkv=8, d=128, keys=131072),
                                   dict(n_seq=1, n_tokens=16000, hq=32, hkv=8, d=128, keys=60000, hints=(1, 60000, 0))])
def test_prompts_beside_single_tokens_need_little_workspace(sizes):
    """Rows whose keys are not cut need no room for the pieces of those whose are.  64 MB are the pieces of 32 rows of 128 for
    each of 4096 workgroups."""
    assert _need(**sizes) <= 128 << 20


def test_workspaces_are_bounded():
    """A row's keys are cut only as far as places on the chip are free: 4096 pieces of 32 rows or 512 of 128, of the own and of the prefix's keys, beside one
    piece a row or tile of each."""
    import random
    rng = random.Random(5)
    for _ in range(4000):
        n_seq, hkv, d = round(2 ** rng.uniform(0, 11)), rng.choice([1, 2, 8, 16]), rng.choice([64, 96, 128, 256])
        hq, n_tokens = hkv * rng.choice([1, 2, 7, 8, 40]), max(1, round(2 ** rng.uniform(0, 16)))
        keys, groups = round(2 ** rng.uniform(0, 20)), rng.choice([0, 1, max(1, n_seq // 4), n_seq])
        prefix = round(2 ** rng.uniform(0, 17)) if groups else 0
        hints = tuple(rng.choice([0, 1, round(2 ** rng.uniform(0, 17))]) for _ in range(3))
        sums = 2 * 4096 * 33 + 2 * 512 * 129 + 2 * n_tokens * hq + 2 * 129 * hkv * (n_seq + groups)
        assert _need(n_seq, n_tokens, hq, hkv, d, keys, groups=groups, prefix=prefix, hints=hints) <= sums * (4 * d + 8), (n_seq, n_tokens, hq, hkv, d, keys, groups, prefix, hints)


def test_vocabularies_beyond_the_limit():
    """Tokens are counted in 32 bits, up to a tile past the last."""
    L = P.load()
    n = C.c_size_t()
    for vocab in (2 ** 30 + 1, 2 ** 31 - 8192, 2 ** 31 - 1):
        assert L.ivf_beam_workspace(1, 1, vocab, 1, C.byref(n)) == -5
        assert L.ivf_beam_step(OK, vocab, 0, 1, 1, vocab, OK, None, 2, 1, OK, OK, OK, OK, None, 0, OK, 1 << 40, None) == -5
    assert L.ivf_beam_workspace(1, 1, 2 ** 30, 1, C.byref(n)) == 0 and 0 < n.value < 1 << 20


def test_what_is_read_is_not_written():
    """A state's destination that begins where the state does, and outputs in the place of inputs that other workgroups may still read."""
    L = P.load()
    n = C.c_size_t()
    assert L.ivf_beam_workspace(3, 2, 10, 2, C.byref(n)) == 0

    def call(out=OK, fin=2 * OK, state=None):
        states = (BeamStateArg * 1)(state) if state else None
        return L.ivf_beam_step(OK, 10, 0, 3, 2, 10, 3 * OK, 4 * OK, 2, 2, out, 5 * OK, 6 * OK, fin, states, 1 if state else 0, OK, n.value, None)
    assert call(out=3 * OK) == -1 and b"scores" in L.ivf_last_error()
    assert call(fin=4 * OK) == -1 and b"done" in L.ivf_last_error()
    assert call(state=BeamStateArg(7 * OK, 7 * OK, 8, 8, 8)) == -1 and b"state 0" in L.ivf_last_error()


@pytest.mark.parametrize("n_tokens,hq", [(3, 4), (3, 2), (600, 4)])
def test_workspaces_of_attention_are_checked(n_tokens, hq):
    """Steps whose keys are cut into pieces: a workspace that is missing or a byte too small."""
    n = C.c_size_t()
    step, cache = _step(table_stride=1000, n_tokens=n_tokens), _cache(n_pages=4000)
    assert P.load().ivf_attend_workspace(step, cache, hq, 0, 0, C.byref(n)) == 0 and n.value > 0
    for kw in (dict(nbytes=n.value - 1), dict(nbytes=0), dict(ws=None)):
        assert _attend(step=step, cache=cache, hq=hq, **kw) == -1 and b"workspace" in P.load().ivf_last_error()

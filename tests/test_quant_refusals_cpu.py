"""What the calls of a quantised cache and of drafted tokens refuse, before any work is enqueued (no GPU)."""
import ctypes as C

import pytest
import torch

import paper_2502_20969_amd as P
import paper_2502_20969_amd.binding as B
from paper_2502_20969_amd.binding import KvCacheArg, KvStepArg, RowsArg
from test_answer_devices_cpu import On, _i32, _step as _on_step, _stream, _zeros

OK = 1 << 20            # an aligned address that no test lets a kernel see


def _cache(**kw):
    a = KvCacheArg(OK, OK, 10, 16 * 2 * 64, 2 * 64, 64, 16, 2, 64, P.IVF_E4M3, OK, OK, 32, 2, 1, P.IVF_BF16)
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


def _append(step=None, cache=None, k=None, v=None):
    return P.load().ivf_kv_append(step or _step(), cache or _cache(), k or _rows(), v or _rows(), OK, 10, 64, 0, None, None, None, 0, None)


def _attend(step=None, cache=None, q=None, out=None, ws=OK, nbytes=1 << 40):
    return P.load().ivf_attend(step or _step(), cache or _cache(), q or _rows(), 4, out or _rows(), None, 0.125, 0, 0, ws, nbytes, None)


def _read(step=None, cache=None, off=OK, rows=3, k=None, v=None):
    return P.load().ivf_kv_read(step or _step(), cache or _cache(), off, None, rows, k or _rows(), v or _rows(), None)


BAD = [dict(k_scale=None), dict(v_scale=None), dict(row_dtype=0), dict(row_dtype=P.IVF_E4M3), dict(row_dtype=-1), dict(page_stride=2040), dict(token_stride=136),
       dict(head_stride=72), dict(k=OK + 8), dict(v=None), dict(page=12), dict(n_pages=0), dict(dtype=4), dict(dtype=P.IVF_F32)]


@pytest.mark.parametrize("kw", BAD)
def test_caches(kw):
    n = C.c_size_t()
    assert _append(cache=_cache(**kw)) == -1 and _attend(cache=_cache(**kw)) == -1 and _read(cache=_cache(**kw)) == -1
    assert P.load().ivf_attend_workspace(_step(), _cache(**kw), 4, 0, 0, C.byref(n)) == -1


@pytest.mark.parametrize("kw", [dict(scale_page_stride=1 << 30), dict(scale_token_stride=-(1 << 31)), dict(page_stride=1 << 30), dict(token_stride=1 << 31), dict(n_pages=1 << 40)])
def test_caches_beyond_the_limits(kw):
    assert _append(cache=_cache(**kw)) == -5 and _attend(cache=_cache(**kw)) == -5 and _read(cache=_cache(**kw)) == -5


def test_16_bit_caches_need_no_scales():
    """What stands behind dtype is not looked at for them."""
    n = C.c_size_t()
    cache = _cache(dtype=P.IVF_F16, k_scale=None, v_scale=None, row_dtype=77, scale_page_stride=1 << 40)
    assert P.load().ivf_attend_workspace(_step(), cache, 4, 0, 0, C.byref(n)) == 0
    assert _read(cache=cache, rows=0) == -1 and b"n_rows" in P.load().ivf_last_error()


def test_widths():
    assert _append(cache=_cache(d=72)) == -1 and _append(cache=_cache(d=1040)) == -5
    for d in (32, 80, 112, 512):
        assert _attend(cache=_cache(d=d)) == -5


def test_reads():
    for rows in (RowsArg(None, 128, 64), RowsArg(OK + 4, 128, 64), RowsArg(OK, 132, 64), RowsArg(OK, 128, 60)):
        assert _read(k=rows) == -1 and _read(v=rows) == -1
    assert _read(off=None) == -1 and _read(rows=0) == -1 and _read(rows=-1) == -1 and _read(rows=1 << 31) == -5
    assert _read(cache=_cache(d=40)) == -1 and _read(cache=_cache(n_heads=1 << 24, d=1024)) == -5
    assert _read(step=_step(len=None)) == -1 and _read(step=_step(n_seq=0)) == -1
    L = P.load()
    assert L.ivf_kv_read(None, _cache(), OK, None, 3, _rows(), _rows(), None) == -1 and L.ivf_kv_read(_step(), None, OK, None, 3, _rows(), _rows(), None) == -1
    assert L.ivf_kv_read(_step(), _cache(), OK, None, 3, None, _rows(), None) == -1


def _verify(step=None, logits=OK, stride=100, dtype=1, vocab=100, scale=1.0, tokens=2 * OK, uniform=3 * OK, draft=None, draft_stride=100, accepted=4 * OK,
            follows=5 * OK, lens=6 * OK, ws=OK, nbytes=1 << 40):
    return P.load().ivf_verify_draft(step or _step(), logits, stride, dtype, vocab, scale, tokens, uniform, draft, draft_stride, accepted, follows, lens, ws,
                                     nbytes, None)


def test_verifications():
    L = P.load()
    n = C.c_size_t()
    for sizes in ((0, 2, 10), (2, 0, 10), (2, 2, 0)):
        assert L.ivf_verify_workspace(*sizes, C.byref(n)) == -1
    for sizes in ((2, 2, 2 ** 30 + 1), (2 ** 24 + 1, 2, 10), (2, 2 ** 24 + 1, 10)):
        assert L.ivf_verify_workspace(*sizes, C.byref(n)) == -5
    assert L.ivf_verify_workspace(2, 3, 10, None) == -1 and L.ivf_verify_workspace(2, 3, 100, C.byref(n)) == 0 and n.value > 0
    for kw in (dict(logits=None), dict(tokens=None), dict(accepted=None), dict(follows=None), dict(lens=None), dict(stride=99), dict(dtype=3), dict(dtype=-1),
               dict(logits=OK + 1), dict(logits=OK + 2, dtype=0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(uniform=None),
               dict(draft=OK, draft_stride=99), dict(draft=OK + 2), dict(ws=None), dict(ws=OK + 8), dict(nbytes=n.value - 1), dict(vocab=0),
               dict(step=_step(q_off=None)), dict(step=_step(len=None)), dict(step=_step(n_seq=0)), dict(step=_step(n_tokens=0))):
        assert _verify(**kw) == -1, kw
    assert _verify(vocab=2 ** 30 + 1, stride=2 ** 31) == -5
    assert L.ivf_verify_draft(None, OK, 100, 1, 100, 1.0, OK, OK, None, 0, OK, OK, OK, OK, 1 << 40, None) == -1


def test_launches_beyond_the_limits():
    """A launch has fewer than 2^32 threads: 512 a sequence, 256 for four tiles of 2048 entries of a row, 256 for sixteen rows that are read back, 256 a token
    that is appended."""
    L, n = P.load(), C.c_size_t()
    for sizes, want in (((2 ** 23, 2, 10), -5), ((2 ** 23 - 1, 2, 10), 0), ((2, 2 ** 24, 10), -5), ((2, 2 ** 24 - 1, 10), 0), ((2, 2 ** 23, 8193), -5),
                        ((2, 2 ** 23 - 1, 8193), 0), ((2 ** 22, 2, 3 * 8192 + 1), -5), ((2 ** 22 - 1, 2, 4 * 8192), 0), ((2, 127, 2 ** 30), 0), ((2, 128, 2 ** 30), -5)):
        assert L.ivf_verify_workspace(*sizes, C.byref(n)) == want, sizes
    for step in (_step(n_seq=2 ** 23), _step(n_tokens=2 ** 24)):
        assert _verify(step=step) == -5 and _verify(step=step, draft=7 * OK) == -5
    assert _read(rows=2 ** 28) == -5 and _read(rows=2 ** 63 - 1) == -5 and _append(step=_step(n_tokens=2 ** 24)) == -5


def test_what_is_read_is_not_written():
    """Outputs in the place of inputs that other workgroups may still read, and of each other; only the lengths may be taken back in place."""
    for kw in (dict(accepted=5 * OK), dict(follows=6 * OK), dict(lens=4 * OK), dict(accepted=2 * OK), dict(follows=3 * OK), dict(lens=2 * OK), dict(accepted=OK),
               dict(follows=OK), dict(lens=3 * OK)):
        assert _verify(**kw) == -1, kw


# ---- the binding: tensors elsewhere, and of other shapes and types (stand-ins say where they are) ---------------------
@pytest.fixture
def reached(monkeypatch):
    import types
    calls = []

    def workspace(*a):
        a[-1]._obj.value = 4096
        return 0
    lib = types.SimpleNamespace(ivf_kv_append=lambda *a: (calls.append("append"), 0)[1], ivf_attend=lambda *a: (calls.append("attend"), 0)[1],
                                ivf_kv_read=lambda *a: (calls.append("read"), 0)[1], ivf_verify_draft=lambda *a: (calls.append("verify"), 0)[1],
                                ivf_attend_workspace=workspace, ivf_verify_workspace=workspace, ivf_last_error=lambda: b"")
    monkeypatch.setattr(B, "load", lambda: lib)
    monkeypatch.setattr(B, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(B, "_new", lambda stream, shape, dtype, kept=True: On(torch.zeros(shape, dtype=dtype)))
    monkeypatch.setattr(B, "_device_now", lambda: 0)
    B.ivf_verify_workspace.cache_clear()
    yield calls
    B.ivf_verify_workspace.cache_clear()


def _q8(device=0, codes=torch.uint8, scales=torch.uint8, dtype=torch.float16, **other):
    t = dict(k=_zeros(4, 16, 2, 64, dtype=codes, device=device), v=_zeros(4, 16, 2, 64, dtype=codes, device=device),
             k_scale=_zeros(4, 16, 2, dtype=scales, device=device), v_scale=_zeros(4, 16, 2, dtype=scales, device=device), dtype=dtype)
    t.update(other)
    return P.KvCache(**t)


def _call(name, step=None, **kw):
    cache = kw.pop("cache", None) or _q8()
    if name == "append":
        a = dict(k=_zeros(3, 2, 64), v=_zeros(3, 2, 64), q=_zeros(3, 4, 64), q_out=_zeros(3, 4, 64))
        return P.ivf_kv_append(step or _on_step(), cache, **{**a, **kw})
    if name == "attend":
        return P.ivf_attend(step or _on_step(), cache, **{**dict(q=_zeros(3, 4, 64), out=_zeros(3, 4, 64)), **kw})
    if name == "read":
        return P.ivf_kv_read(step or _on_step(), cache, **{**dict(out_off=_i32(3), k=_zeros(9, 2, 64), v=_zeros(9, 2, 64), first=_i32(2)), **kw})
    f32 = dict(dtype=torch.float32)
    a = dict(logits=_zeros(3, 50), tokens=_i32(3), uniform=_zeros(3, **f32), draft=_zeros(3, 50, **f32), lens_out=_i32(2), workspace=_zeros(4096, dtype=torch.uint8))
    return P.ivf_verify_draft(step or _on_step(), **{**a, **kw})


def test_calls_on_one_device_reach_the_library(reached):
    for name in ("append", "attend", "read", "verify"):
        _call(name)
    _call("read", first=None)
    _call("verify", draft=None, lens_out=None, workspace=None)
    _call("verify", uniform=None, draft=None, scale=0.0)
    _call("append", cache=_q8(codes=torch.float8_e4m3fn, scales=torch.float8_e8m0fnu))
    assert reached == ["append", "attend", "read", "verify", "read", "verify", "verify", "append"]


@pytest.mark.parametrize("other", [-1, 1])
def test_tensors_elsewhere(reached, other):
    at = lambda *shape, dtype=torch.float16: _zeros(*shape, dtype=dtype, device=other)
    f32, i32, u8 = torch.float32, torch.int32, torch.uint8
    bad = [lambda: _q8(k_scale=at(4, 16, 2, dtype=u8)), lambda: _q8(v_scale=at(4, 16, 2, dtype=u8)), lambda: _q8(v=at(4, 16, 2, 64, dtype=u8)),
           lambda: _call("append", k=at(3, 2, 64)), lambda: _call("attend", q=at(3, 4, 64)), lambda: _call("attend", out=at(3, 4, 64)),
           lambda: _call("read", out_off=at(3, dtype=i32)), lambda: _call("read", first=at(2, dtype=i32)), lambda: _call("read", k=at(9, 2, 64)),
           lambda: _call("read", v=at(9, 2, 64)), lambda: _call("verify", logits=at(3, 50)), lambda: _call("verify", tokens=at(3, dtype=i32)),
           lambda: _call("verify", uniform=at(3, dtype=f32)), lambda: _call("verify", draft=at(3, 50, dtype=f32)), lambda: _call("verify", lens_out=at(2, dtype=i32)),
           lambda: _call("verify", workspace=at(4096, dtype=u8))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    assert reached == []


def test_other_devices_than_the_current_one(reached):
    bad = [lambda: _call(name, step=_on_step(1)) for name in ("append", "attend", "read", "verify")]
    bad += [lambda: _call(name, cache=_q8(1)) for name in ("append", "attend", "read")]
    bad += [lambda: _call(name, stream=_stream(1)) for name in ("append", "attend", "read", "verify")]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    assert reached == []


def test_shapes_and_types(reached):
    f32 = torch.float32
    bad = [lambda: _q8(k_scale=None), lambda: _q8(v_scale=None), lambda: _q8(dtype=None), lambda: _q8(k_scale=None, v_scale=None),
           lambda: _q8(codes=torch.float16), lambda: _q8(codes=torch.int8), lambda: _q8(scales=torch.int8), lambda: _q8(scales=f32),
           lambda: _q8(v_scale=_zeros(4, 16, 2, dtype=torch.float8_e8m0fnu)), lambda: _q8(k_scale=_zeros(4, 16, 3, dtype=torch.uint8)),
           lambda: _q8(v_scale=On(torch.zeros(4, 2, 16, dtype=torch.uint8).transpose(1, 2))), lambda: _q8(dtype=torch.uint8),
           lambda: P.KvCache(_zeros(4, 16, 2, 64, dtype=torch.uint8), _zeros(4, 16, 2, 64, dtype=torch.uint8)),
           lambda: _call("append", k=_zeros(3, 2, 64, dtype=torch.bfloat16)), lambda: _call("attend", q=_zeros(3, 4, 64, dtype=torch.uint8)),
           lambda: _call("read", out_off=_i32(4)), lambda: _call("read", first=_i32(3)), lambda: _call("read", k=_zeros(9, 3, 64)),
           lambda: _call("read", v=_zeros(8, 2, 64)), lambda: _call("read", out_off=_zeros(3, dtype=torch.int64)),
           lambda: _call("verify", logits=_zeros(4, 50)), lambda: _call("verify", logits=_zeros(3, 50, dtype=torch.float64)), lambda: _call("verify", tokens=_i32(2)),
           lambda: _call("verify", logits=On(torch.zeros(3, 100)[:, ::2])), lambda: _call("verify", uniform=_zeros(3)), lambda: _call("verify", uniform=_zeros(4, dtype=f32)),
           lambda: _call("verify", draft=_zeros(3, 50)), lambda: _call("verify", draft=_zeros(3, 51, dtype=f32)), lambda: _call("verify", draft=_zeros(2, 50, dtype=f32)),
           lambda: _call("verify", lens_out=_i32(3)), lambda: _call("verify", workspace=On(torch.zeros(8192, dtype=torch.uint8)[::2]))]
    for call in bad:
        with pytest.raises((ValueError, TypeError)):
            call()
    assert reached == []

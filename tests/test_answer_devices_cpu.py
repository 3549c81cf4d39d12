"""Tensors on another device than the call's are refused before the library is reached (no GPU: stand-ins say where they are)."""
import types

import pytest
import torch

import paper_2502_20969_amd as P
import paper_2502_20969_amd.binding as B


class On:
    """A tensor that claims to be on a CUDA device, or on none (-1)."""

    def __init__(self, t, device=0):
        self._t, self._device = t, device

    def __getattr__(self, name):
        return getattr(self._t, name)

    def __getitem__(self, i):
        return On(self._t[i], self._device)

    def get_device(self):
        return self._device

    @property
    def is_cuda(self):
        return self._device >= 0

    @property
    def device(self):
        return torch.device("cuda", self._device) if self._device >= 0 else torch.device("cpu")


def _zeros(*shape, dtype=torch.float16, device=0):
    return On(torch.zeros(*shape, dtype=dtype), device)


def _i32(*shape, device=0):
    return _zeros(*shape, dtype=torch.int32, device=device)


@pytest.fixture
def reached(monkeypatch):
    """Names of the calls that reach a library which does nothing."""
    calls = []

    def call(name, status=0):
        return lambda *a: (calls.append(name), status)[1]

    def workspace(*a):
        a[-1]._obj.value = 4096
        return 0
    lib = types.SimpleNamespace(ivf_kv_append=call("append"), ivf_attend=call("attend"), ivf_beam_step=call("beam"), ivf_attend_workspace=workspace,
                                ivf_beam_workspace=workspace, ivf_last_error=lambda: b"")
    monkeypatch.setattr(B, "load", lambda: lib)
    monkeypatch.setattr(B, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(B, "_new", lambda stream, shape, dtype, kept=True: On(torch.zeros(shape, dtype=dtype)))
    monkeypatch.setattr(B, "_device_now", lambda: 0)
    B.ivf_beam_workspace.cache_clear()
    yield calls
    B.ivf_beam_workspace.cache_clear()


def _step(device=0, **other):
    t = dict(q_off=_i32(3, device=device), lens=_i32(2, device=device), table=_i32(2, 4, device=device), group_off=_i32(2, device=device),
             prefix_lens=_i32(1, device=device), prefix_table=_i32(1, 4, device=device))
    t.update(other)
    return P.KvStep(page=16, n_tokens=3, **t)


def _cache(device=0):
    return P.KvCache(_zeros(4, 16, 2, 64, device=device), _zeros(4, 16, 2, 64, device=device))


def _stream(device):
    return types.SimpleNamespace(cuda_stream=0, device_index=device)


@pytest.mark.parametrize("other", [-1, 1])
def test_caches_and_steps(other):
    with pytest.raises(ValueError):
        P.KvCache(_zeros(4, 16, 2, 64), _zeros(4, 16, 2, 64, device=other))
    for name, shape in dict(q_off=(3,), lens=(2,), table=(2, 4), group_off=(2,), prefix_lens=(1,), prefix_table=(1, 4)).items():
        with pytest.raises(ValueError):
            _step(**{name: _i32(*shape, device=other)})
    with pytest.raises(ValueError):
        _step(device=-1)


def _append(step=None, cache=None, **kw):
    a = dict(k=_zeros(3, 2, 64), v=_zeros(3, 2, 64), q=_zeros(3, 4, 64), q_out=_zeros(3, 4, 64), rotary=_zeros(9, 64, dtype=torch.float32), positions=_i32(3))
    a.update(kw)
    return P.ivf_kv_append(step or _step(), cache or _cache(), **a)


def _attend(step=None, cache=None, **kw):
    a = dict(q=_zeros(3, 4, 64), out=_zeros(3, 4, 64), lse=_zeros(3, 4, dtype=torch.float32), workspace=_zeros(4096, dtype=torch.uint8))
    a.update(kw)
    return P.ivf_attend(step or _step(), cache or _cache(), **a)


def _beams(states=None, **kw):
    a = dict(logits=_zeros(2, 3, 50), scores=_zeros(2, 3, dtype=torch.float32), done=_zeros(2, 3, dtype=torch.bool), workspace=_zeros(4096, dtype=torch.uint8))
    a.update(kw)
    return P.ivf_beam_step(**a, states=[(_i32(6, 5), _i32(6, 5))] if states is None else states)


def test_calls_on_one_device_reach_the_library(reached):
    _append()
    _attend()
    _attend(workspace=None, stream=_stream(0))
    _beams()
    _beams(workspace=None)
    assert reached == ["append", "attend", "attend", "beam", "beam"]


@pytest.mark.parametrize("other", [-1, 1])
def test_tensors_elsewhere(reached, other):
    at = lambda *shape, dtype=torch.float16: _zeros(*shape, dtype=dtype, device=other)
    bad = [lambda: _append(k=at(3, 2, 64)), lambda: _append(v=at(3, 2, 64)), lambda: _append(q=at(3, 4, 64)), lambda: _append(q_out=at(3, 4, 64)),
           lambda: _append(rotary=at(9, 64, dtype=torch.float32)), lambda: _append(positions=at(3, dtype=torch.int32)),
           lambda: _attend(q=at(3, 4, 64)), lambda: _attend(out=at(3, 4, 64)), lambda: _attend(lse=at(3, 4, dtype=torch.float32)),
           lambda: _attend(workspace=at(4096, dtype=torch.uint8)),
           lambda: _beams(logits=at(2, 3, 50)), lambda: _beams(scores=at(2, 3, dtype=torch.float32)), lambda: _beams(done=at(2, 3, dtype=torch.bool)),
           lambda: _beams(workspace=at(4096, dtype=torch.uint8)),
           lambda: _beams([(at(6, 5, dtype=torch.int32), _i32(6, 5))]), lambda: _beams([(_i32(6, 5), at(6, 5, dtype=torch.int32))])]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    assert reached == []


def test_other_devices_than_the_current_one(reached):
    bad = [lambda: _append(step=_step(1)), lambda: _append(cache=_cache(1)), lambda: _attend(step=_step(1)), lambda: _attend(cache=_cache(1)),
           lambda: _attend(_step(1), _cache(1), q=_zeros(3, 4, 64, device=1), out=_zeros(3, 4, 64, device=1), lse=None, workspace=_zeros(4096, dtype=torch.uint8, device=1)),
           lambda: _append(stream=_stream(1)), lambda: _attend(stream=_stream(1)), lambda: _beams(stream=_stream(1))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    assert reached == []


def test_workspaces_with_holes(reached):
    for call in (_attend, _beams):
        with pytest.raises(ValueError):
            call(workspace=On(torch.zeros(8192, dtype=torch.uint8)[::2]))
    assert reached == []


@pytest.mark.parametrize("names", [("prefix_lens", "prefix_table"), ("prefix_lens",), ("prefix_table",), ("group_off",), ("group_off", "prefix_lens"), ("group_off", "prefix_table")])
def test_parts_of_a_prefix_alone(names):
    shapes = dict(group_off=(2,), prefix_lens=(1,), prefix_table=(1, 4))
    with pytest.raises(ValueError):
        _step(**{name: _i32(*shapes[name]) if name in names else None for name in shapes})

"""The binding of the calls that put a prompt into a paged cache, on the CPU: tensors that say they are on a device, a
library that notes what it is asked for."""
import types
import weakref

import pytest
import torch

from paper_2606_31315_amd import _lib as L

I32 = torch.int32


class OnDevice(torch.Tensor):
    is_cuda = True

    def get_device(self):
        return 0

    @classmethod
    def __torch_function__(cls, func, types, args=(), kwargs=None):
        with torch._C.DisableTorchFunctionSubclass():
            return func(*args, **(kwargs or {}))


def dev(*s, dt=torch.bfloat16):
    return torch.zeros(*s, dtype=dt).as_subclass(OnDevice)


@pytest.fixture
def asked(monkeypatch):
    """The calls made: (name, the shape's fields)."""
    out = []

    def noted(name):
        def call(ref, *args):
            out.append((name, {f: getattr(ref._obj, f) for f, _ in ref._obj._fields_}))
            return 0
        return call

    real = L.lib()
    monkeypatch.setattr(L, "lib", lambda: types.SimpleNamespace(
        **{n: noted(n) for n in ("sd_qk_norm_rope", "sd_kv_append_rope_paged", "sd_chunk_attn_paged")},
        sd_chunk_attn_workspace_size=real.sd_chunk_attn_workspace_size, sd_last_error=real.sd_last_error))
    monkeypatch.setattr(L, "_cur_device", lambda: 0)
    monkeypatch.setattr(L, "_raw_stream", lambda device: 5)
    monkeypatch.setattr(L, "_call_cache", {})
    monkeypatch.setattr(L, "_prompt_cache", {}, raising=False)
    return out


def _rope(**kw):
    return L.qk_norm_rope(dev(5, 4, 128), dev(5, 2, 128), dev(5, dt=I32), dev(64, dt=torch.float32), **kw)


def _append(**kw):
    pool = dev(9, 2, 16, 128)
    return L.kv_append_rope_paged(dev(5, 4, 128), dev(5, 2, 128), dev(5, 2, 128), pool, pool, dev(3, 4, dt=I32),
                                  dev(3, dt=I32), dev(4, dt=I32), dev(64, dt=torch.float32), **kw)


@pytest.mark.parametrize("call", [_rope, _append])
@pytest.mark.parametrize("name", ["eps", "rot_scale"])
def test_numbers_in_tensors_are_read_at_each_call(asked, call, name):
    """A 0-d tensor that is changed between two calls counts as it stands at each."""
    x = torch.tensor(0.25)
    call(**{name: x})
    x.fill_(0.5)
    call(**{name: x})
    assert [f[name] for _, f in asked] == [0.25, 0.5]


def test_a_workspace_that_is_grown_out_of_is_given_back_first(monkeypatch):
    empty, held, sizes = torch.empty, [], []

    def make(n, device=None, **k):
        assert not held or held[-1]() is None, "the smaller buffer is still held"
        sizes.append(n)
        buf = empty(n, **k)
        held.append(weakref.ref(buf))
        return buf

    monkeypatch.setattr(torch, "empty", make)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(L, "_stream", lambda stream: 5)
    ws, cuda = L.StreamWorkspace(), torch.device("cuda", 0)
    for n in (1000, 5000, 3000, 9000):
        assert ws.get(n, cuda, None).numel() >= n
    assert sizes == [1000, 5000, 9000]


def test_prompts_of_many_lengths_leave_the_per_step_calls_entries(asked):
    """The table of the per-step calls is cleared when it is full: the prompt calls do not fill it."""
    keep = L._call_cache["attn"] = object()
    pool, table, lens, off, ws = dev(9, 2, 16, 128), dev(3, 4, dt=I32), dev(3, dt=I32), dev(4, dt=I32), dev(1 << 22, dt=torch.uint8)
    for n in range(2 * L._CALL_CACHE_MAX):
        L.chunk_attn_paged(dev(1 + n % 8, 4, 128), pool, pool, table, lens, lens, off, 0, max_ctx=n % 60, max_chunk=3 + n // 60,
                           workspace=ws)
        _rope(eps=float(n))
    assert L._call_cache == {"attn": keep} and len(L._prompt_cache) <= L._CALL_CACHE_MAX

"""What the calls that put a prompt into a paged cache refuse, on the host before any device access: the C
entry points by status code, the binding by exception."""
import contextlib
import ctypes
import threading
import types

import pytest
import torch

from paper_2606_31315_amd import _lib as L

P = ctypes.c_void_p


def rope_shape(**kw):
    sh = L.SdRopeShape(2, 20, 32, 8, 128, 128, 0, L.SD_BF16, 1e-6, 0.0, 0, 0, 0, 0, 0)
    for k, v in kw.items():
        setattr(sh, k, v)
    return sh


def rope(sh, **kw):
    p = dict(q=4096, k=8192, pos=16, f=32, qw=4096, kw=4096, qo=12288, ko=16384)
    p.update(kw)
    return L.lib().sd_qk_norm_rope(ctypes.byref(sh) if sh is not None else None,
                                   *(P(p[x]) for x in ("q", "k", "pos", "f", "qw", "kw", "qo", "ko")), None)


def append(sh, page=16, pages=10, most=4, **kw):
    p = dict(table=16, q=4096, k=8192, v=8192, ctx=16, off=16, f=32, qw=4096, kw=4096, qo=12288, kp=16384, vp=20480)
    p.update(kw)
    return L.lib().sd_kv_append_rope_paged(ctypes.byref(sh) if sh is not None else None, page, pages, most, *(
        P(p[x]) for x in ("table", "q", "k", "v", "ctx", "off", "f", "qw", "kw", "qo", "kp", "vp")), None)


@pytest.mark.parametrize("call", [rope, append])
@pytest.mark.parametrize("field,value,code", [
    ("total_q", -1, L.SD_ERR_INVALID_ARG), ("num_seqs", -1, L.SD_ERR_INVALID_ARG),
    ("num_q_heads", -1, L.SD_ERR_INVALID_ARG), ("num_kv_heads", -1, L.SD_ERR_INVALID_ARG),
    ("num_q_heads", 65537, L.SD_ERR_INVALID_ARG), ("head_dim", 96, L.SD_ERR_UNSUPPORTED),
    ("rot_dim", -16, L.SD_ERR_INVALID_ARG), ("rot_dim", 24, L.SD_ERR_INVALID_ARG),
    ("rot_dim", 144, L.SD_ERR_INVALID_ARG), ("interleaved", 2, L.SD_ERR_INVALID_ARG),
    ("dtype", 2, L.SD_ERR_INVALID_ARG), ("eps", -1.0, L.SD_ERR_INVALID_ARG),
    ("eps", float("nan"), L.SD_ERR_INVALID_ARG), ("eps", float("inf"), L.SD_ERR_INVALID_ARG),
    ("rot_scale", float("inf"), L.SD_ERR_INVALID_ARG), ("rot_scale", float("nan"), L.SD_ERR_INVALID_ARG),
    ("q_stride", 4088, L.SD_ERR_INVALID_ARG), ("q_stride", -4096, L.SD_ERR_INVALID_ARG),
    ("q_stride", 4100, L.SD_ERR_INVALID_ARG), ("k_stride", 1000, L.SD_ERR_INVALID_ARG),
    ("q_out_stride", 64, L.SD_ERR_INVALID_ARG), ("q_stride", (1 << 32) + 8, L.SD_ERR_INVALID_ARG),
])
def test_shape_errors(call, field, value, code):
    assert call(rope_shape(**{field: value})) == code
    assert L.lib().sd_last_error().decode()


def test_rope_pointer_errors():
    assert rope(None) == L.SD_ERR_INVALID_ARG
    for x in ("q", "k", "pos", "f", "qo", "ko"):
        assert rope(rope_shape(), **{x: None}) == L.SD_ERR_INVALID_ARG, x
    for x in ("q", "k", "qo", "ko", "qw", "kw"):
        assert rope(rope_shape(), **{x: 4104}) == L.SD_ERR_INVALID_ARG, x
    assert rope(rope_shape(num_q_heads=0, num_kv_heads=0)) == L.SD_ERR_INVALID_ARG
    assert rope(rope_shape(k_out_stride=8)) == L.SD_ERR_INVALID_ARG
    assert rope(rope_shape(total_q=0), q=None, k=None, pos=None) == L.SD_OK


def test_append_errors():
    assert append(None) == L.SD_ERR_INVALID_ARG
    for x in ("table", "q", "k", "v", "ctx", "off", "f", "qo", "kp", "vp"):
        assert append(rope_shape(), **{x: None}) == L.SD_ERR_INVALID_ARG, x
    for x in ("q", "k", "v", "qo", "kp", "vp", "qw", "kw"):
        assert append(rope_shape(), **{x: 4104}) == L.SD_ERR_INVALID_ARG, x
    for kw in (dict(page=8), dict(page=24), dict(page=8192), dict(pages=0), dict(most=0), dict(page=4096, most=1 << 20)):
        assert append(rope_shape(), **kw) == L.SD_ERR_INVALID_ARG, kw
    assert append(rope_shape(num_kv_heads=0)) == L.SD_ERR_INVALID_ARG
    assert append(rope_shape(v_stride=512)) == L.SD_ERR_INVALID_ARG
    assert append(rope_shape(num_seqs=0)) == L.SD_OK
    assert append(rope_shape(total_q=0), q=None) == L.SD_OK


def chunk_shape(**kw):
    sh = L.SdAttnShape(4, 32, 8, 128, 4096, 900, 3000, 1000, L.SD_BF16, 0.0)
    for k, v in kw.items():
        setattr(sh, k, v)
    return sh


def chunk_ws(sh):
    n = ctypes.c_size_t(0)
    return L.lib().sd_chunk_attn_workspace_size(ctypes.byref(sh) if sh is not None else None, ctypes.byref(n)), n.value


def chunk(sh, page=16, pages=10, most=256, mask=0, ws_bytes=None, ws=256, **kw):
    p = dict(table=16, q=4096, k=8192, v=8192, ctx=16, len=16, off=16, out=12288)
    p.update(kw)
    n = chunk_ws(sh)[1] if ws_bytes is None else ws_bytes
    return L.lib().sd_chunk_attn_paged(ctypes.byref(sh) if sh is not None else None, page, pages, most, *(
        P(p[x]) for x in ("table", "q", "k", "v", "ctx", "len", "off")), mask, P(p["out"]), P(ws), n, None)


@pytest.mark.parametrize("field,value,code", [
    ("num_seqs", -1, L.SD_ERR_INVALID_ARG), ("num_q_heads", 0, L.SD_ERR_INVALID_ARG),
    ("num_kv_heads", 5, L.SD_ERR_INVALID_ARG), ("head_dim", 96, L.SD_ERR_UNSUPPORTED),
    ("max_block", 0, L.SD_ERR_INVALID_ARG), ("max_block", 4097, L.SD_ERR_INVALID_ARG), ("max_ctx", 4097, L.SD_ERR_INVALID_ARG),
    ("max_ctx", -1, L.SD_ERR_INVALID_ARG), ("total_q", 4001, L.SD_ERR_INVALID_ARG),
    ("total_q", -1, L.SD_ERR_INVALID_ARG), ("dtype", L.SD_F32, L.SD_ERR_UNSUPPORTED),
    ("dtype", 7, L.SD_ERR_INVALID_ARG), ("scale", float("nan"), L.SD_ERR_INVALID_ARG),
    ("scale", -1.0, L.SD_ERR_INVALID_ARG), ("scale", float("inf"), L.SD_ERR_INVALID_ARG),
])
def test_chunk_shape_errors(field, value, code):
    assert chunk_ws(chunk_shape(**{field: value}))[0] == code
    assert chunk(chunk_shape(**{field: value}), ws_bytes=1 << 40) == code


def test_chunk_errors():
    assert chunk_ws(None)[0] == L.SD_ERR_INVALID_ARG
    assert L.lib().sd_chunk_attn_workspace_size(ctypes.byref(chunk_shape()), None) == L.SD_ERR_INVALID_ARG
    assert chunk_ws(chunk_shape(num_q_heads=257, num_kv_heads=1))[0] == L.SD_ERR_UNSUPPORTED
    assert chunk_ws(chunk_shape(num_q_heads=256, num_kv_heads=1))[0] == L.SD_OK
    for sh in (chunk_shape(), chunk_shape(max_block=16, total_q=64)):  # the chunk kernel, the block kernels
        rc, n = chunk_ws(sh)
        assert rc == L.SD_OK and n > 0
        for x in ("table", "q", "k", "v", "ctx", "len", "off", "out"):
            assert chunk(sh, **{x: None}) == L.SD_ERR_INVALID_ARG, x
        for x in ("q", "k", "v", "out"):
            assert chunk(sh, **{x: 4104}) == L.SD_ERR_INVALID_ARG, x
        assert chunk(sh, mask=2) == L.SD_ERR_INVALID_ARG
        assert chunk(sh, ws=128) == L.SD_ERR_INVALID_ARG
        assert chunk(sh, ws=None) == L.SD_ERR_INVALID_ARG
        assert chunk(sh, ws_bytes=n - 1) == L.SD_ERR_WORKSPACE
        for kw in (dict(page=8), dict(page=24), dict(pages=0), dict(most=255)):
            assert chunk(sh, **kw) == L.SD_ERR_INVALID_ARG, kw
    assert chunk(chunk_shape(num_seqs=0, total_q=0)) == L.SD_OK
    assert chunk(chunk_shape(total_q=0), q=None) == L.SD_OK


def test_lengths_near_the_end_of_32_bits():
    """The kernels' key index looks some steps ahead of the last key."""
    top = 2 ** 31 - 16
    for block in (1, 5000):
        for ctx, code in ((top - block, L.SD_ERR_INVALID_ARG), (2 ** 31 - 512 - block, L.SD_ERR_INVALID_ARG),
                          (2 ** 31 - 513 - block, L.SD_OK)):
            sh = chunk_shape(num_seqs=1, total_q=1, max_kv_len=top, max_ctx=ctx, max_block=block)
            assert chunk_ws(sh)[0] == code, (block, ctx)


def _t(*shape, dt=torch.bfloat16):
    return torch.zeros(*shape, dtype=dt)


def test_binding_refuses_wrong_shapes_and_host_tensors():
    q, k, pos, f = _t(5, 4, 128), _t(5, 2, 128), _t(5, dt=torch.int32), _t(64, dt=torch.float32)
    for bad in (dict(q=_t(6, 4, 128)), dict(q=_t(5, 4, 64)), dict(positions=pos[:4]), dict(q=_t(5, 512)), dict(q=None, k=None), dict(q=[1]), dict(positions=None),
                dict(inv_freq=3.0), dict(q_weight=f), dict(k=None, k_out=k)):
        with pytest.raises((ValueError, TypeError)):
            L.qk_norm_rope(**{"q": q, "k": k, "positions": pos, "inv_freq": f, **bad})
    with pytest.raises(ValueError, match="device tensor"):
        L.qk_norm_rope(q, k, pos, f)
    pool, table, lens, off = _t(9, 2, 16, 128), _t(3, 4, dt=torch.int32), _t(3, dt=torch.int32), _t(4, dt=torch.int32)
    a = dict(q=q, k_new=k, v_new=k, k_pages=pool, v_pages=pool, block_table=table, ctx_lens=lens, q_offsets=off, inv_freq=f)
    for bad in (dict(), dict(v_pages=pool[:4]), dict(k_pages=pool[0]), dict(q_offsets=lens)):
        with pytest.raises((ValueError, TypeError)):
            L.kv_append_rope_paged(**{**a, **bad})
    c = dict(q=q, k_pages=pool, v_pages=pool, block_table=table, ctx_lens=lens, chunk_lens=lens, q_offsets=off,
             mask_mode=0, max_ctx=0, max_chunk=5)
    for bad in (dict(), dict(chunk_lens=off), dict(q=_t(5, 4, 64)), dict(out=_t(4, 4, 128))):
        with pytest.raises((ValueError, TypeError)):
            L.chunk_attn_paged(**{**c, **bad})


def test_row_strides():
    """_rows takes slices of packed rows and refuses heads apart, rows that overlap, other types."""
    class OnDevice(torch.Tensor):
        is_cuda = True
    x = torch.zeros(6, 10 * 128, dtype=torch.bfloat16).as_subclass(OnDevice)
    rows = lambda t, H, dt=torch.bfloat16: L._rows(t, "q", dt, t.device, None, H, 128)  # noqa: E731
    assert rows(x[:, :512].unflatten(1, (4, 128)), 4) == 1280
    assert rows(x[:1, :512].unflatten(1, (4, 128)), 4) == 512
    assert rows(x[:, :128].unflatten(1, (1, 128)), 1) == 1280
    with pytest.raises(ValueError, match="side by side"):
        rows(x.unflatten(1, (10, 128))[:, ::2], 5)
    with pytest.raises(ValueError, match="side by side"):
        rows(x[:1, :512].expand(6, 512).unflatten(1, (4, 128)), 4)
    with pytest.raises(TypeError):
        rows(x[:, :512].unflatten(1, (4, 128)), 4, torch.float32)


def test_binding_takes_meta_tensors_to_the_device_check():
    """Right shapes without memory stop at the device check, in every call."""
    m = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device="meta")  # noqa: E731
    i = lambda *s: m(*s, dt=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="device tensor"):
        L.qk_norm_rope(m(5, 4, 128), m(5, 2, 128), i(5), m(64, dt=torch.float32))
    with pytest.raises(ValueError, match="device tensor"):
        L.kv_append_rope_paged(m(5, 4, 128), m(5, 2, 128), m(5, 2, 128), m(9, 2, 16, 128), m(9, 2, 16, 128), i(3, 4), i(3),
                               i(4), m(64, dt=torch.float32))
    with pytest.raises(ValueError, match="device tensor"):
        L.chunk_attn_paged(m(5, 4, 128), m(9, 2, 16, 128), m(9, 2, 16, 128), i(3, 4), i(3), i(3), i(4), 0, max_ctx=0, max_chunk=5)


def test_chunk_attn_refuses_a_workspace_the_card_cannot_use(monkeypatch):
    """A workspace in host memory, or one with gaps, is refused before the library is called."""
    class OnDevice(torch.Tensor):
        is_cuda = True

    def dev(*s, dt=torch.bfloat16):
        return torch.zeros(*s, dtype=dt).as_subclass(OnDevice)

    monkeypatch.setattr(L, "lib", lambda: pytest.fail("the library was called"))
    i32 = torch.int32
    args = (dev(5, 4, 128), dev(9, 2, 16, 128), dev(9, 2, 16, 128), dev(3, 4, dt=i32), dev(3, dt=i32), dev(3, dt=i32),
            dev(4, dt=i32), 0)
    for ws, what in ((torch.zeros(1 << 16, dtype=torch.uint8), "workspace must be a device tensor"),
                     (dev(1 << 12, 16, dt=torch.uint8)[:, ::2], "workspace must be contiguous"), (7, "workspace must be a torch")):
        with pytest.raises((ValueError, TypeError), match=what):
            L.chunk_attn_paged(*args, max_ctx=0, max_chunk=5, workspace=ws)


def test_new_outputs_belong_to_the_call_s_stream(monkeypatch):
    """Where a stream is given, the outputs that a call makes are allocated on it; a stream of another device is refused."""
    on, current = [], [None]

    @contextlib.contextmanager
    def enter(stream):
        current.append(stream)
        yield
        current.pop()

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

    empty, empty_like = torch.empty, torch.empty_like
    calls = types.SimpleNamespace(**{f: lambda *a: 0 for f in ("sd_qk_norm_rope", "sd_kv_append_rope_paged", "sd_chunk_attn_paged")},
                                  sd_chunk_attn_workspace_size=L.lib().sd_chunk_attn_workspace_size)
    monkeypatch.setattr(L, "lib", lambda: calls)
    monkeypatch.setattr(L, "_cur_device", lambda: 0)
    monkeypatch.setattr(L, "_call_cache", {})
    monkeypatch.setattr(torch.cuda, "stream", enter)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: on.append(current[-1]) or empty(*a, **k))
    monkeypatch.setattr(torch, "empty_like", lambda *a, **k: on.append(current[-1]) or empty_like(*a, **k))
    i32, s = torch.int32, types.SimpleNamespace(cuda_stream=5, device_index=0)
    q, k, pool, table, lens, off = dev(5, 4, 128), dev(5, 2, 128), dev(9, 2, 16, 128), dev(3, 4, dt=i32), dev(3, dt=i32), dev(4, dt=i32)
    f, pos, ws = dev(64, dt=torch.float32), dev(5, dt=i32), dev(1 << 20, dt=torch.uint8)
    run = (lambda st: L.qk_norm_rope(q, k, pos, f, stream=st),
           lambda st: L.kv_append_rope_paged(q, k, k, pool, pool, table, lens, off, f, stream=st),
           lambda st: L.chunk_attn_paged(q, pool, pool, table, lens, lens, off, 0, max_ctx=0, max_chunk=5, workspace=ws, stream=st))
    for call, outputs in zip(run, (2, 1, 1)):
        on.clear()
        call(s)
        assert on == [s] * outputs
        with pytest.raises(ValueError, match="stream is one of cuda:1"):
            call(types.SimpleNamespace(cuda_stream=6, device_index=1))


def test_host_threads_share_no_workspace(monkeypatch):
    """Two threads' calls on one stream are several launches each, and may mix: each thread has its own buffer."""
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: empty(*a, **k))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(L, "_stream", lambda stream: 5)
    ws, dev, got = L.StreamWorkspace(), torch.device("cuda", 0), {}
    go = threading.Barrier(2)  # both alive, so that no buffer is one that the other gave back

    def work(i):
        if i == 1:
            go.wait()
        got[i] = ws.get(1000, dev, None), ws.get(900, dev, None)
        if i == 0:
            go.wait()
        go.wait()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert got[0][0] is got[0][1] and got[1][0] is got[1][1]
    assert got[0][0].data_ptr() != got[1][0].data_ptr()

"""Host-side refusals of the norms of queries and keys with the rotation and of sliding-window attention: codes for
bad sizes, types, pointers and workspaces, before anything is launched."""
import ctypes

import pytest

FAKE = ctypes.c_void_p(0x10000)       # aligned, never dereferenced: the call returns first
ODD = ctypes.c_void_p(0x10004)
i32, f32, vp, sz = ctypes.c_int32, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t


class Rope(ctypes.Structure):
    _fields_ = [(n, i32) for n in ("B", "T", "H", "Hk", "n", "pairs", "interleaved", "dtype")] + [("eps", f32)]


class Window(ctypes.Structure):
    _fields_ = [(n, i32) for n in ("B", "T", "Tk", "H", "Hk", "d", "window", "sinks", "dtype")] + [("scale", f32)]


@pytest.fixture(scope="module")
def lib():
    import paper_2602_10743_amd as K
    lib = K._load()
    R, W = ctypes.POINTER(Rope), ctypes.POINTER(Window)
    lib.kla_qk_norm_rope_workspace.argtypes = [R]
    lib.kla_qk_norm_rope_workspace.restype = sz
    lib.kla_qk_norm_rope_forward.argtypes = [R] + [vp] * 9
    lib.kla_qk_norm_rope_backward.argtypes = [R] + [vp] * 13 + [sz, vp]
    for n in ("saved_bytes", "workspace", "backward_workspace"):
        getattr(lib, "kla_window_attn_" + n).argtypes = [W]
        getattr(lib, "kla_window_attn_" + n).restype = sz
    lib.kla_window_attn_forward.argtypes = [W] + [vp] * 9 + [sz, vp]
    lib.kla_window_attn_backward.argtypes = [W] + [vp] * 11 + [sz, vp]
    lib.kla_window_attn_step_workspace.argtypes = [i32] * 7
    lib.kla_window_attn_step_workspace.restype = sz
    lib.kla_window_attn_step.argtypes = [i32] * 7 + [f32] + [vp] * 8 + [sz, vp]
    return lib


def put(args, i, x):
    return args[:i] + [x] + args[i + 1:]


def rope(**o):
    return ctypes.byref(Rope(**{**dict(B=2, T=8, H=4, Hk=2, n=64, pairs=32, interleaved=0, dtype=1, eps=1e-6), **o}))


def window(**o):
    return ctypes.byref(Window(**{**dict(B=2, T=8, Tk=8, H=4, Hk=2, d=64, window=4, sinks=1, dtype=1, scale=0.125), **o}))


def test_rope(lib):
    # q k wq wk freq positions q_out k_out
    ok = [FAKE, FAKE, None, None, FAKE, None, FAKE, FAKE]
    fwd = lambda a, **o: lib.kla_qk_norm_rope_forward(rope(**o), *a, None)
    for bad in (dict(B=0), dict(T=-1), dict(H=0), dict(Hk=0), dict(n=48), dict(pairs=-8), dict(pairs=12), dict(pairs=40),
                dict(interleaved=2), dict(eps=-1.0), dict(eps=float("nan")), dict(H=1 << 18), dict(H=(1 << 31) - 1, Hk=1)):
        assert fwd(ok, **bad) == 2, bad
        assert lib.kla_qk_norm_rope_workspace(rope(**bad)) == 0
    assert fwd(ok, dtype=2) == 3 and lib.kla_qk_norm_rope_forward(None, *ok, None) == 1
    for i in (0, 1, 4, 6, 7):
        assert fwd(put(ok, i, None)) == 1, i
    for i in range(8):
        assert fwd(put(ok, i, ODD)) == 4, i
    assert fwd([None] * 4 + [FAKE] + [None] * 3, T=0) == 0
    # q k wq wk freq positions dq_out dk_out dq dk dwq dwk ws
    ok = [FAKE, FAKE, None, None, FAKE, None] + [FAKE] * 4 + [None, None, FAKE]
    bwd = lambda a, ws=1 << 30, **o: lib.kla_qk_norm_rope_backward(rope(**o), *a, ws, None)
    assert bwd(ok, n=24) == 2 and bwd(ok, dtype=5) == 3
    for i in (0, 1, 4, 6, 7, 8, 9):
        assert bwd(put(ok, i, None)) == 1, i
    for i in range(13):
        assert bwd(put(ok, i, ODD)) == 4, i
    need = lib.kla_qk_norm_rope_workspace(rope())
    assert need > 0 and bwd(put(ok, 12, None)) == 5 and bwd(ok, ws=need - 1) == 5


def test_window(lib):
    # q k v len y saved cache_k cache_v ws
    ok = [FAKE] * 3 + [None, FAKE] + [None] * 4
    fwd = lambda a, n=0, **o: lib.kla_window_attn_forward(window(**o), *a, n, None)
    bads = (dict(B=0), dict(T=-1), dict(Tk=7), dict(H=3), dict(H=0), dict(Hk=0), dict(d=48), dict(window=0), dict(window=-3),
            dict(sinks=-1), dict(sinks=65), dict(window=1 << 30), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
            dict(scale=float("nan")), dict(H=1 << 17), dict(Tk=(1 << 28) + 1), dict(B=1 << 23), dict(B=1 << 15, Tk=1 << 20))
    for bad in bads:
        assert fwd(ok, **bad) == 2, bad
        for q in (lib.kla_window_attn_saved_bytes, lib.kla_window_attn_workspace, lib.kla_window_attn_backward_workspace):
            assert q(window(**bad)) == 0, bad
    assert fwd(ok, dtype=2) == 3 and lib.kla_window_attn_forward(None, *ok, 0, None) == 1
    for i in (0, 1, 2, 4):
        assert fwd(put(ok, i, None)) == 1, i
    for i in range(9):
        assert fwd(put(ok, i, ODD) if i not in (6, 7) else put(put(ok, 6, FAKE), 7, FAKE)[:i] + [ODD] + put(put(ok, 6, FAKE), 7, FAKE)[i + 1:]) == 4, i
    assert fwd(put(ok, 6, FAKE)) == 1 and fwd(put(ok, 7, FAKE)) == 1   # one cache without the other
    long = dict(B=1, T=4, Tk=8192, window=8192)
    need = lib.kla_window_attn_workspace(window(**long))
    assert need > 0 and fwd(ok, **long) == 5 and fwd(put(ok, 8, FAKE), need - 1, **long) == 5
    # q k v len y saved dy dq dk dv ws
    ok = [FAKE] * 3 + [None] + [FAKE] * 7
    bwd = lambda a, n=1 << 40, **o: lib.kla_window_attn_backward(window(**o), *a, n, None)
    for bad in bads:
        assert bwd(ok, **bad) == 2, bad
    for i in (0, 1, 2, 4, 5, 6, 7, 8, 9):
        assert bwd(put(ok, i, None)) == 1, i
    for i in range(11):
        assert bwd(put(ok, i, ODD)) == 4, i
    need = lib.kla_window_attn_backward_workspace(window())
    assert need > 0 and bwd(put(ok, 10, None)) == 5 and bwd(ok, need - 1) == 5
    assert lib.kla_window_attn_backward_workspace(window(T=4096, Tk=4096)) > lib.kla_window_attn_backward_workspace(
        window(T=4096, Tk=4096, sinks=0)) > 0


def test_step(lib):
    # q k v pos cache_k cache_v y ws
    ok = [FAKE] * 7 + [None]
    base = dict(S=2, H=4, Hk=2, d=64, window=4, sinks=1, dtype=1)
    step = lambda a, n=0, scale=0.1, **o: lib.kla_window_attn_step(*{**base, **o}.values(), scale, *a, n, None)
    for bad in (dict(S=0), dict(S=1 << 19), dict(H=3), dict(Hk=0), dict(d=8), dict(window=0), dict(sinks=65), dict(sinks=-1),
                dict(window=1 << 30), dict(H=1 << 17)):
        assert step(ok, **bad) == 2, bad
        assert lib.kla_window_attn_step_workspace(*{**base, **bad}.values()) == 0
    assert step(ok, dtype=2) == 3 and step(ok, scale=0.0) == 2 and step(ok, scale=float("nan")) == 2
    for i in range(7):
        assert step(put(ok, i, None)) == 1, i
    for i in range(8):
        assert step(put(ok, i, ODD)) == 4, i
    need = lib.kla_window_attn_step_workspace(*{**base, "window": 8192}.values())
    assert need > 0 and step(ok, window=8192) == 5 and step(put(ok, 7, FAKE), need - 1, window=8192) == 5


def test_binding_refuses_cpu_tensors():
    import torch
    import paper_2602_10743_amd as K
    x = torch.zeros(1, 4, 2, 16)
    with pytest.raises(ValueError, match="GPU"):
        K.kla_qk_norm_rope(x, x)
    with pytest.raises(ValueError, match="GPU"):
        K.kla_qk_norm_rope_forward(x, x)
    with pytest.raises(ValueError, match="GPU"):
        K.kla_window_attn(x, x, x, 2)
    with pytest.raises(ValueError, match="GPU"):
        K.kla_window_attn_forward(x, x, x, 2)
    with pytest.raises(ValueError, match="GPU"):
        K.kla_window_attn_step(x[0], x[0], x[0], x, x, torch.zeros(4, dtype=torch.int32))

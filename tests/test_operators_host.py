"""Host-side refusals of linear attention, layer norm and the token log probabilities: codes for bad
sizes, types, pointers and workspaces, before anything is launched."""
import ctypes

import pytest

FAKE = ctypes.c_void_p(0x10000)       # aligned, never dereferenced: the call returns first
ODD = ctypes.c_void_p(0x10004)


@pytest.fixture(scope="module")
def lib():
    import paper_2602_10743_amd as K
    lib = K._load()
    sz, vp, i32, i64, f32 = ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    D = ctypes.POINTER(K._Desc)
    lib.kla_linear_attn_workspace.argtypes = lib.kla_linear_attn_backward_workspace.argtypes = [D]
    lib.kla_linear_attn_workspace.restype = lib.kla_linear_attn_backward_workspace.restype = sz
    lib.kla_linear_attn_forward.argtypes = [D] + [vp] * 9 + [sz, vp]
    lib.kla_linear_attn_backward.argtypes = [D] + [vp] * 13 + [sz, vp]
    lib.kla_linear_attn_step.argtypes = [i32] * 5 + [vp] * 7
    lib.kla_layer_norm_workspace.argtypes = [i32]
    lib.kla_layer_norm_workspace.restype = sz
    lib.kla_layer_norm_forward.argtypes = [i64, i32, i32, vp, vp, vp, f32, vp, vp, vp, vp]
    lib.kla_layer_norm_backward.argtypes = [i64, i32, i32] + [vp] * 9 + [sz, vp]
    lib.kla_token_logp_workspace.argtypes = [i32, i64, i32, i32]
    lib.kla_token_logp_workspace.restype = sz
    lib.kla_token_logp_forward.argtypes = [i32, i64, i32, i32, i32] + [vp] * 8 + [sz, vp]
    lib.kla_token_logp_backward.argtypes = [i32, i64, i32, i32] + [vp] * 8
    return lib


def desc(B=1, T=8, H=1, dk=16, dv=16, dtype=0):
    import paper_2602_10743_amd as K
    return ctypes.byref(K._Desc(B, T, H, dk, dv, dtype))


def put(args, i, x):
    return args[:i] + [x] + args[i + 1:]


def test_linear_attn(lib):
    # q k v g s0 len y sT ws
    ok = [FAKE] * 4 + [None, None, FAKE, None, None]
    fwd = lambda d, a, n=0: lib.kla_linear_attn_forward(d, *a, n, None)
    assert fwd(desc(dk=24), ok) == 2 and fwd(desc(B=0), ok) == 2 and fwd(desc(T=-1), ok) == 2
    assert fwd(desc(H=1 << 24, dk=32), ok) == 2           # row offsets of a chunk past 32 bits
    assert fwd(desc(B=(1 << 20) + 1, H=1), ok) == 2       # a launch's threads past 32 bits
    assert fwd(desc(dtype=3), ok) == 3 and fwd(None, ok) == 1
    for i in (0, 1, 2, 3, 6):
        assert fwd(desc(), put(ok, i, None)) == 1, i
    for i in range(9):
        assert fwd(desc(), put(ok, i, ODD)) == 4, i
    long = desc(T=4096)
    need = lib.kla_linear_attn_workspace(long)
    assert need > 0 and lib.kla_linear_attn_backward_workspace(long) >= need
    assert fwd(long, ok) == 5 and fwd(long, put(ok, 8, FAKE), need - 1) == 5
    assert lib.kla_linear_attn_workspace(desc(dk=24)) == 0
    # q k v g s0 len dy dsT dq dk dv ds0 ws
    ok = [FAKE] * 4 + [None, None, FAKE, None, FAKE, FAKE, FAKE, None, None]
    bwd = lambda d, a, n=0: lib.kla_linear_attn_backward(d, *a, n, None)
    assert bwd(desc(dv=8), ok) == 2 and bwd(long, ok) == 5
    for i in (0, 1, 2, 3, 6, 8, 9, 10):
        assert bwd(desc(), put(ok, i, None)) == 1, i
    for i in range(13):
        assert bwd(desc(), put(ok, i, ODD)) == 4, i
    ok = [FAKE] * 6
    step = lambda a, S=2, H=1, dk=16, dv=16, t=0: lib.kla_linear_attn_step(S, H, dk, dv, t, *a, None)
    assert step(ok, dk=48) == 2 and step(ok, S=0) == 2 and step(ok, S=1 << 20, H=4) == 2 and step(ok, t=2) == 3
    for i in range(6):
        assert step(put(ok, i, None)) == 1 and step(put(ok, i, ODD)) == 4, i


def test_layer_norm(lib):
    # x w bias eps out mean rstd
    fwd = lambda a, rows=2, n=8, t=0, eps=1e-5: lib.kla_layer_norm_forward(rows, n, t, a[0], a[1], a[2], eps, *a[3:], None)
    ok = [FAKE, FAKE, None, FAKE, None, None]
    assert fwd(ok, n=0) == 2 and fwd(ok, n=16385) == 2 and fwd(ok, rows=-1) == 2 and fwd(ok, eps=-1.0) == 2
    assert fwd(ok, rows=1 << 61) == 2 and fwd(ok, t=2) == 3
    for i in (0, 1, 3):
        assert fwd(put(ok, i, None)) == 1, i
    for i in range(6):
        assert fwd(put(ok, i, ODD)) == 4, i
    # x w mean rstd dout dx dw dbias ws
    bwd = lambda a, n=8, ws=1 << 30: lib.kla_layer_norm_backward(2, n, 0, *a, ws, None)
    ok = [FAKE] * 7 + [None, FAKE]
    assert bwd(ok, n=0) == 2
    for i in range(7):
        assert bwd(put(ok, i, None)) == 1, i
    for i in range(9):
        assert bwd(put(ok, i, ODD)) == 4, i
    assert bwd(put(ok, 8, None)) == 5 and bwd(ok, ws=lib.kla_layer_norm_workspace(8) - 1) == 5
    assert lib.kla_layer_norm_workspace(0) == 0


def test_token_logp(lib):
    # logits target logp entropy stat top_logp top_index ws
    fwd = lambda a, S=1, n=2, V=50, top=0, t=0, ws=0: lib.kla_token_logp_forward(S, n, V, top, t, *a, ws, None)
    ok = [FAKE] * 3 + [None] * 5
    assert fwd(ok, S=0) == 2 and fwd(ok, n=-1) == 2 and fwd(ok, V=0) == 2 and fwd(ok, top=33) == 2 and fwd(ok, top=-1) == 2
    assert fwd(ok, V=4, top=5) == 2 and fwd(ok, S=4, n=1 << 22) == 2 and fwd(ok, t=2) == 3
    for i in range(3):
        assert fwd(put(ok, i, None)) == 1, i
    assert fwd(ok, top=1) == 1
    for i in range(8):
        assert fwd(put(ok, i, ODD)) == 4, i
    need = lib.kla_token_logp_workspace(1, 1, 100000, 0)
    assert need > 0 and fwd(ok, n=1, V=100000) == 5 and fwd(put(ok, 7, FAKE), n=1, V=100000, ws=need - 1) == 5
    assert lib.kla_token_logp_workspace(1, 1, 100000, 8) > need and lib.kla_token_logp_workspace(1, 1, 0, 0) == 0
    assert fwd([None] * 8, n=0) == 0
    # logits target stat entropy dlogp dentropy dlogits
    bwd = lambda a, V=50: lib.kla_token_logp_backward(1, 2, V, 0, *a, None)
    ok = [FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE]
    assert bwd(ok, V=0) == 2
    for i in (0, 1, 2, 3, 6):
        assert bwd(put(ok, i, None)) == 1, i
    for i in range(7):
        assert bwd(put(ok, i, ODD)) == 4, i


def test_binding_refuses_cpu_tensors():
    import torch
    import paper_2602_10743_amd as K
    x = torch.zeros(1, 4, 2, 16)
    with pytest.raises(ValueError, match="GPU"):
        K.kla_linear_attn_forward(x, x, x, torch.zeros(2))
    with pytest.raises(ValueError, match="GPU"):
        K.kla_linear_attn_step(x[0], x[0], x[0], torch.zeros(2), torch.zeros(4, 2, 16, 16))
    with pytest.raises(ValueError, match="GPU"):
        K.kla_layer_norm(x, torch.ones(16))
    with pytest.raises(ValueError, match="GPU"):
        K.kla_token_logp(x, torch.zeros(2, dtype=torch.int64))

"""Host-only checks of the gated recurrence's and the norm's entry points: every call here is refused before anything is launched."""
import ctypes

import pytest

from paper_2312_00752_b200 import binding as K

a = ctypes.c_void_p(4096)
odd = ctypes.c_void_p(4097)


def _gated(batch=2, L=100, D=64, io=K.SSM_BF16, flags=0, **ld):
    return K.ssm_gated_problem_t(batch, L, D, io, flags, *[ld.get(k, 0) for k in ("x", "gate", "in_gate", "dx", "dgate", "din_gate")])


def _fwd(p, **over):
    dec, save = p.flags & 1, p.flags & 4
    v = dict(x=a, gate=a, in_gate=a if dec else None, A=a if dec else None, reset=None, h0=None, y=a, h_last=None,
             saved=a if save else None)
    v.update(over)
    return K.load_library().ssm_gated_fwd(ctypes.byref(p), *v.values(), None)


def _bwd(p, ws=a, n=1 << 40, **over):
    dec, save = p.flags & 1, p.flags & 4
    only = a if dec else None
    v = dict(x=a, gate=a, in_gate=only, A=only, reset=None, h0=None, dy=a, dh_last=None, saved=a if save else None, dx=a,
             dgate=a, din_gate=only, dA=only, dh0=None)
    v.update(over)
    return K.load_library().ssm_gated_bwd(ctypes.byref(p), *v.values(), ws, n, None)


def _step(p, **over):
    only = a if p.flags & 1 else None
    v = dict(x=a, gate=a, in_gate=only, A=only, reset=None, h=a, y=a)
    v.update(over)
    return K.load_library().ssm_gated_step(ctypes.byref(p), *v.values(), None)


@pytest.mark.parametrize("bad,code", [
    (dict(batch=0), 1), (dict(L=0), 1), (dict(D=-1), 1), (dict(flags=2), 1), (dict(flags=8), 1), (dict(io=2), 2),
    (dict(x=63), 1), (dict(gate=1), 1), (dict(dx=-64), 1), (dict(in_gate=64), 1), (dict(din_gate=64), 1), (dict(x=1 << 60), 2),
    (dict(batch=1 << 30, D=1 << 12), 2), (dict(batch=1 << 20, L=1 << 30, D=1 << 10), 2),
])
def test_invalid_gated_problems_are_refused(bad, code):
    p = _gated(**bad)
    lib = K.load_library()
    assert lib.ssm_gated_saved_state_bytes(ctypes.byref(p)) == 0 and lib.ssm_gated_bwd_workspace_bytes(ctypes.byref(p)) == 0
    assert _fwd(p) == code and _bwd(p) == code
    if bad.get("L") is None:
        p.L = 1
        assert _step(p) in (1, 2)
    assert lib.ssm_gated_fwd(None, a, a, None, None, None, None, a, None, None, None) == 1


@pytest.mark.parametrize("flags", [0, 1, 4, 5])
def test_missing_superfluous_and_misaligned_gated_arguments(flags):
    p = _gated(flags=flags)
    for name in ("x", "gate", "y"):
        assert _fwd(p, **{name: None}) == 1 and _fwd(p, **{name: odd}) == 1
    for name in ("in_gate", "A"):
        assert _fwd(p, **{name: None if flags & 1 else a}) == 1 and _bwd(p, **{name: None if flags & 1 else a}) == 1
    for name in ("h0", "h_last"):
        assert _fwd(p, **{name: ctypes.c_void_p(4098)}) == 1
    assert _fwd(p, saved=None if flags & 4 else a) == 1 and _bwd(p, saved=None if flags & 4 else a) == 1
    for name in ("x", "gate", "dy", "dx", "dgate"):
        assert _bwd(p, **{name: None}) == 1 and _bwd(p, **{name: odd}) == 1
    for name in ("din_gate", "dA"):
        assert _bwd(p, **{name: None if flags & 1 else a}) == 1
    for name in ("dh_last", "dh0", "h0"):
        assert _bwd(p, **{name: ctypes.c_void_p(4098)}) == 1
    need = K.load_library().ssm_gated_bwd_workspace_bytes(ctypes.byref(p))
    assert (need > 0) == (flags != 4)
    if need:
        assert _bwd(p, None, 0) == 3 and _bwd(p, a, need - 1) == 3 and _bwd(p, ctypes.c_void_p(4104), need) == 3


def test_a_step_has_one_row_per_entry():
    assert _step(_gated(L=2)) == 1 and _step(_gated(L=1, flags=4)) == 1
    for name in ("x", "gate", "h", "y"):
        assert _step(_gated(L=1), **{name: None}) == 1 and _step(_gated(L=1), **{name: odd}) == 1
    assert _step(_gated(L=1), A=a) == 1 and _step(_gated(L=1, flags=1), in_gate=None) == 1


def test_saved_states_and_workspace_sizes():
    lib = K.load_library()
    size = lambda **kw: lib.ssm_gated_saved_state_bytes(ctypes.byref(_gated(**kw)))
    assert 0 < size(L=1) <= size(L=100) <= size(L=5000) and size(L=100, D=1) > 0
    assert size(L=1 << 24, D=8192, batch=1) >= (1 << 24) // 64 * 8192 * 4      # (past 32 bits)
    need = lambda **kw: lib.ssm_gated_bwd_workspace_bytes(ctypes.byref(_gated(**kw)))
    assert need(flags=4) == 0 and need(flags=0) >= size() and need(flags=1) > need(flags=5) > 0


def _norm(rows=10, D=64, io=K.SSM_BF16, res=K.SSM_BF16, flags=0, eps=1e-5):
    return K.ssm_norm_problem_t(rows, D, io, res, flags, eps)


def _nfwd(p, **over):
    v = dict(x=a, residual=a if p.flags & 4 else None, weight=a, bias=a if p.flags & 2 else None, y=a, residual_out=None, stats=None)
    v.update(over)
    return K.load_library().ssm_norm_fwd(ctypes.byref(p), *v.values(), None)


def _nbwd(p, ws=a, n=1 << 40, **over):
    v = dict(s=a, weight=a, dy=a, stats=a, dresidual_out=None, dx=a, dresidual=None, dweight=a, dbias=a if p.flags & 2 else None)
    v.update(over)
    return K.load_library().ssm_norm_bwd(ctypes.byref(p), *v.values(), ws, n, None)


@pytest.mark.parametrize("bad,code", [
    (dict(rows=0), 1), (dict(D=0), 1), (dict(flags=8), 1), (dict(io=3, res=3), 2), (dict(res=5), 2), (dict(eps=-1.0), 1),
    (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(res=K.SSM_F32), 1), (dict(io=K.SSM_F32, flags=4), 2),
    (dict(rows=1 << 40), 2),
])
def test_invalid_norm_problems_are_refused(bad, code):
    p = _norm(**bad)
    assert K.load_library().ssm_norm_bwd_workspace_bytes(ctypes.byref(p)) == 0
    assert _nfwd(p) == code and _nbwd(p) == code


@pytest.mark.parametrize("flags", [0, 1, 2, 4, 7])
def test_missing_superfluous_and_misaligned_norm_arguments(flags):
    p = _norm(flags=flags)
    for name in ("x", "weight", "y"):
        assert _nfwd(p, **{name: None}) == 1 and _nfwd(p, **{name: odd}) == 1
    assert _nfwd(p, residual=None if flags & 4 else a) == 1 and _nfwd(p, bias=None if flags & 2 else a) == 1
    if not flags & 4:
        assert _nfwd(p, residual_out=a) == 1 and _nbwd(p, dresidual_out=a) == 1
    assert _nfwd(p, stats=ctypes.c_void_p(4098)) == 1
    for name in ("s", "weight", "dy", "stats", "dx", "dweight"):
        assert _nbwd(p, **{name: None}) == 1 and _nbwd(p, **{name: odd}) == 1
    assert _nbwd(p, dbias=None if flags & 2 else a) == 1
    assert _nbwd(p, dresidual=a) == 1                       # dx is the gradient of both
    need = K.load_library().ssm_norm_bwd_workspace_bytes(ctypes.byref(p))
    assert need > 0 and _nbwd(p, None, 0) == 3 and _nbwd(p, a, need - 1) == 3 and _nbwd(p, ctypes.c_void_p(4104), need) == 3


def test_bindings_refuse_host_tensors():
    import torch
    x, v = torch.zeros(2, 3, 4), torch.zeros(4)
    for call in (lambda: K.ssm_gated_fwd(x, x), lambda: K.ssm_gated_bwd(x, x, None, None, x), lambda: K.ssm_gated_step(x[0], x[0], None, None, x[0]),
                 lambda: K.ssm_norm_fwd(x, v), lambda: K.ssm_norm_bwd(x, v, x, x), lambda: K.ssm_gated_fwd(None, x), lambda: K.ssm_norm_fwd(3, v)):
        with pytest.raises(K.SsmScanError):
            call()

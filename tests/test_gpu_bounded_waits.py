"""Waits between the blocks of a cluster (gated recurrence) and for a row's copies (norm, long rows) that run out: the call ends, NaN
marks everything that was waited for, and the calls after it are none the worse.  The test hooks withhold what is waited for."""
import ctypes
import time

import pytest

from paper_2312_00752_b200 import binding as K
from tests.test_gpu_gated import device, make

a = ctypes.c_void_p(4096)


def test_the_step_has_no_such_hook():
    p = K.ssm_gated_problem_t(2, 1, 64, K.SSM_BF16, K.SSM_GATED_FLAG_TEST_WITHHOLD, *[0] * 6)
    assert K.load_library().ssm_gated_step(ctypes.byref(p), a, a, None, None, None, a, a, None) == 1
    assert K.load_library().ssm_gated_bwd_workspace_bytes(ctypes.byref(p)) > 0


def _p(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _done(code):
    import torch
    assert code == K.SSM_OK
    start = time.monotonic()
    torch.cuda.synchronize()
    assert time.monotonic() - start < 5.0


def _nan(t):
    import torch
    return bool(torch.isnan(t).all())


@pytest.mark.gpu
@pytest.mark.parametrize("decay", [False, True])
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("batch,L,D", [(1, 5000, 64), (2, 3000, 322), (3, 700, 33), (1, 20001, 1536)])
@pytest.mark.parametrize("packed", [False, True])
def test_blocks_that_wait_for_one_that_sends_nothing(packed, batch, L, D, io, decay):
    import torch
    lib, s = K.load_library(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    d = device(make(batch, L, D, io, decay, seed=1), io)
    reset = None
    if packed:                      # (a reset behind the first round of every block's tiles, which must not bring the numbers back)
        reset = torch.zeros(batch, L, dtype=torch.bool, device="cuda")
        reset[:, -1] = True
    flags = (K.SSM_GATED_FLAG_DECAY if decay else 0) | K.SSM_GATED_FLAG_SAVE_STATES
    name = {"bf16": K.SSM_BF16, "f32": K.SSM_F32}[io]
    held, ordinary = (ctypes.byref(K.ssm_gated_problem_t(batch, L, D, name, flags | f, *[0] * 6)) for f in (K.SSM_GATED_FLAG_TEST_WITHHOLD, 0))
    last = torch.zeros(batch, D, device="cuda")
    y, saved = K.ssm_gated_fwd(d["x"], d["gate"], d["in_gate"], d["A"], reset=reset, h0=d["h0"], h_last=last, save_states=True)
    grads = K.ssm_gated_bwd(d["x"], d["gate"], d["in_gate"], d["A"], d["dy"], saved, reset=reset, h0=d["h0"], dh_last=d["dh_last"], want_dh0=True)
    torch.cuda.synchronize()
    grads = {k: v for k, v in grads.items() if v is not None}
    y2, last2, saved2 = torch.zeros_like(y), torch.zeros_like(last), torch.zeros_like(saved)
    g2 = {k: torch.zeros_like(v) for k, v in grads.items()}
    ws = torch.empty(lib.ssm_gated_bwd_workspace_bytes(held), dtype=torch.uint8, device="cuda")

    def forward(problem):
        _done(lib.ssm_gated_fwd(problem, _p(d["x"]), _p(d["gate"]), _p(d["in_gate"]), _p(d["A"]), _p(reset), _p(d["h0"]), _p(y2), _p(last2),
                                _p(saved2), s))

    def backward(problem):
        _done(lib.ssm_gated_bwd(problem, _p(d["x"]), _p(d["gate"]), _p(d["in_gate"]), _p(d["A"]), _p(reset), _p(d["h0"]), _p(d["dy"]),
                                _p(d["dh_last"]), _p(saved), _p(g2["dx"]), _p(g2["dgate"]), _p(g2.get("din_gate")), _p(g2.get("dA")), _p(g2["dh0"]),
                                _p(ws) if ws.numel() else None, ws.numel(), s))

    for _ in range(2):
        forward(held)
        assert _nan(y2[:, :L - 1] if packed else y2) and _nan(last2)
        backward(held)
        # (in front of the reset at the last step, what its run of eight steps holds comes from no other block)
        assert all(_nan(g2[k][:, :L - 8] if packed else g2[k]) for k in ("dx", "dgate", "din_gate") if k in g2)
        assert _nan(g2["dh0"]) and (not decay or _nan(g2["dA"]))
        forward(ordinary)
        backward(ordinary)
        assert torch.equal(y2, y) and torch.equal(last2, last) and torch.equal(saved2, saved)
        assert all(torch.equal(g2[k], grads[k]) for k in grads)


@pytest.mark.gpu
def test_one_block_for_all_of_a_sequence_waits_for_nobody():
    import torch
    d = device(make(8, 16, 5120, "bf16", True, seed=2), "bf16")
    ref = K.ssm_gated_fwd(d["x"], d["gate"], d["in_gate"], d["A"])
    y = torch.empty_like(ref)
    p = K.ssm_gated_problem_t(8, 16, 5120, K.SSM_BF16, K.SSM_GATED_FLAG_DECAY | K.SSM_GATED_FLAG_TEST_WITHHOLD, *[0] * 6)
    _done(K.load_library().ssm_gated_fwd(ctypes.byref(p), _p(d["x"]), _p(d["gate"]), _p(d["in_gate"]), _p(d["A"]), None, None, _p(y), None, None,
                                         ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)))
    assert torch.equal(y, ref)


@pytest.mark.gpu
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("rows,D,io,res", [(5, 5120, "bf16", None), (1300, 5120, "bf16", "bf16"), (900, 4096, "bf16", "f32"), (700, 2052, "f32", "f32"),
                                           (2000, 8192, "bf16", None)])
def test_rows_whose_copies_stay_away(rows, D, io, res, bias, rms):
    import torch
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    lib, st = K.load_library(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    g = torch.Generator(device="cuda").manual_seed(3)
    n = lambda t: torch.randn(rows, D, generator=g, device="cuda").to(t)
    s, dy, w = n(types[res or io]), n(types[io]), torch.rand(D, generator=g, device="cuda")
    down = None if res is None else n(types[res])
    stats = torch.stack([torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")], 1).contiguous()
    ref = K.ssm_norm_bwd(s, w, dy, stats, down, rms=rms, has_bias=bias)
    names = [k for k in ("dx", "dresidual", "dweight", "dbias") if ref[k] is not None and not (k == "dresidual" and res in (None, io))]
    out = {k: torch.zeros_like(ref[k]) for k in names}
    flags = (K.SSM_NORM_FLAG_RMS if rms else 0) | (K.SSM_NORM_FLAG_HAS_BIAS if bias else 0) | (K.SSM_NORM_FLAG_HAS_RESIDUAL if res else 0)
    kind = {"bf16": K.SSM_BF16, "f32": K.SSM_F32}
    held, ordinary = (ctypes.byref(K.ssm_norm_problem_t(rows, D, kind[io], kind[res or io], flags | f, 0.0)) for f in (K.SSM_NORM_FLAG_TEST_WITHHOLD, 0))
    ws = torch.empty(lib.ssm_norm_bwd_workspace_bytes(held), dtype=torch.uint8, device="cuda")

    def backward(problem):
        _done(lib.ssm_norm_bwd(problem, _p(s), _p(w), _p(dy), _p(stats), _p(down), _p(out["dx"]), _p(out.get("dresidual")), _p(out["dweight"]),
                               _p(out.get("dbias")), _p(ws), ws.numel(), st))

    for _ in range(2):
        backward(held)
        assert all(_nan(v) for v in out.values())
        backward(ordinary)
        assert all(torch.equal(out[k], ref[k]) for k in names)

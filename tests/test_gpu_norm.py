"""Norm with residual add on the GPU against its float64 oracle.

Tolerances: a stored value is rounded once (at most eps / 2 relative) and carries the error of the float32 arithmetic before it.  A row's
sums are of D <= 10000 terms in float32, added in many short chains: relative error below 1e-6 of the sum of their magnitudes;
with a handful of roundings after them, E = 1e-5 of the largest value covers y; ds is a difference of r q, r mean(q) and
r xh mean(q xh), each rounded by itself, which may all but cancel (a row of one value with rms: xh^2 = 1 - eps r^2, so that
1e-4 of the terms is left), so that E goes by the sum of the terms' magnitudes.  dweight and dbias are sums over the rows:
E = 1e-5 of the sum of their terms' magnitudes (chains of at most some hundred additions, 2^-24 each)."""
import numpy as np
import pytest

from paper_2312_00752_b200 import synth
from tests.test_gpu_gated import HALF, close

pytestmark = pytest.mark.gpu


def make(rows, D, io, res, seed=0, mean=0.0):
    rng = np.random.default_rng(seed)
    n = lambda kind, *s: synth.round_to_io(rng.standard_normal(s) + mean, kind)
    return {"x": n(io, rows, D), "residual": None if res is None else n(res, rows, D), "dy": synth.round_to_io(rng.standard_normal((rows, D)), io),
            "weight": (1 + 0.2 * rng.standard_normal(D)).astype(np.float32), "bias": (0.2 * rng.standard_normal(D)).astype(np.float32),
            "dresidual_out": None if res is None else n(res, rows, D)}


def device(case, io, res):
    import torch
    kind = {"bf16": torch.bfloat16, "f32": torch.float32, None: None}
    types = {"x": kind[io], "dy": kind[io], "residual": kind[res], "dresidual_out": kind[res]}
    return {k: None if v is None else torch.from_numpy(v).cuda().to(types.get(k, torch.float32)) for k, v in case.items()}


def check(case, io, res, rms, bias, eps=1e-5, dev=None, down=True):
    import torch
    from oracle import norm_oracle as NO
    from paper_2312_00752_b200 import binding as K
    d = device(case, io, res) if dev is None else dev
    b = d["bias"] if bias else None
    got = list(K.ssm_norm_fwd(d["x"], d["weight"], b, d["residual"], rms=rms, eps=eps, save_stats=True))
    y, stats = got[0], got[-1]
    s = d["x"]
    if res is not None:
        s = got[1]
        exact = case["x"].astype(np.float64) + case["residual"]
        err = np.abs(s.double().cpu().numpy().reshape(exact.shape) - exact) - HALF[res] * (1 + 2.0 ** -14) * np.abs(exact)
        assert s.dtype == d["residual"].dtype and err.max() <= 0
    held = s.double().cpu().numpy().reshape(-1, s.shape[-1])
    ref, rs = NO.norm_fwd(held, case["weight"], case["bias"] if bias else None, rms, eps)
    assert y.dtype == d["x"].dtype
    close(y.reshape(ref.shape), ref, io, 1e-5)
    close(stats.reshape(-1, 2)[:, 1], rs[:, 1], "f32", 1e-5)
    close(stats.reshape(-1, 2)[:, 0], rs[:, 0], "f32", 1e-6, max(1.0, np.abs(held).max()))
    dro = d["dresidual_out"] if down else None
    g = K.ssm_norm_bwd(s, d["weight"], d["dy"], stats, dro, rms=rms, has_bias=bias)
    rg = NO.norm_bwd(held, case["weight"], case["dy"], case["dresidual_out"] if down else None, rms, eps)
    close(g["dx"].reshape(ref.shape), rg["ds"], io, 1e-5, rg["ds_terms"].max())
    if res is not None and res != io:
        close(g["dresidual"].reshape(ref.shape), rg["ds"], res, 1e-5, rg["ds_terms"].max())
    else:
        assert g["dresidual"] is g["dx"] or g["dresidual"].data_ptr() == g["dx"].data_ptr()
    close(g["dweight"], rg["dweight"], "f32", 1e-5, rg["dweight_terms"].max())
    if bias:
        close(g["dbias"], rg["dbias"], "f32", 1e-5, rg["dbias_terms"].max())
    else:
        assert g["dbias"] is None
    return (*got, *[v for v in g.values() if v is not None])


KINDS = [("bf16", None), ("bf16", "bf16"), ("bf16", "f32"), ("f32", None), ("f32", "f32")]
SHAPES = [(1, 64), (1, 1), (3, 2), (5, 7), (2, 31), (4, 33), (7, 100), (33, 96), (300, 64), (17, 256), (9, 1001), (5, 1002),
          (6, 2048), (150, 520), (3, 5120), (2, 8192), (2, 10007), (700, 136), (1500, 24),
          # more rows than blocks at once, in registers and through the ring; rows of whole pairs; rows of no kernel but the long ones'
          (1400, 1024), (1300, 4096), (900, 1802), (5, 5002), (2, 17000)]


@pytest.mark.parametrize("rms,bias", [(False, True), (True, False), (True, True), (False, False)])
@pytest.mark.parametrize("io,res", KINDS)
@pytest.mark.parametrize("rows,D", SHAPES)
def test_forward_backward(rows, D, io, res, rms, bias):
    if D == 1 and not rms:        # a row of one value is its own mean: s - m = 0
        return
    check(make(rows, D, io, res, seed=D), io, res, rms, bias)


@pytest.mark.parametrize("io,res", KINDS)
def test_rows_of_one_value_give_the_bias(io, res):
    import torch
    from paper_2312_00752_b200 import binding as K
    d = device(make(5, 1, io, res), io, res)
    got = K.ssm_norm_fwd(d["x"], d["weight"], d["bias"], d["residual"], save_stats=True)
    assert torch.equal(got[0], d["bias"].to(d["x"].dtype).expand(5, 1))
    g = K.ssm_norm_bwd(got[1] if res else d["x"], d["weight"], d["dy"], got[-1], has_bias=True)
    # dy w - mean(dy w), the product rounded once in the mean and perhaps not at all beside it: 2^-24 of it, times r = eps^-1/2
    bound = 2.0 ** -22 * 1e-5 ** -0.5 * float((d["dy"].float() * d["weight"]).abs().max())
    assert float(g["dx"].float().abs().max()) <= bound and bool((g["dweight"] == 0).all())


@pytest.mark.parametrize("res", [None, "bf16", "f32"])
def test_nothing_arrives_at_the_residual(res):
    check(make(40, 160, "bf16", res, seed=3), "bf16", res, False, True, down=False)


def test_a_mean_far_from_zero():
    # variance by the squares' mean less the mean's square would lose it: 100^2 against 1
    check(make(20, 700, "f32", "f32", seed=4, mean=100.0), "f32", "f32", False, True)


def test_leading_dimensions_outputs_and_unaligned_rows():
    import torch
    from paper_2312_00752_b200 import binding as K
    case = make(24, 264, "bf16", "f32", seed=5)
    base = check(case, "bf16", "f32", True, False)
    d = device(case, "bf16", "f32")
    shaped = {k: v if v is None or v.dim() < 2 else v.view(2, 3, 4, 264) for k, v in d.items()}
    got = check(case, "bf16", "f32", True, False, dev=shaped)
    assert got[2].shape == (2, 3, 4, 2) and all(torch.equal(p.flatten(), q.flatten()) for p, q in zip(base, got))
    out = {"out": torch.empty_like(d["x"]), "residual_out": torch.empty_like(d["residual"]), "stats": torch.empty(24, 2, device="cuda")}
    back = K.ssm_norm_fwd(d["x"], d["weight"], None, d["residual"], rms=True, save_stats=True, **out)
    assert [t.data_ptr() for t in back] == [t.data_ptr() for t in out.values()] and all(torch.equal(p, q) for p, q in zip(base, back))
    moved = {}
    for k, v in d.items():
        if v is not None:
            flat = torch.empty(v.numel() + 1, dtype=v.dtype, device="cuda")
            flat[1:] = v.flatten()
            moved[k] = flat[1:].view_as(v)
    check(case, "bf16", "f32", True, False, dev=moved)
    single = K.ssm_norm_fwd(d["x"][3], d["weight"], rms=True)          # one row without leading dimensions
    assert single.shape == (264,)


def test_values_that_are_not_finite_stay_in_their_row():
    import torch
    from paper_2312_00752_b200 import binding as K
    case = make(50, 200, "bf16", "f32", seed=6)
    clean = check(case, "bf16", "f32", False, True)
    for bad in (float("inf"), float("nan")):
        d = device(case, "bf16", "f32")
        d["x"][7, 11] = bad
        y, s, stats = K.ssm_norm_fwd(d["x"], d["weight"], d["bias"], d["residual"], save_stats=True)
        g = K.ssm_norm_bwd(s, d["weight"], d["dy"], stats, d["dresidual_out"], has_bias=True)
        rest = [i for i in range(50) if i != 7]
        assert bool(torch.isnan(y[7]).all()) and bool(torch.isnan(g["dx"][7]).all())
        assert torch.equal(y[rest], clean[0][rest]) and torch.equal(g["dx"][rest], clean[3][rest])
        assert torch.equal(g["dbias"], clean[-1])


@pytest.mark.parametrize("rows,D,io,res", [(900, 328, "bf16", "f32"), (3000, 1001, "f32", None)])
def test_runs_repeat_bit_for_bit_and_in_a_graph_and_on_a_stream(rows, D, io, res):
    import torch
    from paper_2312_00752_b200 import binding as K
    d = device(make(rows, D, io, res, seed=7), io, res)

    def run(**kw):
        got = list(K.ssm_norm_fwd(d["x"], d["weight"], d["bias"], d["residual"], save_stats=True, **kw))
        g = K.ssm_norm_bwd(got[1] if res else d["x"], d["weight"], d["dy"], got[-1], d["dresidual_out"], has_bias=True, **kw)
        return got + [v for v in g.values()]

    ref = run()
    s, other = torch.cuda.Stream(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for kw in ({}, {"stream": s}):
        torch.cuda.synchronize()               # (what is allocated here belongs to the current stream)
        got = run(**kw)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(ref, got))
    with torch.cuda.stream(s):
        run()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = run()
        graphs.append((graph, got))
    for _, got in graphs:
        for v in got:
            v.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(s):
            graphs[0][0].replay()
        with torch.cuda.stream(other):
            graphs[1][0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for _, got in graphs for p, q in zip(ref, got))


def test_rows_past_32_bits():
    import torch
    from paper_2312_00752_b200 import binding as K
    rows, D = 70001, 32768                                  # 2.3e9 elements
    x = torch.empty(rows, D, dtype=torch.bfloat16, device="cuda").normal_()
    w = torch.rand(D, device="cuda") + 0.5
    y, stats = K.ssm_norm_fwd(x, w, rms=True, save_stats=True)
    g = K.ssm_norm_bwd(x, w, x, stats, rms=True)
    tail = slice(rows - 8, rows)
    y2, stats2 = K.ssm_norm_fwd(x[tail], w, rms=True, save_stats=True)
    g2 = K.ssm_norm_bwd(x[tail], w, x[tail], stats2, rms=True)
    assert torch.equal(y[tail], y2) and torch.equal(stats[tail], stats2) and torch.equal(g["dx"][tail], g2["dx"])
    # sum of x xhat over the rows: x^2 r, r = 1 within 2 %
    assert bool(((g["dweight"] / rows - 1).abs() < 0.05).all())


def test_refusals():
    import torch
    from paper_2312_00752_b200 import binding as K
    x, w = torch.randn(6, 16, device="cuda"), torch.ones(16, device="cuda")
    bf = torch.bfloat16
    y, stats = K.ssm_norm_fwd(x, w, save_stats=True)
    fwd, bwd = K.ssm_norm_fwd, K.ssm_norm_bwd
    bad = [
        lambda: fwd(x.half(), w), lambda: fwd(x, w.to(bf)), lambda: fwd(x, w[:8]), lambda: fwd(x, None), lambda: fwd(x.t(), w), lambda: fwd(x, w.cpu()),
        lambda: fwd(x, w, residual=x.to(bf)), lambda: fwd(x, w, residual=x[:3]), lambda: fwd(x.to(bf), w, residual=x.half()),
        lambda: fwd(x, w, residual_out=x), lambda: fwd(x, w, residual=x, residual_out=x.to(bf)), lambda: fwd(x, w, eps=-1.0),
        lambda: fwd(x, w, eps=float("nan")), lambda: fwd(x, w, w[:3]), lambda: fwd(x[:0], w), lambda: fwd(x[:, :0], w[:0]), lambda: fwd(x, w, out=x.to(bf)),
        lambda: fwd(x, w, save_stats=True, stats=torch.empty(6, device="cuda")), lambda: fwd(x[:, ::2], w[::2].contiguous()),
        lambda: bwd(x, w, x[:3], stats), lambda: bwd(x, w, x, stats[:3]), lambda: bwd(x, w, x, None), lambda: bwd(x.to(bf), w, x, stats),
        lambda: bwd(x, w, x, stats, x.to(bf)), lambda: bwd(x, w, x, stats, outputs={"dresidual": x}), lambda: bwd(x, w, x, stats, outputs={"dweight": w[:3]}),
        lambda: bwd(x, None, x, stats), lambda: bwd(x, w, x.cpu(), stats), lambda: bwd(x, w, None, stats),
    ]
    for call in bad:
        with pytest.raises(K.SsmScanError):
            call()

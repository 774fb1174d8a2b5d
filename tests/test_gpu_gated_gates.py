"""Gates that are nearly closed or nearly open, element by element: each gradient is as good relative to its own size (that of the
terms it is summed from) as it is to the largest one's.

Tolerance: a stored value is rounded once (bf16 2^-8, fp32 2^-24 relative).  Before it: an exponential of |z| log2(e) <= 24 rounded to
float32 is off by 24 * 2^-24 = 1.4e-6 relative and the hardware's by 2^-22 more, reciprocals and reciprocal roots by 2^-22, products of
some ten such: below 2e-5 of the magnitudes of the terms."""
import numpy as np
import pytest

from paper_2312_00752_b200 import synth
from tests.test_gpu_gated import HALF, device

pytestmark = pytest.mark.gpu

E = 2e-5


def _sigma(z):
    e = np.exp(-z)
    return 1.0 / (1.0 + e), e / (1.0 + e)


def _near(got, ref, terms, io):
    got = got.detach().double().cpu().numpy()
    over = np.abs(got - ref) - HALF[io] * np.abs(ref) - E * (1 + HALF[io]) * terms
    assert np.isfinite(got).all() and over.max() <= 0, (np.abs(got - ref) / np.maximum(terms, 1e-300)).max()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("A", [None, -0.4, -3.0])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("batch,L,D", [(2, 40, 64), (1, 700, 66), (1, 24, 33)])
def test_gradients_of_nearly_saturated_gates(batch, L, D, sign, A, io):
    from paper_2312_00752_b200 import binding as K
    rng = np.random.default_rng(L)
    n = lambda *s: synth.round_to_io(rng.standard_normal(s), io)
    between = lambda: synth.round_to_io(sign * (8 + 8 * rng.random((batch, L, D))), io)
    # every step resets: each stands alone, and its gradients are plain products
    case = {"x": n(batch, L, D), "gate": between(), "in_gate": None if A is None else between(),
            "A": None if A is None else (A * (1 - 0.5 * rng.random(D))).astype(np.float32), "reset": np.ones((batch, L), bool), "dy": n(batch, L, D)}
    d = device(case, io)
    y, saved = K.ssm_gated_fwd(d["x"], d["gate"], d["in_gate"], d["A"], reset=d["reset"], save_states=True)
    g = K.ssm_gated_bwd(d["x"], d["gate"], d["in_gate"], d["A"], d["dy"], saved, reset=d["reset"])
    x, gate, mu = (case[k].astype(np.float64) for k in ("x", "gate", "dy"))
    rho, closed = _sigma(gate)
    if A is None:
        want = {"y": rho * x, "dx": mu * rho, "dgate": mu * x * rho * closed}
    else:
        iota, off = _sigma(case["in_gate"].astype(np.float64))
        decay = case["A"].astype(np.float64)
        la = rho * decay
        a, beta = np.exp(la), np.sqrt(-np.expm1(2 * la))
        want = {"y": beta * iota * x, "dx": mu * beta * iota, "din_gate": mu * beta * x * iota * off,
                "dgate": -mu * a * a / beta * iota * x * decay * rho * closed}
    for name, ref in want.items():
        _near(y if name == "y" else g[name], ref, np.abs(ref), io)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("A", [-0.4, -3.0])
@pytest.mark.parametrize("L,D", [(40, 100), (37, 101)])
def test_gates_of_every_size(L, D, A, io):
    # closed gates may flush to 0 what float32 cannot hold as a normal number, and the forward pass drops inputs whose gate is below -44
    from paper_2312_00752_b200 import binding as K
    levels = np.array([-200.0, -95.0, -87.0, -60.0, -30.0, -12.0, -5.0, 0.0, 6.0, 6.25, 12.0, 30.0, 60.0, 87.0, 95.0, 200.0])
    rng = np.random.default_rng(D)
    pick = lambda: rng.choice(levels, (1, L, D)).astype(np.float32)
    n = lambda *s: synth.round_to_io(rng.standard_normal(s), io)
    case = {"x": n(1, L, D), "gate": pick(), "in_gate": pick(), "A": (A * (1 - 0.5 * rng.random(D))).astype(np.float32),
            "reset": np.ones((1, L), bool), "dy": n(1, L, D)}
    d = device(case, io)
    y, saved = K.ssm_gated_fwd(d["x"], d["gate"], d["in_gate"], d["A"], reset=d["reset"], save_states=True)
    g = K.ssm_gated_bwd(d["x"], d["gate"], d["in_gate"], d["A"], d["dy"], saved, reset=d["reset"])
    x, mu, decay = (case[k].astype(np.float64) for k in ("x", "dy", "A"))
    (rho, closed), (iota, off) = (_sigma(case[k].astype(np.float64)) for k in ("gate", "in_gate"))
    la = rho * decay
    a, beta = np.exp(la), np.sqrt(-np.expm1(2 * la))
    lost = 1e-18 * np.abs(x)        # (beta is at least 1e-19, the root of the least normal number; the gate's limit is 1e-19)
    held = np.where(np.abs(la) > 1e-30, np.abs(la), 0.0)          # (below, the step size itself is no normal number any more)
    slope = np.divide(a * a * iota * x * decay * rho * closed, beta, out=np.zeros_like(x), where=held > 0)
    want = {"y": (beta * iota * x, lost), "dx": (mu * beta * iota, 1e-18 * np.abs(mu)),
            "din_gate": (mu * beta * x * iota * off, 1e-18 * np.abs(mu * x)), "dgate": (-mu * slope, 1e-14 * np.abs(mu * x))}
    for name, (ref, floor) in want.items():
        got = (y if name == "y" else g[name]).detach().double().cpu().numpy()
        over = np.abs(got - ref) - HALF[io] * np.abs(ref) - E * (1 + HALF[io]) * np.abs(ref) - floor
        assert np.isfinite(got).all() and over.max() <= 0, (name, over.max(), np.unravel_index(over.argmax(), over.shape))

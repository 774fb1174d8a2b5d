"""The oracles of the gated linear recurrence and of the norm: closed forms, torch's own layer norm, differences."""
import numpy as np
import pytest

from oracle import gated_oracle as GO
from oracle import norm_oracle as NO


def _inputs(batch=2, L=9, D=3, decay=True, seed=0):
    rng = np.random.default_rng(seed)
    n = lambda *s: rng.standard_normal(s)
    x, gate, in_gate = n(batch, L, D), n(batch, L, D), n(batch, L, D)
    A = -np.exp(n(D)) if decay else None
    reset = rng.random((batch, L)) < 0.25
    return x, gate, (in_gate if decay else None), A, reset, n(batch, D), n(batch, L, D), n(batch, D)


def test_convex_form_is_the_selective_scan_of_one_state():
    # A = -1, B = 1, step size softplus(gate), zero-order hold: the selective scan of N = 1 with C = 1
    from oracle import ssm_oracle as O
    x, gate, _, _, _, h0, _, _ = _inputs(decay=False)
    batch, L, D = x.shape
    x, gate = x.astype(np.float32), gate.astype(np.float32)
    delta = np.log1p(np.exp(gate.astype(np.float64))).astype(np.float32)
    one = np.ones((batch, L, 1), np.float32)
    want = O.scan_fwd(x, delta, -np.ones((D, 1), np.float32), one, one, zoh=True)
    got, _ = GO.gated_fwd(x, gate)
    np.testing.assert_allclose(got, want, rtol=0, atol=2e-6)      # delta was rounded to float32


def test_constant_gates_give_geometric_sums():
    z, L = -2.0, 40
    g = 1.0 / (1.0 + np.exp(-z))
    x = np.ones((1, L, 1))
    y, last = GO.gated_fwd(x, np.full((1, L, 1), z), h0=np.full((1, 1), 3.0))
    t = np.arange(1, L + 1)
    np.testing.assert_allclose(y[0, :, 0], 1.0 + 2.0 * (1.0 - g) ** t, rtol=1e-13)
    assert last[0, 0] == y[0, -1, 0]
    A = np.array([-0.5])
    a = np.exp(g * A[0])
    y, _ = GO.gated_fwd(x, np.full((1, L, 1), z), np.full((1, L, 1), z), A)
    np.testing.assert_allclose(y[0, :, 0], np.sqrt(1 - a * a) * g * (1 - a ** t) / (1 - a), rtol=1e-12)


@pytest.mark.parametrize("decay", [False, True])
def test_a_reset_is_a_new_sequence(decay):
    x, gate, in_gate, A, _, h0, _, _ = _inputs(L=12, decay=decay, seed=3)
    reset = np.zeros((2, 12), bool)
    reset[:, 5] = True
    y, last = GO.gated_fwd(x, gate, in_gate, A, reset, h0)
    cut = lambda v, lo, hi: None if v is None else v[:, lo:hi]
    first, _ = GO.gated_fwd(x[:, :5], gate[:, :5], cut(in_gate, 0, 5), A, None, h0)
    second, last2 = GO.gated_fwd(x[:, 5:], gate[:, 5:], cut(in_gate, 5, 12), A)
    assert np.array_equal(y, np.concatenate([first, second], 1)) and np.array_equal(last, last2)


@pytest.mark.parametrize("decay", [False, True])
def test_gated_gradients_against_differences(decay):
    x, gate, in_gate, A, reset, h0, dy, dh_last = _inputs(decay=decay, seed=5)
    args = {"x": x, "gate": gate, "h0": h0}
    if decay:
        args.update(in_gate=in_gate, A=A)

    def loss(**over):
        v = {**args, **over}
        y, last = GO.gated_fwd(v["x"], v["gate"], v.get("in_gate"), v.get("A"), reset, v["h0"])
        return (dy * y).sum() + (dh_last * last).sum()

    got = GO.gated_bwd(x, gate, in_gate, A, dy, reset, h0, dh_last)
    for name, v in args.items():
        num = np.empty_like(v)
        for i in np.ndindex(v.shape):
            up, down = v.copy(), v.copy()
            up[i] += 1e-6
            down[i] -= 1e-6
            num[i] = (loss(**{name: up}) - loss(**{name: down})) / 2e-6
        np.testing.assert_allclose(got["d" + name], num, rtol=0, atol=1e-7, err_msg=name)


@pytest.mark.parametrize("rms", [False, True])
def test_norm_against_torch_and_differences(rms):
    import torch
    rng = np.random.default_rng(7)
    s, w, b, dy, dr = rng.standard_normal((5, 11)), rng.standard_normal(11), rng.standard_normal(11), rng.standard_normal((5, 11)), rng.standard_normal((5, 11))
    ts, tw, tb = (torch.from_numpy(v).requires_grad_() for v in (s, w, b))
    y = torch.nn.functional.rms_norm(ts, (11,), tw, 1e-3) + tb if rms else torch.nn.functional.layer_norm(ts, (11,), tw, tb, 1e-3)
    (y * torch.from_numpy(dy)).sum().add((ts * torch.from_numpy(dr)).sum()).backward()
    got, stats = NO.norm_fwd(s, w, b, rms, 1e-3)
    np.testing.assert_allclose(got, y.detach().numpy(), rtol=1e-12, atol=1e-12)
    g = NO.norm_bwd(s, w, dy, dr, rms, 1e-3)
    for name, t in (("ds", ts), ("dweight", tw), ("dbias", tb)):
        np.testing.assert_allclose(g[name], t.grad.numpy(), rtol=1e-10, atol=1e-12)
    loss = lambda v: (NO.norm_fwd(v, w, b, rms, 1e-3)[0] * dy).sum() + (dr * v).sum()
    for i in np.ndindex(s.shape):
        up, down = s.copy(), s.copy()
        up[i] += 1e-6
        down[i] -= 1e-6
        assert abs((loss(up) - loss(down)) / 2e-6 - g["ds"][i]) <= 1e-6

"""The decay form with parameters A below -1, where the kernels take another way through the gates than for -1 <= A <= 0, alone and
mixed with small ones: forward, gradients, masks, clusters, single tokens against the float64 oracle.

Tolerances as in test_gpu_gated.py, whose derivation goes by the number of steps that a state remembers: it is 150 at most there, and
fewer the larger |A| is.  The retention itself is exp(v) with v = sigma(gate) A rounded to float32: an error of |v| 2^-24 relative,
|v| exp(-|v|) 2^-24 < 2^-25 absolute."""
import numpy as np
import pytest

from tests.test_gpu_gated import check, close, device, make

pytestmark = pytest.mark.gpu


def _A(kind, D, seed=0):
    rng = np.random.default_rng(seed)
    small = 8 * np.log(0.9 + 0.099 * rng.random(D))
    A = {"scan": -(1.0 + np.arange(D) % 16), "wide": -np.exp(np.clip(1.5 * rng.standard_normal(D), -4, 3.4)),
         "one of a warp": np.where(np.arange(D) % 64 == 5 % min(D, 64), -4.0, small),
         "edges": np.resize([-1.0, -1.0 - 2.0 ** -20, -0.25, -0.5, -2.0, -30.0, -88.0, -1e4], D)}[kind]
    return A.astype(np.float32)


def _case(batch, L, D, io, kind, seed, reset=None):
    case = make(batch, L, D, io, True, seed=seed, reset=reset)
    case["A"] = _A(kind, D, seed)
    return case


KINDS = ["scan", "wide", "one of a warp", "edges"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("batch,L,D", [(2, 200, 64), (1, 1, 64), (3, 1, 7), (1, 17, 2), (2, 33, 1), (1, 127, 130), (5, 257, 33), (1, 1025, 256),
                                       (2, 2049, 34), (1, 5000, 65)])
def test_forward_backward(batch, L, D, io, kind):
    check(_case(batch, L, D, io, kind, L), io)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("batch,L,D,reset", [(2, 300, 64, 0.02), (1, 77, 33, 0.5), (2, 40, 64, 1.0), (1, 4100, 48, 0.003), (3, 515, 66, 0.01)])
def test_packed_sequences(batch, L, D, reset, io, kind):
    check(_case(batch, L, D, io, kind, L, reset), io)


@pytest.mark.parametrize("kind", ["wide", "one of a warp"])
@pytest.mark.parametrize("batch,L,D,io,reset", [(4, 260, 5120, "bf16", None), (8, 515, 1600, "bf16", 0.01), (2, 1100, 1536, "f32", 0.01),
                                                (1, 3000, 2560, "bf16", None)])
def test_layer_widths(batch, L, D, io, reset, kind):
    check(_case(batch, L, D, io, kind, L, reset), io)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("batch,L,D,io", [(2, 200, 64, "bf16"), (1, 1300, 33, "f32"), (2, 70, 7, "bf16")])
def test_states_rebuilt_by_backward(batch, L, D, io, kind):
    import torch
    case = _case(batch, L, D, io, kind, 1, 0.01)
    *_, g = check(case, io)
    *_, h = check(case, io, saved_given=False)
    assert all(torch.equal(g[k], h[k]) for k in g if g[k] is not None)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("batch,D,io", [(1, 64, "bf16"), (1, 1, "f32"), (5, 1001, "bf16"), (256, 96, "f32")])
def test_step(batch, D, io, kind):
    from oracle import gated_oracle as GO
    from paper_2312_00752_b200 import binding as K
    case = _case(batch, 1, D, io, kind, 8)
    d = device(case, io)
    h = d["h0"].clone()
    y = K.ssm_gated_step(d["x"][:, 0], d["gate"][:, 0], d["in_gate"][:, 0], d["A"], h)
    _, last = GO.gated_fwd(case["x"], case["gate"], case["in_gate"], case["A"], None, case["h0"])
    close(y, last, io, 1e-5)
    close(h, last, "f32", 1e-5)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_gradients_of_extreme_parameters(io):
    # from next to no decay to all of the state at once; gates of every size
    A = np.resize([-1e-6, -1e-3, -1.0, -80.0, -1e6, -3e38], 66).astype(np.float32)
    case = make(1, 300, 66, io, True, seed=3, reset=0.02)
    case["A"] = A
    check(case, io)


def test_one_channel_of_large_decay_leaves_the_others_as_they_were():
    # a channel below -1 sends its warp the other way: the results of the 63 beside it stay within the arithmetic's error
    import torch
    small = _case(2, 500, 64, "f32", "one of a warp", 4)
    small["A"][5] = -0.5
    large = {**small, "A": small["A"].copy()}
    large["A"][5] = -4.0
    got = [check(c, "f32") for c in (small, large)]
    others = torch.arange(64, device="cuda") != 5
    for a, b in zip((got[0][0], got[0][3]["dx"], got[0][3]["dgate"]), (got[1][0], got[1][3]["dx"], got[1][3]["dgate"])):
        a, b = a[..., others], b[..., others]
        assert float((a - b).abs().max()) <= 1e-4 * float(a.abs().max())

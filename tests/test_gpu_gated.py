"""Gated linear recurrence on the GPU against its float64 oracle.

Tolerances: a stored value is rounded once, at most eps / 2 relative (bf16 2^-8, fp32 2^-24), and carries the error of the
float32 arithmetic before it, E times the array's largest value.  E: gates by hardware exponential and reciprocal are good to a few
2^-22 for |gate| <= 6; the error of a retention counts once for every step that the state remembers, about 1 / (1 - a) <= 150 of
them with the gates below, at 2^-25 each if all rounded the same way: E = 1e-5 for the state; gradients are products of
two such quantities and of sums over as many steps again: E = 1e-4."""
import numpy as np
import pytest

from paper_2312_00752_b200 import synth
from tests import _gpu_util as U

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def close(got, ref, io, E, scale=None):
    got = got.detach().double().cpu().numpy()
    assert got.shape == ref.shape
    scale = np.abs(ref).max() if scale is None else scale
    worst = np.abs(got - ref) - HALF[io] * np.abs(ref) - E * scale
    assert np.isfinite(got).all() and worst.max() <= 0, f"{worst.max()} over, of {np.abs(ref).max()}"


def make(batch, L, D, io, decay, seed=0, reset=None, h0=True):
    rng = np.random.default_rng(seed)
    n = lambda *s: synth.round_to_io(rng.standard_normal(s), io)
    case = {"x": n(batch, L, D), "gate": synth.round_to_io(np.clip(rng.standard_normal((batch, L, D)), -3, 3) - 2 * rng.random(D), io),
            "in_gate": n(batch, L, D) if decay else None,
            "A": (8 * np.log(0.9 + 0.099 * rng.random(D))).astype(np.float32) if decay else None,
            "reset": None if reset is None else rng.random((batch, L)) < reset,
            "h0": rng.standard_normal((batch, D)).astype(np.float32) if h0 else None,
            "dy": n(batch, L, D), "dh_last": rng.standard_normal((batch, D)).astype(np.float32)}
    return case


def device(case, io):
    import torch
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    out = {}
    for k, v in case.items():
        t = None if v is None else torch.from_numpy(np.ascontiguousarray(v)).cuda()
        out[k] = t.to(dt) if k in ("x", "gate", "in_gate", "dy") and t is not None else t
    return out


def check(case, io, dev=None, saved_given=True, **kw):
    """Forward and backward of a case against the oracle; returns what the calls returned."""
    import torch
    from oracle import gated_oracle as GO
    from paper_2312_00752_b200 import binding as K
    d = device(case, io) if dev is None else dev
    last = torch.full((case["x"].shape[0], case["x"].shape[2]), float("nan"), device="cuda")
    y, saved = K.ssm_gated_fwd(d["x"], d["gate"], d["in_gate"], d["A"], reset=d["reset"], h0=d["h0"], h_last=last, save_states=True)
    g = K.ssm_gated_bwd(d["x"], d["gate"], d["in_gate"], d["A"], d["dy"], saved if saved_given else None, reset=d["reset"],
                        h0=d["h0"], dh_last=d["dh_last"], want_dh0=True, **kw)
    ref, ref_last = GO.gated_fwd(case["x"], case["gate"], case["in_gate"], case["A"], case["reset"], case["h0"])
    rg = GO.gated_bwd(case["x"], case["gate"], case["in_gate"], case["A"], case["dy"], case["reset"], case["h0"], case["dh_last"])
    close(y, ref, io, 1e-5)
    close(last, ref_last, "f32", 1e-5)
    for k in ("dx", "dgate", "din_gate"):
        if rg[k] is None:
            assert g[k] is None
        else:
            close(g[k], rg[k], io, 1e-4)
    close(g["dh0"], rg["dh0"], "f32", 1e-4, max(1.0, np.abs(rg["dh0"]).max()))
    if rg["dA"] is None:
        assert g["dA"] is None
    else:
        close(g["dA"], rg["dA"], "f32", 1e-5, rg["dA_terms"].max())
    return y, last, saved, g


SHAPES = [
    (2, 200, 64), (1, 1, 64), (3, 1, 7), (2, 15, 66), (1, 16, 40), (1, 17, 2), (2, 33, 1), (1, 127, 130), (2, 128, 64),
    (1, 129, 96), (5, 257, 33), (1, 1025, 256), (2, 2049, 34), (1, 5000, 65), (1, 9001, 64),
]


@pytest.mark.parametrize("decay", [False, True])
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("batch,L,D", SHAPES)
def test_forward_backward(batch, L, D, io, decay):
    check(make(batch, L, D, io, decay, seed=L), io)


@pytest.mark.parametrize("decay", [False, True])
@pytest.mark.parametrize("batch,L,D,io,reset", [(4, 260, 5120, "bf16", None), (8, 515, 1600, "bf16", 0.01), (2, 1100, 1536, "f32", 0.01),
                                                (1, 3000, 2560, "bf16", None)])
def test_layer_widths(batch, L, D, io, reset, decay):
    # (clusters of other sizes than the shapes above, several rounds each)
    check(make(batch, L, D, io, decay, seed=L, reset=reset), io)


@pytest.mark.parametrize("decay", [False, True])
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("batch,L,D,reset", [(2, 300, 64, 0.02), (1, 77, 33, 0.5), (2, 40, 64, 1.0), (3, 1, 64, 1.0), (1, 4100, 48, 0.003)])
def test_packed_sequences(batch, L, D, reset, io, decay):
    check(make(batch, L, D, io, decay, seed=L, reset=reset), io)


@pytest.mark.parametrize("decay", [False, True])
@pytest.mark.parametrize("batch,L,D,io", [(2, 200, 64, "bf16"), (1, 1300, 33, "f32"), (2, 70, 7, "bf16"), (1, 2500, 64, "f32")])
def test_states_rebuilt_by_backward(batch, L, D, io, decay):
    import torch
    case = make(batch, L, D, io, decay, seed=1, reset=0.01, h0=False)
    *_, g = check(case, io)
    *_, h = check(case, io, saved_given=False)
    assert all(torch.equal(g[k], h[k]) for k in g if g[k] is not None)


def _columns(case, io, D, pad):
    """x, gate, in_gate as column ranges of one buffer, and buffers of the same kind for their gradients."""
    import torch
    d = device(case, io)
    names = [k for k in ("x", "gate", "in_gate") if d[k] is not None]
    batch, L, _ = case["x"].shape
    wide = torch.full((batch, L, len(names) * (D + pad) + pad), float("nan"), dtype=d["x"].dtype, device="cuda")
    grads = torch.full_like(wide, 7.0)
    outputs = {}
    for i, k in enumerate(names):
        at = slice(pad + i * (D + pad), pad + i * (D + pad) + D)
        wide[..., at] = d[k]
        d[k] = wide[..., at]
        outputs["d" + k] = grads[..., at]
    return d, outputs, grads


@pytest.mark.parametrize("decay", [False, True])
@pytest.mark.parametrize("batch,L,D,io,pad", [(2, 150, 64, "bf16", 0), (2, 150, 64, "bf16", 2), (1, 70, 64, "bf16", 3),
                                              (2, 33, 31, "f32", 1), (3, 1, 64, "f32", 0), (1, 1100, 64, "f32", 5)])
def test_column_ranges_of_a_projection(batch, L, D, io, pad, decay):
    import torch
    case = make(batch, L, D, io, decay, seed=2, reset=0.02)
    d, outputs, grads = _columns(case, io, D, pad)
    y, last, saved, g = check(case, io, dev=d, outputs=outputs)
    names = list(outputs)
    assert all(g[k].data_ptr() == outputs[k].data_ptr() for k in names)
    for v in outputs.values():
        v.fill_(7.0)
    assert bool((grads == 7.0).all())                      # nothing was written between the columns
    if pad == 0 or io == "f32" and D % 4:        # (as aligned as the dense ones: the same kernel)
        y2, last2, saved2, g2 = check(case, io)
        assert torch.equal(y, y2) and torch.equal(last, last2) and torch.equal(saved, saved2)
        assert torch.equal(g["dh0"], g2["dh0"]) and (not decay or torch.equal(g["dA"], g2["dA"]))


@pytest.mark.parametrize("decay", [False, True])
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [1, 2, 4])
def test_unaligned_pointers(offset, io, decay):
    import torch
    case = make(2, 300, 64, io, decay, seed=4)
    d = device(case, io)
    for k, v in d.items():
        if v is not None:
            flat = torch.empty(v.numel() + offset, dtype=v.dtype, device="cuda")
            flat[offset:] = v.flatten()
            d[k] = flat[offset:].view_as(v)
    check(case, io, dev=d)


@pytest.mark.parametrize("decay", [False, True])
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_steps_one_by_one_are_the_sequence(io, decay):
    import torch
    from paper_2312_00752_b200 import binding as K
    batch, L, D = 3, 40, 130
    case = make(batch, L, D, io, decay, seed=6, reset=0.1)
    y, last, _, _ = check(case, io)
    d = device(case, io)
    h = d["h0"].clone()
    for t in range(L):
        out = K.ssm_gated_step(d["x"][:, t], d["gate"][:, t], None if not decay else d["in_gate"][:, t], d["A"], h, reset=d["reset"][:, t].contiguous())
        close(out, y[:, t].double().cpu().numpy(), io, 1e-5 + HALF[io])
    close(h, last.double().cpu().numpy(), "f32", 1e-5)


@pytest.mark.parametrize("batch,D,io", [(1, 64, "bf16"), (1, 1, "f32"), (64, 2560, "bf16"), (5, 1001, "bf16"), (256, 96, "f32")])
@pytest.mark.parametrize("decay", [False, True])
def test_step(batch, D, io, decay):
    from oracle import gated_oracle as GO
    from paper_2312_00752_b200 import binding as K
    case = make(batch, 1, D, io, decay, seed=8)
    d = device(case, io)
    h = d["h0"].clone()
    y = K.ssm_gated_step(d["x"][:, 0], d["gate"][:, 0], d["in_gate"][:, 0] if decay else None, d["A"], h)
    _, last = GO.gated_fwd(case["x"], case["gate"], case["in_gate"], case["A"], None, case["h0"])
    close(y, last, io, 1e-5)
    close(h, last, "f32", 1e-5)


@pytest.mark.parametrize("decay", [False, True])
@pytest.mark.parametrize("L", [3, 300, 3000])
def test_a_sequence_in_pieces(L, decay):
    from paper_2312_00752_b200 import binding as K
    import torch
    case = make(2, L, 64, "f32", decay, seed=9, reset=0.01)
    y, last, _, g = check(case, "f32")
    d = device(case, "f32")
    cut = L // 3
    part = lambda lo, hi: [None if d[k] is None else d[k][:, lo:hi].contiguous() for k in ("x", "gate", "in_gate")] + [d["A"]]
    reset = lambda lo, hi: d["reset"][:, lo:hi].contiguous()
    mid, end = torch.empty_like(last), torch.empty_like(last)
    y1 = K.ssm_gated_fwd(*part(0, cut), reset=reset(0, cut), h0=d["h0"], h_last=mid)
    y2 = K.ssm_gated_fwd(*part(cut, L), reset=reset(cut, L), h0=mid, h_last=end)
    close(torch.cat([y1, y2], 1), y.double().cpu().numpy(), "f32", 1e-5)
    g2 = K.ssm_gated_bwd(*part(cut, L), d["dy"][:, cut:].contiguous(), reset=reset(cut, L), h0=mid, dh_last=d["dh_last"], want_dh0=True)
    g1 = K.ssm_gated_bwd(*part(0, cut), d["dy"][:, :cut].contiguous(), reset=reset(0, cut), h0=d["h0"], dh_last=g2["dh0"], want_dh0=True)
    for k in ("dx", "dgate", "din_gate"):
        if g[k] is not None:
            close(torch.cat([g1[k], g2[k]], 1), g[k].double().cpu().numpy(), "f32", 1e-4)
    close(g1["dh0"], g["dh0"].double().cpu().numpy(), "f32", 1e-4, 1.0)


def test_extreme_gates():
    # gates that saturate either way: retention of exactly one step or of all of them; nothing but finite numbers comes out
    import torch
    from oracle import gated_oracle as GO
    from paper_2312_00752_b200 import binding as K
    L, levels = 64, [-200.0, -95.0, -60.0, -30.0, 30.0, 60.0, 95.0, 200.0]
    rng = np.random.default_rng(3)
    for decay in (False, True):
        case = make(1, L, len(levels) ** 2, "f32", decay, seed=10)
        case["gate"] = np.tile(np.repeat(levels, len(levels)), (1, L, 1)).astype(np.float32)
        if decay:
            case["in_gate"] = np.tile(np.tile(levels, len(levels)), (1, L, 1)).astype(np.float32)
        check(case, "f32")
    A = np.array([0.0, -1e-30, -1e-6, -1.0, -80.0, -1e6, -3e38, -1e-3] * 8, np.float32)      # no decay at all .. all at once
    case["gate"] = np.clip(rng.standard_normal((1, L, 64)), -3, 3).astype(np.float32)
    case["A"] = A
    d = device(case, "f32")
    y, saved = K.ssm_gated_fwd(d["x"], d["gate"], d["in_gate"], d["A"], h0=d["h0"], save_states=True)
    close(y, GO.gated_fwd(case["x"], case["gate"], case["in_gate"], A, None, case["h0"])[0], "f32", 1e-5)
    g = K.ssm_gated_bwd(d["x"], d["gate"], d["in_gate"], d["A"], d["dy"], saved, h0=d["h0"])
    assert all(bool(torch.isfinite(v).all()) for k, v in g.items() if v is not None)


@pytest.mark.parametrize("decay", [False, True])
@pytest.mark.parametrize("L", [40, 700, 5000])
def test_infinities_and_nan_stay_in_their_sequence(L, decay):
    import torch
    from paper_2312_00752_b200 import binding as K
    case = make(1, L, 66, "f32", decay, seed=11)
    case["reset"] = np.zeros((1, L), bool)
    cut = L // 2 + 1
    case["reset"][0, cut] = True
    clean, last, _, g = check(case, "f32")
    at = L // 3
    for bad in (float("inf"), float("-inf"), float("nan")):
        d = device(case, "f32")
        d["x"][0, at, 5] = bad
        h = torch.empty_like(last)
        y, saved = K.ssm_gated_fwd(d["x"], d["gate"], d["in_gate"], d["A"], reset=d["reset"], h0=d["h0"], h_last=h, save_states=True)
        ok = torch.ones_like(clean, dtype=torch.bool)
        ok[0, at:cut, 5] = False
        assert torch.equal(y[ok], clean[ok]) and torch.equal(h, last)
        hit = y[0, at:cut, 5]
        assert bool(torch.isnan(hit).all()) if bad != bad else bool((hit == bad).all())
        b = K.ssm_gated_bwd(d["x"], d["gate"], d["in_gate"], d["A"], d["dy"], saved, reset=d["reset"], h0=d["h0"], dh_last=d["dh_last"])
        assert torch.equal(b["dx"], g["dx"])               # (no state is in it)
        assert torch.equal(b["dgate"][ok], g["dgate"][ok])
        # a gradient that is not finite does not pass the reset backwards
        d = device(case, "f32")
        d["dy"][0, L - 2, 7] = bad
        b = K.ssm_gated_bwd(d["x"], d["gate"], d["in_gate"], d["A"], d["dy"], None, reset=d["reset"], h0=d["h0"], dh_last=d["dh_last"])
        ok = torch.ones_like(clean, dtype=torch.bool)
        ok[0, cut:L - 1, 7] = False
        assert all(torch.equal(b[k][ok], g[k][ok]) for k in ("dx", "dgate"))
        # an infinite state before the first step is kept, whatever the product of the retentions is
        d = device(case, "f32")
        d["h0"][0, 3] = bad
        y = K.ssm_gated_fwd(d["x"], d["gate"], d["in_gate"], d["A"], h0=d["h0"], h_last=h)
        assert bool(torch.isnan(y[0, :, 3]).all()) if bad != bad else bool((y[0, :, 3] == bad).all())


def test_rows_past_32_bits():
    import torch
    from paper_2312_00752_b200 import binding as K
    L, D, ld = 70000, 64, 32768
    case = make(1, L, D, "bf16", False, seed=12)
    d = device(case, "bf16")
    wide = torch.empty(1, L, ld, dtype=torch.bfloat16, device="cuda")      # 2.3e9 elements
    grads = torch.empty_like(wide)
    at = {"x": slice(100, 164), "gate": slice(ld - 64, ld)}
    for k, s in at.items():
        wide[..., s] = d[k]
    y, saved = K.ssm_gated_fwd(d["x"], d["gate"], save_states=True, h0=d["h0"])
    y2, saved2 = K.ssm_gated_fwd(wide[..., at["x"]], wide[..., at["gate"]], save_states=True, h0=d["h0"])
    assert torch.equal(y, y2) and torch.equal(saved, saved2)
    g = K.ssm_gated_bwd(d["x"], d["gate"], None, None, d["dy"], saved, h0=d["h0"])
    K.ssm_gated_bwd(wide[..., at["x"]], wide[..., at["gate"]], None, None, d["dy"], saved, h0=d["h0"],
                    outputs={"dx": grads[..., at["x"]], "dgate": grads[..., at["gate"]]})
    assert torch.equal(grads[..., at["x"]], g["dx"]) and torch.equal(grads[..., at["gate"]], g["dgate"])


@pytest.mark.parametrize("decay", [False, True])
def test_runs_repeat_bit_for_bit_and_in_a_graph_and_on_a_stream(decay):
    import torch
    from paper_2312_00752_b200 import binding as K
    case = make(2, 900, 320, "bf16", decay, seed=13, reset=0.01)
    d = device(case, "bf16")

    def run(saved_given=True, **kw):
        last = torch.empty(2, 320, device="cuda")
        y, saved = K.ssm_gated_fwd(d["x"], d["gate"], d["in_gate"], d["A"], reset=d["reset"], h0=d["h0"], h_last=last, save_states=True, **kw)
        g = K.ssm_gated_bwd(d["x"], d["gate"], d["in_gate"], d["A"], d["dy"], saved if saved_given else None, reset=d["reset"],
                            h0=d["h0"], dh_last=d["dh_last"], want_dh0=True, **kw)
        return [y, last, saved, *[v for v in g.values() if v is not None]]

    ref = run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for kw in ({}, {"saved_given": False}, {"stream": s}):
        torch.cuda.synchronize()               # (what is allocated here belongs to the current stream)
        got = run(**kw)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(ref, got))
    with torch.cuda.stream(s):
        run(False)
    graphs = []
    for _ in range(2):                     # two graphs, replayed side by side: neither works in the other's scratch
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = run(False)
        graphs.append((graph, got))
    for _, got in graphs:
        for v in got:
            v.zero_()
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(s):
            graphs[0][0].replay()
        with torch.cuda.stream(other):
            graphs[1][0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for _, got in graphs for p, q in zip(ref, got))


def test_refusals():
    import torch
    from paper_2312_00752_b200 import binding as K
    bf = torch.bfloat16
    x = torch.randn(2, 10, 8, device="cuda")
    gate, A, h = torch.randn_like(x), -torch.ones(8, device="cuda"), torch.zeros(2, 8, device="cuda")
    fwd, bwd, step = K.ssm_gated_fwd, K.ssm_gated_bwd, K.ssm_gated_step
    bad = [
        lambda: fwd(x, gate.to(bf)), lambda: fwd(x, gate[:, :9]), lambda: fwd(x.half(), gate.half()), lambda: fwd(x, None),
        lambda: fwd(x, gate, gate), lambda: fwd(x, gate, None, A), lambda: fwd(x, gate, gate, A.double()), lambda: fwd(x, gate, gate, A[:7]),
        lambda: fwd(x.transpose(0, 1), gate.transpose(0, 1)), lambda: fwd(x.transpose(1, 2), gate.transpose(1, 2)),
        lambda: fwd(x, gate[:, :1].expand(2, 10, 8)), lambda: fwd(x, gate[:1].expand(2, 10, 8)), lambda: fwd(x, gate[..., ::2]),
        lambda: fwd(x[:, ::2][:, :4], gate[:, :4]), lambda: fwd(x[0], gate[0]), lambda: fwd(x, gate.cpu()),
        lambda: fwd(x, gate, reset=torch.zeros(2, 9, device="cuda", dtype=torch.bool)), lambda: fwd(x, gate, reset=torch.zeros(2, 10, device="cuda")),
        lambda: fwd(x, gate, h0=h.to(bf)), lambda: fwd(x, gate, h0=h[:1]), lambda: fwd(x, gate, h_last=h.t()), lambda: fwd(x, gate, out=x[..., :7]),
        lambda: fwd(x, gate, out=torch.empty(2, 8, 10, device="cuda").transpose(1, 2)), lambda: fwd(x, gate, h0=h.cpu()),
        lambda: fwd(x, gate, save_states=True, saved_states=torch.empty(3, device="cuda")), lambda: fwd(x[:0], gate[:0]), lambda: fwd(x[:, :0], gate[:, :0]),
        lambda: bwd(x, gate, None, None, None), lambda: bwd(x, gate, None, None, x.to(bf)), lambda: bwd(x, gate, None, None, x, torch.empty(5, device="cuda")),
        lambda: bwd(x, gate, None, None, x, outputs={"dx": x[:, :5]}), lambda: bwd(x, gate, None, None, x, dh_last=h[:, :4]),
        lambda: bwd(x, gate, None, None, x, outputs={"dgate": torch.empty(2, 8, 10, device="cuda").transpose(1, 2)}),
        lambda: step(x, gate, None, None, h), lambda: step(x[:, 0], gate[:, 0], None, None, None), lambda: step(x[:, 0], gate[:, 0], None, None, h[:1]),
        lambda: step(x[:, 0], gate[:, 0], None, None, h, reset=torch.zeros(3, device="cuda", dtype=torch.bool)),
    ]
    for call in bad:
        with pytest.raises(K.SsmScanError):
            call()
    every = fwd(x, gate)                        # (rows of every second batch entry or step lie evenly spaced or are refused)
    wide = torch.randn(4, 10, 8, device="cuda")
    with pytest.raises(K.SsmScanError):
        fwd(wide[::2], gate)
    assert torch.equal(fwd(x[:, ::2], gate[:, ::2].contiguous()), fwd(x[:, ::2].contiguous(), gate[:, ::2].contiguous())) and every.shape == x.shape


def test_against_differences_of_the_call_itself():
    import torch
    from paper_2312_00752_b200 import binding as K
    case = make(1, 50, 4, "f32", True, seed=14, reset=0.05)
    d = device(case, "f32")
    y, last, _, g = check(case, "f32")

    def loss(**over):
        v = {**d, **over}
        h = torch.empty_like(last)
        out = K.ssm_gated_fwd(v["x"], v["gate"], v["in_gate"], v["A"], reset=d["reset"], h0=v["h0"], h_last=h)
        return float((out.double() * d["dy"].double()).sum() + (h.double() * d["dh_last"].double()).sum())

    rng = np.random.default_rng(0)
    for name in ("x", "gate", "in_gate", "A", "h0"):
        way = torch.from_numpy(rng.standard_normal(d[name].shape)).cuda()
        eps = 2.0 ** -10
        up, down = ((d[name].double() + s * eps * way).float() for s in (1, -1))
        num = (loss(**{name: up}) - loss(**{name: down})) / (2 * eps)
        want = float((g["d" + name].double() * way).sum())
        # differences of sums of a few hundred terms of size 1, each good to 1e-6, over 2^-9; and eps^2 of the third derivative
        assert abs(num - want) <= 2e-2 + 1e-3 * abs(want), (name, num, want)


def test_results_of_a_call_on_another_stream_are_no_memory_that_the_current_one_still_writes():
    import torch
    from paper_2312_00752_b200 import binding as K
    x, gate, w = torch.randn(4, 1000, 64, device="cuda"), torch.randn(4, 1000, 64, device="cuda"), torch.ones(64, device="cuda")
    s = torch.cuda.Stream()
    run = lambda **kw: (K.ssm_gated_fwd(x, gate, **kw), K.ssm_norm_fwd(x, w, **kw))
    ref = run()
    run(stream=s)
    torch.cuda.synchronize()
    late = [torch.empty_like(x) for _ in range(8)]
    torch.cuda._sleep(400_000_000)                # the writes below wait behind this, a fifth of a second
    for v in late:
        v.fill_(7.0)
    v = late = None                               # (their memory is free again for the current stream, in its order)
    got = run(stream=s)
    s.synchronize()
    assert not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ref, got))

"""The operators of a residual block as they are used together: norm with residual add, projection, short convolution, gated
recurrence, projection back; a prompt and then tokens one by one against the whole sequence at once, and the block's gradients
against float64 autograd of its definition."""
import pytest

pytestmark = pytest.mark.gpu

E, W = 96, 4


def _parameters(D, dtype, seed=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s, dt=torch.float32, scale=1.0: torch.randn(*s, generator=g, device="cuda").mul(scale).to(dt)
    return {"norm": 1 + 0.1 * n(D), "into": n(D, 3 * E, dt=dtype, scale=D ** -0.5), "taps": n(E, W, scale=0.5), "bias": 0.1 * n(E),
            "A": -(0.01 + 0.5 * torch.rand(E, generator=g, device="cuda")), "back": n(E, D, dt=dtype, scale=E ** -0.5)}


def _block(p, x, residual, cache=None, reset=None):
    """One block on (batch, L, D): what goes to the next block, and the residual stream; `cache` is carried along."""
    import torch
    from paper_2312_00752_b200 import binding as K
    y, residual = K.ssm_norm_fwd(x, p["norm"], None, residual, rms=True)
    wide = y @ p["into"]
    v, gate, in_gate = wide.split(E, dim=-1)
    v = v.contiguous()
    last = torch.empty(x.shape[0], E, device="cuda")
    prev = h0 = None
    if cache is not None and cache:
        prev, h0 = cache["conv"], cache["h"]
    c = K.ssm_conv1d_fwd(v, p["taps"], p["bias"], x_prev=prev)
    h = K.ssm_gated_fwd(c, gate, in_gate, p["A"], reset=reset, h0=h0, h_last=last)
    if cache is not None:
        before = v if prev is None else torch.cat([prev, v], 1)
        cache.update(conv=before[:, -(W - 1):].contiguous(), h=last)
    return h @ p["back"], residual


def _token(p, x, residual, cache):
    """The block on one token, (batch, D)."""
    import torch
    from paper_2312_00752_b200 import binding as K
    y, residual = K.ssm_norm_fwd(x, p["norm"], None, residual, rms=True)
    v, gate, in_gate = (y @ p["into"]).split(E, dim=-1)
    v = v.contiguous()[:, None]
    c = K.ssm_conv1d_fwd(v, p["taps"], p["bias"], x_prev=cache["conv"])
    cache["conv"] = torch.cat([cache["conv"], v], 1)[:, 1:].contiguous()
    h = K.ssm_gated_step(c[:, 0], gate, in_gate, p["A"], cache["h"])
    return h @ p["back"], residual


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_prompt_and_tokens_are_the_sequence(io):
    import torch
    dtype = torch.bfloat16 if io == "bf16" else torch.float32
    batch, L, D, layers = 2, 37, 64, 3
    torch.backends.cuda.matmul.allow_tf32 = False
    ps = [_parameters(D, dtype, seed=k) for k in range(layers)]
    x = torch.randn(batch, L, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(9)).to(dtype)

    def whole(x):
        out, res = x, torch.zeros(batch, x.shape[1], D, device="cuda")
        for p in ps:
            out, res = _block(p, out, res)
        return res + out.float()

    def tokens(x, prompt):
        caches = [{} for _ in ps]
        out, res = x[:, :prompt].contiguous(), torch.zeros(batch, prompt, D, device="cuda")
        for p, c in zip(ps, caches):
            out, res = _block(p, out, res, c)
        got = [res + out.float()]
        for t in range(prompt, x.shape[1]):
            out, res = x[:, t].contiguous(), torch.zeros(batch, D, device="cuda")
            for p, c in zip(ps, caches):
                out, res = _token(p, out, res, c)
            got.append((res + out.float())[:, None])
        return torch.cat(got, 1)

    want, got = whole(x), tokens(x, 20)
    # float32: the same sums in other orders.  bf16: every layer rounds its norm, projection, convolution, state and result, the
    # matrix products of one token and of many may add in other orders and round the other way: one step (2^-7) of the
    # values at some of these five places in each of three layers
    tol = {"f32": 1e-4, "bf16": 15 * 2.0 ** -7}[io]
    scale = float(want.abs().max())
    assert scale > 1 and float((got - want).abs().max()) <= tol * scale
    assert float((got - want).norm() / want.norm()) <= {"f32": 1e-5, "bf16": 15 * 2.0 ** -8}[io]


def test_gradients_of_a_block_against_autograd_of_its_definition():
    import torch
    from paper_2312_00752_b200 import binding as K
    torch.backends.cuda.matmul.allow_tf32 = False
    batch, L, D = 2, 70, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")
    p = _parameters(D, torch.float32)
    x, residual, dout, dres = n(batch, L, D), n(batch, L, D), n(batch, L, D), n(batch, L, D)
    reset = torch.rand(batch, L, generator=g, device="cuda") < 0.05
    # forward and backward by the library
    y, s, stats = K.ssm_norm_fwd(x, p["norm"], None, residual, rms=True, save_stats=True)
    wide = y @ p["into"]
    v, gate, in_gate = wide.split(E, dim=-1)
    v = v.contiguous()
    c = K.ssm_conv1d_fwd(v, p["taps"], p["bias"])
    h, saved = K.ssm_gated_fwd(c, gate, in_gate, p["A"], reset=reset, save_states=True)
    out = h @ p["back"]
    dh = dout @ p["back"].t()
    dwide = torch.empty_like(wide)
    dv, dgate, din = dwide.split(E, dim=-1)
    gg = K.ssm_gated_bwd(c, gate, in_gate, p["A"], dh, saved, reset=reset, outputs={"dgate": dgate, "din_gate": din})
    gc = K.ssm_conv1d_bwd(v, p["taps"], p["bias"], gg["dx"])
    dv.copy_(gc["dx"])
    gn = K.ssm_norm_bwd(s, p["norm"], dwide @ p["into"].t(), stats, dres, rms=True)
    got = {"x": gn["dx"], "norm": gn["dweight"], "into": y.flatten(0, 1).t() @ dwide.flatten(0, 1), "taps": gc["dw"], "bias": gc["dbias"],
           "A": gg["dA"], "back": h.flatten(0, 1).t() @ dout.flatten(0, 1)}
    # its definition, in float64
    leaves = {k: t.double().requires_grad_() for k, t in {"x": x, **p}.items()}
    q = leaves
    s64 = q["x"] + residual.double()
    w64 = (s64 * torch.rsqrt(s64.square().mean(-1, keepdim=True) + 1e-5) * q["norm"]) @ q["into"]
    v64, g64, i64 = w64.split(E, dim=-1)
    pad = torch.nn.functional.pad(v64, (0, 0, W - 1, 0))
    c64 = torch.nn.functional.silu(sum(pad[:, k:k + L] * q["taps"][:, k] for k in range(W)) + q["bias"])
    la = torch.sigmoid(g64) * q["A"]
    u = torch.sqrt(-torch.expm1(2 * la)) * torch.sigmoid(i64) * c64
    state, hs = torch.zeros(batch, E, dtype=torch.float64, device="cuda"), []
    for t in range(L):
        state = torch.exp(la[:, t]) * torch.where(reset[:, t, None], 0.0, state) + u[:, t]
        hs.append(state)
    h64 = torch.stack(hs, 1)
    o64 = h64 @ q["back"]
    ((o64 * dout.double()).sum() + (s64 * dres.double()).sum()).backward()
    o64 = o64.detach()
    assert float((out - o64).norm() / o64.norm()) <= 1e-5
    for k, t in got.items():
        ref = leaves[k].grad
        assert float((t.double() - ref).norm() / ref.norm()) <= 1e-4, k

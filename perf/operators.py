"""The operators of a residual block around the scan, as measurable cases: the gated linear recurrence and the norm with
its residual add, each in a plain form of elementary torch operations and as the library's calls.

A case is a dict of plain values:

* `op`       "gated" (forward, carried state in and out), "gated_train" (forward that saves its states, then backward),
             "gated_step" (one decoding step), "norm" (forward) or "norm_train" (forward, then backward).
* `io`       element type of the activations: "bf16" or "f32".
* `batch`, `L`, `D`: shape of a recurrence; `rows`, `D`: shape of a norm.
* `form`     of a recurrence: "convex" (h = (1 - g) h + g x, g = sigmoid(gate): the gating that a selective scan of one
             state reduces to) or "decay" (a = exp(sigmoid(gate) A), h = a h + sqrt(1 - a^2) sigmoid(in_gate) x).
* `packed`   sequences of uneven lengths lie one behind the other in a row; a mask tells where each begins.
* `split`    x, gate (and in_gate) are column ranges of one projection's result: rows further apart than D.
* `rms`      a norm without mean and bias; otherwise a layer norm.
* `residual` "none", or the element type of the residual stream that x is added to.

Values: x, dy ~ N(0, 1); gate, in_gate ~ N(0, 1), the former moved by a channel's offset, so that a channel remembers from
a few steps to some hundreds; A = 8 log(a) with a uniform in 0.9 .. 0.999.
"""
from __future__ import annotations

import math

import torch

own = False

_IO = {"bf16": torch.bfloat16, "f32": torch.float32}
_GATED = {"io": "bf16", "form": "decay", "packed": False, "split": False}
_NORM = {"io": "bf16", "rms": False, "residual": "none"}


def _gated(op, batch, L, D, **kw):
    return {"op": op, "batch": batch, "L": L, "D": D, **_GATED, **kw}


def _norm(op, rows, D, **kw):
    return {"op": op, "rows": rows, "D": D, **_NORM, **kw}


def listed():
    cases = {
        # one token of one sequence through a layer of 2.8B width: the smallest call, a launch and little else
        "step_b1": _gated("gated_step", 1, 1, 5120),
        # one token of a decoding batch, in full precision
        "step_b64_f32": _gated("gated_step", 64, 1, 5120, form="convex", io="f32"),
        # prefill of a batch at 2.8B width, the three inputs cut from one projection
        "prefill_convex": _gated("gated", 4, 2048, 5120, form="convex", split=True),
        # one long document at 130M width, continuing from a carried state: few channels, many steps
        "long_decay": _gated("gated", 1, 131072, 1536),
        # nothing divides anything
        "odd_f32": _gated("gated", 3, 1237, 1001, io="f32"),
        # training of a wide layer on packed documents
        "train_decay": _gated("gated_train", 8, 2048, 2560, packed=True, split=True),
        # full-precision training at 130M width
        "train_convex_f32": _gated("gated_train", 2, 2048, 1536, form="convex", io="f32"),
        # the norm in front of a layer while one token is decoded, residual stream in full precision
        "norm_token": _norm("norm", 1, 2560, rms=True, residual="f32"),
        # the same for a batch's prefill, residual stream in bf16
        "norm_prefill": _norm("norm", 8192, 2560, residual="bf16"),
        # training at 2.8B width, residual stream in full precision
        "norm_train_rms": _norm("norm_train", 8192, 2560, rms=True, residual="f32"),
        # training, layer norm with bias over the inner width, no residual
        "norm_train_wide": _norm("norm_train", 8192, 5120),
        # nothing divides anything, in full precision
        "norm_train_odd_f32": _norm("norm_train", 3711, 1001, io="f32"),
    }
    return [{"name": name, **c} for name, c in cases.items()]


def _log(rng, lo, hi, multiple=1):
    """A whole number in [lo, hi], uniform over its logarithm, rounded to a multiple."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi // multiple, max(-(-lo // multiple), round(v / multiple))) * multiple


def _width(rng, lo, hi):
    """A channel count: multiples of 64 as models have them, more rarely of 8, of 2 or anything."""
    return _log(rng, lo, hi, rng.choice((64, 64, 64, 8, 8, 2, 1)))


def draw(rng):
    kind = rng.choice(("step", "prefill", "prefill", "long", "train", "train", "odd", "norm", "norm_train", "norm_train"))
    io = rng.choice(("bf16", "bf16", "f32"))
    form, packed, split = rng.choice(("convex", "decay")), rng.random() < 0.4, rng.random() < 0.5
    if kind == "step":
        return _gated("gated_step", _log(rng, 1, 256), 1, _width(rng, 512, 8192), form=form, io=io)
    if kind == "long":
        return _gated("gated", 1, _log(rng, 16384, 131072), _log(rng, 256, 1536, 64), form=form, packed=packed)
    if kind == "odd":
        return _gated(rng.choice(("gated", "gated_train")), rng.randint(1, 4), _log(rng, 1, 2048) | 1,
                      _log(rng, 33, 1536) | 1, form=form, io=io, packed=packed, split=split)
    if kind in ("prefill", "train"):
        batch = rng.randint(1, 8)
        L = _log(rng, 17, (16384 if io == "bf16" else 8192) // batch)
        return _gated("gated" if kind == "prefill" else "gated_train", batch, L, _width(rng, 512, 2560), form=form, io=io,
                      packed=packed, split=split)
    residual = rng.choice(("none", "f32", "f32" if io == "f32" else "bf16"))
    return _norm(kind, _log(rng, 1, 8192), _width(rng, 64, 5120), io=io, rms=rng.random() < 0.5, residual=residual)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    io, D = _IO[case["io"]], case["D"]

    def normal(*shape, dtype=io):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    s = {"op": case["op"]}
    if case["op"] in ("norm", "norm_train"):
        rows = case["rows"]
        s["rms"], s["eps"] = case["rms"], 1e-5
        s["x"] = normal(rows, D)
        s["residual"] = None if case["residual"] == "none" else normal(rows, D, dtype=_IO[case["residual"]]).mul_(2.0)
        s["weight"] = 1.0 + 0.2 * normal(D, dtype=torch.float32)
        s["bias"] = None if case["rms"] else 0.2 * normal(D, dtype=torch.float32)
        if case["op"] == "norm_train":
            s["dy"] = normal(rows, D)
            s["dresidual_out"] = None if s["residual"] is None else normal(rows, D, dtype=s["residual"].dtype)
        return s

    batch, L, decay = case["batch"], case["L"], case["form"] == "decay"
    shape = (batch, D) if case["op"] == "gated_step" else (batch, L, D)
    n = 3 if decay else 2
    if case["split"]:
        parts = normal(*shape[:-1], n * D).split(D, dim=-1)
    else:
        parts = [normal(*shape) for _ in range(n)]
    s["x"], s["gate"], s["in_gate"] = parts[0], parts[1], parts[2] if decay else None
    if decay:
        s["A"] = 8.0 * torch.log(0.9 + 0.099 * uniform(D))
    else:
        s["A"] = None
        s["gate"] -= (5.0 * uniform(D)).to(io)
    if case["op"] == "gated_step":
        s["h"] = normal(batch, D, dtype=torch.float32)
        return s
    s["reset"] = None
    if case["packed"]:
        s["reset"] = uniform(batch, L) < 1.0 / 300.0      # (the first sequence of a row may continue from h0)
    s["h0"] = normal(batch, D, dtype=torch.float32)
    s["h_last"] = torch.empty(batch, D, device="cuda")
    if case["op"] == "gated_train":
        s["dy"] = normal(batch, L, D)
    return s


# ------------------------------------------------------------------------------------------- the plain forms (32 bits)
def _shift(v, k, fill):
    """v a further k steps down the second axis, `fill` in front."""
    return torch.cat([torch.full_like(v[:, :k], fill), v[:, :-k]], dim=1)


def _scan(a, u):
    """h_t = a_t h_{t-1} + u_t from zero, by doubling: after the step of width k an element stands for 2 k steps.  (The loop
    runs over the logarithm of the length; a product of exponentials would leave the range of 32 bits.)"""
    k = 1
    while k < u.shape[1]:
        u = torch.addcmul(u, a, _shift(u, k, 0.0))
        a = a * _shift(a, k, 1.0)
        k *= 2
    return u


def _gates(x, gate, in_gate, A):
    """Retention a, input u and what the gradients need: g (convex) or rho, iota, beta (decay)."""
    if A is None:
        g = torch.sigmoid(gate)
        return torch.sigmoid(-gate), g * x, (g,)
    rho, iota = torch.sigmoid(gate), torch.sigmoid(in_gate)
    la = rho * A
    beta = torch.sqrt(-torch.expm1(2.0 * la))
    return torch.exp(la), beta * iota * x, (rho, iota, beta)


def _f32(s, *names):
    return [None if s[n] is None else s[n].float() for n in names]


def _plain_states(s):
    x, gate, in_gate, A = _f32(s, "x", "gate", "in_gate", "A")
    a, u, parts = _gates(x, gate, in_gate, A)
    keep = a if s["reset"] is None else torch.where(s["reset"][:, :, None], 0.0, a)
    first = torch.addcmul(u[:, :1], keep[:, :1], s["h0"][:, None])
    h = _scan(keep, torch.cat([first, u[:, 1:]], dim=1))
    return x, gate, in_gate, A, a, keep, parts, h


def _plain_gated(s):
    h = _plain_states(s)[-1]
    return {"y": h.to(s["x"].dtype), "h_last": h[:, -1].clone()}


def _plain_gated_train(s):
    io = s["x"].dtype
    x, gate, in_gate, A, a, keep, parts, h = _plain_states(s)
    prev = torch.cat([s["h0"][:, None], h[:, :-1]], dim=1)
    if s["reset"] is not None:
        prev = torch.where(s["reset"][:, :, None], 0.0, prev)
    after = torch.cat([keep[:, 1:], torch.ones_like(keep[:, :1])], dim=1)      # what carries the adjoint back from t + 1
    mu = _scan(after.flip(1), s["dy"].float().flip(1)).flip(1)
    out = {"y": h.to(io), "dh0": keep[:, 0] * mu[:, 0]}
    if A is None:
        (g,) = parts
        out["dx"] = (mu * g).to(io)
        out["dgate"] = (mu * (x - prev) * g * a).to(io)
        return out
    rho, iota, beta = parts
    out["dx"] = (mu * beta * iota).to(io)
    out["din_gate"] = (mu * beta * x * iota * torch.sigmoid(-in_gate)).to(io)
    dla = mu * (a * prev - a * a * iota * x / beta)
    out["dgate"] = (dla * A * rho * torch.sigmoid(-gate)).to(io)
    out["dA"] = (dla * rho).sum(dim=(0, 1))
    return out


def _plain_step(s):
    x, gate, in_gate, A = _f32(s, "x", "gate", "in_gate", "A")
    a, u, _ = _gates(x, gate, in_gate, A)
    s["h"].copy_(torch.addcmul(u, a, s["h"]))
    return {"y": s["h"].to(s["x"].dtype), "h": s["h"]}


def _plain_norm(s):
    io = s["x"].dtype
    total = s["x"].float()
    out = {}
    if s["residual"] is not None:
        kept = (total + s["residual"].float()).to(s["residual"].dtype)
        out["residual_out"], total = kept, kept.float()
    centred = total if s["rms"] else total - total.mean(dim=-1, keepdim=True)
    rstd = torch.rsqrt(centred.square().mean(dim=-1, keepdim=True) + s["eps"])
    xhat = centred * rstd
    y = xhat * s["weight"]
    out["y"] = (y if s["bias"] is None else y + s["bias"]).to(io)
    return out, xhat, rstd


def _plain_norm_train(s):
    io, dy = s["x"].dtype, s["dy"].float()
    out, xhat, rstd = _plain_norm(s)
    q = dy * s["weight"]
    ds = q - xhat * (q * xhat).mean(dim=-1, keepdim=True)
    if not s["rms"]:
        ds = ds - q.mean(dim=-1, keepdim=True)
    ds = ds * rstd
    if s["residual"] is not None:
        ds = ds + s["dresidual_out"].float()
        out["dresidual"] = ds.to(s["residual"].dtype)
    out["dx"] = ds.to(io)
    out["dweight"] = (dy * xhat).sum(dim=0)
    if s["bias"] is not None:
        out["dbias"] = dy.sum(dim=0)
    return out


# --------------------------------------------------------------------------------------------------- the library's calls
def _own(s):
    from paper_2312_00752_b200 import binding as K
    if s["op"] == "gated_step":
        return {"y": K.ssm_gated_step(s["x"], s["gate"], s["in_gate"], s["A"], s["h"]), "h": s["h"]}
    if s["op"] == "gated":
        y = K.ssm_gated_fwd(s["x"], s["gate"], s["in_gate"], s["A"], reset=s["reset"], h0=s["h0"], h_last=s["h_last"])
        return {"y": y, "h_last": s["h_last"]}
    if s["op"] == "gated_train":
        y, saved = K.ssm_gated_fwd(s["x"], s["gate"], s["in_gate"], s["A"], reset=s["reset"], h0=s["h0"], save_states=True)
        grads = K.ssm_gated_bwd(s["x"], s["gate"], s["in_gate"], s["A"], s["dy"], saved, reset=s["reset"], h0=s["h0"],
                                want_dh0=True)
        return {"y": y, **grads}
    train = s["op"] == "norm_train"
    got = K.ssm_norm_fwd(s["x"], s["weight"], s["bias"], s["residual"], rms=s["rms"], eps=s["eps"], save_stats=train)
    got = list(got) if isinstance(got, tuple) else [got]
    out = {"y": got.pop(0)}
    if s["residual"] is not None:
        out["residual_out"] = got.pop(0)
    if train:
        summed = out.get("residual_out", s["x"])
        grads = K.ssm_norm_bwd(summed, s["weight"], s["dy"], got.pop(0), s["dresidual_out"], rms=s["rms"],
                               has_bias=s["bias"] is not None)
        if s["residual"] is None:
            del grads["dresidual"]
        out.update(grads)
    return out


def run(state):
    if own:
        return _own(state)
    op = state["op"]
    if op == "gated_step":
        return _plain_step(state)
    if op == "gated":
        return _plain_gated(state)
    if op == "gated_train":
        return _plain_gated_train(state)
    return _plain_norm_train(state) if op == "norm_train" else _plain_norm(state)[0]


def work(case):
    io = 2 if case["io"] == "bf16" else 4
    D = case["D"]
    if case["op"] in ("norm", "norm_train"):
        n = case["rows"] * D
        res = {"none": 0, "bf16": 2, "f32": 4}[case["residual"]]
        train = case["op"] == "norm_train"
        params = (1 if case["rms"] else 2) * D * 4
        # x and the residual in, y and the sum out; dy and the sum's gradient in, the gradients of x and of the residual out
        # (where the residual has the activations' type the two gradients are one array)
        per = 2 * io + 2 * res + (2 * io + res + (res if res != io else 0) if train else 0)
        return {"bytes": n * per + params * (2 if train else 1), "flops": n * (20 if train else 8)}
    n = case["batch"] * case["L"] * D
    decay = case["form"] == "decay"
    ins = 3 if decay else 2
    state = case["batch"] * D * 4 * 2
    params = D * 4 if decay else 0
    mask = case["batch"] * case["L"] if case["packed"] else 0
    if case["op"] == "gated_train":
        return {"bytes": n * io * (2 * ins + 2) + state + 2 * params + mask, "flops": n * (60 if decay else 30)}
    return {"bytes": n * io * (ins + 1) + state + params + mask, "flops": n * (25 if decay else 12)}


# --------------------------------------------------------------------------------- the definition, in 64 bits, step by step
def _exact_norm(s, train):
    x, w = s["x"].double(), s["weight"].double()
    out = {}
    total = x
    if s["residual"] is not None:
        total = (x + s["residual"].double()).to(s["residual"].dtype).double()
        out["residual_out"] = total
    D = total.shape[-1]
    m = torch.zeros_like(total[:, :1]) if s["rms"] else total.sum(-1, keepdim=True) / D
    sigma = ((total.pow(2).sum(-1, keepdim=True) - D * m * m) / D + s["eps"]).sqrt()
    xh = (total - m) / sigma
    out["y"] = xh * w + (0.0 if s["bias"] is None else s["bias"].double())
    if train:
        dy = s["dy"].double()
        # the Jacobian of (s - m) / sigma, applied to dy w
        q = dy * w
        ds = q / sigma - (total - m) * (q * (total - m)).sum(-1, keepdim=True) / (D * sigma.pow(3))
        if not s["rms"]:
            ds = ds - (q.sum(-1, keepdim=True) / D) / sigma
        if s["residual"] is not None:
            ds = ds + s["dresidual_out"].double()
            out["dresidual"] = ds
        out["dx"] = ds
        out["dweight"] = torch.einsum("rd,rd->d", dy, xh)
        if s["bias"] is not None:
            out["dbias"] = torch.einsum("rd->d", dy)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm", "norm_train"):
        return _exact_norm(s, case["op"] == "norm_train")
    x, gate = s["x"].double(), s["gate"].double()
    e = torch.exp(-gate)
    rho = 1.0 / (1.0 + e)                    # the gate, 1 - rho = e / (1 + e)
    if s["A"] is None:
        a, w = e / (1.0 + e), rho
    else:
        A, iota = s["A"].double(), 1.0 / (1.0 + torch.exp(-s["in_gate"].double()))
        a = torch.exp(A * rho)
        beta = torch.sqrt(-torch.expm1(2.0 * A * rho))
        w = beta * iota
    u = w * x
    if case["op"] == "gated_step":
        h = a * s["h"].double() + u
        return {"y": h, "h": h}
    keep = a if s["reset"] is None else a * (~s["reset"])[:, :, None].double()
    h = s["h0"].double()
    states = torch.empty_like(u)
    for t in range(case["L"]):
        h = torch.addcmul(u[:, t], keep[:, t], h, out=states[:, t])
    if case["op"] == "gated":
        return {"y": states, "h_last": h}
    dh = torch.zeros_like(h)
    mu = torch.empty_like(u)
    dy = s["dy"].double()
    for t in reversed(range(case["L"])):
        dh = torch.add(dy[:, t], dh, out=mu[:, t]) * keep[:, t]
    prev = torch.cat([s["h0"].double()[:, None], states[:, :-1]], dim=1)
    if s["reset"] is not None:
        prev = prev * (~s["reset"])[:, :, None].double()
    out = {"y": states, "dh0": dh, "dx": mu * w}
    if s["A"] is None:
        out["dgate"] = mu * (x - prev) * a * rho
    else:
        da = mu * (prev - iota * x * a / beta)                    # d beta / d a = -a / beta
        out["din_gate"] = mu * u * (1.0 - iota)
        out["dgate"] = da * a * A * rho * (e / (1.0 + e))
        out["dA"] = (da * a * rho).sum(dim=(0, 1))
    return out

"""Plain 64-bit forms of what stands around the recurrence (selective scan, short convolution,
norms), token by token and row by row, differentiable, and the tolerances their kernels are held to.

Tolerances (relative L2), derived before the first run:
- bf16 results: everything ahead of the result's own rounding is fp32, so that rounding alone is
  allowed: uniform in +- 2^-8 of a value's power of two, 2^-8 / sqrt(3) of the value at most (ROUNDED
  of packed_ref, with its allowance for few values), plus the fp32 bound.
- fp32 results: a decay exp(D A) is off by 2^-22 at most (2 units in the last place and the
  argument's rounding) and a state is a sum over the tokens that it remembers, a thousand at the
  slowest steps used here; with random signs sqrt(1000) 2^-22 = 7.5e-6 of it.  Sums over T <= 2000
  rows or over states add sqrt(T) 2^-24 = 2.7e-6 of a typical sum.  In quadrature below 8e-6; 2e-5
  as for the other fp32 results.
"""
import torch

from packed_ref import F32_TOL, ROUNDED, rel

BF16, F32 = torch.bfloat16, torch.float32


def allowed(x, ref):
    if x.dtype == F32:
        return F32_TOL
    return ROUNDED * (1 + 3 / (2 * ref.numel()) ** 0.5) + F32_TOL


def close(x, ref, what):
    assert x.shape == ref.shape, f"{what}: {tuple(x.shape)}, not {tuple(ref.shape)}"
    assert torch.isfinite(x).all(), f"{what}: not finite"
    if ref.numel():
        r, most = rel(x, ref), allowed(x, ref)
        assert r <= most, f"{what}: relative L2 {r:.3e} > {most:.3e}"


def close_each(x, ref, lens, what):
    """Every sequence's rows by themselves."""
    at = 0
    for i, n in enumerate(lens):
        close(x[at:at + n], ref[at:at + n], f"{what} of sequence {i} ({n} rows)")
        at += n


def silu(x):
    return x * torch.sigmoid(x)


def sliced(x, pad):
    """The same values as a slice of rows wider by `pad` elements, NaN around it."""
    if not pad:
        return x
    wide = torch.full((x.shape[0], x[0].numel() + 2 * pad), float("nan"), dtype=x.dtype, device=x.device)
    wide[:, pad:-pad] = x.reshape(x.shape[0], -1)
    return wide[:, pad:-pad].view(x.shape) if x.dim() == 2 else wide[:, pad:-pad].unflatten(1, x.shape[1:])


# ---- selective scan ------------------------------------------------------------------------

SSM = ("x", "dt", "A", "B", "C", "D", "z", "dt_bias")


def ssm_inputs(lens, D, N, G, dtype, seed=0, gate=True, skip=True, bias=True, rows_behind=0, pad=0,
               device="cuda"):
    gen = torch.Generator().manual_seed(seed)
    T = sum(lens) + rows_behind
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    low = torch.exp(-7.0 + 4.6 * torch.rand(D, generator=gen, dtype=torch.float64))
    x = {"x": r(T, D), "dt": r(T, D), "A": -torch.arange(1, N + 1) * torch.exp(0.1 * r(D, N)),
         "B": r(T, G, N), "C": r(T, G, N), "D": r(D) if skip else None,
         "z": r(T, D) if gate else None, "dt_bias": torch.log(torch.expm1(low)) if bias else None,
         "dout": r(T, D)}
    x = {n: t if t is None else t.to(F32 if n in ("A", "D", "dt_bias") else dtype).to(device)
         for n, t in x.items()}
    for n in ("x", "dt", "B", "C", "z"):
        if x[n] is not None:
            x[n] = sliced(x[n], pad)
    return x


def ssm_ref(x, lens, state=None, softplus=True):
    """(out, last states) in float64; rows behind the last sequence are zero.  Differentiable."""
    v = {n: None if x[n] is None else x[n].double() for n in SSM}
    T, D = v["x"].shape
    G, N = v["B"].shape[1:]
    group = torch.arange(D, device=v["x"].device) // (D // G)
    step = v["dt"] if v["dt_bias"] is None else v["dt"] + v["dt_bias"]
    if softplus:
        step = torch.nn.functional.softplus(step, threshold=40.0)
    outs, lasts, at = [], [], 0
    for i, n in enumerate(lens):
        h = (torch.zeros(D, N, dtype=torch.float64, device=group.device) if state is None
             else state[i].double())
        for t in range(at, at + n):
            h = (torch.exp(step[t][:, None] * v["A"]) * h
                 + (step[t] * v["x"][t])[:, None] * v["B"][t, group])
            outs.append((h * v["C"][t, group]).sum(-1))
        lasts.append(h)
        at += n
    zero = torch.zeros(D, dtype=torch.float64, device=group.device)
    out = torch.stack(outs + [zero] * (T - at))
    rows = torch.arange(T, device=group.device)[:, None] < at
    if v["D"] is not None:
        out = out + torch.where(rows, v["D"] * v["x"], 0.0)
    if v["z"] is not None:
        out = out * torch.where(rows, silu(v["z"]), 0.0)
    return out, torch.stack(lasts)


def gradients(f, x, names, sent):
    """d sum(sent_i f(x)_i) / dx by automatic differentiation of the definition; None for inputs that
    are not given."""
    leaves = {n: x[n].double().detach().requires_grad_() if n in names and x[n] is not None else x[n]
              for n in x}
    outs = f(leaves)
    loss = sum((o * s.double()).sum() for o, s in zip(outs, sent))
    given = [n for n in names if x[n] is not None]
    got = dict(zip(given, torch.autograd.grad(loss, [leaves[n] for n in given])))
    return [got.get(n) for n in names]


# ---- short convolution -----------------------------------------------------------------------

CONV = ("x", "w", "bias")


def conv_inputs(lens, D, W, dtype, seed=0, bias=True, rows_behind=0, pad=0, device="cuda"):
    gen = torch.Generator().manual_seed(seed)
    T = sum(lens) + rows_behind
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    x = {"x": r(T, D).to(dtype), "w": r(D, W).to(F32), "bias": r(D).to(F32) if bias else None,
         "dout": r(T, D).to(dtype)}
    x = {n: t if t is None else t.to(device) for n, t in x.items()}
    x["x"] = sliced(x["x"], pad)
    return x


def conv_ref(x, lens, state=None, act=True):
    """(out, last rows) in float64, for the rows of the sequences.  Differentiable."""
    v, w = x["x"].double(), x["w"].double()
    D, W = w.shape
    outs, lasts, at = [], [], 0
    for i, n in enumerate(lens):
        ahead = (torch.zeros(W - 1, D, dtype=torch.float64, device=v.device) if state is None
                 else state[i].double())
        rows = torch.cat([ahead, v[at:at + n]])
        for t in range(n):
            p = (rows[t:t + W] * w.t()).sum(0)
            if x["bias"] is not None:
                p = p + x["bias"].double()
            outs.append(silu(p) if act else p)
        lasts.append(rows[n:])
        at += n
    out = torch.stack(outs) if outs else v[:0]
    return out, torch.stack(lasts)


# ---- norms -------------------------------------------------------------------------------------

NORM = ("x", "res", "z", "w", "scale")


def norm_inputs(T, H, d, dtype, heads=None, gate=False, res=False, scale=False, seed=0, pad=0,
                device="cuda"):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    par = (d,) if heads is None else (heads, d)
    x = {"x": r(T, H, d).to(dtype), "res": (2 * r(T, H, d)).to(dtype) if res else None,
         "z": r(T, H, d).to(dtype) if gate else None, "w": (1 + 0.3 * r(*par)).to(F32),
         "scale": (0.5 + 0.2 * r(*par)).to(F32) if scale else None, "dout": r(T, H, d).to(dtype),
         "dtotal": r(T, H, d).to(dtype) if res else None}
    x = {n: t if t is None else t.to(device) for n, t in x.items()}
    for n in ("x", "res", "z"):
        if x[n] is not None:
            x[n] = sliced(x[n], pad)
    return x


def norm_ref(x, eps):
    """(out, total or None) in float64.  Differentiable."""
    r, w = x["x"].double(), x["w"].double()
    if x["res"] is not None:
        s = 1.0 if x["scale"] is None else x["scale"].double()
        r = x["res"].double() + s * r
    out = r / torch.sqrt((r * r).mean(-1, keepdim=True) + eps) * w
    if x["z"] is not None:
        out = out * silu(x["z"].double())
    return out, (r if x["res"] is not None else None)

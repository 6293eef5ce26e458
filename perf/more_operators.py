"""What a recurrent layer needs around and beside the gated delta rule, for measuring: the short
causal convolution in front of it, the selective state space scan (whole sequences, training step,
one token) and the norm behind it, with its gate, or ahead of it, with the residual sum.

A case with `own` false is computed in plain torch operations, in 32 bits; with `own` true by the
library's entry points.  `exact` computes the same from the operators' definitions in 64 bits.

Sequences of a batch are packed one after the other: rows [T][channels], with the lengths of the
sequences in the case ("8*4096" stands for eight of 4096).

Inputs: the scan's input is silu(N(0, 1)), as the convolution leaves it; its steps are
softplus(N(0, 1) + bias) with softplus(bias) log-uniform in [0.001, 0.1] per channel, and
A = -n exp(0.1 N(0, 1)), n = 1 .. N, as such layers are initialised and a little trained; B, C, the
gate and dout ~ N(0, 1).  x, the gate and, in the scan, the step's and B's and C's rows are slices of
wider projections, as a layer has them.  The convolution's taps are uniform in +- 1 / sqrt(width).
The residual stream is N(0, 9), what is added to it N(0, 1) times a scale in [0.1, 1] per channel.
"""
import math

import torch

own = False
DEVICE = "cuda"


def _conv(name, call, dtype, lens, D, W=4, silu=True):
    return {"name": name, "call": call, "dtype": dtype, "lens": lens, "D": D, "W": W, "silu": silu}


def _ssm(name, call, dtype, lens, D, N=16, G=1, gate=True):
    return {"name": name, "call": call, "dtype": dtype, "lens": lens, "D": D, "N": N, "G": G,
            "gate": gate}


def _norm(name, call, dtype, T, H, d, gate, res):
    return {"name": name, "call": call, "dtype": dtype, "T": T, "H": H, "d": d, "gate": gate,
            "res": res}


def listed():
    return [
        # one token of each sequence of a serving batch: latency is all
        _conv("conv_token", "conv_token", "bf16", "64*1", 2048),
        # a prefill batch of long prompts: x, B and C of a layer side by side
        _conv("conv_prompt", "conv_prompt", "bf16", "8*4096", 4096),
        # a training step on packed documents, ragged, down to single tokens
        _conv("conv_train", "conv_train", "bf16", "4096,5003,2900,701,97,20*1", 2048),
        # one token of each sequence of a full serving batch: bound by the state
        _ssm("ssm_token", "ssm_token", "bf16", "256*1", 4096),
        # a few short prompts of different lengths in one call, one of a single token
        _ssm("ssm_prompt_short", "ssm_prompt", "bf16", "37,128,1,300,64", 1024),
        # one long prompt: few channels, many tokens
        _ssm("ssm_prompt_one", "ssm_prompt", "bf16", "8192", 1280),
        # a prefill batch of long prompts: the largest forward
        _ssm("ssm_prompt_long", "ssm_prompt", "bf16", "8*4096", 2048),
        # a language-model training step
        _ssm("ssm_train", "ssm_train", "bf16", "8*1024", 2048),
        # a training step in fp32, ragged, two groups of B and C, no gate
        _ssm("ssm_train_f32", "ssm_train", "f32", "1000,257", 512, 16, 2, False),
        # behind a prefill batch's recurrence: a norm of every head, with the gate
        _norm("norm_gate_prompt", "norm_fwd", "bf16", 32768, 16, 128, True, False),
        # ahead of the next block of a training step: residual sum, scale and norm, and back
        _norm("norm_residual_train", "norm_train", "bf16", 16384, 1, 2048, False, True),
        # the same ahead of a block for one token of each of a few streams
        _norm("norm_residual_token", "norm_fwd", "bf16", 16, 1, 2048, False, True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _text(lens):
    return ",".join(str(n) for n in lens)


def draw(rng):
    call = rng.choice(["conv_token", "conv_prompt", "conv_train", "ssm_token", "ssm_prompt",
                       "ssm_prompt", "ssm_train", "ssm_train", "norm_fwd", "norm_train"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kind, what = call.split("_")
    if kind == "norm":
        d = 8 * _log_int(rng, 4, 512)
        H = 1 if d > 512 else rng.choice([1, 3, 4, 8, 16])
        top = 2 ** 25 >> (dtype == "f32") >> (what == "train")
        T = _log_int(rng, 1, min(20000, top // (H * d)))
        gate, res = rng.choice([(True, False), (False, True), (True, True), (False, False)])
        c = _norm("", call, dtype, T, H, d, gate, res)
    elif what == "token":
        lens = "%d*1" % _log_int(rng, 1, 200)
        D = 8 * _log_int(rng, 8, 400)
        c = (_conv("", call, dtype, lens, D, rng.choice([2, 3, 4])) if kind == "conv" else
             _ssm("", call, dtype, lens, D, rng.choice([8, 16, 16, 32]), 1, rng.random() < 0.7))
    elif kind == "conv":
        lens = [_log_int(rng, 1, 6000) for _ in range(_log_int(rng, 1, 12))]
        D = 8 * _log_int(rng, 8, min(300, 2 ** 22 // sum(lens)))
        c = _conv("", call, dtype, _text(lens), D, rng.choice([2, 3, 4, 4]), rng.random() < 0.8)
    else:
        N = rng.choice([8, 16, 16, 16, 32])
        G = rng.choice([1, 1, 2, 4])
        D = 8 * G * _log_int(rng, 8, 1600 // N // G * 2)
        top = {"ssm_prompt": 3500, "ssm_train": 1000}[call]
        lens = [_log_int(rng, 1, top) for _ in range(_log_int(rng, 1, 8))]
        c = _ssm("", call, dtype, _text(lens), D, N, G, rng.random() < 0.7)
    del c["name"]
    return c


def _lens(text):
    out = []
    for part in text.split(","):
        n, _, m = part.rpartition("*")
        out += [int(m)] * (int(n) if n else 1)
    return out


def _offsets(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return torch.tensor(cu, dtype=torch.int32, device=DEVICE)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[case["dtype"]]

    def randn(*shape):
        return torch.randn(*shape, device=DEVICE, generator=gen)

    def rand(*shape):
        return torch.rand(*shape, device=DEVICE, generator=gen)

    st = {"call": case["call"], "dt": dt}
    if case["call"].startswith("norm"):
        T, H, d = case["T"], case["H"], case["d"]
        st.update(eps=1e-6, x=randn(T, H, d).to(dt), w=1.0 + 0.1 * randn(H, d), z=None, res=None,
                  scale=None)
        if case["gate"]:  # a slice of a projection twice as wide
            st["z"] = randn(T, 2 * H, d).to(dt)[:, H:]
        if case["res"]:
            st.update(res=(3.0 * randn(T, H, d)).to(dt), scale=0.1 + 0.9 * rand(H, d))
        if case["call"] == "norm_train":
            st["dout"] = randn(T, H, d).to(dt)
            if case["res"]:  # what the stream's later users send back
                st["dsum"] = randn(T, H, d).to(dt)
        return st
    lens, D = _lens(case["lens"]), case["D"]
    T = sum(lens)
    st.update(lens=lens, cu=_offsets(lens))
    if case["call"].startswith("conv"):
        W = case["W"]
        st.update(silu=case["silu"], x=randn(T, 2 * D).to(dt)[:, :D],
                  w=(2.0 * rand(D, W) - 1.0) / math.sqrt(W),
                  bias=(2.0 * rand(D) - 1.0) / math.sqrt(W))
        if case["call"] == "conv_token":
            st["state"] = randn(T, W - 1, D).to(dt)
        if case["call"] == "conv_train":
            st["dout"] = randn(T, D).to(dt)
            if own:
                from paper_2606_27748_gb300 import flexattn
                st["ws"] = flexattn.conv_workspace(st["x"], st["w"], st["cu"])
        return st
    N, G = case["N"], case["G"]
    x = randn(T, D)
    low = torch.exp(math.log(0.001) + math.log(100.0) * rand(D))
    bc = randn(T, 2 * G * N).to(dt)
    n = torch.arange(1, N + 1, dtype=torch.float32, device=DEVICE)
    st.update(x=(x * torch.sigmoid(x)).to(dt), delta=randn(T, D).to(dt),
              bias=torch.log(torch.expm1(low)), A=-n * torch.exp(0.1 * randn(D, N)),
              B=bc[:, :G * N].view(T, G, N), C=bc[:, G * N:].view(T, G, N),
              Ds=1.0 + 0.1 * randn(D), z=None)
    if case["gate"]:
        st["z"] = randn(T, 2 * D).to(dt)[:, D:]
    if case["call"] == "ssm_token":
        # the state of a sequence some way on
        st["state"] = 0.3 * randn(T, D, N)
    if case["call"] == "ssm_train":
        st["dout"] = randn(T, D).to(dt)
    if own and case["call"] != "ssm_token":
        from paper_2606_27748_gb300 import flexattn
        st["ws"] = flexattn.ssm_workspace(st["x"], st["B"], st["cu"],
                                          backward=case["call"] == "ssm_train")
    return st


def run(st):
    if own:
        return _run_own(st)
    kind, what = st["call"].split("_")
    if what == "token":
        return _plain_conv_token(st) if kind == "conv" else _plain_ssm_token(st)
    names = {"conv": ("x", "w", "bias"), "ssm": ("x", "delta", "A", "B", "C", "Ds", "z", "bias"),
             "norm": ("x", "res", "z", "w", "scale")}[kind]
    plain = {"conv": _plain_conv, "ssm": _plain_ssm, "norm": _plain_norm}[kind]
    leaves = {n: st[n].float() for n in names if st[n] is not None}
    if what != "train":
        return tuple(y.to(t) for y, t in plain(leaves, st))
    with torch.enable_grad():
        leaves = {n: x.detach().requires_grad_() for n, x in leaves.items()}
        got = plain(leaves, st)
        out = got[:2] if "dsum" in st else got[:1]
        sent = [st["dout"].float()] + ([st["dsum"].float()] if "dsum" in st else [])
        grads = torch.autograd.grad([y for y, _ in out], list(leaves.values()), sent)
    return (*(y.detach().to(t) for y, t in out),
            *(g.to(st[n].dtype) for n, g in zip(leaves, grads)))


def _run_own(st):
    from paper_2606_27748_gb300 import flexattn
    call = st["call"]
    if call == "conv_token":
        return (flexattn.conv_decode(st["x"], st["w"], st["state"], bias=st["bias"],
                                     silu=st["silu"]), st["state"])
    if call.startswith("conv"):
        out, last = flexattn.conv_fwd(st["x"], st["w"], st["cu"], bias=st["bias"],
                                      silu=st["silu"], want_state=call == "conv_prompt")
        if call == "conv_prompt":
            return out, last
        return (out, *flexattn.conv_bwd(st["x"], st["w"], st["cu"], st["dout"], bias=st["bias"],
                                        silu=st["silu"], ws=st["ws"]))
    if call.startswith("norm"):
        out, total, rstd = flexattn.norm_fwd(st["x"], st["w"], z=st["z"], res=st["res"],
                                             scale=st["scale"], eps=st["eps"],
                                             want_rstd=call == "norm_train")
        outs = (out,) if total is None else (out, total)
        if call == "norm_fwd":
            return outs
        dx, dres, dz, dw, dscale = flexattn.norm_bwd(
            st["x"], st["w"], rstd, st["dout"], z=st["z"], res=st["res"], scale=st["scale"],
            dtotal=st.get("dsum"))
        return (*outs, *(g for g in (dx, dres, dz, dw, dscale) if g is not None))
    x = [st[n] for n in ("x", "delta", "A", "B", "C")]
    kw = {"D": st["Ds"], "z": st["z"], "dt_bias": st["bias"]}
    if call == "ssm_token":
        return flexattn.ssm_decode(*x, st["state"], **kw), st["state"]
    if call == "ssm_prompt":
        return flexattn.ssm_fwd(*x, st["cu"], ws=st["ws"], **kw)
    save = flexattn.ssm_save(st["x"], st["B"], st["cu"])
    out, _ = flexattn.ssm_fwd(*x, st["cu"], want_state=False, save=save, ws=st["ws"], **kw)
    dx, ddt, dA, dB, dC, dD, dz, dbias = flexattn.ssm_bwd(*x, st["cu"], st["dout"], save,
                                                          ws=st["ws"], **kw)
    return tuple(g for g in (out, dx, ddt, dA, dB, dC, dD, dz, dbias) if g is not None)


# ---- plain forms -------------------------------------------------------------------------

def _silu(x):
    return x / (1.0 + torch.exp(-x))


def _softplus(x):
    return torch.where(x > 20.0, x, torch.log1p(torch.exp(torch.clamp(x, max=20.0))))


def _padded(x, lens, ahead=0):
    """[T][...] rows as [sequences][ahead + longest][...], zeros elsewhere; and where rows are."""
    at = torch.arange(max(lens) + ahead, device=x.device) - ahead
    n = torch.tensor(lens, device=x.device)
    first = torch.cumsum(n, 0) - n
    inside = (at >= 0) & (at < n[:, None])
    rows = torch.where(inside, first[:, None] + at, 0)
    return torch.where(inside.view(*inside.shape, *([1] * (x.dim() - 1))), x[rows], 0.0), inside


def _plain_conv(x, st):
    """out, and the last W - 1 rows of every sequence (oldest first, zeros ahead of its start)."""
    W = x["w"].shape[1]
    rows, inside = _padded(x["x"], st["lens"], W - 1)
    L = max(st["lens"])
    pre = x["bias"] + sum(x["w"][:, j] * rows[:, j:j + L] for j in range(W))
    out = (_silu(pre) if st["silu"] else pre)[inside[:, W - 1:]]
    last = torch.stack([rows[i, n:n + W - 1] for i, n in enumerate(st["lens"])])
    return (out, st["dt"]), (last, st["dt"])


def _plain_conv_token(st):
    rows = torch.cat([st["state"], st["x"][:, None]], 1)
    pre = st["bias"] + (st["w"].t() * rows.float()).sum(1)
    st["state"].copy_(rows[:, 1:])
    return (_silu(pre) if st["silu"] else pre).to(st["dt"]), st["state"]


def _plain_ssm(x, st):
    """out and the last states, all sequences a token at a time."""
    G = x["B"].shape[1]
    D, N = x["A"].shape
    step = _softplus(x["delta"] + x["bias"])
    (dt, inside), (dx, _), (B, _), (C, _) = (_padded(v, st["lens"]) for v in (
        step, step * x["x"], x["B"], x["C"]))
    n, A = len(st["lens"]), x["A"].view(G, D // G, N)
    dt, dx = (v.view(n, -1, G, D // G, 1) for v in (dt, dx))
    h, out = torch.zeros(n, G, D // G, N, device=dt.device), []
    for t in range(dt.shape[1]):
        h = torch.exp(dt[:, t] * A) * h + dx[:, t] * B[:, t, :, None]
        out.append((h * C[:, t, :, None]).sum(-1))
    out = torch.stack(out, 1).reshape(n, -1, D)[inside] + x["Ds"] * x["x"]
    if "z" in x:
        out = out * _silu(x["z"])
    return (out, st["dt"]), (h.reshape(n, D, N), torch.float32)


def _plain_ssm_token(st):
    x, S, A = st["x"].float(), st["state"], st["A"]
    n, D, N = S.shape
    G = st["B"].shape[1]
    dt = _softplus(st["delta"].float() + st["bias"])
    B, C = (st[m].float()[:, :, None].expand(n, G, D // G, N).reshape(n, D, N) for m in ("B", "C"))
    S *= torch.exp(dt[..., None] * A)
    S += (dt * x)[..., None] * B
    out = (S * C).sum(-1) + st["Ds"] * x
    if st["z"] is not None:
        out = out * _silu(st["z"].float())
    return out.to(st["dt"]), S


def _plain_norm(x, st):
    r = x["x"] if "res" not in x else x["res"] + x["scale"] * x["x"]
    out = r / torch.sqrt((r * r).mean(-1, keepdim=True) + st["eps"]) * x["w"]
    if "z" in x:
        out = out * _silu(x["z"])
    return ((out, st["dt"]),) if "res" not in x else ((out, st["dt"]), (r, st["dt"]))


# ---- what a pass cannot do without -------------------------------------------------------

def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    call = case["call"]
    if call.startswith("norm"):
        T, H, d = case["T"], case["H"], case["d"]
        rows = 2 + case["gate"] + 2 * case["res"]          # x, out; the gate; the stream in and out
        if call == "norm_train":  # the forward's inputs once, dout and gradients of all of them
            rows += 2 + case["gate"] + 2 * case["res"]
        params = H * d * (1 + case["res"]) * (2 if call == "norm_train" else 1)
        return {"bytes": es * rows * T * H * d + 4 * params,
                "flops": (12 if call == "norm_fwd" else 40) * T * H * d}
    lens, D = _lens(case["lens"]), case["D"]
    T, n = sum(lens), len(lens)
    if call.startswith("conv"):
        W = case["W"]
        if call == "conv_train":  # x, out, dout, dx
            return {"bytes": es * 4 * T * D + 8 * D * (W + 1), "flops": T * D * (6 * W + 20)}
        state = es * n * (W - 1) * D * (2 if call == "conv_token" else 1)
        return {"bytes": es * 2 * T * D + 4 * D * (W + 1) + state, "flops": T * D * (2 * W + 6)}
    N, G, gate = case["N"], case["G"], case["gate"]
    rows = (3 + gate) * D + 2 * G * N
    params = 4 * D * (N + 2)
    if call == "ssm_train":  # the forward, dout, and gradients of all inputs
        more = (3 + gate) * D + 2 * G * N
        return {"bytes": es * T * (rows + more) + 2 * params, "flops": T * D * (28 * N + 40)}
    state = 4 * n * D * N * (2 if call == "ssm_token" else 1)
    return {"bytes": es * T * rows + params + state, "flops": T * D * (7 * N + 20)}


# ---- from the definitions, in 64 bits ----------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    kind = case["call"].split("_")[0]
    return {"conv": _exact_conv, "ssm": _exact_ssm, "norm": _exact_norm}[kind](st)


def _gate64(z):
    """silu(z) and its derivative."""
    s = torch.sigmoid(z)
    return z * s, s * (1.0 + z * (1.0 - s))


def _exact_conv(st):
    """One sequence at a time: a sum over rows that are shifted against one another."""
    w, bias = st["w"].double(), st["bias"].double()
    W = w.shape[1]
    outs, lasts, dxs, at = [], [], [], 0
    dw, db = torch.zeros_like(w), torch.zeros_like(bias)
    for i, n in enumerate(st["lens"]):
        x = st["x"][at:at + n].double()
        ahead = (st["state"][i].double() if "state" in st
                 else torch.zeros(W - 1, x.shape[1], dtype=torch.float64, device=x.device))
        x = torch.cat([ahead, x])
        pre = bias.expand(n, -1).clone()
        for j in range(W):
            pre += w[:, j] * x[j:j + n]
        y, slope = _gate64(pre) if st["silu"] else (pre, torch.ones_like(pre))
        outs.append(y)
        lasts.append(x[n:])
        if "dout" in st:
            dp = slope * st["dout"][at:at + n].double()
            dx = torch.zeros_like(x)
            for j in range(W):
                dx[j:j + n] += w[:, j] * dp
                dw[:, j] += (dp * x[j:j + n]).sum(0)
            db += dp.sum(0)
            dxs.append(dx[W - 1:])
        at += n
    if "dout" in st:
        return torch.cat(outs), torch.cat(dxs), dw, db
    return torch.cat(outs), torch.stack(lasts)


def _exact_ssm(st):
    """Token by token over all sequences at once; one that has ended keeps its state."""
    x, raw, A, Bg, Cg = (st[m].double() for m in ("x", "delta", "A", "B", "C"))
    Ds, bias = st["Ds"].double(), st["bias"].double()
    T, D = x.shape
    N, G, lens = A.shape[1], Bg.shape[1], st["lens"]
    group = torch.arange(D, device=x.device) // (D // G)
    raw = raw + bias
    dt = torch.nn.functional.softplus(raw, threshold=40.0)
    n = torch.tensor(lens, device=x.device)
    first = torch.cumsum(n, 0) - n
    order = torch.argsort(n, descending=True, stable=True)  # those still running come first
    first = first[order]
    S = torch.zeros(len(lens), D, N, dtype=torch.float64, device=x.device)
    if "state" in st:
        S = st["state"].double()[order]
    training = "dout" in st
    y, states = torch.zeros_like(x), []
    running = [sum(m > t for m in lens) for t in range(max(lens))]
    for t, m in enumerate(running):
        at = first[:m] + t
        if training:
            states.append(S[:m].clone())
        S[:m] = (torch.exp(dt[at][..., None] * A) * S[:m]
                 + (dt[at] * x[at])[..., None] * Bg[at][:, group])
        y[at] = torch.einsum("mdn,mdn->md", S[:m], Cg[at][:, group]) + Ds * x[at]
    gate, slope = (_gate64(st["z"].double()) if st["z"] is not None
                   else (torch.ones_like(y), torch.zeros_like(y)))
    out = y * gate
    if not training:
        return out, S[torch.argsort(order)]
    dout = st["dout"].double()
    dy, dz = dout * gate, dout * y * slope
    dx, ddt = Ds * dy, torch.zeros_like(x)
    dA, dB, dC = torch.zeros_like(A), torch.zeros_like(Bg), torch.zeros_like(Cg)
    E = torch.zeros_like(S)
    for t in range(len(running) - 1, -1, -1):
        m = running[t]
        at = first[:m] + t
        B, C = Bg[at][:, group], Cg[at][:, group]
        a = torch.exp(dt[at][..., None] * A)
        kept = a * states.pop()
        h = kept + (dt[at] * x[at])[..., None] * B
        Et = E[:m] + dy[at][..., None] * C
        dC[at] = (dy[at][..., None] * h).view(m, G, D // G, N).sum(2)
        dB[at] = ((dt[at] * x[at])[..., None] * Et).view(m, G, D // G, N).sum(2)
        s = (Et * B).sum(-1)
        dx[at] += s * dt[at]
        q = Et * kept
        dA += (q * dt[at][..., None]).sum(0)
        ddt[at] = s * x[at] + (q * A).sum(-1)
        E[:m] = a * Et
    ddt = ddt * torch.sigmoid(raw)
    grads = [dx, ddt, dA, dB, dC, (dy * x).sum(0)]
    return (out, *grads, *([dz] if st["z"] is not None else []), ddt.sum(0))


def _exact_norm(st):
    x, w = st["x"].double(), st["w"].double()
    r = x if st["res"] is None else st["res"].double() + st["scale"].double() * x
    inv = torch.rsqrt(torch.mean(r ** 2, -1, keepdim=True) + st["eps"])
    gate, slope = (_gate64(st["z"].double()) if st["z"] is not None
                   else (torch.ones_like(r), None))
    out = r * inv * w * gate
    outs = (out,) if st["res"] is None else (out, r)
    if "dout" not in st:
        return outs
    g = st["dout"].double()
    dn = g * gate * w
    dr = inv * (dn - r * inv ** 2 * torch.mean(dn * r, -1, keepdim=True))
    dw = (g * gate * r * inv).sum(0)
    dz = [] if slope is None else [g * slope * r * inv * w]
    if st["res"] is None:
        return (*outs, dr, *dz, dw)
    dr = dr + st["dsum"].double()
    return (*outs, st["scale"].double() * dr, dr, *dz, dw, (dr * x).sum(0))

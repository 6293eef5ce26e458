"""The packed-batch operators of this library for measuring their speed and accuracy: the
gated delta rule (whole sequences, training step, one token) and softmax attention over
prompts.

A case with `own` false is computed in plain torch operations, in 32 bits; with `own` true by
the library's entry points.  `exact` computes the same from the operators' definitions, token
by token and row by row, in 64 bits.

Sequences of a batch are packed one after the other: rows [T][heads][d], with the lengths of
the sequences in the case ("8*4096" stands for eight of 4096).

Inputs: q and k are unit vectors with a common component (keys of one text are correlated),
v and dout ~ N(0, 1), beta = sigmoid(N(0, 1)), the log decay g = -A dt with A in [1, 16] per
head and dt log-uniform in [0.001, 0.1] per token, as such layers are initialised.  For softmax
attention q and k ~ N(0, 1), which spreads the scores as a trained layer's.
"""
import math

import torch

own = False
CHUNK = 64  # rows of the plain delta rule's chunks


def _delta(name, call, dtype, lens, H, Hk, d):
    return {"name": name, "call": call, "dtype": dtype, "lens": lens, "H": H, "Hk": Hk, "d": d}


def _attn(name, dtype, lens_q, lens_k, H, Hk, d, causal=True):
    return {"name": name, "call": "attn", "dtype": dtype, "lens": lens_q, "lens_k": lens_k,
            "H": H, "Hk": Hk, "d": d, "causal": causal}


def listed():
    return [
        # one token for each of a few streams: interactive decoding, latency is all
        _delta("delta_token_small", "delta_token", "bf16", "4*1", 16, 16, 64),
        # one token for each sequence of a full serving batch: bound by the state
        _delta("delta_token_serving", "delta_token", "bf16", "256*1", 16, 8, 128),
        # a few short prompts of different lengths in one call, one of a single token
        _delta("delta_prompt_short", "delta_prompt", "bf16", "37,128,1,300,64", 16, 16, 64),
        # a prefill batch of long prompts, two value heads to a key head: the largest forward
        _delta("delta_prompt_long", "delta_prompt", "bf16", "8*4096", 16, 8, 128),
        # prompts in fp32, one ragged
        _delta("delta_prompt_f32", "delta_prompt", "f32", "1000,257", 4, 4, 64),
        # a language-model training step at the library's own head size
        _delta("delta_train", "delta_train", "bf16", "8*2048", 12, 12, 64),
        # a training step on packed documents, ragged, shared key heads
        _delta("delta_train_packed", "delta_train", "bf16", "1500,701,97,1", 8, 4, 128),
        # the same kind of training step in fp32
        _delta("delta_train_f32", "delta_train", "f32", "4*1000", 4, 4, 64),
        # one long prompt through a full-attention layer with grouped heads: the most arithmetic
        _attn("attn_prompt_long", "bf16", "16384", "16384", 16, 4, 128),
        # packed prompts of very different lengths, one key head per head
        _attn("attn_prompt_packed", "bf16", "4000,1531,700,129,64,7,1",
              "4000,1531,700,129,64,7,1", 12, 12, 64),
        # one new token for each sequence against its keys so far
        _attn("attn_token", "bf16", "32*1", "16*8000,16*1777", 16, 4, 128),
        # the distillation's teacher in fp32, small
        _attn("attn_f32", "f32", "1000,300", "1000,300", 4, 4, 64),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _text(lens):
    return ",".join(str(n) for n in lens)


def draw(rng):
    call = rng.choice(["delta_prompt", "delta_prompt", "delta_train", "delta_train",
                       "delta_token", "attn", "attn", "attn"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([64, 128])
    if call == "delta_token":
        H = rng.choice([4, 8, 12, 16])
        c = _delta("", call, dtype, "%d*1" % _log_int(rng, 1, 200), H,
                   H // rng.choice([1, 2]), d)
    elif call == "attn":
        G = rng.choice([1, 1, 2, 3, 4, 8])
        Hk = rng.choice([1, 2, 4]) if G > 2 else rng.choice([2, 4, 8])
        nseq = _log_int(rng, 1, 12)
        top = 1200 if dtype == "f32" else 6000
        lens_q = [_log_int(rng, 1, top) for _ in range(nseq)]
        kind = rng.choice(["same", "same", "longer", "token"])
        if kind == "token":
            lens_q = [1] * nseq
        lens_k = lens_q if kind == "same" else [n + _log_int(rng, 1, top // 2) for n in lens_q]
        c = _attn("", dtype, _text(lens_q), _text(lens_k), G * Hk, Hk, d, rng.random() < 0.8)
    else:
        H = rng.choice([4, 8, 12, 16])
        nseq = _log_int(rng, 1, 8)
        top = {"bf16": 4000, "f32": 1500}[dtype] // (1 if call == "delta_prompt" else 2)
        c = _delta("", call, dtype, _text(_log_int(rng, 1, top) for _ in range(nseq)), H,
                   H // rng.choice([1, 1, 2]), d)
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
    return torch.tensor(cu, dtype=torch.int32, device="cuda")


def _unit(x):
    return x / x.norm(dim=-1, keepdim=True)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[case["dtype"]]
    H, Hk, d = case["H"], case["Hk"], case["d"]

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    lens = _lens(case["lens"])
    T = sum(lens)
    st = {"call": case["call"], "lens": lens, "cu": _offsets(lens), "G": H // Hk,
          "scale": 1.0 / math.sqrt(d)}
    if case["call"] == "attn":
        lens_k = _lens(case["lens_k"])
        Tk = sum(lens_k)
        st.update(lens_k=lens_k, cu_k=_offsets(lens_k), causal=case["causal"],
                  q=randn(T, H, d).to(dt), k=randn(Tk, Hk, d).to(dt), v=randn(Tk, Hk, d).to(dt))
        if own:
            from paper_2606_27748_gb300 import flexattn
            st["ws"] = flexattn.softattn_workspace(st["q"], st["k"], st["cu"])
        return st
    common = randn(1, Hk, d)
    A = torch.rand(1, H, device="cuda", generator=gen) * 15.0 + 1.0
    dt_ = torch.exp(math.log(0.001) + math.log(100.0)
                    * torch.rand(T, H, device="cuda", generator=gen))
    st.update(q=_unit(randn(T, Hk, d) + 0.5 * common).to(dt),
              k=_unit(randn(T, Hk, d) + 0.5 * common).to(dt), v=randn(T, H, d).to(dt),
              beta=torch.sigmoid(randn(T, H)).to(dt), g=(-A * dt_).to(dt))
    if case["call"] == "delta_token":
        # the state of a sequence some way on: entries of the size that unit keys leave
        st["state"] = randn(T, H, d, d) / math.sqrt(d)
    if case["call"] == "delta_train":
        st["dout"] = randn(T, H, d).to(dt)
    if own:
        from paper_2606_27748_gb300 import flexattn
        if case["call"] != "delta_token":
            st["ws"] = flexattn.delta_workspace(st["q"], st["v"], st["cu"],
                                                backward=case["call"] == "delta_train")
    return st


def run(st):
    if own:
        return _run_own(st)
    if st["call"] == "attn":
        return _plain_attention(st)
    if st["call"] == "delta_token":
        return _plain_token(st)
    if st["call"] == "delta_prompt":
        return _plain_delta(*_floats(st), st)
    with torch.enable_grad():
        leaves = [x.requires_grad_() for x in _floats(st)]
        out, _ = _plain_delta(*leaves, st)
        grads = torch.autograd.grad(out, leaves, st["dout"])
    return (out.detach(), *(x.to(st["q"].dtype) for x in grads))


def _run_own(st):
    from paper_2606_27748_gb300 import flexattn
    if st["call"] == "attn":
        return flexattn.softattn_fwd(st["q"], st["k"], st["v"], st["cu"], st["cu_k"],
                                     causal=st["causal"], scale=st["scale"], ws=st["ws"])
    x = [st[n] for n in ("q", "k", "v", "g", "beta")]
    if st["call"] == "delta_token":
        return (flexattn.delta_decode(*x, st["state"], scale=st["scale"]), st["state"])
    if st["call"] == "delta_prompt":
        return flexattn.delta_fwd(*x, st["cu"], scale=st["scale"], ws=st["ws"])
    save = flexattn.delta_save(st["q"], st["v"], st["cu"])
    out, _ = flexattn.delta_fwd(*x, st["cu"], scale=st["scale"], want_state=False, save=save,
                                ws=st["ws"])
    return (out, *flexattn.delta_bwd(*x, st["cu"], st["dout"], save, scale=st["scale"],
                                     ws=st["ws"]))


# ---- plain forms -------------------------------------------------------------------------

def _floats(st):
    return [st[n].float() for n in ("q", "k", "v", "g", "beta")]


def _padded(x, lens, to):
    """[T][...] rows as [sequences][to][...], zeros behind each sequence's end."""
    at = torch.arange(to, device=x.device)
    n = torch.tensor(lens, device=x.device)
    first = torch.cumsum(n, 0) - n
    inside = at < n[:, None]
    rows = torch.where(inside, first[:, None] + at, 0)
    return torch.where(inside.view(*inside.shape, *([1] * (x.dim() - 1))), x[rows], 0.0), inside


def _plain_delta(q, k, v, g, beta, st):
    """(out [T][H][d], last state [sequences][H][d][d]) of the gated delta rule in chunks."""
    lens, G, scale, dt = st["lens"], st["G"], st["scale"], st["v"].dtype
    C, n = CHUNK, len(lens)
    to = -(-max(lens) // C) * C
    q, k = (x.repeat_interleave(G, dim=1) for x in (q, k))
    (q, inside), (k, _), (v, _), (g, _), (beta, _) = (_padded(x, lens, to)
                                                     for x in (q, k, v, g, beta))
    H, d = v.shape[2], v.shape[3]
    q, k, v = (x.transpose(1, 2).reshape(n, H, to // C, C, d) for x in (q, k, v))
    g, beta = (x.transpose(1, 2).reshape(n, H, to // C, C) for x in (g, beta))
    sums = torch.cumsum(g, -1)
    low = torch.ones(C, C, dtype=torch.bool, device=q.device).tril()
    decay = torch.exp(torch.where(low, sums[..., :, None] - sums[..., None, :], 0.0)) * low
    L = (beta[..., None] * decay * (k @ k.transpose(-1, -2))).tril(-1)
    P = scale * decay * (q @ k.transpose(-1, -2))
    # rows of (I + L)^-1 diag(beta) [v | e^sums k], one after the other
    rhs = beta[..., None] * torch.cat([v, torch.exp(sums)[..., None] * k], -1)
    solved = [rhs[..., 0, :]]
    for i in range(1, C):
        done = torch.stack(solved, -2)
        solved.append(rhs[..., i, :] - (L[..., i, None, :i] @ done).squeeze(-2))
    solved = torch.stack(solved, -2)
    uv, w = solved[..., :d], solved[..., d:]
    qd = scale * torch.exp(sums)[..., None] * q
    kd = torch.exp(sums[..., -1:] - sums)[..., None] * k
    last = torch.exp(sums[..., -1])[..., None, None]
    S = torch.zeros(n, H, d, d, device=q.device)
    out = []
    for c in range(to // C):
        u = uv[:, :, c] - w[:, :, c] @ S
        out.append(qd[:, :, c] @ S + P[:, :, c] @ u)
        S = last[:, :, c] * S + kd[:, :, c].transpose(-1, -2) @ u
    out = torch.stack(out, 2).reshape(n, H, to, d).transpose(1, 2)[inside]
    return out.to(dt), S


def _plain_token(st):
    q, k, v, g, beta = _floats(st)
    q, k = (x.repeat_interleave(st["G"], dim=1) for x in (q, k))
    S = st["state"]
    S *= torch.exp(g)[..., None, None]
    u = beta[..., None] * (v - (k[..., None, :] @ S).squeeze(-2))
    S += k[..., :, None] * u[..., None, :]
    out = st["scale"] * (q[..., None, :] @ S).squeeze(-2)
    return out.to(st["v"].dtype), S


def _plain_attention(st):
    """(out [T][H][d], lse [T][H]), blocks of queries at a time."""
    lens, lens_k, G = st["lens"], st["lens_k"], st["G"]
    (q, inside), (k, seen), (v, _) = (_padded(x.float(), n, max(n)) for x, n in (
        (st["q"], lens), (st["k"], lens_k), (st["v"], lens_k)))
    k, v = (x.repeat_interleave(G, dim=2).transpose(1, 2) for x in (k, v))
    q = q.transpose(1, 2) * st["scale"]
    shift = torch.tensor([b - a for a, b in zip(lens, lens_k)], device=q.device)[:, None, None]
    at = torch.arange(k.shape[2], device=q.device)
    step = max(1, 2 ** 29 // (q.shape[0] * q.shape[1] * k.shape[2]))
    out, lse = [], []
    for i in range(0, q.shape[2], step):
        ok = seen[:, None, :]
        if st["causal"]:
            rows = torch.arange(i, min(i + step, q.shape[2]), device=q.device)[:, None]
            ok = ok & (at <= rows + shift)
        s = (q[:, :, i:i + step] @ k.transpose(-1, -2)).masked_fill_(~ok[:, None], -math.inf)
        top = s.amax(-1, keepdim=True)
        s = torch.exp_(s.sub_(top.clamp(min=-1e30)))
        total = s.sum(-1, keepdim=True)
        out.append((s @ v) / total.clamp(min=1e-30))
        lse.append((top + torch.log(total)).squeeze(-1))
    out = torch.cat(out, 2).transpose(1, 2)[inside]
    lse = torch.cat(lse, 2).transpose(1, 2)[inside]
    return out.to(st["q"].dtype), lse


# ---- what a pass cannot do without -------------------------------------------------------

def _pairs(case):
    total = 0
    for a, b in zip(_lens(case["lens"]), _lens(case["lens_k"])):
        if not case["causal"]:
            total += a * b
        else:  # row i sees i + 1 + b - a keys
            first = max(0, a - b)
            m = a - first
            total += m * (first + 1 + b - a) + m * (m - 1) // 2
    return total


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    H, Hk, d = case["H"], case["Hk"], case["d"]
    lens = _lens(case["lens"])
    T, n = sum(lens), len(lens)
    if case["call"] == "attn":
        Tk = sum(_lens(case["lens_k"]))
        return {"bytes": es * d * (2 * T * H + 2 * Tk * Hk) + 4 * T * H,
                "flops": 4 * d * H * _pairs(case)}
    given = es * T * (2 * Hk * d + H * d + 2 * H)
    state = 4 * n * H * d * d
    if case["call"] == "delta_token":
        return {"bytes": given + es * T * H * d + 2 * state, "flops": 6 * d * d * T * H}
    if case["call"] == "delta_prompt":
        return {"bytes": given + es * T * H * d + state, "flops": 6 * d * d * T * H}
    # the forward, then the backward: inputs and dout read again, their gradients written
    return {"bytes": 3 * given + 2 * es * T * H * d, "flops": 20 * d * d * T * H}


# ---- from the definitions, in 64 bits ----------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["call"] == "attn":
        return _exact_attention(st)
    return _exact_delta(st)


def _exact_delta(st):
    """Token by token over all sequences at once; a sequence that has ended keeps its state."""
    q, k, v, g, beta = (st[n].double() for n in ("q", "k", "v", "g", "beta"))
    G, scale, lens = st["G"], st["scale"], st["lens"]
    T, H, d = v.shape
    head = torch.arange(H, device=v.device) // G
    n = torch.tensor(lens, device=v.device)
    first = torch.cumsum(n, 0) - n
    order = torch.argsort(n, descending=True, stable=True)  # those still running come first
    first = first[order]
    S = torch.zeros(len(lens), H, d, d, dtype=torch.float64, device=v.device)
    if "state" in st:
        S = st["state"].double()[order]
    training = st["call"] == "delta_train"
    out, e = torch.zeros_like(v), torch.zeros_like(v)
    states, running = [], [sum(m > t for m in lens) for t in range(max(lens))]
    for t, m in enumerate(running):
        at = first[:m] + t
        kt, qt = k[at][:, head], q[at][:, head]
        if training:
            states.append(S[:m].clone())
        Sa = torch.exp(g[at])[..., None, None] * S[:m]
        e[at] = v[at] - torch.einsum("nhij,nhi->nhj", Sa, kt)
        Sa = Sa + torch.einsum("nhi,nhj->nhij", kt, beta[at][..., None] * e[at])
        S[:m] = Sa
        out[at] = scale * torch.einsum("nhij,nhi->nhj", Sa, qt)
    if not training:
        return out, S[torch.argsort(order)]
    do = st["dout"].double()
    dqh, dkh, dv = torch.zeros_like(v), torch.zeros_like(v), torch.zeros_like(v)
    dg, db = torch.zeros_like(g), torch.zeros_like(g)
    D = torch.zeros_like(S)
    for t in range(len(running) - 1, -1, -1):
        m = running[t]
        at = first[:m] + t
        kt, qt, bt = k[at][:, head], q[at][:, head], beta[at][..., None]
        before = torch.exp(g[at])[..., None, None] * states.pop()
        after = before + torch.einsum("nhi,nhj->nhij", kt, bt * e[at])
        dqh[at] = scale * torch.einsum("nhij,nhj->nhi", after, do[at])
        Dt = D[:m] + scale * torch.einsum("nhi,nhj->nhij", qt, do[at])
        du = torch.einsum("nhij,nhi->nhj", Dt, kt)
        db[at] = (e[at] * du).sum(-1)
        dv[at] = bt * du
        dkh[at] = (torch.einsum("nhij,nhj->nhi", Dt, bt * e[at])
                   - torch.einsum("nhij,nhj->nhi", before, dv[at]))
        Dt = Dt - torch.einsum("nhi,nhj->nhij", kt, dv[at])
        dg[at] = (before * Dt).sum((-1, -2))
        D[:m] = torch.exp(g[at])[..., None, None] * Dt
    dq, dk = (x.view(T, H // G, G, d).sum(2) for x in (dqh, dkh))
    return out, dq, dk, dv, dg, db


def _exact_attention(st):
    """One sequence and a block of its rows at a time."""
    H, d = st["q"].shape[1:]
    out, lse, a, b = [], [], 0, 0
    for nq, nk in zip(st["lens"], st["lens_k"]):
        q = st["q"][a:a + nq].double().view(nq, H // st["G"], st["G"], d)
        k, v = st["k"][b:b + nk].double(), st["v"][b:b + nk].double()
        for i in range(0, nq, 512):
            s = st["scale"] * torch.einsum("ihgd,jhd->hgij", q[i:i + 512], k)
            if st["causal"]:
                i_at = torch.arange(i, i + s.shape[2], device=s.device)[:, None] + nk - nq
                s = s.masked_fill(torch.arange(nk, device=s.device) > i_at, -math.inf)
            z = torch.logsumexp(s, -1)
            p = torch.where(s > -math.inf, torch.exp(s - z[..., None]), 0.0)
            out.append(torch.einsum("hgij,jhd->ihgd", p, v).reshape(-1, H, d))
            lse.append(z.permute(2, 0, 1).reshape(-1, H))
        a, b = a + nq, b + nk
    return torch.cat(out), torch.cat(lse)

"""Plain 64-bit forms of the packed-batch operators, token by token and row by row, and the
tolerances their kernels are held to.

Tolerances (relative L2), derived before the first run:
- fp32 results (fp32 storage; states and log sums in either storage): 2e-5.  One token commits
  an error of about sqrt(d) 2^-24 <= 7e-7 of what it adds (a sum of d <= 128 products), a
  product of bf16 high and low parts one of 2^-17 / sqrt(3) = 4.4e-6 of its operand; decay and
  correction keep the state's error a quadrature sum over the few tens of tokens it remembers
  with random signs, relative to a state that grew the same way: below 4 to 5 times one step's.
- bf16 results: 2 * 2^-8.  The result's own rounding is at most 2^-8 of each value; weights and
  corrections that enter a product as bf16 are off by at most 2^-8 each and add up with random
  signs (rms 2^-8 / sqrt(3) each), so three of them stay below another 2^-8.
"""
import torch

F32_TOL = 2e-5
BF16_TOL = 2 * 2.0 ** -8


def tol(dtype):
    return BF16_TOL if dtype == torch.bfloat16 else F32_TOL


def rel(x, ref):
    x, ref = x.double(), ref.double()
    top = ref.norm()
    return float((x - ref).norm() / top) if top > 0 else float((x - ref).norm())


def check(x, ref, what, dtype=None):
    assert torch.isfinite(x).all(), f"{what}: not finite"
    r = rel(x, ref)
    assert r <= tol(dtype or x.dtype), f"{what}: relative L2 {r:.3e}"


def offsets(lens, device="cuda"):
    return torch.tensor([0, *torch.tensor(lens).cumsum(0).tolist()], dtype=torch.int32,
                        device=device)


def delta_inputs(lens, H, Hk, d, dtype, seed=0, rows_behind=0, device="cuda"):
    """q, k (unit vectors with a common part), v, g, beta, dout, with rows behind the last
    sequence if asked."""
    gen = torch.Generator().manual_seed(seed)
    T = sum(lens) + rows_behind
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    common = 0.5 * r(1, Hk, d)
    x = {"q": unit(r(T, Hk, d) + common), "k": unit(r(T, Hk, d) + common), "v": r(T, H, d),
         "g": -torch.exp(2.0 * r(T, H) - 3.0), "beta": torch.sigmoid(r(T, H)),
         "dout": r(T, H, d)}
    return {n: t.to(dtype).to(device) for n, t in x.items()}


def delta_ref(x, lens, scale, state=None):
    """(out, last states) in float64; rows behind the last sequence are zero.  Differentiable."""
    q, k, v, g, beta = (x[n].double() for n in ("q", "k", "v", "g", "beta"))
    T, H, d = v.shape
    G = H // q.shape[1]
    q, k = q.repeat_interleave(G, 1), k.repeat_interleave(G, 1)
    outs, lasts, at = [], [], 0
    for i, n in enumerate(lens):
        S = (torch.zeros(H, d, d, dtype=torch.float64, device=v.device) if state is None
             else state[i].double())
        for t in range(at, at + n):
            S = torch.exp(g[t])[:, None, None] * S
            e = v[t] - torch.einsum("hij,hi->hj", S, k[t])
            S = S + torch.einsum("hi,hj->hij", k[t], beta[t][:, None] * e)
            outs.append(scale * torch.einsum("hij,hi->hj", S, q[t]))
        lasts.append(S)
        at += n
    outs += [torch.zeros(H, d, dtype=torch.float64, device=v.device)] * (T - at)
    return torch.stack(outs), torch.stack(lasts)


def delta_grads(x, lens, scale):
    """Gradients of sum(dout * out) by automatic differentiation of the definition."""
    names = ("q", "k", "v", "g", "beta")
    leaves = {n: x[n].double().detach().requires_grad_() for n in names}
    out, _ = delta_ref(leaves, lens, scale)
    n = sum(lens)
    return torch.autograd.grad((out[:n] * x["dout"][:n].double()).sum(), [leaves[m] for m in names])


def softattn_ref(q, k, v, lens_q, lens_k, scale, causal):
    """(out, lse) in float64 for the rows of the sequences."""
    H, d = q.shape[1:]
    G = H // k.shape[1]
    outs, lses, a, b = [], [], 0, 0
    for nq, nk in zip(lens_q, lens_k):
        qs = q[a:a + nq].double()
        ks = k[b:b + nk].double().repeat_interleave(G, 1)
        vs = v[b:b + nk].double().repeat_interleave(G, 1)
        s = scale * torch.einsum("ihd,jhd->hij", qs, ks)
        if causal:
            i = torch.arange(nq, device=q.device)[:, None] + nk - nq
            s = s.masked_fill(torch.arange(nk, device=q.device) > i, float("-inf"))
        z = torch.logsumexp(s, -1) if nk else torch.full((H, nq), float("-inf"),
                                                        dtype=torch.float64, device=q.device)
        p = torch.where(s > float("-inf"), torch.exp(s - z[..., None]), 0.0)
        outs.append(torch.einsum("hij,jhd->ihd", p, vs))
        lses.append(z.transpose(0, 1))
        a, b = a + nq, b + nk
    return torch.cat(outs), torch.cat(lses)


# Bounds for one sequence by itself, whose rows would drown in a batch's norm.  Derived before the
# first run, with roundings of random sign (2-norms over hundreds of values):
# - ROUNDED: a result's rounding to bf16 is uniform in +- 2^-8 of its power of two, 2^-8 / sqrt(3) of
#   its value at most;
# - WEIGHTED: the weights of softmax attention are rounded so too, and with random v their errors add
#   up as the output itself does: sqrt(2) of it;
# - GRADIENT: as many roundings as a bf16 gradient's longest chain of rounded operands has (the state or
#   its gradient, E twice, dV, Z) and its own, sqrt(6) of it, at the 1 / sqrt(2) that uniform
#   significands leave of the bound above;
# - SPLIT: bf16 high and low parts leave 2^-17 / sqrt(3) of an operand; three operands on the way to
#   the state (S, beta R, U);
# - PLAIN: fp32 sums of 128 products carry sqrt(128) 2^-24 of a typical sum; a state or an output
#   takes 5 such errors over (see the tolerances above).
ROUNDED = 2.0 ** -8 / 3 ** 0.5
WEIGHTED = 2 ** 0.5 * ROUNDED
GRADIENT = (6 / 2) ** 0.5 * ROUNDED
SPLIT = 3 ** 0.5 * 2.0 ** -17 / 3 ** 0.5
PLAIN = 5 * 128 ** 0.5 * 2.0 ** -24


def check_each(x, ref, lens, bound, what):
    """Every sequence's rows by themselves.  The bounds are for the root of a mean square; that of N
    errors strays by 1 / sqrt(2 N) of it (the squares of a normal variable have a variance of twice
    their mean's square, those of a rounding less), three times which is allowed: 7% for 1000 values,
    but half for the 20 gates of 5 rows of 4 heads."""
    assert torch.isfinite(x[:sum(lens)]).all(), f"{what}: not finite"
    at = 0
    for i, n in enumerate(lens):
        if n:
            r = rel(x[at:at + n], ref[at:at + n])
            most = bound * (1 + 3 / (2 * ref[at:at + n].numel()) ** 0.5)
            assert r <= most, f"{what} of sequence {i} ({n} rows): relative L2 {r:.3e} > {most:.3e}"
        at += n

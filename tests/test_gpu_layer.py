"""The calls of a recurrent layer one after the other, as a model makes them: residual norm, short
convolution, recurrence (selective scan, or the delta rule), gated norm; forward, gradients and single
tokens, against the same chain in 64 bits."""
import pytest
import torch

from paper_2606_27748_gb300 import flexattn as fa
from layer_ref import BF16, F32, conv_ref, norm_ref, ssm_ref
from packed_ref import delta_ref, offsets, rel

pytestmark = pytest.mark.gpu

LENS = (70, 1, 33)
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def library():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    from paper_2606_27748_gb300 import build
    build.build()
    fa.load()


def _ssm_layer(dtype, T, seed=0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    D, N = 128, 16
    act = {"y": r(T, 1, D), "res": 2 * r(T, 1, D), "z": r(T, 1, D), "dt": r(T, D), "B": r(T, 1, N),
           "C": r(T, 1, N), "up": r(T, 1, D), "dtotal": r(T, 1, D)}
    par = {"w1": 1 + 0.1 * r(D), "scale": 0.5 + 0.1 * r(D), "taps": 0.5 * r(D, 4), "bias": 0.5 * r(D),
           "A": -torch.arange(1, N + 1) * torch.exp(0.1 * r(D, N)), "skip": r(D), "dt_bias": r(D) - 3,
           "w2": 1 + 0.1 * r(D)}
    return ({n: t.to(dtype).cuda() for n, t in act.items()}, {n: t.to(F32).cuda() for n, t in par.items()})


def _reference(a, p, lens):
    """(out, total) of the chain in 64 bits."""
    h, total = norm_ref({"x": a["y"], "res": a["res"], "z": None, "w": p["w1"], "scale": p["scale"]}, EPS)
    c, _ = conv_ref({"x": h.flatten(1), "w": p["taps"], "bias": p["bias"]}, lens)
    s, last = ssm_ref({"x": c, "dt": a["dt"], "A": p["A"], "B": a["B"], "C": a["C"], "D": p["skip"],
                       "z": None, "dt_bias": p["dt_bias"]}, lens)
    out, _ = norm_ref({"x": s[:, None], "res": None, "z": a["z"], "w": p["w2"], "scale": None}, EPS)
    return out, total, last


def _forward(a, p, cu, save=None):
    h, total, r1 = fa.norm_fwd(a["y"], p["w1"], res=a["res"], scale=p["scale"], eps=EPS, want_rstd=True)
    h = h.flatten(1)
    c, rows = fa.conv_fwd(h, p["taps"], cu, bias=p["bias"], want_state=True)
    s, last = fa.ssm_fwd(c, a["dt"], p["A"], a["B"], a["C"], cu, D=p["skip"], dt_bias=p["dt_bias"],
                         save=save)
    out, _, r2 = fa.norm_fwd(s[:, None], p["w2"], z=a["z"], eps=EPS, want_rstd=True)
    return out, total, h, c, s, r1, r2, rows, last


# A chain of k bf16 results: each rounding is 2^-8 / sqrt(3) of its value at most and is carried on by
# operators whose gain is of order 1 (norms divide by their own input's size): forward 4 results; a
# gradient has those behind it and 4 of its own, 8 in quadrature, with a factor 2 for gains.
FORWARD = 2 * 4 ** 0.5 * 2.0 ** -8 / 3 ** 0.5
BACKWARD = 2 * 8 ** 0.5 * 2.0 ** -8 / 3 ** 0.5


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_selective_scan_layer(dtype):
    T, cu = sum(LENS), offsets(LENS)
    a, p = _ssm_layer(dtype, T)
    save = fa.ssm_save(a["dt"], a["B"], cu)
    out, total, h, c, s, r1, r2, _, _ = _forward(a, p, cu, save)
    most = FORWARD if dtype == BF16 else 4e-5
    leaves = {n: t.double().requires_grad_() for n, t in {**a, **p}.items()}
    ref, rtotal, _ = _reference(leaves, leaves, LENS)
    assert rel(out, ref.detach()) <= most and rel(total, rtotal.detach()) <= most
    # back through the calls
    ds, _, dz, dw2, _ = fa.norm_bwd(s[:, None], p["w2"], r2, a["up"], z=a["z"], eps=EPS)
    dc, ddt, dA, dB, dC, dskip, _, dtb = fa.ssm_bwd(c, a["dt"], p["A"], a["B"], a["C"], cu,
                                                    ds.flatten(1), save, D=p["skip"], dt_bias=p["dt_bias"])
    dh, dtaps, dbias = fa.conv_bwd(h, p["taps"], cu, dc, bias=p["bias"])
    dy, dres, _, dw1, dscale = fa.norm_bwd(a["y"], p["w1"], r1, dh[:, None], res=a["res"], scale=p["scale"],
                                           eps=EPS, dtotal=a["dtotal"])
    got = {"y": dy, "res": dres, "z": dz, "dt": ddt, "B": dB, "C": dC, "w1": dw1, "scale": dscale,
           "taps": dtaps, "bias": dbias, "A": dA, "skip": dskip, "dt_bias": dtb, "w2": dw2}
    want = torch.autograd.grad((ref * a["up"].double()).sum() + (rtotal * a["dtotal"].double()).sum(),
                               [leaves[n] for n in got])
    most = BACKWARD if dtype == BF16 else 1e-4
    for (n, g), w in zip(got.items(), want):
        assert rel(g, w) <= most, f"d{n}: {rel(g, w):.2e}"


def test_tokens_go_on_where_a_prompt_ended():
    """A prompt, then five single tokens through the layer's states, against the whole sequences."""
    lens, more = (40, 23), 5
    T = sum(lens) + 2 * more
    a, p = _ssm_layer(F32, T, seed=1)
    whole = (lens[0] + more, lens[1] + more)
    ref, _, rlast = _reference(a, p, whole)
    start = (0, whole[0])
    at = torch.cat([torch.arange(b, b + n) for b, n in zip(start, lens)]).cuda()
    out, *_, rows, last = _forward({n: t[at] for n, t in a.items()}, p, offsets(lens))
    assert rel(out, ref[at]) <= 4e-5
    for k in range(more):
        at = torch.tensor([b + n + k for b, n in zip(start, lens)]).cuda()
        t = {n: v[at] for n, v in a.items()}
        h, _, _ = fa.norm_fwd(t["y"], p["w1"], res=t["res"], scale=p["scale"], eps=EPS)
        c = fa.conv_decode(h.flatten(1), p["taps"], rows, bias=p["bias"])
        s = fa.ssm_decode(c, t["dt"], p["A"], t["B"], t["C"], last, D=p["skip"], dt_bias=p["dt_bias"])
        out, _, _ = fa.norm_fwd(s[:, None], p["w2"], z=t["z"], eps=EPS)
        assert rel(out, ref[at]) <= 4e-5, k
    assert rel(last, rlast) <= 4e-5


def test_delta_rule_layer():
    """The same neighbours around the delta rule: convolutions of q, k and v in heads, the gated norm of
    every head behind it."""
    T, cu, H, d = sum(LENS), offsets(LENS), 2, 64
    gen = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64).cuda()  # noqa: E731
    x = {n: (0.3 * r(T, H, d)).to(F32) for n in ("q", "k", "v")}
    taps = {n: (0.5 * r(H * d, 4)).to(F32) for n in x}
    g, beta = (-0.1 * r(T, H).abs()).to(F32), torch.sigmoid(r(T, H)).to(F32)
    z, w = r(T, H, d).to(F32), (1 + 0.1 * r(d)).to(F32)
    c = {n: fa.conv_fwd(x[n], taps[n], cu)[0] for n in x}
    k = c["k"] / c["k"].norm(dim=-1, keepdim=True)
    o, _ = fa.delta_fwd(c["q"], k, c["v"], g, beta, cu)
    out, _, _ = fa.norm_fwd(o, w, z=z, eps=EPS)
    ref = {n: conv_ref({"x": x[n].flatten(1), "w": taps[n], "bias": None}, LENS)[0].view(T, H, d) for n in x}
    ref["k"] = ref["k"] / ref["k"].norm(dim=-1, keepdim=True)
    o, _ = delta_ref({**ref, "g": g, "beta": beta}, LENS, d ** -0.5)
    want, _ = norm_ref({"x": o, "res": None, "z": z, "w": w, "scale": None}, EPS)
    assert rel(out, want) <= 4e-5

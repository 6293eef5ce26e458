"""Gated and residual norms (flex_norm_fwd / _bwd) against their definition in 64 bits."""
import pytest
import torch

from paper_2606_27748_gb300 import flexattn
from layer_ref import BF16, F32, NORM, close, gradients, norm_inputs, norm_ref
from packed_ref import offsets

pytestmark = pytest.mark.gpu

EPS = 1e-5
FORMS = [dict(), dict(gate=True), dict(res=True), dict(res=True, scale=True),
         dict(gate=True, res=True, scale=True)]
# rows, heads, size: one unit a head to rows of four blocks' worth, and more rows than groups
SIZES = [(1, 1, 8), (7, 3, 16), (33, 4, 128), (5, 1, 1000), (3, 2, 4104), (2, 1, 8192), (900, 16, 64)]


@pytest.fixture(scope="module", autouse=True)
def library():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    from paper_2606_27748_gb300 import build
    build.build()
    flexattn.load()


def _fwd(x, **kw):
    return flexattn.norm_fwd(x["x"], x["w"], z=x["z"], res=x["res"], scale=x["scale"], eps=EPS, **kw)


def _bwd(x, rstd, **kw):
    return flexattn.norm_bwd(x["x"], x["w"], rstd, x["dout"], z=x["z"], res=x["res"], scale=x["scale"],
                             eps=EPS, dtotal=x["dtotal"], **kw)


def _check(x, out, total, got):
    ref, rtotal = norm_ref(x, EPS)
    close(out, ref, "out")
    sent = [x["dout"]]
    if rtotal is None:
        assert total is None
    else:
        close(total, rtotal, "total")
        sent.append(x["dtotal"])
    ref = gradients(lambda v: [o for o in norm_ref(v, EPS) if o is not None], x, NORM, sent)
    for name, g, r in zip(("dx", "dres", "dz", "dw", "dscale"), got, ref):
        if r is None:
            assert g is None, name
        else:
            close(g, r, name)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(f) or "plain")
@pytest.mark.parametrize("own", [False, True], ids=["shared", "own"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_norm(size, own, form, dtype):
    T, H, d = size
    x = norm_inputs(T, H, d, dtype, heads=H if own else None, pad=8, **form)
    out, total, rstd = _fwd(x, want_rstd=True)
    _check(x, out, total, _bwd(x, rstd))


def test_rows_of_the_sequences_only_and_in_place():
    lens = (20, 0, 11)
    x = norm_inputs(50, 4, 64, BF16, heads=4, gate=True, res=True, scale=True, seed=1)
    for n in ("x", "res", "z", "dout", "dtotal"):
        x[n][31:] = float("nan")
    cu = offsets(lens)
    keep = {n: torch.full_like(x["x"], 7.0) for n in ("out", "total", "dx", "dres", "dz")}
    rstd = torch.full((50, 4), 7.0, device="cuda")
    out, total, _ = _fwd(x, cu=cu, out=keep["out"], total=keep["total"], rstd=rstd)
    got = _bwd(x, rstd, cu=cu, **{n: keep[n] for n in ("dx", "dres", "dz")})
    for t in (*keep.values(), rstd):
        assert (t[31:] == 7).all()
    y = {n: t[:31] if n in ("x", "res", "z", "dout", "dtotal") else t for n, t in x.items()}
    _check(y, out[:31], total[:31], [g[:31] if g.dim() == 3 else g for g in got])
    stream = x["res"].clone()
    out2, same, _ = _fwd({**x, "res": stream}, cu=cu, total=stream)
    assert same is stream and torch.equal(stream[:31], total[:31]) and torch.equal(out2[:31], out[:31])


def test_no_rows_and_no_upstream_of_the_stream():
    x = norm_inputs(12, 2, 64, F32, res=True, scale=True, seed=2)
    empty = offsets((0, 0))
    out = torch.full_like(x["x"], 7.0)
    _, _, rstd = _fwd(x, want_rstd=True)
    _fwd(x, cu=empty, out=out)
    assert (out == 7).all()
    got = _bwd(x, rstd, cu=empty)
    assert (got[3] == 0).all() and (got[4] == 0).all()
    x["dtotal"] = None
    got = _bwd(x, rstd)
    ref = gradients(lambda v: norm_ref(v, EPS)[:1], x, NORM, [x["dout"]])
    for g, r in zip(got, ref):
        assert (g is None) == (r is None)
        if r is not None:
            close(g, r, "gradient")


def test_zeros_and_one_row_of_nan():
    x = norm_inputs(9, 1, 128, F32, gate=True, seed=3)
    x["x"][4] = 0.0
    x["x"][6, 0, 5] = float("nan")
    out, _, rstd = _fwd(x, want_rstd=True)
    assert (out[4] == 0).all() and torch.isnan(out[6]).all()
    assert torch.isfinite(out[:6]).all() and torch.isfinite(out[7:]).all()
    dx = _bwd(x, rstd)[0]
    assert torch.isfinite(dx[:6]).all() and torch.isfinite(dx[7:]).all()


def test_results_repeat_and_replay():
    x, y = (norm_inputs(700, 2, 256, BF16, gate=True, res=True, scale=True, seed=s) for s in (4, 5))

    def both(v, ws=None, stream=None):
        out, total, rstd = _fwd(v, want_rstd=True, stream=stream)
        return out, total, rstd, *_bwd(v, rstd, ws=ws, stream=stream)

    first = both(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    there = both(x, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, there))
    held = {n: t.clone() for n, t in x.items()}
    ws = flexattn.norm_workspace(x["x"], x["w"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(held, ws)
    for v in (y, x):
        for n in held:
            held[n].copy_(v[n])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, both(v)))


def test_gradients_against_differences():
    x = norm_inputs(6, 2, 32, F32, heads=2, gate=True, res=True, scale=True, seed=6)
    _, _, rstd = _fwd(x, want_rstd=True)
    got = _bwd(x, rstd)

    def loss(v):
        out, total = norm_ref(v, EPS)
        return float((out * x["dout"].double()).sum() + (total * x["dtotal"].double()).sum())

    gen = torch.Generator().manual_seed(0)
    for name, g in zip(NORM, got):
        way = torch.randn(x[name].shape, generator=gen, dtype=torch.float64).cuda()
        up, down = ({**x, name: x[name].double() + s * way} for s in (1e-5, -1e-5))
        slope = (loss(up) - loss(down)) / 2e-5
        assert abs(float((g.double() * way).sum()) - slope) <= 2e-5 * float(g.double().norm() * way.norm()), name


# More than two rounds of every group of threads, at each number of threads a group (past 32 with block
# barriers between) and of 16-byte units a thread.
ROUNDS = [(BF16, 2600, 1, 512), (BF16, 1300, 1, 1000), (BF16, 650, 2, 2048), (BF16, 700, 1, 4096),
          (BF16, 620, 1, 8192), (F32, 650, 2, 1024), (F32, 700, 1, 2048), (F32, 620, 1, 4096),
          (F32, 310, 2, 8192)]


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(f) or "plain")
@pytest.mark.parametrize("own", [False, True], ids=["shared", "own"])
@pytest.mark.parametrize("dtype,T,H,d", ROUNDS, ids=str)
def test_many_rounds(dtype, T, H, d, own, form):
    x = norm_inputs(T, H, d, dtype, heads=H if own else None, seed=7, pad=8, **form)
    out, total, rstd = _fwd(x, want_rstd=True)
    _check(x, out, total, _bwd(x, rstd))


@pytest.mark.parametrize("dtype,T,H,d", ROUNDS, ids=str)
def test_rounds_that_some_groups_sit_out(dtype, T, H, d):
    """The last sequence ends where a part of a block's groups, or of the blocks, has a row left."""
    x = norm_inputs(T, H, d, dtype, heads=H, gate=True, res=True, scale=True, seed=8)
    for rows in (T - 7, T // 2 + 1, 1):
        y = {n: t.clone() if n in ("x", "res", "z", "dout", "dtotal") else t for n, t in x.items()}
        for n in ("x", "res", "z", "dout", "dtotal"):
            y[n][rows:] = float("nan")
        cu = offsets((rows,))
        out, total, rstd = _fwd(y, cu=cu, want_rstd=True)
        got = _bwd(y, rstd, cu=cu)
        z = {n: t[:rows] if n in ("x", "res", "z", "dout", "dtotal") else t for n, t in x.items()}
        _check(z, out[:rows], total[:rows], [g[:rows] if g.dim() == 3 else g for g in got])

"""Rows more than 2^31 elements behind the first: the last sequence of a batch that large, against the same
sequence by itself or its definition."""
import pytest
import torch

from paper_2606_27748_gb300 import flexattn as fa
from layer_ref import BF16, F32, SSM, close, gradients, ssm_ref
from packed_ref import offsets

pytestmark = pytest.mark.gpu

D, LAST = 2048, 90
T = 2 ** 31 // D + 400  # elements of one tensor pass 31 bits
LENS = (T - LAST - 300, 300, LAST)


@pytest.fixture(scope="module", autouse=True)
def library():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    from paper_2606_27748_gb300 import build
    build.build()
    fa.load()


def _rows(seed, *shape):
    """[T, ...] of which the last rows are random, the others a value that leaves sums small."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.full((T, *shape), 0.001, dtype=BF16, device="cuda")
    x[-400:] = torch.randn(400, *shape, device="cuda", generator=gen).to(BF16)
    return x


def _par(seed, *shape):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=gen)


def test_convolution():
    x, dout, w, b = _rows(1, D), _rows(2, D), _par(3, D, 4), _par(4, D)
    cu = offsets(LENS)
    out, last = fa.conv_fwd(x, w, cu, bias=b, want_state=True)
    dx, dw, db = fa.conv_bwd(x, w, cu, dout, bias=b)
    one = offsets((LAST,))
    xs, ds = x[-LAST:].clone(), dout[-LAST:].clone()
    o1, l1 = fa.conv_fwd(xs, w, one, bias=b, want_state=True)
    assert torch.equal(out[-LAST:], o1) and torch.equal(last[2], l1[0])
    assert torch.equal(dx[-LAST:], fa.conv_bwd(xs, w, one, ds, bias=b)[0])
    assert torch.isfinite(dw).all() and torch.isfinite(db).all()


def test_norm():
    x, z, res, dout, up = (_rows(s, 16, 128) for s in (5, 6, 7, 8, 9))
    w, s = 1 + 0.1 * _par(10, 16, 128), _par(11, 16, 128)
    out, total, rstd = fa.norm_fwd(x, w, z=z, res=res, scale=s, want_rstd=True)
    got = fa.norm_bwd(x, w, rstd, dout, z=z, res=res, scale=s, dtotal=up)
    end = lambda t: t[-LAST:].clone()  # noqa: E731
    o1, t1, r1 = fa.norm_fwd(end(x), w, z=end(z), res=end(res), scale=s, want_rstd=True)
    assert torch.equal(out[-LAST:], o1) and torch.equal(total[-LAST:], t1) and torch.equal(rstd[-LAST:], r1)
    g1 = fa.norm_bwd(end(x), w, r1, end(dout), z=end(z), res=end(res), scale=s, dtotal=end(up))
    for a, b in zip(got[:3], g1[:3]):
        assert torch.equal(a[-LAST:], b)


def test_selective_scan():
    x = {"x": _rows(12, D), "dt": _rows(13, D), "A": -torch.exp(0.1 * _par(14, D, 16)), "B": _rows(15, 1, 16),
         "C": _rows(16, 1, 16), "D": _par(17, D), "z": _rows(18, D), "dt_bias": _par(19, D) - 4.0,
         "dout": _rows(20, D)}
    cu = offsets(LENS)
    five, opt = [x[n] for n in ("x", "dt", "A", "B", "C")], {n: x[n] for n in ("D", "z", "dt_bias")}
    save = fa.ssm_save(x["x"], x["B"], cu)
    out, last = fa.ssm_fwd(*five, cu, save=save, **opt)
    got = fa.ssm_bwd(*five, cu, x["dout"], save, **opt)
    y = {n: t[-LAST:].clone() if t.shape[0] == T else t for n, t in x.items()}
    ref, rlast = ssm_ref(y, (LAST,))
    close(out[-LAST:], ref, "out")
    close(last[2:], rlast, "last state")
    want = gradients(lambda v: ssm_ref(v, (LAST,))[:1], y, SSM, [y["dout"]])
    for n, g, r in zip(SSM, got, want):
        if g.shape[0] == T:
            close(g[-LAST:], r, "d" + n)
        else:
            assert torch.isfinite(g).all(), n

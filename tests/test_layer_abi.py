"""Entry points around the recurrence: what the host refuses (no GPU needed: no compute call is
made)."""
import ctypes

import pytest
import torch

from paper_2606_27748_gb300 import flexattn
from paper_2606_27748_gb300.flexattn import (FLEX_EINVAL, FLEX_EUNSUPPORTED, FLEX_EWORKSPACE,
                                             FlexConv, FlexNorm, FlexSsm)

P = ctypes.c_void_p(1 << 20)  # never dereferenced: validation fails first
OFF = ctypes.c_void_p((1 << 20) + 2)
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    from paper_2606_27748_gb300 import build
    build.build()
    return flexattn.load()


# ---- selective scan ------------------------------------------------------------------------

FWD = ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "cu", "S0", "S1", "out", "save", "ws")
BWD = ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "cu", "dout", "save", "dx", "ddt", "dA", "dB",
       "dC", "dD", "dz", "ddt_bias", "ws")
TOKEN = ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "S", "out")


def _ssm(**kw):
    x = dict(n=3, T=100, D=64, G=1, N=16, dtype=1, softplus=1, x_stride=64, dt_stride=64,
             b_stride=16, c_stride=16, z_stride=64)
    x.update(kw)
    return FlexSsm(*(x[name] for name, _ in FlexSsm._fields_))


def _call(f, names, s, n=BIG, scratch=True, **kw):
    given = {"S0": None, "save": P if "dout" in names else None}
    args = [kw.get(name, given.get(name, P)) for name in names]
    return f(ctypes.byref(s) if s else None, *args, *([n, None] if scratch else [None]))


def _fwd(lib, s, **kw):
    return _call(lib.flex_ssm_fwd, FWD, s, **kw)


def _bwd(lib, s, **kw):
    return _call(lib.flex_ssm_bwd, BWD, s, **kw)


def _token(lib, s, **kw):
    return _call(lib.flex_ssm_decode, TOKEN, s, scratch=False, **kw)


@pytest.mark.parametrize("kw", [dict(n=0), dict(T=0), dict(D=0), dict(G=0), dict(N=0), dict(G=3),
                                dict(dtype=2), dict(x_stride=56), dict(dt_stride=68),
                                dict(b_stride=8), dict(c_stride=20)], ids=str)
def test_ssm_bad_shapes(lib, kw):
    s = _ssm(**kw)
    assert _fwd(lib, s) == _bwd(lib, s) == _token(lib, s) == FLEX_EINVAL
    assert lib.flex_ssm_workspace_bytes(ctypes.byref(s), 1) == 0
    assert lib.flex_ssm_save_bytes(ctypes.byref(s)) == 0


@pytest.mark.parametrize("kw", [dict(N=4), dict(N=24), dict(N=64), dict(D=68, x_stride=72, dt_stride=72),
                                dict(n=65536), dict(T=1 << 30), dict(D=65544)], ids=str)
def test_ssm_unsupported_shapes(lib, kw):
    s = _ssm(**kw)
    assert _fwd(lib, s) == _bwd(lib, s) == _token(lib, s) == FLEX_EUNSUPPORTED
    assert lib.flex_ssm_workspace_bytes(ctypes.byref(s), 0) == 0


@pytest.mark.parametrize("name", FWD)
def test_ssm_fwd_pointers(lib, name):
    assert _fwd(lib, _ssm(), **{name: OFF if name != "cu" else ctypes.c_void_p((1 << 20) + 1)}) == FLEX_EINVAL
    if name not in ("D", "z", "dt_bias", "S0", "S1", "save"):
        assert _fwd(lib, _ssm(), **{name: None}) == FLEX_EINVAL


@pytest.mark.parametrize("name", BWD)
def test_ssm_bwd_pointers(lib, name):
    assert _bwd(lib, _ssm(), **{name: OFF if name != "cu" else ctypes.c_void_p((1 << 20) + 1)}) == FLEX_EINVAL
    assert _bwd(lib, _ssm(), **{name: None}) == FLEX_EINVAL  # (a gradient goes with its input)


@pytest.mark.parametrize("name", TOKEN)
def test_ssm_decode_pointers(lib, name):
    s = _ssm(T=3)
    assert _token(lib, s, **{name: OFF}) == FLEX_EINVAL
    if name not in ("D", "z", "dt_bias"):
        assert _token(lib, s, **{name: None}) == FLEX_EINVAL
    assert _token(lib, _ssm()) == FLEX_EINVAL  # T != n


def test_ssm_gate_stride_save_and_workspace(lib):
    assert _fwd(lib, _ssm(z_stride=56)) == FLEX_EINVAL
    assert _fwd(lib, _ssm(), S0=P, save=P) == FLEX_EINVAL  # training starts from the zero state
    s = _ssm()
    b = ctypes.byref(s)
    need = [lib.flex_ssm_workspace_bytes(b, k) for k in (0, 1)]
    assert 256 <= need[0] <= need[1]
    assert _fwd(lib, s, n=255) == FLEX_EWORKSPACE and _fwd(lib, s, n=need[0] - 1) == FLEX_EWORKSPACE
    assert _bwd(lib, s, n=need[1] - 1) == FLEX_EWORKSPACE
    assert lib.flex_ssm_save_bytes(b) == (100 // 8 + 3) * 64 * 16 * 4


def test_ssm_binding_refuses():
    x, B = torch.zeros(10, 64), torch.zeros(10, 1, 16)
    A, cu = torch.zeros(64, 16), torch.tensor([0, 10], dtype=torch.int32)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        flexattn.ssm_fwd(x, x, A, B, B, cu)  # not on the GPU
    cpu = x.get_device()
    shape = flexattn._packed_ssm(x, x, B, B, None, 1, True, cpu)
    assert (shape.T, shape.D, shape.G, shape.N, shape.x_stride, shape.b_stride) == (10, 64, 1, 16, 64, 16)
    wide = torch.zeros(10, 96)
    assert flexattn._packed_ssm(wide[:, 8:72], x, B, B, wide[:, :64], 1, True, cpu).x_stride == 96
    for bad in (dict(x=x[:, None]), dict(B=B[:, 0]), dict(dt=x[:9]), dict(dt=x.double()), dict(C=B[:, :, :8]),
                dict(x=x[:0], dt=x[:0], B=B[:0], C=B[:0]), dict(z=x[:, :32]),
                dict(x=torch.zeros(64, 10).t())):
        args = dict(x=x, dt=x, B=B, C=B, z=None)
        args.update(bad)
        with pytest.raises(ValueError):
            flexattn._packed_ssm(*args.values(), 1, True, cpu)
    with pytest.raises(TypeError):
        flexattn._packed_ssm(*(t.half() for t in (x, x, B, B)), None, 1, True, cpu)


# ---- short convolution -------------------------------------------------------------------------

CONV_FWD = ("x", "w", "bias", "cu", "S0", "S1", "out")
CONV_BWD = ("x", "w", "bias", "cu", "dout", "dx", "dw", "dbias", "ws")
CONV_TOKEN = ("x", "w", "bias", "S", "out")


def _conv(**kw):
    x = dict(n=3, T=100, D=64, W=4, dtype=1, silu=1, x_stride=64)
    x.update(kw)
    return FlexConv(*(x[name] for name, _ in FlexConv._fields_))


def _plain_call(f, names, s, *more, **kw):
    at = {n: ctypes.c_void_p((1 << 20) + 4096 * i) for i, n in enumerate(names)}
    at["S0"] = None
    return f(ctypes.byref(s) if s else None, *(kw.get(n, at[n]) for n in names), *more, None)


def _conv_calls(lib, s, n=BIG, **kw):
    return [_plain_call(lib.flex_conv_fwd, CONV_FWD, s, **kw),
            _plain_call(lib.flex_conv_bwd, CONV_BWD, s, n, **kw),
            _plain_call(lib.flex_conv_decode, CONV_TOKEN, s, **kw)]


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), FLEX_EINVAL), (dict(T=0), FLEX_EINVAL), (dict(D=0), FLEX_EINVAL), (dict(W=0), FLEX_EINVAL),
    (dict(dtype=3), FLEX_EINVAL), (dict(x_stride=56), FLEX_EINVAL), (dict(x_stride=66), FLEX_EINVAL),
    (dict(W=1), FLEX_EUNSUPPORTED), (dict(W=5), FLEX_EUNSUPPORTED), (dict(D=60), FLEX_EUNSUPPORTED),
    (dict(n=65536), FLEX_EUNSUPPORTED), (dict(T=1 << 30), FLEX_EUNSUPPORTED),
    (dict(D=65544), FLEX_EUNSUPPORTED)], ids=str)
def test_conv_shapes(lib, kw, status):
    s = _conv(**kw)
    assert _conv_calls(lib, s) == [status] * 3
    assert lib.flex_conv_workspace_bytes(ctypes.byref(s)) == 0


def test_conv_pointers_and_workspace(lib):
    s, one = _conv(), _conv(T=3)
    assert _conv_calls(lib, None) == [FLEX_EINVAL] * 3
    for f, names, shape, more in ((lib.flex_conv_fwd, CONV_FWD, s, ()),
                                  (lib.flex_conv_bwd, CONV_BWD, s, (BIG,)),
                                  (lib.flex_conv_decode, CONV_TOKEN, one, ())):
        for name in names:
            off = ctypes.c_void_p((1 << 20) + 1)
            assert _plain_call(f, names, shape, *more, **{name: off}) == FLEX_EINVAL, name
            if name not in ("S0", "S1", "bias") or (name == "bias" and "dbias" in names):
                assert _plain_call(f, names, shape, *more, **{name: None}) == FLEX_EINVAL, name
    assert _plain_call(lib.flex_conv_decode, CONV_TOKEN, s) == FLEX_EINVAL  # T != n
    assert _plain_call(lib.flex_conv_fwd, CONV_FWD, s, S0=P, S1=P) == FLEX_EINVAL  # one buffer
    assert _plain_call(lib.flex_conv_fwd, CONV_FWD, s, x=P, out=P) == FLEX_EINVAL
    assert _plain_call(lib.flex_conv_bwd, CONV_BWD, s, BIG, x=P, dx=P) == FLEX_EINVAL
    assert _plain_call(lib.flex_conv_bwd, CONV_BWD, s, BIG, dout=P, dx=P) == FLEX_EINVAL
    need = lib.flex_conv_workspace_bytes(ctypes.byref(s))
    assert need > 256
    assert _plain_call(lib.flex_conv_bwd, CONV_BWD, s, need - 1) == FLEX_EWORKSPACE


# ---- norms -------------------------------------------------------------------------------------

NORM_FWD = ("x", "w", "z", "res", "scale", "end", "out", "total", "rstd")
NORM_BWD = ("x", "w", "z", "res", "scale", "end", "rstd", "dout", "dtotal", "dx", "dres", "dz", "dw",
            "dscale", "ws")


def _norm(**kw):
    x = dict(T=100, H=4, d=64, dtype=1, heads=1, x_stride=256, z_stride=256, res_stride=256, eps=1e-6)
    x.update(kw)
    return FlexNorm(*(x[name] for name, _ in FlexNorm._fields_))


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), FLEX_EINVAL), (dict(H=0), FLEX_EINVAL), (dict(d=0), FLEX_EINVAL), (dict(heads=2), FLEX_EINVAL),
    (dict(dtype=-1), FLEX_EINVAL), (dict(eps=-1.0), FLEX_EINVAL), (dict(eps=float("nan")), FLEX_EINVAL),
    (dict(x_stride=248), FLEX_EINVAL), (dict(z_stride=260), FLEX_EINVAL), (dict(res_stride=0), FLEX_EINVAL),
    (dict(d=60), FLEX_EUNSUPPORTED), (dict(H=1, d=8200, x_stride=8200), FLEX_EUNSUPPORTED),
    (dict(H=1025), FLEX_EUNSUPPORTED), (dict(T=1 << 30), FLEX_EUNSUPPORTED),
    (dict(T=(1 << 30) - 1, H=3), FLEX_EUNSUPPORTED)], ids=str)
def test_norm_shapes(lib, kw, status):
    s = _norm(**kw)
    assert _plain_call(lib.flex_norm_fwd, NORM_FWD, s) == status
    assert _plain_call(lib.flex_norm_bwd, NORM_BWD, s, BIG) == status
    if "z_stride" not in kw and "res_stride" not in kw:  # (strides of what the size does not know)
        assert lib.flex_norm_workspace_bytes(ctypes.byref(s)) == 0


def test_norm_pointers_and_workspace(lib):
    s = _norm()
    fwd = lambda **kw: _plain_call(lib.flex_norm_fwd, NORM_FWD, s, **kw)  # noqa: E731
    bwd = lambda n=BIG, **kw: _plain_call(lib.flex_norm_bwd, NORM_BWD, s, n, **kw)  # noqa: E731
    assert _plain_call(lib.flex_norm_fwd, NORM_FWD, None) == FLEX_EINVAL
    off = ctypes.c_void_p((1 << 20) + 2)
    for name in NORM_FWD:
        assert fwd(**{name: off}) == FLEX_EINVAL, name
    for name in ("x", "w", "out", "total", "res"):  # (total goes with res, scale wants it)
        assert fwd(**{name: None}) == FLEX_EINVAL, name
    for name in NORM_BWD:
        assert bwd(**{name: off}) == FLEX_EINVAL, name
    for name in ("x", "w", "rstd", "dout", "dx", "dres", "dz", "dw", "dscale", "ws", "z", "res", "scale"):
        assert bwd(**{name: None}) == FLEX_EINVAL, name
    assert bwd(scale=None, dscale=None) == FLEX_EINVAL  # dres is dx, which is not given then
    need = lib.flex_norm_workspace_bytes(ctypes.byref(s))
    assert bwd(need - 1) == FLEX_EWORKSPACE
    assert bwd(need - 1, scale=None, dscale=None, dx=None) == FLEX_EWORKSPACE


def test_conv_and_norm_bindings_refuse():
    x, w, cu = torch.zeros(10, 64), torch.zeros(64, 4), torch.tensor([0, 10], dtype=torch.int32)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        flexattn.conv_fwd(x, w, cu)  # not on the GPU
    cpu = x.get_device()
    s = flexattn._packed_conv(torch.zeros(10, 96)[:, :64].view(10, 4, 16), w, 1, True, cpu)
    assert (s.T, s.D, s.W, s.x_stride) == (10, 64, 4, 96)
    for bad in (x[:0], x[0], torch.zeros(64, 10).t()):
        with pytest.raises(ValueError):
            flexattn._packed_conv(bad, w, 1, True, cpu)
    y, p = torch.zeros(10, 4, 64), torch.zeros(64)
    s = flexattn._packed_norm(y, p, None, y, 1e-6, cpu)
    assert (s.T, s.H, s.d, s.heads, s.res_stride) == (10, 4, 64, 1, 256)
    assert flexattn._packed_norm(y, torch.zeros(4, 64), None, None, 1e-6, cpu).heads == 4
    for args in ((x, p, None, None), (y, torch.zeros(1, 4, 64), None, None), (y, p, y[:9], None),
                 (y, p, None, y.double()), (y[:0], p, None, None)):
        with pytest.raises(ValueError):
            flexattn._packed_norm(*args, 1e-6, cpu)
    with pytest.raises(ValueError):
        flexattn._plain(torch.zeros(65), "w", flexattn._params(p, s), torch.float32, cpu)


# ---- outputs over their inputs ---------------------------------------------------------------

def _apart(names):
    return {n: ctypes.c_void_p((1 << 20) + 4096 * i) for i, n in enumerate(names)}


def _over(call, names, pairs, strides, make, rows):
    """Every output over an input: refused where the input is a slice of wider rows, by any of
    several rows; `call` gets one byte of workspace too little, so no launch is reached."""
    for out, inp in pairs:
        at = _apart(names)
        at[out] = at[inp]
        wide = {strides[inp]: 2 * make()[strides[inp]]}
        assert call(make(**wide), at) == FLEX_EINVAL, (out, inp)
        if rows:  # a single row, and rows of no wider ones, are in place
            assert call(make(), at) == FLEX_EWORKSPACE, (out, inp)
            assert call(make(**wide, **rows), at) == FLEX_EWORKSPACE, (out, inp)


def test_ssm_output_over_a_slice(lib):
    def make(**kw):
        return {**dict(n=3, T=100, D=64, G=1, N=16, dtype=1, softplus=1, x_stride=64, dt_stride=64,
                       b_stride=16, c_stride=16, z_stride=64), **kw}

    def fwd(kw, at):
        s = FlexSsm(*kw.values())
        need = lib.flex_ssm_workspace_bytes(ctypes.byref(s), 0)
        return _fwd(lib, s, n=need - 1, **{**at, "S0": None})

    def bwd(kw, at):
        s = FlexSsm(*kw.values())
        need = lib.flex_ssm_workspace_bytes(ctypes.byref(s), 1)
        return _bwd(lib, s, n=need - 1, **at)

    strides = {"x": "x_stride", "dt": "dt_stride", "z": "z_stride"}
    one = dict(n=1, T=1)
    _over(fwd, FWD, [("out", i) for i in strides], strides, make, one)
    _over(bwd, BWD, [(o, i) for o in ("dx", "ddt", "dz") for i in strides], strides, make, one)
    token = lambda kw, at: _token(lib, FlexSsm(*kw.values()), **at)  # noqa: E731
    _over(token, TOKEN, [("out", i) for i in strides], strides, lambda **kw: make(T=3, **kw), None)


def test_conv_token_over_a_slice(lib):
    make = lambda **kw: {**dict(n=3, T=3, D=64, W=4, dtype=1, silu=1, x_stride=64), **kw}  # noqa: E731
    token = lambda kw, at: _plain_call(lib.flex_conv_decode, CONV_TOKEN, FlexConv(*kw.values()), **at)  # noqa: E731
    _over(token, CONV_TOKEN, [("out", "x")], {"x": "x_stride"}, make, None)


def test_norm_output_over_a_slice(lib):
    def make(**kw):
        return {**dict(T=100, H=4, d=64, dtype=1, heads=1, x_stride=256, z_stride=256, res_stride=256,
                       eps=1e-6), **kw}

    def bwd(kw, at):
        s = FlexNorm(*kw.values())
        need = lib.flex_norm_workspace_bytes(ctypes.byref(s))
        return _plain_call(lib.flex_norm_bwd, NORM_BWD, s, need - 1, **at)

    strides = {"x": "x_stride", "z": "z_stride", "res": "res_stride"}
    fwd = lambda kw, at: _plain_call(lib.flex_norm_fwd, NORM_FWD, FlexNorm(*kw.values()), **at)  # noqa: E731
    _over(fwd, NORM_FWD, [(o, i) for o in ("out", "total") for i in strides], strides, make, None)
    _over(bwd, NORM_BWD, [(o, i) for o in ("dx", "dres", "dz") for i in strides], strides, make, dict(T=1))

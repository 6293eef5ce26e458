"""Entry points around the recurrence: what the host refuses (no GPU needed: no compute call is
made)."""
import ctypes

import pytest
import torch

from paper_2606_27748_gb300 import flexattn
from paper_2606_27748_gb300.flexattn import (FLEX_EINVAL, FLEX_EUNSUPPORTED, FLEX_EWORKSPACE,
                                             FlexSsm)

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
                                dict(n=65536), dict(T=(1 << 30) + 1), dict(D=65544)], ids=str)
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
    assert lib.flex_ssm_save_bytes(b) == (100 // 16 + 3) * 64 * 16 * 4


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

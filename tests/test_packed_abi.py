"""Packed-batch entry points: what the host refuses (no GPU needed: no compute call is made)."""
import ctypes

import pytest
import torch

from paper_2606_27748_gb300 import flexattn
from paper_2606_27748_gb300.flexattn import (FLEX_EINVAL, FLEX_EUNSUPPORTED, FLEX_EWORKSPACE,
                                             FlexPacked)


@pytest.fixture(scope="module")
def lib():
    from paper_2606_27748_gb300 import build
    build.build()
    return flexattn.load()


def _shape(**kw):
    x = dict(n=3, T=100, Tk=100, H=4, Hk=2, d=64, dtype=1, q_stride=256, k_stride=256, v_stride=256)
    x.update(kw)
    return FlexPacked(*(x[name] for name, _ in FlexPacked._fields_))


P = ctypes.c_void_p(1 << 20)  # never dereferenced: validation fails first
BIG = 1 << 40


def _fwd(lib, s, q=P, k=P, v=P, g=P, beta=P, cu=P, S0=None, S1=None, out=P, save=None, ws=P, n=BIG):
    return lib.flex_delta_fwd(ctypes.byref(s) if s else None, q, k, v, g, beta, cu, 1.0, S0, S1,
                              out, save, ws, n, None)


def _bwd(lib, s, save=P, dout=P, dq=P, dk=P, dv=P, dg=P, dbeta=P, ws=P, n=BIG):
    return lib.flex_delta_bwd(ctypes.byref(s), P, P, P, P, P, P, 1.0, dout, save, dq, dk, dv, dg,
                              dbeta, ws, n, None)


def _attn(lib, s, q=P, k=P, v=P, cu_q=P, cu_k=P, out=P, lse=P, ws=P, n=BIG):
    return lib.flex_softattn_fwd(ctypes.byref(s) if s else None, q, k, v, cu_q, cu_k, 1.0, 1, out,
                                 lse, ws, n, None)


BAD = [dict(n=0), dict(T=0, Tk=0), dict(Tk=0), dict(H=0), dict(Hk=0), dict(Hk=3), dict(dtype=2),
       dict(q_stride=120), dict(k_stride=0), dict(v_stride=100), dict(q_stride=260)]
UNSUPPORTED = [dict(d=32), dict(d=96), dict(n=65536), dict(H=2048, Hk=2048, q_stride=1 << 20,
                                                           k_stride=1 << 20, v_stride=1 << 20)]


@pytest.mark.parametrize("kw", BAD, ids=str)
def test_bad_shapes(lib, kw):
    s = _shape(**kw)
    assert _fwd(lib, s) == FLEX_EINVAL and _bwd(lib, s) == FLEX_EINVAL
    assert _attn(lib, s) == FLEX_EINVAL
    assert lib.flex_delta_workspace_bytes(ctypes.byref(s), 1) == 0
    assert lib.flex_delta_save_bytes(ctypes.byref(s)) == 0
    assert lib.flex_softattn_workspace_bytes(ctypes.byref(s)) == 0


@pytest.mark.parametrize("kw", UNSUPPORTED, ids=str)
def test_unsupported_shapes(lib, kw):
    s = _shape(**kw)
    assert _fwd(lib, s) == FLEX_EUNSUPPORTED and _bwd(lib, s) == FLEX_EUNSUPPORTED
    assert _attn(lib, s) == FLEX_EUNSUPPORTED
    assert lib.flex_softattn_workspace_bytes(ctypes.byref(s)) == 0


def test_row_counts_differ(lib):
    s = _shape(Tk=90)
    assert _fwd(lib, s) == FLEX_EINVAL  # the delta rule has one key per row
    assert lib.flex_softattn_workspace_bytes(ctypes.byref(s)) > 0
    wide = _shape(H=130, Hk=2, q_stride=130 * 64)
    assert _attn(lib, wide) == FLEX_EUNSUPPORTED  # more than 64 heads to a key head


@pytest.mark.parametrize("name", ["q", "k", "v", "g", "beta", "cu", "out", "ws"])
def test_delta_fwd_pointers(lib, name):
    assert _fwd(lib, _shape(), **{name: None}) == FLEX_EINVAL
    assert _fwd(lib, _shape(), **{name: ctypes.c_void_p((1 << 20) + 1)}) == FLEX_EINVAL


@pytest.mark.parametrize("name", ["save", "dout", "dq", "dk", "dv", "dg", "dbeta", "ws"])
def test_delta_bwd_pointers(lib, name):
    assert _bwd(lib, _shape(), **{name: None}) == FLEX_EINVAL
    assert _bwd(lib, _shape(), **{name: ctypes.c_void_p((1 << 20) + 1)}) == FLEX_EINVAL


@pytest.mark.parametrize("name", ["q", "k", "v", "cu_q", "cu_k", "out", "ws"])
def test_softattn_pointers(lib, name):
    assert _attn(lib, _shape(), **{name: None}) == FLEX_EINVAL
    assert _attn(lib, _shape(), **{name: ctypes.c_void_p((1 << 20) + 1)}) == FLEX_EINVAL


def test_states_save_and_workspaces(lib):
    s = _shape()
    off = ctypes.c_void_p((1 << 20) + 8)
    assert _fwd(lib, None) == FLEX_EINVAL and _attn(lib, None) == FLEX_EINVAL
    assert _fwd(lib, s, S0=off) == FLEX_EINVAL and _fwd(lib, s, S1=off) == FLEX_EINVAL
    assert _fwd(lib, s, save=off) == FLEX_EINVAL
    assert _fwd(lib, s, S0=P, save=P) == FLEX_EINVAL  # training starts from the zero state
    b = ctypes.byref(s)
    assert _fwd(lib, s, n=lib.flex_delta_workspace_bytes(b, 0) - 1) == FLEX_EWORKSPACE
    assert _bwd(lib, s, n=lib.flex_delta_workspace_bytes(b, 1) - 1) == FLEX_EWORKSPACE
    assert lib.flex_delta_workspace_bytes(b, 1) >= lib.flex_delta_workspace_bytes(b, 0) >= 256
    assert _attn(lib, s, n=lib.flex_softattn_workspace_bytes(b) - 1) == FLEX_EWORKSPACE
    assert _attn(lib, s, lse=ctypes.c_void_p((1 << 20) + 2)) == FLEX_EINVAL


def test_decode(lib):
    f = lib.flex_delta_decode
    one, more = _shape(T=3, Tk=3), _shape()
    assert f(ctypes.byref(more), P, P, P, P, P, 1.0, P, P, None) == FLEX_EINVAL  # T != n
    for i in range(7):
        args = [P] * 5 + [1.0] + [P] * 2
        args[i + (i >= 5)] = None
        assert f(ctypes.byref(one), *args, None) == FLEX_EINVAL


def test_binding_refuses_what_is_not_on_the_gpu_or_does_not_fit():
    q, v = torch.zeros(10, 2, 64), torch.zeros(10, 4, 64)
    g, cu = torch.zeros(10, 4), torch.tensor([0, 10], dtype=torch.int32)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        flexattn.delta_fwd(q, q, v, g, g, cu)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        flexattn.softattn_fwd(v, q, q, cu)
    cpu, f32 = q.get_device(), torch.float32
    rows = torch.zeros(10, 64, 4).transpose(1, 2)
    with pytest.raises(ValueError):  # heads not contiguous
        flexattn._rows(rows, "q", rows.shape, f32, cpu)
    with pytest.raises(ValueError):  # another shape, another type, another device
        flexattn._rows(q, "q", (10, 3, 64), f32, cpu)
    with pytest.raises(ValueError):
        flexattn._rows(q, "q", q.shape, torch.bfloat16, cpu)
    with pytest.raises(ValueError):
        flexattn._rows(q, "q", q.shape, f32, 0)
    wide = torch.zeros(10, 3 * 128)
    assert flexattn._rows(wide[:, 128:256].view(10, 2, 64), "q", (10, 2, 64), f32, cpu) == 384
    for bad in (torch.zeros(3, dtype=torch.int64), torch.zeros(1, dtype=torch.int32),
                torch.zeros(2, 2, dtype=torch.int32)):
        with pytest.raises(ValueError):
            flexattn._offsets(bad, "cu", cpu)
    with pytest.raises(ValueError):
        flexattn._plain(torch.zeros(3, 4), "g", (3, 5), f32, cpu)
    with pytest.raises(ValueError):
        flexattn._plain(torch.zeros(4, 3).t(), "g", (3, 4), f32, cpu)
    with pytest.raises(ValueError):
        flexattn._rank3(torch.zeros(3, 4), "q")
    with pytest.raises(TypeError):
        flexattn._dtype_code(torch.zeros(3, dtype=torch.float16))


def test_results_on_another_stream_come_from_its_own_memory(monkeypatch):
    """With `stream=`, a result's block comes from that stream's pool (another's block may still be
    at work there) and is marked as used on the caller's stream."""
    import contextlib
    inside, marked = [], []

    class Tensor:
        def __init__(self):
            self.of = inside[-1] if inside else "current"

        def record_stream(self, s):
            marked.append(s)

    @contextlib.contextmanager
    def stream(s):
        inside.append(s)
        yield
        inside.pop()

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream",
                        lambda device=None: inside[-1] if inside else "current")
    monkeypatch.setattr(torch, "empty", lambda *a, **k: Tensor())
    t = flexattn._new("side", (3,), torch.float32, "cuda")
    assert t.of == "side" and marked == ["current"]
    assert flexattn._new(None, (3,), torch.float32, "cuda").of == "current" and len(marked) == 1


def test_workspaces(lib, monkeypatch):
    """A forward that saves asks for the header alone; only the header is cleared."""
    s = _shape()
    assert _fwd(lib, s, save=P, n=255) == FLEX_EWORKSPACE
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: empty(*a, **k).fill_(7))
    ws = flexattn._workspace(1000, "", "cpu")
    assert (ws[:256] == 0).all() and (ws[256:] == 7).all()
    with pytest.raises(flexattn.FlexError):
        flexattn._workspace(0, "", "cpu")

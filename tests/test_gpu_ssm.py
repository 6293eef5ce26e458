"""Selective state space scan over packed sequences (flex_ssm_fwd / _bwd / _decode) against its
definition in 64 bits, token by token."""
import pytest
import torch

from paper_2606_27748_gb300 import flexattn
from layer_ref import (BF16, F32, SSM, close, close_each, gradients, ssm_inputs, ssm_ref)
from packed_ref import offsets

pytestmark = pytest.mark.gpu

LENS = [(1,), (2, 0, 3), (15, 16, 17), (0, 130, 1, 0), (200, 17, 128, 5)]
# channels, states, groups: whole blocks of 64 (or 32) channels, ragged ones, several to a group
SHAPES = [(64, 16, 1), (8, 8, 1), (200, 16, 2), (72, 32, 1), (136, 8, 2)]
GRADS = ("dx", "ddt", "dA", "dB", "dC", "dD", "dz", "ddt_bias")


@pytest.fixture(scope="module", autouse=True)
def library():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    from paper_2606_27748_gb300 import build
    build.build()
    flexattn.load()


def _opt(x):
    return {n: x[n] for n in ("D", "z", "dt_bias")}


def _five(x):
    return [x[n] for n in ("x", "dt", "A", "B", "C")]


def _fwd(x, cu, **kw):
    return flexattn.ssm_fwd(*_five(x), cu, **_opt(x), **kw)


def _train(x, cu, **kw):
    save = flexattn.ssm_save(x["x"], x["B"], cu)
    save.fill_(255)
    out, _ = _fwd(x, cu, save=save, want_state=False, **kw)
    return out, flexattn.ssm_bwd(*_five(x), cu, x["dout"], save, **_opt(x), **kw)


def _check_grads(got, x, lens, **kw):
    n = sum(lens)
    sent = x["dout"].clone()
    sent[n:] = 0
    ref = gradients(lambda v: ssm_ref(v, lens, **kw)[:1], x, SSM, [sent])
    for name, g, r in zip(GRADS, got, ref):
        if r is None:
            assert g is None, name
        elif name in ("dA", "dD", "ddt_bias"):
            close(g, r, name)
        else:
            close_each(g, r, lens, name)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_forward(lens, shape, dtype):
    D, N, G = shape
    x = ssm_inputs(lens, D, N, G, dtype, pad=8)
    out, last = _fwd(x, offsets(lens))
    ref, rlast = ssm_ref(x, lens)
    close_each(out, ref, lens, "out")
    close(last, rlast, "last state")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_gradients(lens, shape, dtype):
    D, N, G = shape
    x = ssm_inputs(lens, D, N, G, dtype, seed=1, pad=8)
    out, got = _train(x, offsets(lens))
    close_each(out, ssm_ref(x, lens)[0], lens, "out")
    _check_grads(got, x, lens)


@pytest.mark.parametrize("gate,skip,bias,softplus", [(False, True, True, True), (True, False, True, True),
                                                     (True, True, False, True), (False, False, False, False)])
def test_what_may_be_left_out(gate, skip, bias, softplus):
    lens = (40, 7)
    x = ssm_inputs(lens, 72, 16, 1, F32, seed=2, gate=gate, skip=skip, bias=bias)
    if not softplus:
        x["dt"] = x["dt"].abs() * 0.1
    cu = offsets(lens)
    out, last = _fwd(x, cu, softplus=softplus)
    ref, rlast = ssm_ref(x, lens, softplus=softplus)
    close_each(out, ref, lens, "out")
    close(last, rlast, "last state")
    _, got = _train(x, cu, softplus=softplus)
    _check_grads(got, x, lens, softplus=softplus)


@pytest.mark.parametrize("lens", [(700,), (1, 900, 0, 333)], ids=str)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_long_sequences_in_blocks(lens, dtype):
    """Few channels: sequences are cut into blocks of 64 tokens whose ends are joined."""
    x = ssm_inputs(lens, 64, 16, 1, dtype, seed=3)
    cu = offsets(lens)
    state = torch.randn(len(lens), 64, 16, device="cuda")
    out, last = _fwd(x, cu, state=state)
    ref, rlast = ssm_ref(x, lens, state=state)
    close_each(out, ref, lens, "out")
    close(last, rlast, "last state")
    _, got = _train(x, cu)
    _check_grads(got, x, lens)
    # in place
    both = state.clone()
    out2, same = _fwd(x, cu, state=both, last_state=both)
    assert same is both and torch.equal(both, last) and torch.equal(out2, out)


def test_a_prompt_in_pieces_and_its_tokens():
    """A prompt's two pieces, then single tokens, give what the whole prompt gives."""
    lens = (90, 41)
    x = ssm_inputs(lens, 136, 16, 2, F32, seed=4)
    ref, rlast = ssm_ref(x, lens)
    pick = lambda a, b: torch.cat([torch.arange(a, b), torch.arange(90 + min(a, 41), 90 + min(b, 41))])  # noqa: E731
    rows, state = [], None
    for a, b in ((0, 30), (30, 36)):
        at = pick(a, b).cuda()
        y = {n: (t[at] if n in ("x", "dt", "B", "C", "z", "dout") else t) for n, t in x.items()}
        out, state = _fwd(y, offsets((b - a, b - a)), state=state)
        close(out, ref[at], f"rows {a} to {b}")
    for t in range(36, 41):
        at = torch.tensor([t, 90 + t]).cuda()
        y = {n: (v[at] if n in ("x", "dt", "B", "C", "z", "dout") else v) for n, v in x.items()}
        out = flexattn.ssm_decode(*_five(y), state, **_opt(y))
        close(out, ref[at], f"token {t}")
    close(state[1], rlast[1], "last state")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,D,N,G", [(1, 8, 8, 1), (3, 200, 16, 2), (9, 72, 32, 1), (70, 64, 16, 1)])
def test_token(n, D, N, G, dtype):
    x = ssm_inputs((1,) * n, D, N, G, dtype, seed=5, pad=8)
    S = torch.randn(n, D, N, device="cuda")
    ref, rlast = ssm_ref(x, (1,) * n, state=S)
    out = flexattn.ssm_decode(*_five(x), S, **_opt(x))
    close(out, ref, "out")
    close(S, rlast, "state")


def test_rows_behind_the_last_sequence_are_left():
    lens = (50, 9)
    x = ssm_inputs(lens, 72, 16, 1, BF16, seed=6, rows_behind=21)
    for n in ("x", "dt", "B", "C", "z", "dout"):
        x[n][59:] = float("nan")
    cu = offsets(lens)
    keep = {n: torch.full_like(x[m], 7.0) for n, m in (("out", "x"), ("dx", "x"), ("ddt", "x"),
                                                       ("dz", "x"), ("dB", "B"), ("dC", "C"))}
    out, last = _fwd(x, cu, out=keep.pop("out"))
    assert (out[59:] == 7).all()
    save = flexattn.ssm_save(x["x"], x["B"], cu)
    _fwd(x, cu, save=save, want_state=False)
    got = flexattn.ssm_bwd(*_five(x), cu, x["dout"], save, **_opt(x), **keep)
    for t in keep.values():
        assert (t[59:] == 7).all()
    y = {n: (t[:59] if n in ("x", "dt", "B", "C", "z", "dout") else t) for n, t in x.items()}
    close_each(out[:59], ssm_ref(y, lens)[0], lens, "out")
    close(last, ssm_ref(y, lens)[1], "last state")
    _check_grads([g[:59] if g.shape[0] == 80 else g for g in got], y, lens)


def test_nan_stays_in_its_sequence():
    lens = (20, 30, 10)
    x = ssm_inputs(lens, 64, 16, 1, BF16, seed=7)
    cu = offsets(lens)
    clean, last = _fwd(x, cu)
    for n in ("x", "dt", "B", "z"):
        y = dict(x)
        y[n] = x[n].clone()
        y[n][25] = float("nan")
        out, l2 = _fwd(y, cu)
        assert torch.equal(out[:25], clean[:25]) and torch.equal(out[50:], clean[50:])
        assert torch.isnan(out[25]).all()
        assert torch.equal(l2[0], last[0]) and torch.equal(l2[2], last[2])
        assert torch.isnan(out[26:50]).all() == (n != "z")


def test_results_repeat_and_replay():
    """The same bits again, on another stream, and from a captured graph whose inputs have changed."""
    lens = (300, 64, 1)
    cu = offsets(lens)
    x, y = (ssm_inputs(lens, 136, 16, 1, BF16, seed=s) for s in (8, 9))
    first = _train(x, cu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = _train(x, cu, stream=None)
    save = flexattn.ssm_save(x["x"], x["B"], cu)
    side.wait_stream(torch.cuda.current_stream())
    out, _ = _fwd(x, cu, save=save, want_state=False, stream=side)
    there = (out, flexattn.ssm_bwd(*_five(x), cu, x["dout"], save, **_opt(x), stream=side))
    torch.cuda.synchronize()
    for o in (again, there):
        assert torch.equal(o[0], first[0])
        assert all(torch.equal(a, b) for a, b in zip(o[1], first[1]))
    held = {n: t.clone() for n, t in x.items()}
    ws = flexattn.ssm_workspace(x["x"], x["B"], cu, backward=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _train(held, cu, ws=ws)
    for v in (y, x):
        for n in held:
            held[n].copy_(v[n])
        graph.replay()
        torch.cuda.synchronize()
        want = _train(v, cu)
        assert torch.equal(got[0], want[0])
        assert all(torch.equal(a, b) for a, b in zip(got[1], want[1]))


def test_gradients_against_differences():
    """Along random directions: central differences of the definition's loss."""
    lens = (33, 5)
    x = ssm_inputs(lens, 16, 8, 2, F32, seed=10)
    _, got = _train(x, offsets(lens))
    loss = lambda v: float((ssm_ref(v, lens)[0] * x["dout"].double()).sum())  # noqa: E731
    gen = torch.Generator().manual_seed(0)
    for name, g in zip(SSM, got):
        way = torch.randn(x[name].shape, generator=gen, dtype=torch.float64).cuda()
        step = 1e-5
        up, down = ({**x, name: x[name].double() + s * way} for s in (step, -step))
        slope = (loss(up) - loss(down)) / (2 * step)
        # a gradient off by 2e-5 of its norm moves its part along a unit direction by that at most
        assert abs(float((g.double() * way).sum()) - slope) <= 2e-5 * float(g.double().norm() * way.norm()), name


def test_extreme_steps():
    """Steps so long that nothing is left of the state, and so short that nothing changes."""
    lens = (40,)
    x = ssm_inputs(lens, 64, 16, 1, F32, seed=11)
    x["dt"][5] = 60.0
    x["dt"][6] = 500.0
    x["dt"][20:24] = -60.0
    x["dt"][30] = -200.0
    cu = offsets(lens)
    out, last = _fwd(x, cu)
    ref, rlast = ssm_ref(x, lens)
    close(out, ref, "out")
    close(last, rlast, "last state")
    _, got = _train(x, cu)
    _check_grads(got, x, lens)


def test_sequences_without_rows():
    """No rows at all: the states stay, the parameters' gradients are 0, rows are left alone."""
    lens, cu = (0, 0), offsets((0, 0))
    x = ssm_inputs((5,), 64, 16, 1, F32, seed=12)
    state = torch.randn(2, 64, 16, device="cuda")
    out = torch.full_like(x["x"], 7.0)
    _, last = _fwd(x, cu, state=state, out=out)
    assert (out == 7).all() and torch.equal(last, state)
    _, last = _fwd(x, cu, out=out)
    assert (last == 0).all() and (out == 7).all()
    save = flexattn.ssm_save(x["x"], x["B"], cu)
    got = flexattn.ssm_bwd(*_five(x), cu, x["dout"], save, **_opt(x), dx=out)
    assert (out == 7).all()
    for g in (got[2], got[5], got[7]):
        assert (g == 0).all()
    assert lens == (0, 0)


def test_many_sequences_of_a_token_and_one_long():
    """Sequences that share no block, between them one of many blocks."""
    lens = (1,) * 130 + (500,) + (2,) * 70
    x = ssm_inputs(lens, 72, 16, 1, BF16, seed=13, pad=8)
    cu = offsets(lens)
    state = torch.randn(len(lens), 72, 16, device="cuda")
    out, last = _fwd(x, cu, state=state)
    ref, rlast = ssm_ref(x, lens, state=state)
    close(out, ref, "out")
    close(last, rlast, "last states")
    _, got = _train(x, cu)
    sent = x["dout"]
    ref = gradients(lambda v: ssm_ref(v, lens)[:1], x, SSM, [sent])
    for name, g, r in zip(GRADS, got, ref):
        close(g, r, name)


def test_calls_with_their_own_workspaces_side_by_side():
    """Two calls on two streams, each with a workspace and save buffer of its own."""
    lens = (700, 90)
    cu = offsets(lens)
    x, y = (ssm_inputs(lens, 64, 16, 1, BF16, seed=s) for s in (14, 15))
    want = [_train(v, cu) for v in (x, y)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for v, s in zip((x, y), streams):
            with torch.cuda.stream(s):
                got.append(_train(v, cu))
        torch.cuda.synchronize()
        for w, g in zip(want, got):
            assert torch.equal(w[0], g[0]) and all(torch.equal(a, b) for a, b in zip(w[1], g[1]))


def test_outputs_over_their_inputs():
    """out may be x or z, and dx the incoming gradient: every value is read before it is replaced."""
    lens = (300, 40)
    cu = offsets(lens)
    x = ssm_inputs(lens, 64, 16, 1, BF16, seed=16)
    want, last = _fwd(x, cu)
    for n in ("x", "z"):
        y = {m: t.clone() for m, t in x.items()}
        out, l2 = _fwd(y, cu, out=y[n])
        assert out is y[n] and torch.equal(out, want) and torch.equal(l2, last)
    _, grads = _train(x, cu)
    save = flexattn.ssm_save(x["x"], x["B"], cu)
    _fwd(x, cu, save=save, want_state=False)
    up = x["dout"].clone()
    got = flexattn.ssm_bwd(*_five(x), cu, up, save, **_opt(x), dx=up)
    assert all(torch.equal(a, b) for a, b in zip(got, grads))


def test_steps_of_zero_change_nothing():
    """Tokens of step 0 leave the state bit for bit, however many and wherever a tile ends; so does a
    single one."""
    lens = (37, 16, 1)
    x = ssm_inputs(lens, 72, 16, 1, F32, seed=17)
    x["dt"].fill_(float("-inf"))
    state = torch.randn(3, 72, 16, device="cuda")
    _, last = _fwd(x, offsets(lens), state=state)
    assert torch.equal(last, state)
    tok = {n: (t[:3].clone() if n in ("x", "dt", "B", "C", "z") else t) for n, t in x.items()}
    S = state.clone()
    flexattn.ssm_decode(*_five(tok), S, **_opt(tok))
    assert torch.equal(S, state)


@pytest.mark.parametrize("cu", [(3, 10, 4, 40), (-5, 7, 900, 40), (0, 50, 20, 33)], ids=str)
def test_offsets_that_are_none(cu):
    """Whatever the offsets hold, nothing outside the tensors is touched: the rows around stay."""
    x = ssm_inputs((40,), 64, 16, 1, F32, seed=18)
    cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
    wide = {n: torch.full((40 + 64, *s), 7.0, device="cuda") for n, s in (
        ("out", (64,)), ("dx", (64,)), ("ddt", (64,)), ("dz", (64,)), ("dB", (1, 16)), ("dC", (1, 16)))}
    mid = {n: t[32:72] for n, t in wide.items()}
    state = torch.zeros(3, 64, 16, device="cuda")
    save = flexattn.ssm_save(x["x"], x["B"], cu)
    save.zero_()
    _fwd(x, cu, out=mid["out"], state=state)
    _fwd(x, cu, out=mid["out"], want_state=False, save=save)
    mid.pop("out")
    flexattn.ssm_bwd(*_five(x), cu, x["dout"], save, **_opt(x), **mid)
    for n, t in wide.items():
        assert (t[:32] == 7).all() and (t[72:] == 7).all(), n


# Tokens x blocks of 64 channels large enough for blocks of more than 32 tokens backward (64, 64, 64, 96) and
# forward of 128 (the last; the others stay whole), with sequences of one and of many blocks.
LARGE = [(2048, 16, 2, (900, 1, 0, 333, 64, 202)), (2048, 8, 1, (1211, 1, 1, 1, 287)),
         (2048, 32, 4, (65, 700, 3, 128, 604)), (4096, 16, 1, (1203, 97))]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D,N,G,lens", LARGE, ids=str)
def test_blocks_of_more_tokens(D, N, G, lens, dtype):
    x = ssm_inputs(lens, D, N, G, dtype, seed=19, pad=8)
    out, got = _train(x, offsets(lens))
    _, last = _fwd(x, offsets(lens))
    ref, rlast = ssm_ref(x, lens)
    close_each(out, ref, lens, "out")
    close(last, rlast, "last states")
    _check_grads(got, x, lens)


def test_nan_of_c_stays_in_its_row():
    lens = (20, 30, 10)
    x = ssm_inputs(lens, 64, 16, 1, BF16, seed=7)
    cu = offsets(lens)
    clean, last = _fwd(x, cu)
    x["C"][25] = float("nan")
    out, l2 = _fwd(x, cu)
    assert torch.isnan(out[25]).all() and torch.equal(l2, last)
    assert torch.equal(out[:25], clean[:25]) and torch.equal(out[26:], clean[26:])

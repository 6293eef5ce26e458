"""Short causal convolution over packed sequences (flex_conv_fwd / _bwd / _decode) against its
definition in 64 bits."""
import pytest
import torch

from paper_2606_27748_gb300 import flexattn
from layer_ref import BF16, F32, CONV, close, close_each, conv_inputs, conv_ref, gradients, silu
from packed_ref import offsets

pytestmark = pytest.mark.gpu

LENS = [(1,), (2, 0, 3), (0, 31, 1, 33, 0, 0), (5, 4, 3, 2, 1, 1, 1), (300, 17, 128)]


@pytest.fixture(scope="module", autouse=True)
def library():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    from paper_2606_27748_gb300 import build
    build.build()
    flexattn.load()


def _grads(x, lens, got, act=True):
    n = sum(lens)
    ref = gradients(lambda v: conv_ref(v, lens, act=act)[:1], x, CONV, [x["dout"][:n]])
    close_each(got[0], ref[0], lens, "dx")
    close(got[1], ref[1], "dw")
    if ref[2] is None:
        assert got[2] is None
    else:
        close(got[2], ref[2], "dbias")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D,W", [(8, 4), (64, 2), (200, 3), (1032, 4)])
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_convolution(lens, D, W, dtype):
    x = conv_inputs(lens, D, W, dtype, pad=8)
    cu = offsets(lens)
    out, last = flexattn.conv_fwd(x["x"], x["w"], cu, bias=x["bias"], want_state=True)
    ref, rlast = conv_ref(x, lens)
    close_each(out, ref, lens, "out")
    assert torch.equal(last.double(), rlast)
    _grads(x, lens, flexattn.conv_bwd(x["x"], x["w"], cu, x["dout"], bias=x["bias"]))


@pytest.mark.parametrize("act,bias", [(False, True), (True, False), (False, False)])
def test_what_may_be_left_out(act, bias):
    lens = (40, 7)
    x = conv_inputs(lens, 72, 4, F32, seed=1, bias=bias)
    cu = offsets(lens)
    out, last = flexattn.conv_fwd(x["x"], x["w"], cu, bias=x["bias"], silu=act)
    assert last is None
    close_each(out, conv_ref(x, lens, act=act)[0], lens, "out")
    _grads(x, lens, flexattn.conv_bwd(x["x"], x["w"], cu, x["dout"], bias=x["bias"], silu=act), act)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("W", [2, 3, 4])
def test_pieces_and_tokens(W, dtype):
    """A state carries a sequence over: pieces of 0, 1, 2 and more rows, then single tokens."""
    D, lens = 136, (12, 9)
    x = conv_inputs(lens, D, W, dtype, seed=2)
    ref, rlast = conv_ref(x, lens)
    state = torch.zeros(2, W - 1, D, dtype=dtype, device="cuda")
    at = [0, 0]
    for piece in ((5, 0), (0, 1), (2, 2), (1, 3)):
        rows = torch.cat([torch.arange(b + a, b + a + n) for b, a, n in zip((0, 12), at, piece)]).cuda()
        out, state = flexattn.conv_fwd(x["x"][rows], x["w"], offsets(piece), bias=x["bias"], state=state,
                                       want_state=True)
        close(out, ref[rows], f"piece {piece}")
        at = [a + n for a, n in zip(at, piece)]
    assert at == [8, 6]
    for k in range(3):
        rows = torch.tensor([8 + k, 12 + 6 + k]).cuda()
        out = flexattn.conv_decode(x["x"][rows], x["w"], state, bias=x["bias"])
        close(out, ref[rows], f"token {k}")
    assert torch.equal(state[1].double(), rlast[1])


def test_heads_many_sequences_and_rows_behind():
    lens = tuple(1 + i % 3 for i in range(500))
    x = conv_inputs(lens, 64, 4, BF16, seed=3, rows_behind=30)
    n = sum(lens)
    for k in ("x", "dout"):
        x[k][n:] = float("nan")
    cu = offsets(lens)
    rows, up = x["x"].view(-1, 4, 16), x["dout"].view(-1, 4, 16)
    out, dx = torch.full_like(rows, 7.0), torch.full_like(rows, 7.0)
    flexattn.conv_fwd(rows, x["w"], cu, bias=x["bias"], out=out)
    got = flexattn.conv_bwd(rows, x["w"], cu, up, bias=x["bias"], dx=dx)
    assert (out[n:] == 7).all() and (dx[n:] == 7).all()
    y = {**x, "x": x["x"][:n], "dout": x["dout"][:n]}
    close(out[:n].flatten(1), conv_ref(y, lens)[0], "out")
    _grads(y, lens, (got[0][:n].flatten(1), *got[1:]))


def test_state_and_its_successor_are_two_buffers():
    lens = (4, 4)
    x = conv_inputs(lens, 64, 4, BF16)
    state = torch.zeros(2, 3, 64, dtype=BF16, device="cuda")
    with pytest.raises(flexattn.FlexError):
        flexattn.conv_fwd(x["x"], x["w"], offsets(lens), state=state, last_state=state)


def test_nan_stays_in_its_sequence_and_window():
    lens = (20, 30, 10)
    x = conv_inputs(lens, 64, 4, BF16, seed=4)
    cu = offsets(lens)
    clean, _ = flexattn.conv_fwd(x["x"], x["w"], cu, bias=x["bias"])
    x["x"][48] = float("nan")
    out, _ = flexattn.conv_fwd(x["x"], x["w"], cu, bias=x["bias"])
    assert torch.equal(out[:48], clean[:48]) and torch.isnan(out[48:50]).all()
    assert torch.equal(out[50:], clean[50:])


def test_results_repeat_and_replay():
    lens = (300, 64, 1)
    cu = offsets(lens)
    x, y = (conv_inputs(lens, 136, 4, BF16, seed=s) for s in (8, 9))

    def both(v, ws=None, stream=None):
        out, _ = flexattn.conv_fwd(v["x"], v["w"], cu, bias=v["bias"], stream=stream)
        return out, *flexattn.conv_bwd(v["x"], v["w"], cu, v["dout"], bias=v["bias"], ws=ws, stream=stream)

    first = both(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    there = both(x, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, there))
    held = {n: t.clone() for n, t in x.items()}
    ws = flexattn.conv_workspace(x["x"], x["w"], cu)
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
    lens = (9, 1, 4)
    x = conv_inputs(lens, 16, 4, F32, seed=10)
    got = flexattn.conv_bwd(x["x"], x["w"], offsets(lens), x["dout"], bias=x["bias"])
    loss = lambda v: float((conv_ref(v, lens)[0] * x["dout"].double()).sum())  # noqa: E731
    gen = torch.Generator().manual_seed(0)
    for name, g in zip(CONV, got):
        way = torch.randn(x[name].shape, generator=gen, dtype=torch.float64).cuda()
        up, down = ({**x, name: x[name].double() + s * way} for s in (1e-5, -1e-5))
        slope = (loss(up) - loss(down)) / 2e-5
        assert abs(float((g.double() * way).sum()) - slope) <= 2e-5 * float(g.double().norm() * way.norm()), name


def test_out_is_another_buffer():
    lens = (9,)
    x = conv_inputs(lens, 64, 4, BF16)
    cu = offsets(lens)
    with pytest.raises(flexattn.FlexError):
        flexattn.conv_fwd(x["x"], x["w"], cu, out=x["x"])
    with pytest.raises(flexattn.FlexError):
        flexattn.conv_bwd(x["x"], x["w"], cu, x["dout"], dx=x["dout"])


def test_sequences_without_rows():
    cu = offsets((0, 0, 0))
    x = conv_inputs((5,), 64, 4, F32)
    state, out = torch.randn(3, 3, 64, device="cuda"), torch.full_like(x["x"], 7.0)
    _, last = flexattn.conv_fwd(x["x"], x["w"], cu, bias=x["bias"], state=state, out=out, want_state=True)
    assert torch.equal(last, state) and (out == 7).all()
    _, last = flexattn.conv_fwd(x["x"], x["w"], cu, out=out, want_state=True)
    assert (last == 0).all()
    got = flexattn.conv_bwd(x["x"], x["w"], cu, x["dout"], bias=x["bias"], dx=out)
    assert (out == 7).all() and (got[1] == 0).all() and (got[2] == 0).all()


@pytest.mark.parametrize("cu", [(3, 10, 4, 40), (-5, 7, 900, 40), (0, 50, 20, 33)], ids=str)
def test_offsets_that_are_none(cu):
    """Whatever the offsets hold, nothing outside the tensors is touched: the rows around stay."""
    x = conv_inputs((40,), 64, 4, F32, seed=11)
    cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
    out, dx = (torch.full((104, 64), 7.0, device="cuda") for _ in range(2))
    state = torch.zeros(3, 3, 64, device="cuda")
    flexattn.conv_fwd(x["x"], x["w"], cu, bias=x["bias"], state=state, out=out[32:72], want_state=True)
    flexattn.conv_bwd(x["x"], x["w"], cu, x["dout"], bias=x["bias"], dx=dx[32:72])
    for t in (out, dx):
        assert (t[:32] == 7).all() and (t[72:] == 7).all()


def _packed_ref(x, lens):
    """conv_ref's out without a loop over rows: tap W - 1 - k of all rows at once, masked where the row
    k ahead lies in the sequence ahead."""
    v, w = x["x"].double(), x["w"].double()
    at = torch.cat([torch.arange(n) for n in lens]).to(v.device)[:, None]
    W = w.shape[1]
    p = sum(torch.where(at >= k, torch.roll(v, k, 0), 0.0) * w[:, W - 1 - k] for k in range(W))
    return silu(p + x["bias"].double())


# Rows of a thread's run, by rows x channels: 8, 16 and 32 (4 above).  Sequences end inside runs and
# batches of rows, at their first and last rows among others.
RUNS = [(8, 2048, (1203, 1, 2, 0, 3, 777, 515)), (8, 1032, (2403, 8, 1, 1, 2, 0, 1500, 1093)),
        (16, 2048, (2403, 1, 1, 2, 0, 1500, 16, 1093)), (32, 2048, (4097, 5, 0, 1, 2903, 31, 670, 97, 1, 1, 2192))]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("run,D,lens", RUNS, ids=str)
def test_long_runs(run, D, lens, W, dtype):
    """All outputs of batches large enough for runs of 8 rows and more, where most rows are taken without
    looking at the offsets.  Sums over 10000 rows are off by sqrt(10000) 2^-24 = 6e-6 of a typical sum if
    they were one chain, a third of the bound."""
    x = conv_inputs(lens, D, W, dtype, seed=12, pad=8)
    cu = offsets(lens)
    ws = flexattn.conv_workspace(x["x"], x["w"], cu)
    assert (ws.numel() - 256) // (4 * (W + 1) * D) == -(-sum(lens) // (8 * run))
    out, last = flexattn.conv_fwd(x["x"], x["w"], cu, bias=x["bias"], want_state=True)
    close_each(out, _packed_ref(x, lens), lens, "out")
    for i, end in enumerate(cu[1:].tolist()):
        n = min(lens[i], W - 1)
        assert torch.equal(last[i, W - 1 - n:], x["x"][end - n:end]) and (last[i, :W - 1 - n] == 0).all()
    got = flexattn.conv_bwd(x["x"], x["w"], cu, x["dout"], bias=x["bias"], ws=ws)
    ref = gradients(lambda v: [_packed_ref(v, lens)], x, CONV, [x["dout"]])
    close_each(got[0], ref[0], lens, "dx")
    close(got[1], ref[1], "dw")
    close(got[2], ref[2], "dbias")

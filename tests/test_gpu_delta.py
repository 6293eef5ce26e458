"""Gated delta rule over packed sequences (flex_delta_fwd / _bwd / _decode) against its
definition in 64 bits, token by token."""
import pytest
import torch

from paper_2606_27748_gb300 import flexattn
from packed_ref import check, delta_grads, delta_inputs, delta_ref, offsets, rel, tol

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
NAMES = ("q", "k", "v", "g", "beta")
LENS = [(1,), (2, 0, 3), (63, 64, 65), (0, 130, 1, 0), (200, 17, 128, 5)]
HEADS = [(1, 1), (4, 2), (3, 1)]


@pytest.fixture(scope="module", autouse=True)
def library():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    from paper_2606_27748_gb300 import build
    build.build()
    flexattn.load()


def _fwd(x, cu, **kw):
    return flexattn.delta_fwd(*(x[n] for n in NAMES), cu, **kw)


def _bwd(x, cu, **kw):
    save = flexattn.delta_save(x["q"], x["v"], cu)
    _fwd(x, cu, save=save, want_state=False, **kw)
    return flexattn.delta_bwd(*(x[n] for n in NAMES), cu, x["dout"], save, **kw)


@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("H,Hk", HEADS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_forward(lens, H, Hk, d, dtype):
    x = delta_inputs(lens, H, Hk, d, dtype)
    out, last = _fwd(x, offsets(lens))
    ro, rs = delta_ref(x, lens, d ** -0.5)
    check(out, ro, "out")
    check(last, rs, "last state", F32)


@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("H,Hk", HEADS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_backward(lens, H, Hk, d, dtype):
    x = delta_inputs(lens, H, Hk, d, dtype, seed=1)
    got = _bwd(x, offsets(lens))
    for name, y, r in zip(NAMES, got, delta_grads(x, lens, d ** -0.5)):
        if sum(lens) == 1 and name == "g":  # the only row decays a zero state: exactly 0, which
            assert float(y.abs().max()) <= 1e-5  # two equal sums leave to fp32 rounding
            continue
        check(y, r, "d" + name)


def test_backward_against_differences():
    """Central differences of the kernel's own fp32 forward along a direction of each input, a
    step of h = 2% of the input's norm: the cubic term is h^2 / 6 = 7e-5 of the slope times a
    curvature of order 10, the outputs' rounding 1e-6 / h = 5e-5: 5e-3 allows both."""
    lens, H, Hk, d = (70, 33), 2, 1, 64
    cu = offsets(lens)
    x = delta_inputs(lens, H, Hk, d, F32, seed=2)
    got = _bwd(x, cu)
    gen = torch.Generator(device="cuda").manual_seed(3)
    for name, y in zip(NAMES, got):
        step = torch.randn(x[name].shape, device="cuda", generator=gen)
        step = step * (step * y > 0)  # a direction along which the slope does not cancel
        slope = float((step.double() * y.double()).sum())
        h = 2e-2 * float(x[name].norm() / step.norm())
        L = [float((_fwd({**x, name: x[name] + s * h * step}, cu)[0].double()
                    * x["dout"].double()).sum()) for s in (1, -1)]
        assert abs((L[0] - L[1]) / (2 * h) - slope) <= 5e-3 * abs(slope), name


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_first_state_and_in_place(d, dtype):
    lens, H, Hk = (0, 70, 1, 129), 4, 2
    x, cu = delta_inputs(lens, H, Hk, d, dtype, seed=4), offsets(lens)
    S0 = torch.randn(len(lens), H, d, d, device="cuda") / d ** 0.5
    ro, rs = delta_ref(x, lens, 0.3, S0)
    out, last = _fwd(x, cu, scale=0.3, state=S0)
    check(out, ro, "out")
    check(last, rs, "last state", F32)
    assert torch.equal(last[0], S0[0])  # an empty sequence keeps its state
    S = S0.clone()
    out2, last2 = _fwd(x, cu, scale=0.3, state=S, last_state=S)
    assert last2 is S and torch.equal(S, last) and torch.equal(out2, out)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_pieces_and_single_tokens_continue_a_prompt(d, dtype):
    """A prompt in two pieces, then token by token, gives what one call gives."""
    H, Hk, n, lens = 4, 2, 3, (150, 150, 150)
    x = delta_inputs(lens, H, Hk, d, dtype, seed=5)
    ro, rs = delta_ref(x, lens, d ** -0.5)
    by_seq = {m: t.view(n, 150, *t.shape[1:]) for m, t in x.items()}
    piece = lambda a, b: {m: t[:, a:b].reshape(-1, *t.shape[2:]).contiguous() for m, t in by_seq.items()}  # noqa: E731
    o1, S = _fwd(piece(0, 67), offsets((67,) * n))
    o2, S = _fwd(piece(67, 140), offsets((73,) * n), state=S)
    o3 = []
    for t in range(140, 150):
        tok = piece(t, t + 1)
        o3.append(flexattn.delta_decode(*(tok[m] for m in NAMES), S))
    got = torch.cat([o1.view(n, 67, H, d), o2.view(n, 73, H, d), torch.stack(o3, 1)], 1)
    check(got.reshape(-1, H, d), ro, "out")
    check(S, rs, "state", F32)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,H,Hk,d", [(1, 1, 1, 64), (5, 4, 2, 128), (33, 6, 3, 64)])
def test_decode(n, H, Hk, d, dtype):
    lens = (1,) * n
    x = delta_inputs(lens, H, Hk, d, dtype, seed=6)
    S0 = torch.randn(n, H, d, d, device="cuda") / d ** 0.5
    ro, rs = delta_ref(x, lens, 0.7, S0)
    S = S0.clone()
    out = flexattn.delta_decode(*(x[m] for m in NAMES), S, scale=0.7)
    check(out, ro, "out")
    check(S, rs, "state", F32)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_slices_of_one_projection_and_rows_behind(dtype):
    """q, k, v as slices of one wide tensor; rows behind the last sequence hold NaN, are not read
    into a result and keep what the outputs held."""
    lens, H, Hk, d = (40, 90), 4, 2, 64
    T = sum(lens) + 9
    x, cu = delta_inputs(lens, H, Hk, d, dtype, seed=7, rows_behind=9), offsets(lens)
    for t in x.values():
        t[sum(lens):] = float("nan")
    wide = torch.cat([x[m].reshape(T, -1) for m in ("q", "k", "v")], 1)
    a = Hk * d
    y = dict(x, q=wide[:, :a].view(T, Hk, d), k=wide[:, a:2 * a].view(T, Hk, d),
             v=wide[:, 2 * a:].view(T, H, d))
    fill = lambda s: torch.full(s, 7.0, dtype=dtype, device="cuda")  # noqa: E731
    out = fill((T, H, d))
    save = flexattn.delta_save(y["q"], y["v"], cu)
    _, last = _fwd(y, cu, out=out, save=save)
    grads = {"d" + m: fill(x[m].shape) for m in NAMES}
    flexattn.delta_bwd(*(y[m] for m in NAMES), cu, x["dout"], save, **grads)
    inner = {m: t[:sum(lens)].contiguous() for m, t in x.items()}
    ro, rs = delta_ref(inner, lens, d ** -0.5)
    check(out[:sum(lens)], ro, "out")
    check(last, rs, "last state", F32)
    for m, r in zip(NAMES, delta_grads(inner, lens, d ** -0.5)):
        check(grads["d" + m][:sum(lens)], r, "d" + m)
    for t in (out, *grads.values()):
        assert (t[sum(lens):] == 7.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("case", ["reset", "no_decay", "beta_0", "beta_1_same_keys", "fast_decay"])
def test_gates_at_their_ends(case, dtype):
    """-inf forgets everything, 0 keeps everything, beta 0 writes nothing; equal keys with beta 1
    overwrite each other; gates that underflow within a few tokens."""
    lens, H, Hk, d = (140, 65), 2, 1, 64
    x, cu = delta_inputs(lens, H, Hk, d, dtype, seed=8), offsets(lens)
    if case == "reset":
        x["g"][::29] = float("-inf")
    elif case == "no_decay":
        x["g"].zero_()
    elif case == "beta_0":
        x["beta"][::2] = 0
    elif case == "beta_1_same_keys":
        x["beta"].fill_(1)
        x["k"][:] = x["k"][:1]
    else:
        x["g"].fill_(-60.0)
    out, last = _fwd(x, cu)
    ro, rs = delta_ref(x, lens, d ** -0.5)
    check(out, ro, "out")
    check(last, rs, "last state", F32)
    got, ref = _bwd(x, cu), delta_grads(x, lens, d ** -0.5)
    for name, y, r in zip(NAMES, got, ref):
        # dg is made of terms of up to 10, each held to the tolerance of the type, of which next
        # to nothing is left: e^-60 of them; or, with one unit key k and beta 1, S_{t-1} = k w^T
        # while D_t - k dv_t^T = (I - k k^T) D_t is orthogonal to k, so their product is 0 (up to
        # |k|^2 - 1).  So its error is at most 10 times the tolerance: 2e-4 in fp32, whose sums
        # keep 2e-5 of each term, 8e-2 in bf16, whose products keep 2 * 2^-8 of each.
        if name == "g" and case in ("fast_decay", "beta_1_same_keys"):
            assert float((y.double() - r).abs().max()) <= 10 * tol(dtype)
            continue
        check(y, r, "d" + name)


def test_repeats_bit_for_bit_on_another_stream_and_in_a_graph():
    lens, H, Hk, d = (300, 77), 4, 2, 64
    x, cu = delta_inputs(lens, H, Hk, d, BF16, seed=9), offsets(lens)
    save = flexattn.delta_save(x["q"], x["v"], cu)
    ws = flexattn.delta_workspace(x["q"], x["v"], cu, backward=True)

    def both():
        out, last = _fwd(x, cu, save=save, ws=ws)
        return (out, last, *flexattn.delta_bwd(*(x[m] for m in NAMES), cu, x["dout"], save, ws=ws))

    first = [t.clone() for t in both()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = both()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for n in NAMES:
        x[n].copy_(x[n].flip(0))
    graph.replay()
    flipped = [t.clone() for t in held]
    assert all(torch.equal(a, b) for a, b in zip(flipped, both()))
    assert not torch.equal(flipped[0], first[0])
    flexattn.check_status(ws)


def test_rows_of_one_sequence_do_not_depend_on_the_batch():
    """A sequence alone and inside a batch: within the rounding of the storage."""
    lens, H, Hk, d = (100, 260, 31), 2, 2, 128
    x, cu = delta_inputs(lens, H, Hk, d, BF16, seed=10), offsets(lens)
    out, last = _fwd(x, cu)
    one = {m: t[100:360].contiguous() for m, t in x.items()}
    o1, s1 = _fwd(one, offsets((260,)))
    assert rel(out[100:360], o1) <= tol(BF16) and rel(last[1], s1[0]) <= tol(F32)


def test_offsets_out_of_range_stay_inside():
    """Offsets beyond the tensors are clamped: the call touches no row that is not there."""
    lens, H, Hk, d = (50, 30), 2, 1, 64
    x = delta_inputs(lens, H, Hk, d, F32, seed=11)
    out, _ = _fwd(x, torch.tensor([0, 50, 900], dtype=torch.int32, device="cuda"))
    ref, _ = _fwd(x, offsets(lens))
    assert torch.equal(out, ref)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_nan_of_the_next_sequence_stays_there(d, dtype):
    """A chunk's tiles reach into the next sequence, all of whose inputs are NaN."""
    lens, H, Hk = (70, 90), 2, 2
    x, cu = delta_inputs(lens, H, Hk, d, dtype, seed=12), offsets(lens)
    for t in x.values():
        t[70:] = float("nan")
    out, last = _fwd(x, cu)
    grads = _bwd(x, cu)
    one = {m: t[:70].contiguous() for m, t in x.items()}
    ro, rs = delta_ref(one, lens[:1], d ** -0.5)
    check(out[:70], ro, "out")
    check(last[0], rs[0], "last state", F32)
    for m, y, r in zip(NAMES, grads, delta_grads(one, lens[:1], d ** -0.5)):
        check(y[:70], r, "d" + m)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_a_prompt_among_single_tokens(dtype):
    lens, H, Hk, d = (1, 500) + (1,) * 9 + (0, 33), 2, 1, 64
    x, cu = delta_inputs(lens, H, Hk, d, dtype, seed=13), offsets(lens)
    out, last = _fwd(x, cu)
    ro, rs = delta_ref(x, lens, d ** -0.5)
    check(out, ro, "out")
    check(last, rs, "last state", F32)
    for m, y, r in zip(NAMES, _bwd(x, cu), delta_grads(x, lens, d ** -0.5)):
        check(y, r, "d" + m)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_rows_far_apart(dtype):
    """Row strides that put the last rows more than 2^31 elements behind the first."""
    lens, H, Hk, d = (130, 20), 2, 1, 64
    T, stride = 150, (1 << 24) + 8
    x, cu = delta_inputs(lens, H, Hk, d, dtype, seed=14), offsets(lens)
    # three views of one long buffer, 512 elements apart inside each row
    long = torch.empty((T - 1) * stride + 2048, dtype=dtype, device="cuda")
    y = dict(x)
    for i, m in enumerate(("q", "k", "v")):
        t = x[m]
        y[m] = torch.as_strided(long, t.shape, (stride, d, 1), storage_offset=512 * i)
        y[m].copy_(t)
    a, b = _fwd(x, cu), _fwd(y, cu)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert all(torch.equal(u, w) for u, w in zip(_bwd(x, cu), _bwd(y, cu)))


def test_calls_on_a_stream_of_their_own():
    """`stream=` without a workspace: the call's scratch belongs to that stream."""
    lens, H, Hk, d = (300, 77), 4, 2, 64
    x, cu = delta_inputs(lens, H, Hk, d, BF16, seed=15), offsets(lens)
    want = _fwd(x, cu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(4):
        got.append(_fwd(x, cu, stream=side))
        torch.zeros(1 << 22, device="cuda")  # would land in scratch released too early
    torch.cuda.current_stream().wait_stream(side)
    for out, last in got:
        assert torch.equal(out, want[0]) and torch.equal(last, want[1])


@pytest.mark.parametrize("dtype,rows", [(F32, 5), (BF16, 5), (BF16, 70)], ids=str)
def test_sequences_that_are_all_empty(dtype, rows):
    H, Hk, d = 2, 1, 64
    x, cu = delta_inputs((0, 0), H, Hk, d, dtype, seed=16, rows_behind=rows), offsets((0, 0))
    out = torch.full((rows, H, d), 7.0, dtype=dtype, device="cuda")
    save = flexattn.delta_save(x["q"], x["v"], cu)
    _, last = _fwd(x, cu, out=out, save=save)
    grads = {"d" + m: torch.full_like(x[m], 7.0) for m in NAMES}
    flexattn.delta_bwd(*(x[m] for m in NAMES), cu, x["dout"], save, **grads)
    assert (last == 0).all()
    assert all((t == 7.0).all() for t in (out, *grads.values()))
    S0 = torch.randn(2, H, d, d, device="cuda")
    assert torch.equal(_fwd(x, cu, state=S0)[1], S0)


@pytest.mark.parametrize("dtype,lens,fwd,bwd", [(F32, (100, 30), 1, 4), (BF16, (3, 4), 1, 4),
                                                (BF16, (100, 30), 2, 2)], ids=str)
def test_launch_counts(dtype, lens, fwd, bwd):
    x, cu = delta_inputs(lens, 2, 1, 64, dtype, seed=17), offsets(lens)
    save = flexattn.delta_save(x["q"], x["v"], cu)
    n = [flexattn.kernel_launches()]
    _fwd(x, cu, save=save)
    n.append(flexattn.kernel_launches())
    flexattn.delta_bwd(*(x[m] for m in NAMES), cu, x["dout"], save)
    n.append(flexattn.kernel_launches())
    k = len(lens)
    flexattn.delta_decode(*(x[m][:k].contiguous() for m in NAMES),
                          torch.zeros(k, 2, 64, 64, device="cuda"))
    n.append(flexattn.kernel_launches())
    assert [b - a for a, b in zip(n, n[1:])] == [fwd, bwd, 1]


@pytest.mark.parametrize("d", [64, 128])
def test_gate_gradients_of_long_sequences_stay_exact(d):
    """dg is a sum over the tokens that follow, whose terms nearly cancel.  At most 64 of them are
    added to an exact <D, S>, each three products with a rounding each: sqrt(64) * 3 * 2^-24 =
    1.5e-6 of the terms, which are of dg's own size, whatever the length."""
    lens, H, Hk = (1500, 64, 65, 600), 2, 1
    x = delta_inputs(lens, H, Hk, d, F32, seed=21)
    got = _bwd(x, offsets(lens))[3].double()
    ref = delta_grads(x, lens, d ** -0.5)[3]
    assert float((got - ref).norm() / ref.norm()) <= 1.5e-6


@pytest.mark.parametrize("d", [64, 128])
def test_scans_of_few_and_of_many_sequences_agree(d):
    """Blocks are narrower where few sequences leave SMs idle; no sum depends on it."""
    lens, H, Hk = (70,) * 20, 4, 2
    x, cu = delta_inputs(lens, H, Hk, d, F32, seed=22), offsets(lens)
    out, last = _fwd(x, cu)
    ro, rs = delta_ref(x, lens, d ** -0.5)
    check(out, ro, "out")
    check(last, rs, "last state", F32)
    got = _bwd(x, cu)
    for name, y, r in zip(NAMES, got, delta_grads(x, lens, d ** -0.5)):
        check(y, r, "d" + name)
    one = {n: t[:70] for n, t in x.items()}
    for a, b in zip((*_fwd(one, cu[:2]), *_bwd(one, cu[:2])), (out, last, *got)):
        assert torch.equal(a, b[:len(a)])


@pytest.mark.parametrize("dtype,lens", [(F32, (1,)), (F32, (1, 1, 0, 1, 1)), (F32, (1, 130, 2, 64, 65)),
                                        (BF16, (1,)), (BF16, (1, 1, 0, 1, 1)), (BF16, (1, 2, 4, 1))], ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_the_gate_of_a_first_token_has_no_gradient(d, dtype, lens):
    """dg_t = a_t <S_{t-1}, ..>: ahead of a sequence's first token the state is 0, so dg is 0."""
    x = delta_inputs(lens, 3, 1, d, dtype, seed=23)
    dg = _bwd(x, offsets(lens))[3]
    at = torch.tensor([0, *torch.tensor(lens).cumsum(0).tolist()])[:-1][torch.tensor(lens) > 0]
    assert (dg[at.cuda()] == 0).all()
    if sum(lens) > len(lens):
        check(dg, delta_grads(x, lens, d ** -0.5)[3], "dg")


@pytest.mark.parametrize("dtype,lens", [(F32, (200, 5, 64)), (BF16, (6, 4, 3)), (BF16, (200, 65))], ids=str)
@pytest.mark.parametrize("every", [1, 3, 70])
@pytest.mark.parametrize("d", [64, 128])
def test_the_gate_of_a_reset_has_no_gradient(d, every, dtype, lens):
    """A gate of -inf: a_t = 0, and with it dg_t.  The others' dg: in fp32 the bound of
    test_gate_gradients_of_long_sequences_stay_exact, in bf16 its storage's."""
    x = delta_inputs(lens, 2, 1, d, dtype, seed=24)
    x["g"][::every] = float("-inf")
    dg = _bwd(x, offsets(lens))[3]
    assert (dg[::every] == 0).all()
    if every > 1:
        ref = delta_grads(x, lens, d ** -0.5)[3]
        assert rel(dg, ref) <= (1.5e-6 if dtype == F32 else tol(BF16))


@pytest.mark.parametrize("d,n", [(64, 17), (64, 70), (128, 9), (128, 65)])
def test_blocks_that_follow_each_other_on_an_sm(d, n):
    """Many times as many walks as SMs, each of one or two chunks, whose blocks take over shared
    and tensor memory from one another: every copy of a sequence has the same results."""
    H, copies = 4, 150
    x = delta_inputs((n,) * 4, H, 2, d, BF16, seed=25)
    many = {m: t.repeat(copies, *([1] * (t.dim() - 1))) for m, t in x.items()}
    cu = offsets((n,) * (4 * copies))
    got = (*_fwd(many, cu), *_bwd(many, cu))
    for y in got:
        y = y.view(copies, -1)
        assert torch.equal(y, y[:1].expand_as(y))
    ro, rs = delta_ref(x, (n,) * 4, d ** -0.5)
    for y, r in zip(got, (ro, rs, *delta_grads(x, (n,) * 4, d ** -0.5))):
        check(y[:len(r)], r, "first copy", F32 if y is got[1] else BF16)


@pytest.mark.parametrize("d", [64, 128])
def test_gradients_of_many_heads_to_a_key_head(d):
    """A block takes the heads of a key head one after the other through the same columns of tensor
    memory: the gates' and values' gradients do not depend on which head came before."""
    H, lens = 8, (70, 200, 5)
    x = delta_inputs(lens, H, 1, d, BF16, seed=26)
    cu = offsets(lens)
    got, turned = _bwd(x, cu), _bwd({m: t.flip(1) if m not in ("q", "k") else t for m, t in x.items()}, cu)
    for y, z in zip(got[2:], turned[2:]):
        assert torch.equal(y, z.flip(1))
    for name, y, r in zip(NAMES, got, delta_grads(x, lens, d ** -0.5)):
        check(y, r, "d" + name)


def _held_busy(shapes):
    """Blocks of these shapes that the allocator hands out again at once, which the current stream
    only comes to overwrite after some 20 ms of products."""
    a = torch.randn(8192, 8192, device="cuda")
    blocks = [torch.empty(s, dtype=t, device="cuda") for s, t in shapes for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(2):
        a = a @ a
    for t in blocks:
        t.fill_(float("nan"))


def test_results_on_a_stream_of_their_own_share_no_block_with_pending_work():
    lens, H, Hk, d = (300, 77), 4, 2, 64
    x, cu = delta_inputs(lens, H, Hk, d, BF16, seed=27), offsets(lens)
    T, side = sum(lens), torch.cuda.Stream()
    save = flexattn.delta_save(x["q"], x["v"], cu)
    out, last = _fwd(x, cu, save=save)
    grads = _bwd(x, cu)
    S = torch.zeros(2, H, d, d, device="cuda")
    tok = [x[n][:2].contiguous() for n in NAMES]
    one = flexattn.delta_decode(*tok, S.clone())
    torch.cuda.synchronize()
    _held_busy([((T, H, d), BF16), ((T, Hk, d), BF16), ((T, H), BF16), ((2, H, d), BF16),
                ((2, H, d, d), F32)])
    got = [*_fwd(x, cu, save=save, stream=side)]
    got += flexattn.delta_bwd(*(x[n] for n in NAMES), cu, x["dout"], save, stream=side)
    got.append(flexattn.delta_decode(*tok, S, stream=side))
    torch.cuda.current_stream().wait_stream(side)
    for y, want in zip(got, (out, last, *grads, one)):
        assert torch.equal(y, want)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("what", ["g", "beta", "k", "v"])
@pytest.mark.parametrize("d", [64, 128])
def test_a_nan_inside_a_sequence_goes_on_to_its_end_and_nowhere_else(d, what, dtype):
    """A NaN of one head (of one key head: k) at one token: that sequence's rows from there on are
    NaN, the chunks of 64 tokens before it, the other heads and the other sequences what they were."""
    lens, H, Hk, at = (300, 70), 4, 2, 150
    x, cu = delta_inputs(lens, H, Hk, d, dtype, seed=28), offsets(lens)
    ro, rs = delta_ref(x, lens, d ** -0.5)
    ref = delta_grads(x, lens, d ** -0.5)
    if what in ("g", "beta"):
        x[what][at, 3] = float("nan")
    else:
        x[what][at, 1 if what == "k" else 3] = float("nan")
    out, last = _fwd(x, cu)
    grads = _bwd(x, cu)
    heads = [2, 3] if what == "k" else [3]
    clean = [h for h in range(H) if h not in heads]
    assert torch.isnan(out[at:300, heads]).all() and torch.isnan(last[0, heads]).all()
    before = at if dtype == F32 else at // 64 * 64
    check(out[:before], ro[:before], "out ahead")
    check(out[300:], ro[300:], "next sequence")
    check(out[:, clean], ro[:, clean], "other heads")
    check(last[1], rs[1], "next state", F32)
    check(last[:, clean], rs[:, clean], "other states", F32)
    for name, y, r in zip(NAMES, grads, ref):
        check(y[300:], r[300:], "d" + name)
        same = [0] if name in ("q", "k") else clean
        check(y[:, same], r[:, same], "d" + name)
    assert torch.isnan(grads[0][at + 1:300, 1]).all()  # dq_t = scale S_t dout_t
    if what != "v":  # dv_t = beta_t D_t^T k_t, and D depends on everything but v
        assert torch.isnan(grads[2][:at, heads]).all()


@pytest.mark.parametrize("gate,many", [(float("-inf"), 1), (float("-inf"), 8), (float("-inf"), 32),
                                       (float("-inf"), 56), (-20.0, 40), (-3.0, 40)], ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_tokens_behind_resets_are_as_accurate_as_others(d, gate, many):
    """Resets or strong decays at a chunk's start, then slow decays: what follows them is held to
    the bounds of any other sequence, forward and backward."""
    lens, H, Hk = (64, 130), 4, 2
    x, cu = delta_inputs(lens, H, Hk, d, BF16, seed=29), offsets(lens)
    at = torch.arange(194, device="cuda")
    at = torch.where(at < 64, at, at - 64) % 64
    x["g"] = torch.where((at < many)[:, None], gate, x["g"].clamp(-0.1, -0.01)).to(BF16)
    out, last = _fwd(x, cu)
    ro, rs = delta_ref(x, lens, d ** -0.5)
    for i, (a, b) in enumerate(((0, 64), (64, 194))):
        check(out[a:b], ro[a:b], "out")
        check(last[i], rs[i], "last state", F32)
    for name, y, r in zip(NAMES, _bwd(x, cu), delta_grads(x, lens, d ** -0.5)):
        check(y, r, "d" + name)


@pytest.mark.parametrize("dtype,lens", [(F32, (130, 70)), (BF16, (130, 70)), (BF16, (3, 2))], ids=str)
def test_workspaces_start_from_their_header_alone(dtype, lens):
    """Whatever else a workspace holds (NaN here) reaches no result; a forward that saves takes one of
    256 bytes and allocates no more."""
    H, Hk, d = 4, 2, 64
    x, cu = delta_inputs(lens, H, Hk, d, dtype, seed=30), offsets(lens)
    want = (*_fwd(x, cu), *_bwd(x, cu))
    ws = flexattn.delta_workspace(x["q"], x["v"], cu, backward=True)
    got = []
    for call in (lambda: _fwd(x, cu, ws=ws), lambda: _bwd(x, cu, ws=ws)):
        ws[256:] = 0xff
        got += call()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    flexattn.check_status(ws)
    save = flexattn.delta_save(x["q"], x["v"], cu)
    first = _fwd(x, cu, save=save, ws=ws)[0]
    out = torch.empty_like(x["v"])
    small = torch.zeros(256, dtype=torch.uint8, device="cuda")
    _fwd(x, cu, save=save, out=out, want_state=False, ws=small)
    assert torch.equal(out, first)
    torch.cuda.reset_peak_memory_stats()
    held = torch.cuda.memory_allocated()
    _fwd(x, cu, save=save, out=out, want_state=False)
    most = torch.cuda.max_memory_allocated()  # (the comparison allocates)
    assert most - held <= 512 and torch.equal(out, first)


@pytest.mark.parametrize("lens", [(200, 17, 128, 5), (64, 400, 63, 30)], ids=str)
@pytest.mark.parametrize("H,Hk", [(4, 4), (8, 4)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_every_sequence_by_itself(lens, H, Hk, d, dtype):
    from packed_ref import GRADIENT, PLAIN, ROUNDED, SPLIT, check_each
    x, cu = delta_inputs(lens, H, Hk, d, dtype, seed=31), offsets(lens)
    out, last = _fwd(x, cu)
    ro, rs = delta_ref(x, lens, d ** -0.5)
    check_each(out, ro, lens, PLAIN if dtype == F32 else ROUNDED, "out")
    check_each(last, rs, (1,) * len(lens), PLAIN if dtype == F32 else SPLIT, "last state")
    for name, y, r in zip(NAMES, _bwd(x, cu), delta_grads(x, lens, d ** -0.5)):
        check_each(y, r, lens, PLAIN if dtype == F32 else GRADIENT, "d" + name)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_as_many_sequences_as_a_call_takes(dtype):
    """65535 single tokens from the zero state: out = scale (q.k) beta v, the state k (beta v)^T."""
    n, d = 65535, 64
    x = delta_inputs((1,) * n, 2, 1, d, dtype, seed=33)
    cu = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    out, last = _fwd(x, cu)
    q, k, v, beta = (x[m].double() for m in ("q", "k", "v", "beta"))
    u = beta[..., None] * v
    check(out, d ** -0.5 * (q * k).sum(-1, keepdim=True) * u, "out")
    for i in (0, 1, 31999, n - 1):
        check(last[i], k[i, 0][None, :, None] * u[i][:, None, :], "state", F32)
    dq, dk, dv, dg, db = _bwd(x, cu)
    du = d ** -0.5 * (q * k).sum(-1, keepdim=True) * x["dout"].double()
    check(dv, beta[..., None] * du, "dv")
    check(db, (v * du).sum(-1), "dbeta")
    w = d ** -0.5 * (u * x["dout"].double()).sum((1, 2))[:, None, None]
    check(dq, w * k, "dq")
    check(dk, w * q, "dk")
    assert (dg == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_as_many_heads_as_a_call_takes(dtype):
    lens, H, Hk, d = (70, 3), 1024, 16, 64
    x, cu = delta_inputs(lens, H, Hk, d, dtype, seed=34), offsets(lens)
    out, last = _fwd(x, cu)
    ro, rs = delta_ref(x, lens, d ** -0.5)
    check(out, ro, "out")
    check(last, rs, "last state", F32)
    for name, y, r in zip(NAMES, _bwd(x, cu), delta_grads(x, lens, d ** -0.5)):
        check(y, r, "d" + name)


@pytest.mark.parametrize("H,Hk,d", [(4, 4, 64), (8, 4, 64), (4, 2, 128)])
def test_bf16_gradients_are_near_their_own_rounding(H, Hk, d):
    """E and the pairs' weights Z enter the gradients' products as bf16 high and low parts.  What is
    rounded on the way (the state, its gradient, dV, and what the walk multiplies) leaves no more
    than two roundings' worth beside a result's own: sqrt(3) of one, at the 1 / sqrt(2) that uniform
    significands leave of the largest."""
    from packed_ref import ROUNDED, check_each
    lens = (512, 200, 333)
    x, cu = delta_inputs(lens, H, Hk, d, BF16, seed=32), offsets(lens)
    for name, y, r in zip(NAMES, _bwd(x, cu), delta_grads(x, lens, d ** -0.5)):
        check_each(y, r, lens, (3 / 2) ** 0.5 * ROUNDED, "d" + name)


@pytest.mark.parametrize("H,Hk,d", [(4, 4, 64), (8, 4, 64), (4, 2, 128)])
@pytest.mark.parametrize("first", [False, True])
def test_last_states_of_bf16_prompts_are_near_fp32(H, Hk, d, first):
    """What a chunk adds to the state enters its product in three bf16 parts, which leave 2^-26 of it;
    M and (d = 128) beta R in two leave 2^-17 / sqrt(3) of the corrections, which are a fraction of
    what is added (0.14 to 0.25 of it, emulated): 1.1e-6, with fp32 sums of 64 products,
    8 2^-24 = 4.8e-7 each, in quadrature 1.2e-6."""
    lens = (512, 200, 333)
    x, cu = delta_inputs(lens, H, Hk, d, BF16, seed=35), offsets(lens)
    S0 = torch.randn(3, H, d, d, device="cuda") / d ** 0.5 if first else None
    last = _fwd(x, cu, state=S0)[1]
    rs = delta_ref(x, lens, d ** -0.5, S0)[1]
    for i in range(3):
        assert rel(last[i], rs[i]) <= 1.2e-6

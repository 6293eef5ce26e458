"""Softmax attention over packed sequences (flex_softattn_fwd) against its definition in 64
bits, and beside the operators it is used with."""
import pytest
import torch

from paper_2606_27748_gb300 import flexattn
from packed_ref import check, delta_inputs, offsets, softattn_ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def library():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    from paper_2606_27748_gb300 import build
    build.build()
    flexattn.load()


def _inputs(lens_q, lens_k, H, Hk, d, dtype, seed=0, behind=0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen).to(dtype).cuda()  # noqa: E731
    return (r(sum(lens_q) + behind, H, d), r(sum(lens_k) + behind, Hk, d),
            r(sum(lens_k) + behind, Hk, d))


def _check(q, k, v, lens_q, lens_k, causal, scale=None, **kw):
    out, lse = flexattn.softattn_fwd(q, k, v, offsets(lens_q), offsets(lens_k), causal=causal,
                                     scale=scale, **kw)
    ro, rz = softattn_ref(q, k, v, lens_q, lens_k, scale or q.shape[2] ** -0.5, causal)
    n = sum(lens_q)
    empty = torch.isinf(rz)
    assert (lse[:n][empty] == float("-inf")).all() and (out[:n][empty] == 0).all()
    check(out[:n], ro, "out")
    check(lse[:n][~empty], rz[~empty], "lse")
    return out, lse


SAME = [(1,), (2, 0, 3), (127, 128, 129), (0, 300, 1, 0), (513, 64, 90)]


@pytest.mark.parametrize("lens", SAME, ids=str)
@pytest.mark.parametrize("H,Hk", [(1, 1), (4, 2), (3, 1), (7, 1), (16, 2)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_prompts(lens, H, Hk, d, dtype, causal):
    _check(*_inputs(lens, lens, H, Hk, d, dtype), lens, lens, causal)


@pytest.mark.parametrize("lens_q,lens_k", [
    ((1, 1, 1), (1, 700, 64)),          # one token each
    ((1,), (5000,)),                    # one token against a long prompt: the keys are split
    ((70, 3, 130), (200, 3, 1000)),     # the next pieces of prompts
    ((100, 5, 64), (30, 0, 64)),        # rows that see no key
    ((64, 64), (0, 64)),                # a sequence without keys
    ((300, 2), (2000, 3000)),           # ranges of keys that end at different rows
    ((5, 6, 7), (20000, 130, 1)),       # a sequence far longer than the average
], ids=str)
@pytest.mark.parametrize("H,Hk,d", [(4, 4, 64), (8, 1, 128), (6, 2, 128), (64, 1, 64)])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_fewer_or_more_queries_than_keys(lens_q, lens_k, H, Hk, d, dtype, causal):
    _check(*_inputs(lens_q, lens_k, H, Hk, d, dtype, seed=1), lens_q, lens_k, causal)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_slices_and_what_lies_outside(dtype):
    """q, k, v as slices of one projection; NaN in the rows behind the last sequence."""
    lens, H, Hk, d = (100, 75), 4, 2, 64
    q, k, v = _inputs(lens, lens, H, Hk, d, dtype, seed=2, behind=60)
    for t in (q, k, v):
        t[175:] = float("nan")
    T = q.shape[0]
    wide = torch.cat([t.reshape(T, -1) for t in (q, k, v)], 1)
    a, b = H * d, (H + Hk) * d
    q, k, v = wide[:, :a].view(T, H, d), wide[:, a:b].view(T, Hk, d), wide[:, b:].view(T, Hk, d)
    out = torch.full((T, H, d), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((T, H), 7.0, device="cuda")
    _check(q, k, v, lens, lens, True, out=out, lse=lse)
    assert (out[175:] == 7.0).all() and (lse[175:] == 7.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_row_strides_off_the_head_size(dtype):
    """Rows padded by 16 bytes: no multiple of a head's bytes."""
    lens, H, Hk, d = (130, 70), 4, 2, 128
    q, k, v = _inputs(lens, lens, H, Hk, d, dtype, seed=10)
    pad = 16 // q.element_size()

    def padded(t):
        w = torch.full((t.shape[0], t.shape[1] * d + pad), float("nan"), dtype=dtype, device="cuda")
        w[:, :-pad] = t.reshape(t.shape[0], -1)
        return w[:, :-pad].view(*t.shape)

    _check(padded(q), padded(k), padded(v), lens, lens, True)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("split", [False, True])
def test_nan_of_the_next_sequence_stays_there(dtype, split):
    """A sequence's last tile of keys reaches into the next sequence's rows."""
    lens_q, lens_k = ((1, 1), (1000, 40)) if split else ((90, 40), (90, 40))
    q, k, v = _inputs(lens_q, lens_k, 2, 2, 64, dtype, seed=3)
    k[lens_k[0]:] = float("nan")
    v[lens_k[0]:] = float("inf")
    out, lse = flexattn.softattn_fwd(q, k, v, offsets(lens_q), offsets(lens_k))
    n = lens_q[0]
    ro, rz = softattn_ref(q, k, v, lens_q[:1], lens_k[:1], 64 ** -0.5, True)
    check(out[:n], ro, "out")
    check(lse[:n], rz, "lse")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("scale", [0.0, 30.0, -1.0])
def test_score_sizes(dtype, scale):
    """Equal scores, scores of several thousands (all but one weight underflow), negative scale."""
    lens = (150, 200)
    q, k, v = _inputs(lens, lens, 2, 1, 64, dtype, seed=4)
    out, lse = flexattn.softattn_fwd(q, k, v, offsets(lens), scale=scale)
    ro, rz = softattn_ref(q, k, v, lens, lens, scale, True)
    # a score of size s carries s 2^-24 sqrt(d) of fp32 rounding, which the weight takes over
    extra = 2000.0 * 2.0 ** -24 * 8 if scale == 30.0 else 0.0
    from packed_ref import rel, tol
    assert rel(out, ro) <= tol(dtype) + extra and rel(lse, rz) <= tol(F32)


def test_largest_weight_first_and_last():
    """The running maximum rises at the first or at the last block of keys by hundreds."""
    lens = (600,)
    for at in (0, 599):
        q, k, v = _inputs(lens, lens, 2, 2, 64, BF16, seed=5)
        k[at] = 12 * q[599, :].float().mean(0, keepdim=True).to(BF16)
        k[at] += 8 * k[at].sign()
        _check(q, k, v, lens, lens, False)


def test_other_stream_graph_and_repeat():
    lens, lens_k = (200, 1, 64), (200, 900, 64)
    cu, cu_k = offsets(lens), offsets(lens_k)
    q, k, v = _inputs(lens, lens_k, 8, 2, 128, BF16, seed=6)
    ws = flexattn.softattn_workspace(q, k, cu)
    run = lambda: flexattn.softattn_fwd(q, k, v, cu, cu_k, ws=ws)  # noqa: E731
    first = [t.clone() for t in run()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    q.copy_(q.flip(0))
    graph.replay()
    flipped = [t.clone() for t in held]
    assert all(torch.equal(a, b) for a, b in zip(flipped, run()))
    assert not torch.equal(flipped[0], first[0])
    flexattn.check_status(ws)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("H,Hk", [(4, 4), (8, 1)])
def test_a_prompt_among_single_tokens(H, Hk, dtype):
    lens_q, lens_k = (1, 400) + (1,) * 20 + (0, 2), (900, 400) + (70,) * 20 + (5, 600)
    _check(*_inputs(lens_q, lens_k, H, Hk, 64, dtype, seed=11), lens_q, lens_k, True)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_many_sequences(dtype, causal):
    """More sequences than are put in order by their work."""
    lens = tuple((7 * i) % 40 for i in range(150)) + (260,)
    _check(*_inputs(lens, lens, 2, 1, 64, dtype, seed=12), lens, lens, causal)
    tok = (1,) * len(lens)
    lens_k = tuple(n + 1 for n in lens)
    _check(*_inputs(tok, lens_k, 2, 1, 64, dtype, seed=13), tok, lens_k, causal)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_rows_far_apart(dtype):
    """Row strides that put the last rows more than 2^31 elements behind the first."""
    lens, H, Hk, d, stride = (130, 20), 2, 1, 64, (1 << 24) + 8
    q, k, v = _inputs(lens, lens, H, Hk, d, dtype, seed=14)
    long = torch.empty(149 * stride + 2048, dtype=dtype, device="cuda")

    def far(t, at):
        y = torch.as_strided(long, t.shape, (stride, d, 1), storage_offset=at)
        y.copy_(t)
        return y

    a = flexattn.softattn_fwd(q, k, v, offsets(lens))
    b = flexattn.softattn_fwd(far(q, 0), far(k, 512), far(v, 1024), offsets(lens))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_calls_on_a_stream_of_their_own():
    """`stream=` without a workspace: the call's scratch belongs to that stream."""
    lens, lens_k = (1, 2), (3000, 900)
    q, k, v = _inputs(lens, lens_k, 8, 2, 128, BF16, seed=15)
    cu, cu_k = offsets(lens), offsets(lens_k)
    want = flexattn.softattn_fwd(q, k, v, cu, cu_k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(4):
        got.append(flexattn.softattn_fwd(q, k, v, cu, cu_k, stream=side))
        torch.zeros(1 << 22, device="cuda")  # would land in scratch released too early
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(o, want[0]) and torch.equal(z, want[1]) for o, z in got)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_sequences_that_are_all_empty(dtype):
    q, k, v = _inputs((0, 0), (5, 0), 2, 1, 64, dtype, seed=16, behind=40)
    out = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    flexattn.softattn_fwd(q, k, v, offsets((0, 0)), offsets((5, 0)), out=out, lse=lse)
    assert (out == 7.0).all() and (lse == 7.0).all()


def test_teacher_of_the_distillation_loss():
    """lse is the normaliser that the distillation's teacher uses: with the frequencies at zero
    the kernel's weights are uniform and the loss is log N for any teacher, and a packed call of
    equal lengths gives the [B, H, N, d] softmax."""
    B, H, N, d = 2, 4, 130, 64
    gen = torch.Generator().manual_seed(7)
    q, k, v = (torch.randn(B, H, N, d, generator=gen).to(BF16).cuda() for _ in range(3))
    W = torch.zeros(H, 64, d, device="cuda")
    loss = flexattn.awd_loss(q, k, W, causal=False)
    assert (loss - torch.log(torch.tensor(float(N)))).abs().max() < 1e-2
    rows = lambda t: t.transpose(1, 2).reshape(B * N, H, d).contiguous()  # noqa: E731
    out, lse = flexattn.softattn_fwd(rows(q), rows(k), rows(v), offsets((N,) * B), causal=False)
    s = torch.einsum("bhid,bhjd->bhij", q.double(), k.double()) / d ** 0.5
    want = torch.softmax(s, -1) @ v.double()
    check(out, rows(want), "out", BF16)
    check(lse, torch.logsumexp(s, -1).transpose(1, 2).reshape(B * N, H), "lse", F32)


def test_a_mixed_stack_on_one_packed_batch():
    """A delta-rule layer, then a full-attention layer, on one packed batch; then one token more
    through both, from the state and from the keys so far."""
    from packed_ref import delta_ref
    lens, H, Hk, d = (90, 33, 128), 4, 2, 64
    cu = offsets(lens)
    x = delta_inputs(lens, H, Hk, d, BF16, seed=8)
    args = [x[n] for n in ("q", "k", "v", "g", "beta")]
    mid, S = flexattn.delta_fwd(*args, cu)
    out, _ = flexattn.softattn_fwd(mid, mid[:, :Hk], mid[:, Hk:], cu)
    rm, rs = delta_ref(x, lens, d ** -0.5)
    check(mid, rm, "first layer")
    ro, _ = softattn_ref(mid, mid[:, :Hk], mid[:, Hk:], lens, lens, d ** -0.5, True)
    check(out, ro, "second layer")
    new = delta_inputs((1,) * 3, H, Hk, d, BF16, seed=9)
    tok = flexattn.delta_decode(*(new[n] for n in ("q", "k", "v", "g", "beta")), S)
    rt, _ = delta_ref(new, (1,) * 3, d ** -0.5, rs)
    check(tok, rt, "token, first layer")
    lens_k = tuple(n + 1 for n in lens)
    rows = torch.cat([torch.cat([a, b]) for a, b in zip(mid.split(lens), tok.split(1))])
    o, _ = flexattn.softattn_fwd(tok, rows[:, :Hk], rows[:, Hk:], offsets((1,) * 3), offsets(lens_k))
    r, _ = softattn_ref(tok, rows[:, :Hk], rows[:, Hk:], (1,) * 3, lens_k, d ** -0.5, True)
    check(o, r, "token, second layer")


@pytest.mark.parametrize("lens_q,lens_k", [
    ((512, 512), (512, 512)),           # two ranges; the first one of rows 0-127 has no block
    ((300,), (300,)), ((700, 40), (700, 900)),
    ((256,), (1100,)), ((130, 130), (1300, 1290)),
], ids=str)
@pytest.mark.parametrize("H,Hk,d", [(2, 2, 64), (2, 2, 128), (4, 1, 128), (4, 1, 64)])
def test_ranges_without_keys_beside_others(lens_q, lens_k, H, Hk, d):
    """Causal, keys split: of a block's two tiles one may have no key in a range.  Many calls one
    behind the other, whose blocks take over shared memory from one another, agree."""
    q, k, v = _inputs(lens_q, lens_k, H, Hk, d, BF16, seed=17)
    ws = flexattn.softattn_workspace(q, k, offsets(lens_q))
    out, lse = _check(q, k, v, lens_q, lens_k, True, ws=ws)
    cu, cu_k = offsets(lens_q), offsets(lens_k)
    for o, z in [flexattn.softattn_fwd(q, k, v, cu, cu_k, ws=ws) for _ in range(20)]:
        assert torch.equal(o, out) and torch.equal(z, lse)
    flexattn.check_status(ws)


def test_results_on_a_stream_of_their_own_share_no_block_with_pending_work():
    """Blocks of the results' sizes are free again, but the current stream has yet to write them."""
    lens, H, Hk, d = (300, 77), 4, 2, 64
    q, k, v = _inputs(lens, lens, H, Hk, d, BF16, seed=18)
    cu, side = offsets(lens), torch.cuda.Stream()
    want = flexattn.softattn_fwd(q, k, v, cu)
    a = torch.randn(8192, 8192, device="cuda")
    blocks = [torch.empty_like(t) for t in want for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(2):
        a = a @ a
    for t in blocks:
        t.fill_(float("nan"))
    del blocks, t
    got = flexattn.softattn_fwd(q, k, v, cu, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("lens_q,lens_k", [((150, 300), (150, 300)),   # one range of keys
                                           ((700,), (700,)),           # two, on the tensor cores
                                           ((1, 1), (3000, 200))],     # single tokens, many
                         ids=str)
@pytest.mark.parametrize("what", ["q", "k", "inf"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_nan_and_infinite_scores_reach_the_rows_that_see_them(lens_q, lens_k, what, d, dtype):
    """A NaN in a row of q makes that row NaN, one in a key (or a score of +inf) every row that sees
    the key; all other rows are what they are without it."""
    H, Hk, G = 4, 2, 2
    q, k, v = _inputs(lens_q, lens_k, H, Hk, d, dtype, seed=19)
    q[:, :, 0] = q[:, :, 0].abs() + 0.5
    clean, rz = softattn_ref(q, k, v, lens_q, lens_k, d ** -0.5, True)
    cu, cu_k = offsets(lens_q), offsets(lens_k)
    nq, nk = lens_q[0], lens_k[0]
    for at in (0, nk // 2, nk - 1):
        hit = torch.zeros(sum(lens_q), H, dtype=torch.bool, device="cuda")
        x, y = q.clone(), k.clone()
        if what == "q":
            x[at % nq, 1, 5] = float("nan")
            hit[at % nq, 1] = True
        else:
            y[at, 1, 0] = float("nan") if what == "k" else float("inf")
            sees = torch.arange(nq, device="cuda") + nk - nq >= at
            hit[:nq, G:] = sees[:, None]
        out, lse = flexattn.softattn_fwd(x, y, v, cu, cu_k)
        assert torch.isnan(out[hit]).all() and torch.isnan(lse[hit]).all()
        check(out[~hit], clean[~hit], "out")
        check(lse[~hit], rz[~hit], "lse")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_workspaces_start_from_their_header_alone(dtype):
    """Whatever else a workspace holds (NaN here) reaches no result of split keys."""
    lens, lens_k = (1, 2), (3000, 900)
    q, k, v = _inputs(lens, lens_k, 8, 2, 128, dtype, seed=20)
    cu, cu_k = offsets(lens), offsets(lens_k)
    want = flexattn.softattn_fwd(q, k, v, cu, cu_k)
    ws = flexattn.softattn_workspace(q, k, cu)
    assert ws.numel() > 256
    ws[256:] = 0xff
    got = flexattn.softattn_fwd(q, k, v, cu, cu_k, ws=ws)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    flexattn.check_status(ws)


@pytest.mark.parametrize("lens_q,lens_k,causal", [
    ((200, 17, 128, 5), (200, 17, 128, 5), True), ((300, 1, 64), (300, 1000, 64), True),
    ((5, 6, 7), (20000, 130, 1), False),     # a sequence far longer than the average
    ((1,) * 6, (4000, 3, 700, 128, 129, 1), True), ((700, 300), (3000, 900), False),
], ids=str)
@pytest.mark.parametrize("H,Hk", [(8, 8), (8, 2)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_every_sequence_by_itself(lens_q, lens_k, causal, H, Hk, d, dtype):
    from packed_ref import PLAIN, WEIGHTED, check_each
    q, k, v = _inputs(lens_q, lens_k, H, Hk, d, dtype, seed=21)
    out, lse = flexattn.softattn_fwd(q, k, v, offsets(lens_q), offsets(lens_k), causal=causal)
    ro, rz = softattn_ref(q, k, v, lens_q, lens_k, d ** -0.5, causal)
    check_each(out, ro, lens_q, PLAIN if dtype == F32 else WEIGHTED, "out")
    # (a row of one key has lse = its score, which may be next to 0)
    assert float((lse - rz).abs().max()) <= PLAIN * (1 + float(rz.abs().max()))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_as_many_sequences_as_a_call_takes(dtype):
    """65535 single tokens that see one key each: its value, and its score as the log sum."""
    n, H, Hk, d = 65535, 2, 1, 64
    one = (1,) * n
    q, k, v = _inputs(one, one, H, Hk, d, dtype, seed=22)
    out, lse = flexattn.softattn_fwd(q, k, v, torch.arange(n + 1, dtype=torch.int32, device="cuda"))
    assert torch.equal(out, v.expand(n, H, d))
    check(lse, d ** -0.5 * (q.double() * k.double()).sum(-1), "lse")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens_q,lens_k", [((70, 3), (70, 300)), ((1, 1), (700, 40))], ids=str)
def test_as_many_heads_as_a_call_takes(lens_q, lens_k, dtype):
    _check(*_inputs(lens_q, lens_k, 1024, 16, 64, dtype, seed=23), lens_q, lens_k, True)


def test_calls_of_both_operators_on_two_streams_at_once():
    """Their blocks share SMs, and with them shared and tensor memory; each call's results are what
    they are alone, also from two graphs replayed at once."""
    lens, H, Hk, d = (300, 64, 513, 90) * 4, 4, 2, 64
    cu = offsets(lens)
    x = delta_inputs(lens, H, Hk, d, BF16, seed=24)
    args = [x[n] for n in ("q", "k", "v", "g", "beta")]
    q, k, v = _inputs(lens, lens, H, Hk, d, BF16, seed=25)
    tok = tuple(1 for _ in lens)
    cu1 = offsets(tok)
    q1 = q[:len(lens)].contiguous()
    save = flexattn.delta_save(x["q"], x["v"], cu)

    def delta():
        out, last = flexattn.delta_fwd(*args, cu, save=save)
        return (out, last, *flexattn.delta_bwd(*args, cu, x["dout"], save))

    def attention():
        return (*flexattn.softattn_fwd(q, k, v, cu), *flexattn.softattn_fwd(q1, k, v, cu1, cu))

    want = delta(), attention()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    held = []
    torch.cuda.synchronize()
    for g, f in zip(graphs, (delta, attention)):
        with torch.cuda.graph(g):
            held.append(f())
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = ([], [])
    for _ in range(10):
        for i, f in enumerate((delta, attention)):
            with torch.cuda.stream(sides[i]):
                got[i].append(f())
    torch.cuda.synchronize()
    for _ in range(10):
        for s, g in zip(sides, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for i in range(2):
        for y in (*got[i], held[i]):
            assert all(torch.equal(a, b) for a, b in zip(y, want[i]))

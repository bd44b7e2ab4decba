"""The vocabulary head's loss and its gradient on the GPU against 64 bits, and against differences of the loss."""
import pytest

from tests.parity import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests.loss_reference import Reference, inputs  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def lede():
    from paper_2606_03113_amd import lede as m
    return m


def close(got, want, tol, what):
    got = got.double()
    ok = ((got - want).abs() <= tol) | (torch.isnan(got) & torch.isnan(want))
    assert bool(ok.all()), (what, float(((got - want).abs() / tol)[~ok].max()), ok.logical_not().nonzero()[:3].tolist())


def check(hidden, head, targets, weights, **kw):
    m = lede()
    r = m.op_head_loss(hidden, head, targets)
    ref = Reference(hidden, head, targets, weights)
    close(r.lse, ref.lse, ref.lse_tol, "lse")
    close(r.loss, ref.loss, ref.loss_tol, "loss")
    dh, dw = m.op_head_loss_grad(hidden, head, targets, r.lse, weights, **kw)
    if dh is not None:
        close(dh, *ref.d_hidden(), "d_hidden")
    if dw is not None:
        close(dw, *ref.d_head(), "d_head")
    return r, dh, dw, ref


SHAPES = [(1, 1, 8), (1, 50, 8), (2, 255, 16), (3, 257, 24), (5, 1000, 64), (64, 513, 72), (65, 300, 200), (128, 256, 128), (129, 703, 136), (200, 2048, 256),
          (256, 1024, 512), (257, 1001, 264), (300, 5000, 64), (32, 1024, 256), (700, 90, 1032), (17, 20000, 40)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,K", SHAPES)
def test_loss_and_gradient(M, V, K, dtype):
    say("head loss M=%d V=%d K=%d %s" % (M, V, K, dtype))
    hidden, head, targets, weights = inputs(M, V, K, DT[dtype], M + V + K)
    check(hidden, head, targets, weights)
    check(hidden, head, targets.clamp(0, V - 1), None)


@pytest.mark.parametrize("M,V,K,dtype", [(2100, 40000, 64, "bf16"), (3000, 33001, 72, "bf16"), (1000, 24003, 40, "f32"), (40, 33000, 704, "f32"), (1500, 24003, 40, "f32")])
def test_pieces_of_the_vocabulary(M, V, K, dtype):
    say("head loss in pieces M=%d V=%d K=%d %s" % (M, V, K, dtype))
    hidden, head, targets, weights = inputs(M, V, K, DT[dtype], 5)
    targets[:4] = torch.tensor([0, V - 1, V - 2, V // 2], dtype=torch.int32)
    check(hidden, head, targets, weights)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,K", [(1, 65409, 8), (3, 70001, 40), (16, 66000, 264), (20, 65537, 72), (33, 65600, 520), (64, 131073, 136), (64, 33000, 256), (65, 33001, 64)])
def test_few_rows_of_large_heads(M, V, K, dtype):
    say("head loss, few rows of large heads M=%d V=%d K=%d %s" % (M, V, K, dtype))
    hidden, head, targets, weights = inputs(M, V, K, DT[dtype], M + V + K)
    targets[0] = V - 1
    check(hidden, head, targets, weights)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_of_the_two(dtype):
    m = lede()
    hidden, head, targets, weights = inputs(70, 600, 128, DT[dtype], 9)
    lse = m.op_head_loss(hidden, head, targets).lse
    both = m.op_head_loss_grad(hidden, head, targets, lse, weights)
    a, none = m.op_head_loss_grad(hidden, head, targets, lse, weights, want_head=False)
    none2, b = m.op_head_loss_grad(hidden, head, targets, lse, weights, want_hidden=False)
    assert none is None and none2 is None and torch.equal(a, both[0]) and torch.equal(b, both[1])
    again = m.op_head_loss_grad(hidden, head, targets, lse, weights)
    assert torch.equal(again[0], both[0]) and torch.equal(again[1], both[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [3, 100, 300])
def test_rows_left_out_may_hold_anything(M, dtype):
    """A row without a target or weight has no part in a gradient, even where it holds NaNs and infinities."""
    m = lede()
    hidden, head, targets, weights = inputs(M, 700, 72, DT[dtype], 4)
    targets = targets.clamp(0, 699)
    weights = weights.clamp(min=0.5)
    targets[0], targets[1], targets[M - 1] = -100, 700, -1
    weights[2 % M] = 0.0
    out = [0, 1, M - 1, 2 % M]
    clean = hidden.clone()
    clean[out] = 0
    bad = hidden.clone()
    for i, value in zip(out, (float("nan"), float("inf"), -float("inf"), float("nan"))):
        bad[i, i % 72] = value
        bad[i, 70] = float("nan")
    r, c = m.op_head_loss(bad, head, targets), m.op_head_loss(clean, head, targets)
    rest = [i for i in range(M) if i not in out]
    assert torch.equal(r.lse[rest], c.lse[rest]) and torch.equal(r.loss[rest], c.loss[rest])
    assert r.loss[[0, 1, M - 1]].tolist() == [0.0] * 3 and bool(torch.isnan(r.lse[out]).all())
    got = m.op_head_loss_grad(bad, head, targets, r.lse, weights)
    want = m.op_head_loss_grad(clean, head, targets, c.lse, weights)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and not bool(got[0][out].any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_left_out_have_no_gradient_whatever_the_head_holds(dtype):
    say("head loss, rows left out under a head with a NaN, %s" % dtype)
    m = lede()
    hidden, head, targets, weights = inputs(70, 600, 64, DT[dtype], 21)
    targets[3], targets[69] = -100, 600
    weights[5] = 0.0
    lse = m.op_head_loss(hidden, head, targets).lse
    head[300, 7] = float("nan")
    dh, _ = m.op_head_loss_grad(hidden, head, targets, lse, weights)
    out = torch.zeros(70, dtype=torch.bool, device="cuda")
    out[[3, 5, 69]] = True
    out |= (targets < 0) | (targets >= 600) | (weights == 0)
    assert bool((dh[out] == 0).all()) and bool(torch.isnan(dh[~out]).any(1).all())


@pytest.mark.parametrize("M,V,dtype", [(131075, 300, "f32"), (131075, 300, "bf16"), (1 << 18, 1 << 20, "f32")])
def test_rows_past_a_launch(M, V, dtype):
    say("head loss of many rows M=%d V=%d %s" % (M, V, dtype))
    hidden, head, targets, _ = inputs(M, V, 8, DT[dtype], 22)
    r = lede().op_head_loss(hidden, head, targets)
    rows = torch.tensor([0, 1, 131071, 131072, 131074, M // 2 + 1, M - 1], device="cuda")
    ref = Reference(hidden[rows], head, targets[rows], None)
    close(r.lse[rows], ref.lse, ref.lse_tol, "lse")
    close(r.loss[rows], ref.loss, ref.loss_tol, "loss")
    del r
    torch.cuda.empty_cache()


def test_everything_left_out_and_no_rows():
    m = lede()
    for dtype in DT.values():
        hidden, head, targets, weights = inputs(20, 300, 64, dtype, 2)
        targets[:] = -1
        r = m.op_head_loss(hidden, head, targets)
        assert not bool(r.loss.any()) and bool(torch.isfinite(r.lse).all())
        dh, dw = m.op_head_loss_grad(hidden, head, targets, r.lse, weights)
        assert not bool(dh.any()) and not bool(dw.any())
        none = m.op_head_loss(hidden[:0], head, targets[:0])
        assert none.loss.numel() == 0
        dh, dw = m.op_head_loss_grad(hidden[:0], head, targets[:0], none.lse, weights[:0], out=(torch.empty(0, 64, device="cuda", dtype=dtype),
                                                                                             torch.full((300, 64), 5.0, device="cuda", dtype=dtype)))
        assert not bool(dw.any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_finite_is_said(dtype):
    m = lede()
    hidden, head, targets, _ = inputs(150, 400, 64, DT[dtype], 8)
    clean = m.op_head_loss(hidden, head, targets)
    bad = hidden.clone()
    bad[7, 3], bad[149, 63] = float("nan"), float("nan")
    r = m.op_head_loss(bad, head, targets.clamp(0, 399))
    assert bool(torch.isnan(r.lse[[7, 149]]).all()) and bool(torch.isnan(r.loss[[7, 149]]).all())
    rest = [i for i in range(150) if i not in (7, 149)]
    assert torch.equal(r.lse[rest], clean.lse[rest])
    w = head.clone()
    w[399, 0] = float("nan")
    assert bool(torch.isnan(m.op_head_loss(hidden, w, targets).lse).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_logits(dtype):
    """Logits thousands apart: one token has all of the probability, and its gradient is 0 or its weight."""
    hidden, head, targets, weights = inputs(90, 520, 64, DT[dtype], 3, scale=400.0)
    check(hidden, head, targets, weights)
    # rows far below zero, far above, and a bias that only shifts them
    hidden, head, targets, weights = inputs(90, 520, 64, DT[dtype], 3)
    head = head.clone()
    head[:, 0], hidden[:, 0] = 64.0, torch.linspace(-1000, 1000, 90, device="cuda").to(DT[dtype])
    check(hidden, head, targets, weights)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_workspaces(dtype):
    m = lede()
    hidden, head, targets, weights = inputs(130, 900, 136, DT[dtype], 6)
    want = m.op_head_loss(hidden, head, targets)
    grads = m.op_head_loss_grad(hidden, head, targets, want.lse, weights)
    wide_h, wide_w = torch.full((130, 200), float("nan"), device="cuda", dtype=DT[dtype]), torch.full((900, 160), float("nan"), device="cuda", dtype=DT[dtype])
    h, w = wide_h[:, 8:144], wide_w[:, 16:152]
    h.copy_(hidden)
    w.copy_(head)
    code = 1 if dtype == "bf16" else 0
    need = m.load().lede_op_head_loss_bytes(code, 130, 900, 136), m.load().lede_op_head_loss_grad_bytes(code, 130, 900, 136)
    ws = [torch.full((n + 256,), 171, dtype=torch.uint8, device="cuda") for n in need]
    got = m.op_head_loss(h, w, targets, workspace=ws[0][:need[0]])
    assert torch.equal(got.loss, want.loss) and torch.equal(got.lse, want.lse)
    oh, ow = torch.full((130, 144), 3.0, device="cuda", dtype=DT[dtype]), torch.full((902, 152), 3.0, device="cuda", dtype=DT[dtype])
    m.op_head_loss_grad(h, w, targets, got.lse, weights, out=(oh[:, :136], ow[1:901, 8:144]), workspace=ws[1][:need[1]])
    assert torch.equal(oh[:, :136], grads[0]) and torch.equal(ow[1:901, 8:144], grads[1])
    oh[:, :136], ow[1:901, 8:144] = 3.0, 3.0
    assert bool((oh == 3.0).all()) and bool((ow == 3.0).all())
    for x, n in zip(ws, need):
        assert bool((x[n:] == 171).all())
    assert bool(torch.isnan(wide_h[:, :8]).all()) and bool(torch.isnan(wide_w[:, 152:]).all())


def test_gradient_against_differences():
    """The loss along a line: its difference quotient is what the gradient says, up to the quotient's own error (known
    from 64 bits) and the losses' rounding."""
    m = lede()
    hidden, head, targets, weights = inputs(60, 400, 128, torch.float32, 12)
    targets = targets.clamp(0, 399)
    r = m.op_head_loss(hidden, head, targets)
    dh, dw = m.op_head_loss_grad(hidden, head, targets, r.lse, weights)
    g = torch.Generator(device="cuda").manual_seed(1)
    for which in (0, 1):
        d = torch.randn((hidden, head)[which].shape, device="cuda", generator=g)
        d /= d.norm()
        eps = 0.5

        def at(sign, f):
            x = [hidden, head]
            x[which] = x[which] + sign * eps * d
            return f(*x)

        op = [float((m.op_head_loss(*x, targets).loss.double() * weights.double()).sum()) for x in (at(1, lambda *a: a), at(-1, lambda *a: a))]
        refs = [at(s, lambda *a: Reference(*a, targets, weights)) for s in (1, -1)]
        true = [float((x.loss * weights.double()).sum()) for x in refs]
        slope = float(((dh, dw)[which].double() * d.double()).sum())
        ref0 = Reference(hidden, head, targets, weights)
        want, tol = (ref0.d_hidden, ref0.d_head)[which]()
        true_slope = float((want * d.double()).sum())
        curve = abs((true[0] - true[1]) / (2 * eps) - true_slope)
        rounding = float(sum((x.loss_tol * weights.double()).sum() for x in refs)) / (2 * eps) + float((tol * d.double().abs()).sum())
        say("slope %g, quotient %g, curve %g, rounding %g" % (slope, (op[0] - op[1]) / (2 * eps), curve, rounding))
        assert abs((op[0] - op[1]) / (2 * eps) - slope) <= curve + rounding


def test_scores_agree_with_those_of_logits():
    """-loss is the log probability that op_logprobs gives for the same logits, formed apart."""
    m = lede()
    hidden, head, targets, _ = inputs(40, 3000, 64, torch.float32, 14)
    targets = targets.clamp(0, 2999)
    ref = Reference(hidden, head, targets)
    z = (ref.h @ ref.w.t()).float()
    lp = m.op_logprobs(z, targets).logprobs
    r = m.op_head_loss(hidden, head, targets)
    assert bool(((r.loss + lp).abs().double() <= ref.loss_tol + 2.0 ** -20 * (ref.loss + 10)).all())


def test_quantised_projection_into_the_loss():
    """Rows through a 4-bit product into the loss and back, as an exit layer's head is trained on them."""
    m = lede()
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(50, 192, device="cuda", generator=g).to(torch.bfloat16)
    codes, scales = m.op_quantize(torch.randn(136, 192, device="cuda", generator=g) * 0.1, 64)
    hidden = m.op_quant_linear(m.QuantMatrix(codes, scales, 192, 64), x)
    _, head, targets, weights = inputs(50, 777, 136, torch.bfloat16, 15)
    check(hidden, head, targets, weights)


def test_in_a_graph():
    """A captured loss with its gradient, replayed over new contents against the eager call."""
    m = lede()
    for dtype, (M, V, K) in (("bf16", (200, 3000, 128)), ("f32", (40, 700, 64)), ("bf16", (2100, 33000, 64))):
        hidden, head, targets, weights = inputs(M, V, K, DT[dtype], 16)

        def both():
            r = m.op_head_loss(hidden, head, targets)
            return (r.loss, r.lse) + m.op_head_loss_grad(hidden, head, targets, r.lse, weights)

        both()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            got = both()
        for i in range(4):
            h, w, t, g = inputs(M, V, K, DT[dtype], 20 + i)
            for a, b in ((hidden, h), (head, w), (targets, t), (weights, g)):
                a.copy_(b)
            want = both()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), (dtype, i)


def test_two_streams_at_once():
    m = lede()
    hidden, head, targets, weights = inputs(300, 4000, 256, torch.bfloat16, 18)
    lse = m.op_head_loss(hidden, head, targets).lse
    want = m.op_head_loss_grad(hidden, head, targets, lse, weights)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            r = m.op_head_loss(hidden, head, targets)
            got.append(m.op_head_loss_grad(hidden, head, targets, r.lse, weights))
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[0]) and torch.equal(b, want[1]) for a, b in got)


def test_head_past_4_gib():
    """A head of more than 2^32 bytes, its last rows among the targets."""
    m = lede()
    V, K = 520000, 4160
    say("head of %.1f GiB" % (V * K * 2 / 2 ** 30))
    head = torch.zeros(V, K, device="cuda", dtype=torch.bfloat16)
    hidden = torch.zeros(3, K, device="cuda", dtype=torch.bfloat16)
    hidden[:, ::2] = 1.0
    head[V - 1, ::2] = 0.01
    head[V - 300, ::2] = -0.01
    targets = torch.tensor([V - 1, 5, V - 300], dtype=torch.int32, device="cuda")
    r = m.op_head_loss(hidden, head, targets)
    a, b = 0.01, -0.01
    a, b = (float(torch.tensor(x, dtype=torch.bfloat16)) * K / 2 for x in (a, b))
    z = torch.tensor([0.0, a, b], dtype=torch.float64)
    count = torch.tensor([V - 2.0, 1.0, 1.0], dtype=torch.float64)
    lse = float((z + count.log()).logsumexp(0))
    assert abs(float(r.lse[0]) - lse) < 1e-4 and torch.allclose(r.loss.cpu().double(), torch.tensor([lse - a, lse, lse - b], dtype=torch.float64), atol=1e-4)
    dh, dw = m.op_head_loss_grad(hidden, head, targets, r.lse)
    p = [float(torch.tensor(x - lse, dtype=torch.float64).exp()) for x in (0.0, a, b)]
    col = dw[:, 0].double().cpu()
    for v, want in ((0, 3 * p[0]), (5, 3 * p[0] - 1), (V - 1, 3 * p[1] - 1), (V - 300, 3 * p[2] - 1), (V - 2, 3 * p[0])):
        assert abs(float(col[v]) - want) <= 2.0 ** -7 * (abs(want) + abs(3 * p[1]) * (v == V - 1)) + 1e-9, v
    assert not bool(dw[:, 1].any()) and bool(torch.isfinite(dh).all())

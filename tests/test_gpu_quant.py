"""4-bit matrices on the GPU against their plain fp64 counterparts: rounding, packing, products."""
import numpy as np
import pytest

from tests import quant_reference as ref
from tests.parity import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def lede():
    from paper_2606_03113_amd import lede as m
    return m


def gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def rounded(a, dtype):
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DT[dtype])
    return t.to("cuda"), t.double().numpy()


def random_matrix(r, N, K, group):
    codes = r.integers(0, 16, (N, K)).astype(np.uint8)
    scales = ref.bf16(np.exp(r.uniform(-8, -2, (N, -(-K // group)))).astype(np.float32) * r.choice([1, 1, 1, -1], (N, -(-K // group))).astype(np.float32))
    m = lede().QuantMatrix(gpu(ref.pack_rows(codes)), gpu(scales).to(torch.bfloat16), K, group)
    return m, codes, scales, ref.values(codes, scales, group)


# ---- rounding ----------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,group", [(1, 1, 32), (3, 31, 32), (5, 33, 32), (17, 128, 64), (2, 300, 128), (9, 1001, 64), (33, 255, 32)])
def test_quantize(N, K, group, dtype):
    say("quantize %d x %d group %d %s" % (N, K, group, dtype))
    r = np.random.default_rng(N + K)
    d, w = rounded(r.standard_normal((N, K)) * np.exp(r.uniform(-30, 30, (N, 1))), dtype)
    codes, scales = lede().op_quantize(d, group)
    want, ws = ref.quantize(w, group)
    assert np.array_equal(scales.float().cpu().numpy(), ws)
    assert np.array_equal(codes.cpu().numpy(), ref.pack_rows(want))


def test_quantize_ties_and_extremes():
    m = lede()
    r = np.random.default_rng(1)
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.0, 0.5, 4.9999995, 5.0000005])
    rows = [np.resize(np.concatenate([mids, -mids]), 64) * s for s in (1.0, 0.0078125, 2.0 ** 100, 2.0 ** -120, 1.0078125)]
    rows += [np.full(64, 0.0), np.full(64, 1e-45), np.full(64, -3.4e38), np.full(64, 1e-39)]
    bad = r.standard_normal((4, 64))
    bad[0, 3], bad[1, 40], bad[2, 63], bad[3, 0] = np.nan, np.inf, -np.inf, np.nan
    w = np.concatenate([np.array(rows), bad]).astype(np.float32)
    codes, scales = m.op_quantize(gpu(w), 32)
    want, ws = ref.quantize(w, 32)
    s = scales.float().cpu().numpy()
    assert np.array_equal(s, ws, equal_nan=True) and np.isnan(s).sum() == 4
    assert np.array_equal(codes.cpu().numpy(), ref.pack_rows(want))


def test_quantize_strided_rows():
    m = lede()
    r = np.random.default_rng(3)
    full = gpu(r.standard_normal((20, 333)).astype(np.float32))
    part = full[::2, 5:205]
    a, b = m.op_quantize(part, 64), m.op_quantize(part.contiguous(), 64)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---- products ----------------------------------------------------------------------------

SHAPES = [(1, 16, 128), (1, 1, 1), (1, 7, 33), (3, 688, 256), (16, 33, 130), (17, 100, 257), (5, 64, 4097), (33, 48, 96), (64, 515, 512), (65, 17, 640),
          (130, 40, 1025), (2, 4096, 31), (1, 300, 11008), (48, 1030, 2048), (256, 129, 384)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_linear(M, N, K, group, dtype):
    say("quant linear M=%d N=%d K=%d group=%d %s" % (M, N, K, group, dtype))
    m = lede()
    r = np.random.default_rng(M * 7 + N + K)
    q, codes, scales, w = random_matrix(r, N, K, group)
    d, x = rounded(r.standard_normal((M, K)) * np.exp(r.uniform(-2, 2, (M, 1))), dtype)
    for y_dtype in ("f32", "bf16"):
        y = m.op_quant_linear(q, d, dtype=DT[y_dtype])
        want, tol = ref.linear(x, w, group, dtype, y_dtype)
        err = np.abs(y.double().cpu().numpy() - want)
        assert (err <= tol).all(), (float((err / tol).max()), np.argwhere(err > tol)[:3])


def test_one_hot_rows_read_every_weight():
    """Rows of the identity give each weight itself."""
    m = lede()
    r = np.random.default_rng(9)
    for N, K, group, dtype in ((37, 200, 32, "bf16"), (16, 256, 128, "f32"), (50, 129, 64, "bf16")):
        q, codes, scales, w = random_matrix(r, N, K, group)
        eye = torch.eye(K, device="cuda", dtype=DT[dtype])
        y = m.op_quant_linear(q, eye, dtype=torch.float32).double().cpu().numpy()
        assert np.array_equal(y, w.T)
        for k in (0, K // 2, K - 1):
            assert np.array_equal(m.op_quant_linear(q, eye[k:k + 1], dtype=torch.float32).double().cpu().numpy()[0], w[:, k])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_alignment(dtype):
    m = lede()
    r = np.random.default_rng(12)
    q, _, _, w = random_matrix(r, 70, 260, 64)
    base = torch.randn(50, 701, device="cuda").to(DT[dtype])
    for x in (base[:, 3:263], base[::3, 8:268], base[7:8, 1:261], base[5:45:2, 440:700], base[:20, :260]):
        want = m.op_quant_linear(q, x.contiguous())
        room = torch.full((x.shape[0] + 2, 100), 7.0, device="cuda", dtype=DT[dtype])
        out = room[1:-1, 11:81]
        assert m.op_quant_linear(q, x, out=out) is out
        assert torch.equal(out, want)
        room[1:-1, 11:81] = 7.0
        assert bool((room == 7.0).all())       # nothing beside the rows


def test_no_rows():
    q = random_matrix(np.random.default_rng(2), 20, 64, 32)[0]
    assert lede().op_quant_linear(q, torch.empty(0, 64, device="cuda")).shape == (0, 20)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [1, 5, 40, 80])
def test_what_is_not_finite_stays(M, dtype):
    """With its row of x, with its row of W."""
    m = lede()
    r = np.random.default_rng(M)
    q, codes, scales, w = random_matrix(r, 60, 300, 32)
    x = r.standard_normal((M, 300)).astype(np.float32)
    d = gpu(x).to(DT[dtype])
    clean = m.op_quant_linear(q, d)
    for value in (np.nan, np.inf, -np.inf):
        bad = d.clone()
        bad[M // 2, 299] = float(value)
        y = m.op_quant_linear(q, bad)
        rows = [i for i in range(M) if i != M // 2]
        assert torch.equal(y[rows], clean[rows])
        want = value * w[:, 299]
        got = y[M // 2].double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    s = scales.copy()
    s[7, 3], s[59, 9], s[20, 0] = np.nan, np.inf, 0.0
    q2 = m.QuantMatrix(gpu(ref.pack_rows(codes)), gpu(s).to(torch.bfloat16), 300, 32)
    y = m.op_quant_linear(q2, d)
    rows = [i for i in range(60) if i not in (7, 20, 59)]
    assert torch.equal(y[:, rows], clean[:, rows]) and bool(torch.isnan(y[:, 7]).all()) and not bool(torch.isfinite(y[:, 59]).any())
    assert bool(torch.isfinite(y[:, 20]).all())


@pytest.mark.parametrize("M", [1, 20])
def test_nan_with_low_bits_alone(M):
    """An fp32 NaN whose payload lies below bf16's bits is still one."""
    q = random_matrix(np.random.default_rng(4), 16, 32, 32)[0]
    x = torch.ones(M, 32, device="cuda")
    x.view(torch.int32)[0, 5] = 0x7F800001
    y = lede().op_quant_linear(q, x)
    assert bool(torch.isnan(y[0]).all()) and bool(torch.isfinite(y[1:]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [1, 3, 33])
def test_large_and_small_numbers(M, dtype):
    """Sums overflow only where the result does, whatever the scales; nothing is lost down to 2^-90."""
    m = lede()
    K, group = 512, 64
    r = np.random.default_rng(21)
    codes = np.full((4, K), 7, np.uint8)
    for big, scale in ((3.3e38, 2.0 ** -20), (2.0 ** 127, 2.0 ** -100), (2.0 ** -90, 1.0), (2.0 ** -60, 2.0 ** 60), (1e30, 1e-3)):
        s = np.full((4, K // group), scale, np.float32)
        q = m.QuantMatrix(gpu(ref.pack_rows(codes)), gpu(ref.bf16(s)).to(torch.bfloat16), K, group)
        d, x = rounded(big * r.uniform(0.5, 1.0, (M, K)), dtype)
        y = m.op_quant_linear(q, d, dtype=torch.float32).double().cpu().numpy()
        want, tol = ref.linear(x, ref.values(codes, ref.bf16(s), group), group, dtype, "f32")
        assert np.isfinite(want).all() and (np.abs(y - want) <= tol + 1e-30 * (big < 1e-20) * scale).all()


def test_large_matrix_offsets():
    """A matrix whose rows of x lie past 2^32 bytes."""
    m = lede()
    r = np.random.default_rng(8)
    q, _, _, w = random_matrix(r, 20, 64, 32)
    ld = 1 << 22
    base = torch.zeros(513 * ld, device="cuda", dtype=torch.bfloat16)      # 4.3 GB
    x = base.view(513, ld)[:, 100:164]
    x[512] = 1.0
    x[1] = 2.0
    y = m.op_quant_linear(q, x, dtype=torch.float32).double().cpu().numpy()
    want, tol = ref.linear(np.ones((1, 64)), w, 32, "bf16", "f32")
    assert (np.abs(y[512] - want[0]) <= tol[0]).all() and (np.abs(y[1] - 2 * want[0]) <= 2 * tol[0]).all() and not y[2:512].any()


def test_weights_round_trip():
    """Quantised weights multiply as their values do."""
    m = lede()
    r = np.random.default_rng(30)
    dw, w = rounded(r.standard_normal((130, 520)) * 0.05, "bf16")
    codes, scales = m.op_quantize(dw, 128)
    q = m.QuantMatrix(codes, scales, 520, 128)
    c, s = ref.quantize(w, 128)
    dx, x = rounded(r.standard_normal((6, 520)), "bf16")
    want, tol = ref.linear(x, ref.values(c, s, 128), 128, "bf16", "bf16")
    assert (np.abs(m.op_quant_linear(q, dx).double().cpu().numpy() - want) <= tol).all()


def test_in_a_graph_and_on_streams():
    m = lede()
    r = np.random.default_rng(40)
    q = random_matrix(r, 500, 1024, 64)[0]
    x = torch.randn(70, 1024, device="cuda", dtype=torch.bfloat16)
    want = [m.op_quant_linear(q, x[:n]) for n in (1, 9, 70)]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        got = [m.op_quant_linear(q, x[:n]) for n in (1, 9, 70)]
    for i in range(5):
        x.normal_()
        want = [m.op_quant_linear(q, x[:n]) for n in (1, 9, 70)]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    res = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            res.append(m.op_quant_linear(q, x))
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[2]) for a in res)

"""Products in 8-bit integers on the GPU: integers and scales to the bit, products against exact sums.

Tolerances: a sum is a whole number, rounded to fp32, times two scales and plus a bias: four roundings of 2^-24
of the sum's and the bias's magnitudes; then the output's."""
import numpy as np
import pytest

from tests import learner_ref as ref
from tests.test_gpu_learner import B16, U, dt, gen, learner, placed, randn, torch  # noqa: F401

pytestmark = pytest.mark.gpu
F = np.float32


def integers(t):
    """(integers as 64-bit whole numbers, fp32 scales) by the definition, step by step in fp32."""
    x = t.detach().cpu().float().numpy()
    q, s = np.zeros(x.shape, np.int64), np.zeros(len(x), F)
    for r, row in enumerate(x):
        most = F(max(F(abs(row).max(initial=F(0))), F(2.0 ** -100)))
        if not np.isfinite(row).all():
            s[r] = np.nan
            continue
        s[r] = most / F(127)
        q[r] = np.rint(row * F(F(127) * F(F(1) / most))).astype(np.int64)
    return q, s


def product(a, sa, b, sb, bias=None, relu=False):
    """(result in 64 bits, tolerance)."""
    with np.errstate(invalid="ignore"):
        y = (a @ b.T) * sa[:, None].astype(np.float64) * sb.astype(np.float64)
        tol = 4 * U * abs(y)
        if bias is not None:
            y, tol = y + bias, tol + 4 * U * abs(bias)
        return (np.where(y < 0, 0, y) if relu else y), tol


def close(t, want, tol):
    got = ref.f64(t)
    unit = B16 if "bfloat16" in str(t.dtype) else U
    ok = (abs(got - want) <= tol + unit * (abs(want) + tol) + 1e-44) | (np.isnan(got) & np.isnan(want))
    assert ok.all(), (np.argwhere(~ok)[:4], got[~ok][:4], want[~ok][:4])


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 127), (4, 128), (5, 129), (9, 512), (7, 513), (2, 2048), (3, 2055),
                                       (6, 8192), (2, 8200), (3, 16391), (1, 30001), (2, 32777), (300, 40)])
@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_quantize(torch, learner, rows, cols, x):  # noqa: F811
    g = gen(torch, rows + cols)
    t, _ = placed(torch, rows, cols, dt(torch, x), 3, 5)
    t.copy_(randn(torch, g, rows, cols) * torch.exp(4 * randn(torch, g, rows, 1)))
    q = learner.quantize_int8(t)
    want, scales = integers(t)
    assert np.array_equal(q.values[:, :cols].cpu().numpy(), want)
    assert bool((q.values[:, cols:] == 0).all()) and q.values.shape[1] % 128 == 0
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    assert abs(want).max() == 127 or not bool(t.any())
    assert np.array_equal(ref.f64(q.dequantize()), (want.astype(F) * scales[:, None]).astype(np.float64))


def test_quantize_borders(torch, learner):  # noqa: F811
    """Ties to even; rows of zeros, of numbers below 2^-100, of the largest; NaN and infinities."""
    x = torch.zeros(9, 260, device="cuda")
    x[0, :4] = torch.tensor([127.0, 2.5, 3.5, -0.5])
    x[1, 0], x[1, 1] = 1e-40, -2.0 ** -101
    x[2] = 3.4e38
    x[3, 259] = float("nan")
    x[4, 0] = float("-inf")
    x[5, 7] = 1e-30
    q = learner.quantize_int8(x)
    # 127 (1 / 127) rounds to 1 in fp32
    assert F(127) * F(F(1) / F(127)) == 1 and q.values[0, :4].tolist() == [127, 2, 4, 0]
    want, scales = integers(x)
    rows = [0, 1, 2, 5, 6, 7, 8]
    assert np.array_equal(q.values[rows, :260].cpu().numpy(), want[rows])
    assert np.array_equal(q.scales.cpu().numpy(), scales, equal_nan=True)
    w = learner.quantize_int8(torch.randn(70, 260, device="cuda"))
    for y in (learner.linear_int8(x, w, dtype=torch.float32), learner.matmul_int8(q, w, dtype=torch.float32)):
        assert bool(y[3:5].isnan().all()) and bool((y[6:] == 0).all())
        assert bool(y[[0, 1, 5]].isfinite().all()) and not bool(y[2].isnan().any())
        # rows of 3.4e38: their sums times the scale pass fp32's range
        sums = want[2] @ integers(w.dequantize())[0].T
        assert np.array_equal(np.isinf(y[2].cpu().numpy()), abs(sums * np.float64(scales[2])) > 3.4028235e38)
    y = learner.matmul_int8(w, q, relu=True, dtype=torch.float32)
    assert bool(y[:, 3:5].isnan().all()) and bool(y[:, [0, 1, 5, 6, 7, 8]].isfinite().all())


SIZES = [(1, 1, 1), (1, 4096, 300), (3, 17, 130), (16, 300, 1000), (17, 64, 256), (32, 100, 640), (33, 65, 129),
         (57, 1000, 900), (100, 8, 4000), (128, 256, 384), (129, 257, 65), (300, 500, 700), (3, 300, 24000),
         (1, 70, 17000), (32, 1000, 8192), (2, 33, 25088), (520, 1030, 260), (64, 128, 16640)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("x,out,bias,relu", [("f32", "f32", None, False), ("bf16", "bf16", "f32", True),
                                             ("bf16", "f32", "bf16", False), ("f32", "bf16", None, True)])
def test_linear(torch, learner, m, n, k, x, out, bias, relu):  # noqa: F811
    g = gen(torch, m + n + k)
    t, _ = placed(torch, m, k, dt(torch, x), 1, 3)
    t.copy_(randn(torch, g, m, k) * torch.exp(randn(torch, g, m, 1)))
    w = randn(torch, g, n, k, std=0.1)
    b = None if bias is None else torch.cat([randn(torch, g, 1), randn(torch, g, n)]).to(dt(torch, bias))[1:]
    wq = learner.quantize_int8(w)
    want, tol = product(*integers(t), *integers(w), None if b is None else ref.f64(b), relu)
    dst, buf = placed(torch, m, n, dt(torch, out), 3, 5, 7.0)
    assert learner.linear_int8(t, wq, b, relu, out=dst) is dst
    close(dst, want, tol)
    y = learner.matmul_int8(learner.quantize_int8(t), wq, b, relu, dtype=dt(torch, out))
    assert torch.equal(y, dst)   # the same in two calls
    dst.fill_(7.0)
    assert bool((buf == 7.0).all())
    # a token's answer is the same alone and in any batch
    for row in {0, m // 2, m - 1}:
        assert torch.equal(learner.linear_int8(t[row:row + 1], wq, b, relu, dtype=dt(torch, out)), y[row:row + 1])


def test_large_tiles(torch, learner):  # noqa: F811
    """Several of the largest tiles for each compute unit, edges, and parts of k of them: equal to the rows one by
    one, whose kernel is another, and (some) to exact sums."""
    for m, n, k, dtype in ((4500, 4300, 260, torch.bfloat16), (1280, 4096, 22272, torch.float32),
                           (2300, 8200, 1000, torch.float32)):
        g = gen(torch, m)
        x, w = randn(torch, g, m, k, dtype=torch.bfloat16), randn(torch, g, n, k, dtype=torch.bfloat16)
        bias = randn(torch, g, n)
        wq = learner.quantize_int8(w)
        y = learner.linear_int8(x, wq, bias, dtype=dtype)
        for at in (0, 777, m - 5):
            assert torch.equal(learner.linear_int8(x[at:at + 5], wq, bias, dtype=dtype), y[at:at + 5])
        want, tol = product(*integers(x[m - 2:]), *integers(w), ref.f64(bias))
        close(y[m - 2:], want, tol)


def test_offsets_past_32_bits(torch, learner):  # noqa: F811
    """Integers and results of more than 2^32 elements: the last rows as by themselves."""
    k, m = 640, (1 << 32) // 640 + 300
    x = torch.zeros(m, k, device="cuda", dtype=torch.bfloat16)
    x[-256:] = randn(torch, gen(torch, 1), 256, k)
    w = learner.quantize_int8(randn(torch, gen(torch, 2), 650, k))
    y = learner.linear_int8(x, w)
    assert y.numel() > 1 << 32 and bool((y[:300] == 0).all())
    assert torch.equal(y[-256:], learner.linear_int8(x[-256:], w))


def test_largest_sums(torch, learner):  # noqa: F811
    """2^17 products of 127^2 are the largest sum; one more column is refused."""
    k = 1 << 17
    x = torch.full((2, k), 1.0, device="cuda")
    x[1] = -1
    for m in (2, 40):
        a = learner.quantize_int8(x[:1].expand(m, k).contiguous())
        y = learner.matmul_int8(a, learner.quantize_int8(x), dtype=torch.float32)
        s = np.float64(F(1) / F(127))
        want = 127 * 127 * k * s * s
        assert bool(((y[:, 0].double() - want).abs() <= 4 * U * want).all()) and torch.equal(y[:, 0], -y[:, 1])
    from paper_1611_06213_amd import ps
    with pytest.raises(ps.PSError):
        learner.quantize_int8(torch.ones(1, k + 1, device="cuda"))


def test_no_rows_no_terms(torch, learner):  # noqa: F811
    w = learner.quantize_int8(torch.randn(9, 30, device="cuda"))
    assert learner.linear_int8(torch.ones(0, 30, device="cuda"), w).shape == (0, 9)
    none = learner.quantize_int8(torch.ones(0, 30, device="cuda"))
    assert learner.linear_int8(torch.ones(4, 30, device="cuda"), none).shape == (4, 0)
    bias = torch.randn(9, device="cuda")
    empty = learner.quantize_int8(torch.ones(9, 0, device="cuda"))
    for m in (4, 50):
        y = learner.linear_int8(torch.ones(m, 0, device="cuda"), empty, bias, True, dtype=torch.float32)
        assert torch.equal(y, bias.clamp(min=0).expand(m, 9))


def test_streams_and_graphs(torch, learner):  # noqa: F811
    """Split, joined and converting products, captured and replayed with eager work between."""
    g = gen(torch, 3)
    layers = [(learner.quantize_int8(randn(torch, g, n, k)), randn(torch, g, m, k, dtype=torch.bfloat16))
              for m, n, k in ((1, 300, 900), (3, 300, 24000), (100, 70, 5000), (300, 600, 256))]
    xs = [x for _, x in layers]

    def fill(s):
        for i, x in enumerate(xs):
            x.copy_(randn(torch, gen(torch, 10 * s + i), *x.shape))

    def run():
        return [learner.linear_int8(x, w, relu=True) for w, x in layers]

    want = {}
    for s in (1, 2, 3):
        fill(s)
        want[s] = run()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        graphs.append((graph, out))
    for s in (1, 2, 3, 1, 2, 3):
        fill(s)
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        graphs[0][0].replay()
        with torch.cuda.stream(other):
            graphs[1][0].replay()
        eager = run()
        torch.cuda.synchronize()
        for got in (graphs[0][1], graphs[1][1], eager):
            assert all(torch.equal(a, b) for a, b in zip(got, want[s]))


def test_refusals(torch, learner):  # noqa: F811
    from paper_1611_06213_amd import ps
    x = torch.ones(4, 30, device="cuda")
    w = learner.quantize_int8(torch.ones(9, 30, device="cuda"))
    other = learner.quantize_int8(torch.ones(9, 31, device="cuda"))

    def exchanged(**parts):
        q = learner.quantize_int8(torch.ones(9, 30, device="cuda"))
        for k, v in parts.items():
            setattr(q, k, v)
        return q

    bad = [
        (TypeError, lambda: learner.linear_int8(x, x)),
        (TypeError, lambda: learner.linear_int8(x.half(), w)),
        (TypeError, lambda: learner.linear_int8(x, w, dtype=torch.float16)),
        (TypeError, lambda: learner.linear_int8(x, w, x[0, :9].half())),
        (ValueError, lambda: learner.linear_int8(x, other)),
        (ValueError, lambda: learner.linear_int8(x.cpu(), w)),
        (ValueError, lambda: learner.linear_int8(x[:, ::2], w)),
        (ValueError, lambda: learner.linear_int8(x, w, torch.ones(8, device="cuda"))),
        (ValueError, lambda: learner.linear_int8(x, w, out=torch.ones(4, 8, device="cuda"))),
        (ValueError, lambda: learner.matmul_int8(w, other)),
        (TypeError, lambda: learner.matmul_int8(x, w)),
        (ValueError, lambda: learner.matmul_int8(w, exchanged(values=w.values[:8]))),
        (ValueError, lambda: learner.matmul_int8(w, exchanged(values=w.values.to(torch.uint8)))),
        (ValueError, lambda: learner.matmul_int8(w, exchanged(scales=w.scales.double()))),
        (ValueError, lambda: learner.matmul_int8(w, exchanged(scales=torch.ones(18, device="cuda")[::2]))),
        (ValueError, lambda: learner.matmul_int8(w, exchanged(values=w.values.cpu()))),
        (ps.PSError, lambda: learner.linear_int8(x, w, out=x[:, :9])),
        (ps.PSError, lambda: learner.linear_int8(x[:1].expand(4, 30), w)),
        (TypeError, lambda: learner.quantize_int8(x.double())),
        (ValueError, lambda: learner.quantize_int8(x[0])),
    ]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()

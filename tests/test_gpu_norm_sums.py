"""The norms and their gradients where a worker has several rows, against the formulas in 64 bits: sums over rows that
are carried from row to row, gates that begin and end inside workers and between them, and sums that are joined.

Tolerances are those of test_gpu_norms, but for sums over rows. There, a worker adds up the 3 rows that it has at most
(after's over its gates once more), then each thread of a column the sums of at most 32 workers, and the 32 threads' sums:
3 + 3 + 32 + 32 additions one after another, and 20 roundings of a term's factors: 90 u of the sum of magnitudes.
"""
import pytest

from tests import learner_ref as ref
from tests.test_gpu_learner import U, gen, learner, placed, randn, torch  # noqa: F401
from tests.test_gpu_norms import EPS, TYPES, Case, backward, close, depth, forward, rounding

pytestmark = pytest.mark.gpu

# rows, columns, gates: of 25 rows and 834 workers of 3 (100 gates are joined eight a workgroup); of 300; of 2, between
# workers of 3; of 20, of 100 and of 30 rows in workgroups of 3, 16 and 9 waves; of 10 rows in workers of one; rows that
# no worker holds, of 25, of 75, of 25 and (44 workers) of 13 rows
SIZES = [(2500, 130, 100), (2100, 1000, 7), (2600, 130, 1300), (2500, 1000, 2500), (700, 1025, 35), (700, 8192, 7),
         (600, 4100, 20), (130, 700, 13), (700, 8200, 28), (3000, 5, 40), (200, 16384, 8), (130, 33000, 10)]


@pytest.mark.parametrize("rows,cols,gates", SIZES)
@pytest.mark.parametrize("stream,branch,weights", TYPES)
def test_sums_over_rows(torch, learner, rows, cols, gates, stream, branch, weights):  # noqa: F811
    c = Case(torch, rows, cols, gates, True, True, stream, branch, weights, 1.25)
    want = backward(c.ref("h"), c.ref("y"), c.ref("dh"), c.ref("dz"), c.ref("gate"), c.ref("after"), c.ref("before"),
                    c.scale)
    d = depth(cols)
    t = 2 * (d / 2 + 4) * U + (d + 10) * U
    for name in ("gate", "after", "before"):
        value, tol = want[name]
        want[name] = value, tol * ((t + 90 * U) / (t + (rows + 20) * U))
    args = (c.h, c.y, c.dh, c.dz, c.gate, c.after, c.before, c.scale, EPS)
    got = learner.residual_norm_grad(*args, weight_dtype=torch.float32)
    for name, x in got._asdict().items():
        close(x, *want[name], rounding(x))
    again = learner.residual_norm_grad(*args, weight_dtype=torch.float32)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    # into places of the caller's, nothing around them; the vectors' added to what is there
    outs = {"gate": c.out(torch.float32, gates, 2.0), "after": placed(torch, 1, cols, torch.float32, 1, 0, 2.0),
            "before": placed(torch, 1, cols, torch.float32, 1, 0, 2.0)}
    learner.residual_norm_grad(*args, accumulate=True,
                               **{f"{k}_out": v[0] if k == "gate" else v[0][0] for k, v in outs.items()})
    for name, (x, buf) in outs.items():
        value, tol = want[name]
        close(x, value + 2.0, tol + 2 * U * (abs(value) + 2.0), U)
        x.fill_(2.0)
        assert bool((buf == 2.0).all()), name


@pytest.mark.parametrize("rows,cols", [(2500, 130), (2100, 1000), (700, 8192), (700, 8200), (3000, 5)])
@pytest.mark.parametrize("gates", [0, 1])
def test_one_gate_or_none(torch, learner, rows, cols, gates):  # noqa: F811
    """Sums over all rows, without a norm after the block, and with bf16 gradients of the vectors."""
    c = Case(torch, rows, cols, gates, not gates, True, "bf16", "f32", "f32", 0.75)
    want = backward(c.ref("h"), c.ref("y"), None, c.ref("dz"), c.ref("gate"), c.ref("after"), c.ref("before"), c.scale)
    d = depth(cols)
    t = 2 * (d / 2 + 4) * U + (d + 10) * U
    got = learner.residual_norm_grad(c.h, c.y, None, c.dz, c.gate, c.after, c.before, c.scale, EPS,
                                     weight_dtype=torch.bfloat16)
    for name, x in got._asdict().items():
        assert (x is not None) == (name in want), name
        if x is not None:
            value, tol = want[name]
            if name in ("gate", "after", "before"):
                tol = tol * ((t + 90 * U) / (t + (rows + 20) * U))
            close(x, value, tol, rounding(x))


@pytest.mark.parametrize("rows,cols,gates", [(9000, 1000, 9), (9000, 1001, 4500), (3, 16384, 3), (5, 12288, 1),
                                             (7, 12290, 7), (12, 8200, 4)])
@pytest.mark.parametrize("stream,branch,weights", TYPES)
def test_forward(torch, learner, rows, cols, gates, stream, branch, weights):  # noqa: F811
    """Workers of three rows, whose gate changes between them; rows of two eights of columns a thread."""
    c = Case(torch, rows, cols, gates, True, True, stream, branch, weights, 1.25)
    (out, buf), (normed, nbuf) = c.out(c.sd), c.out(c.bd)
    learner.residual_norm(c.x, c.y, c.gate, c.after, c.before, c.scale, EPS, out=out, normed_out=normed)
    wh, wz, th, tz = forward(*(c.ref(k) for k in ("x", "y", "gate", "after", "before")), c.scale)
    close(out, wh, th, rounding(out))
    close(normed, wz, tz, rounding(normed))
    for t, b in ((out, buf), (normed, nbuf)):   # nothing around them
        t.fill_(7.0)
        assert bool((b == 7.0).all())
    z = learner.rms_norm(c.x, c.before, EPS, dtype=c.bd)
    _, want, _, tol = forward(c.ref("x"), None, None, None, c.ref("before"), 1.0)
    close(z, want, tol, rounding(z))


@pytest.mark.parametrize("cols", [1000, 8200, 8203, 16384])
def test_rows_of_a_worker_are_as_alone(torch, learner, cols):  # noqa: F811
    """More rows than workers, whose gate changes inside them: to the bit what calls of one gate's rows give."""
    gates, each = 7, 700
    g = gen(torch, cols)
    x, y = (randn(torch, g, gates * each, cols, dtype=torch.bfloat16) for _ in range(2))
    gate, after, before = randn(torch, g, gates, cols), randn(torch, g, cols), randn(torch, g, cols)
    h, z = learner.residual_norm(x, y, gate, after, before, 0.5)
    normed = learner.rms_norm(x, before)
    for i in range(gates):
        s = slice(i * each, (i + 1) * each)
        h1, z1 = learner.residual_norm(x[s], y[s], gate[i], after, before, 0.5)
        assert torch.equal(h[s], h1) and torch.equal(z[s], z1), i
        assert torch.equal(normed[s], learner.rms_norm(x[s], before)), i

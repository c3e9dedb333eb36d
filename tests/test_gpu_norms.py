"""The norms around a residual block, and their gradients, on the GPU against the formulas in 64 bits.

Tolerances, u = 2^-24. A sum over a row of C columns adds at most D = 8 ceil(C / 8192) + 30 terms one after
another (eight a thread for each 8192 columns, six steps over a wave, sixteen waves): D u of the sum of
magnitudes. 1 / sqrt(sum / C + eps) halves the relative error of a sum of squares and rounds four times:
E = (D / 2 + 4) u.
  h   the branch E + 4 u of its magnitude, the stream and the sum 2 u each, then the output's rounding
  z   what h's error e leaves: its own, and that of h's norm, |e| / |h| over the row; E + 4 u
  gradients: each is a sum of terms with those factors; with t = 2 E + (D + 10) u, t of the sum of the terms'
      magnitudes, (rows + 20) u more for sums over rows; then the output's rounding
"""
import numpy as np
import pytest

from tests import learner_ref as ref
from tests.test_gpu_learner import B16, U, dt, gen, learner, placed, randn, torch  # noqa: F401

pytestmark = pytest.mark.gpu
EPS = 1e-5


def depth(cols):
    return 8 * -(-cols // 8192) + 30


def inv(v):
    return 1 / np.sqrt((v * v).mean(1, keepdims=True) + EPS)


def forward(x, y, gate, after, before, scale):
    """(h, z, their tolerances) in 64 bits, without the outputs' rounding."""
    rows, cols = x.shape
    e = (depth(cols) / 2 + 4) * U
    if y is None:
        h, th = x, np.zeros_like(x)
    else:
        b = y if after is None else y * inv(y) * after
        if gate is not None:
            b = b * np.repeat(gate, rows // len(gate), axis=0)
        h = scale * x + b
        th = (e + 4 * U) * abs(b) + 2 * U * (abs(scale * x) + abs(h))
    r = inv(h)
    w = 1.0 if before is None else before
    size = np.sqrt((h * h).sum(1, keepdims=True)) + 1e-300
    z = h * r * w
    tz = abs(r * w) * th + abs(z) * (e + 4 * U + np.sqrt((th * th).sum(1, keepdims=True)) / size)
    return h, z, th, tz


def backward(h, y, dh, dz, gate, after, before, scale):
    """{name: (gradient, tolerance)} of the formulas, each term's magnitude beside it."""
    rows, cols = h.shape
    d = depth(cols)
    t = 2 * (d / 2 + 4) * U + (d + 10) * U
    tr = t + (rows + 20) * U
    out = {}
    total = np.zeros_like(h) if dh is None else dh
    size = abs(total)
    if dz is not None:
        r = inv(h)
        w = np.ones(cols) if before is None else before
        u = dz * w
        total = total + r * (u - h * (r * r * (u * h).mean(1, keepdims=True)))
        size = size + r * (abs(u) + abs(h) * (r * r * abs(u * h).mean(1, keepdims=True)))
        if before is not None:
            out["before"] = (dz * h * r).sum(0), tr * abs(dz * h * r).sum(0)
    out["x"] = scale * total, (t + U) * abs(scale) * size
    if y is None:
        return out
    g = 1.0 if gate is None else np.repeat(gate, rows // len(gate), axis=0)
    ry = np.ones((rows, 1)) if after is None else inv(y)
    w = 1.0 if after is None else after
    b = y * ry * w
    if gate is not None:
        out["gate"] = tuple(v.reshape(len(gate), -1, cols).sum(1) for v in (total * b, tr * size * abs(b)))
    if after is None:
        out["y"] = total * g, (t + U) * size * abs(g)
        return out
    out["after"] = (total * g * y * ry).sum(0), tr * (size * abs(g * y) * ry).sum(0)
    v = total * g * w
    k = ry * ry * (v * y).mean(1, keepdims=True)
    kk = ry * ry * (size * abs(g * w * y)).mean(1, keepdims=True)
    out["y"] = ry * (v - y * k), 2 * t * ry * (size * abs(g * w) + abs(y) * kk)
    return out


def close(got, want, tol, rounding):
    got = ref.f64(got).reshape(want.shape)
    bad = ~(abs(got - want) <= tol + rounding * (abs(want) + tol) + 1e-38)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], (tol + 0 * want)[bad][:4])


def rounding(t):
    return B16 if "bfloat16" in str(t.dtype) else U


class Case:
    """Inputs in odd places, with sentinels around them."""

    def __init__(self, torch, rows, cols, gates, after, before, stream, branch, weights, scale=1.0, seed=1):
        g = gen(torch, seed * 1000 + rows + cols)
        self.torch, self.rows, self.cols, self.scale = torch, rows, cols, scale
        self.sd, self.bd, self.wd = dt(torch, stream), dt(torch, branch), dt(torch, weights)

        def matrix(dtype, offset, gap, std=1.0):
            m, _ = placed(torch, rows, cols, dtype, offset, gap)
            m.copy_(randn(torch, g, rows, cols, std=std))
            return m

        self.x, self.y = matrix(self.sd, 3, 5, 2.0), matrix(self.bd, 1, 0)
        self.dh, self.dz = matrix(self.sd, 2, 9), matrix(self.bd, 7, 1)
        self.h = matrix(self.sd, 5, 2, 1.5)

        def vector(there, offset):
            return torch.cat([randn(torch, g, offset), 1 + 0.3 * randn(torch, g, cols)]).to(self.wd)[offset:] \
                if there else None

        self.after, self.before = vector(after, 1), vector(before, 3)
        self.gate = None
        if gates:
            self.gate, _ = placed(torch, gates, cols, self.wd, 1, 3)
            self.gate.copy_(randn(torch, g, gates, cols))

    def ref(self, name):
        t = getattr(self, name)
        return None if t is None else ref.f64(t)

    def out(self, dtype, rows=None, value=7.0):
        return placed(self.torch, self.rows if rows is None else rows, self.cols, dtype, 3, 5, value)


SIZES = [(1, 1), (1, 100), (3, 7), (5, 64), (6, 65), (4, 513), (57, 1000), (12, 1025), (33, 2049), (6, 4097),
         (4, 8193), (3, 16390), (300, 24), (1000, 130)]
PARTS = [(0, True, True), (1, True, True), ("all", True, False), ("some", False, True), (1, False, False)]
TYPES = [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "bf16", "f32"), ("bf16", "f32", "bf16")]


def gates_of(kind, rows):
    if kind == "all":
        return rows
    if kind == "some":   # groups that begin and end anywhere in the workers' rows
        return next((d for d in (7, 5, 3, 2) if rows % d == 0), 1)
    return kind


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("gates,after,before", PARTS)
@pytest.mark.parametrize("stream,branch,weights", TYPES)
def test_residual_norm(torch, learner, rows, cols, gates, after, before, stream, branch, weights):  # noqa: F811
    c = Case(torch, rows, cols, gates_of(gates, rows), after, before, stream, branch, weights, 1.25)
    (out, buf), (normed, nbuf) = c.out(c.sd), c.out(c.bd)
    h, z = learner.residual_norm(c.x, c.y, c.gate, c.after, c.before, c.scale, EPS, out=out,
                                 normed_out=normed if before else None)
    assert h is out and (z is normed if before else z is None)
    wh, wz, th, tz = forward(*(c.ref(k) for k in ("x", "y", "gate", "after", "before")), c.scale)
    close(h, wh, th, rounding(h))
    if before:
        close(z, wz, tz, rounding(z))
    for t, b in ((out, buf), (normed, nbuf)):   # nothing around them
        t.fill_(7.0)
        assert bool((b == 7.0).all())
    h2, z2 = learner.residual_norm(c.x, c.y, c.gate, c.after, c.before, c.scale, EPS)
    assert h2.dtype == c.sd and (z2 is None or z2.dtype == c.bd)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("stream,branch,weights", TYPES)
def test_rms_norm(torch, learner, rows, cols, stream, branch, weights):  # noqa: F811
    c = Case(torch, rows, cols, 0, False, True, stream, branch, weights)
    out, buf = c.out(c.bd)
    assert learner.rms_norm(c.x, c.before, EPS, out=out) is out
    _, want, _, tol = forward(c.ref("x"), None, None, None, c.ref("before"), 1.0)
    close(out, want, tol, rounding(out))
    out.fill_(7.0)
    assert bool((buf == 7.0).all())
    z = learner.rms_norm(c.x, None, EPS, dtype=c.bd)
    _, want, _, tol = forward(c.ref("x"), None, None, None, None, 1.0)
    close(z, want, tol, rounding(z))
    assert learner.rms_norm(c.x, c.before).dtype == c.sd
    # backward, with and without what else is known of the stream's gradient
    for dh in (None, c.dh):
        (dx, xbuf), (dw, wbuf) = c.out(c.sd), placed(torch, 1, cols, torch.float32, 1, 0, 7.0)
        got = learner.rms_norm_grad(c.h, c.before, c.dz, EPS, stream_grad=dh, x_out=dx, weight_out=dw[0])
        assert got[0] is dx and got[1].data_ptr() == dw.data_ptr()
        want = backward(c.ref("h"), None, None if dh is None else c.ref("dh"), c.ref("dz"), None, None,
                        c.ref("before"), 1.0)
        close(dx, *want["x"], rounding(dx))
        close(dw[0], *want["before"], U)
        for t, b in ((dx, xbuf), (dw, wbuf)):
            t.fill_(7.0)
            assert bool((b == 7.0).all())


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("gates,after,before", PARTS)
@pytest.mark.parametrize("stream,branch,weights", TYPES)
def test_residual_norm_grad(torch, learner, rows, cols, gates, after, before, stream, branch, weights):  # noqa: F811
    gates = gates_of(gates, rows)
    c = Case(torch, rows, cols, gates, after, before, stream, branch, weights, 1.25)
    want = backward(c.ref("h"), c.ref("y"), c.ref("dh"), c.ref("dz") if before else None, c.ref("gate"),
                    c.ref("after"), c.ref("before"), c.scale)
    args = (c.h, c.y, c.dh, c.dz if before else None, c.gate, c.after, c.before, c.scale, EPS)
    got = learner.residual_norm_grad(*args, weight_dtype=c.wd)
    for name, t in got._asdict().items():
        assert (t is not None) == (name in want), name
        if t is not None:
            assert t.dtype == {"x": c.sd, "y": c.bd}.get(name, c.wd) and t.is_contiguous()
            close(t, *want[name], rounding(t))
    again = learner.residual_norm_grad(*args, weight_dtype=c.wd)
    assert all(a is None or torch.equal(a, b) for a, b in zip(got, again))
    # into places of the caller's, nothing around them; the vectors' added to what is there
    outs = {"x": c.out(c.sd), "y": c.out(c.bd), "gate": c.out(torch.float32, gates, 2.0),
            "after": placed(torch, 1, cols, torch.float32, 1, 0, 2.0),
            "before": placed(torch, 1, cols, torch.float32, 1, 0, 2.0)}
    given = {f"{k}_out": v[0] if k in ("x", "y", "gate") else v[0][0] for k, v in outs.items() if k in want}
    learner.residual_norm_grad(*args, accumulate=True, **given)
    for name in want:
        t, buf = outs[name]
        value, tol = want[name]
        if name not in ("x", "y"):
            value, tol = value + 2.0, tol + 2 * U * (abs(value) + 2.0)
        close(t, value, tol, rounding(t))
        fill = float(buf[0])
        t.fill_(fill)
        assert bool((buf == fill).all())


def test_gradients_are_differences(torch, learner):  # noqa: F811
    """sum(h dh) + sum(z dz) along directions of each argument, by central differences of the forward formulas in 64
    bits, which err by eps^2 times a third derivative (here below 1e-8 of the sums' magnitudes)."""
    c = Case(torch, 21, 70, 7, True, True, "f32", "f32", "f32", 1.25)
    args = {k: c.ref(k) for k in ("x", "y", "gate", "after", "before")}
    h = forward(*args.values(), c.scale)[0]
    dh, dz = c.ref("dh"), c.ref("dz")
    got = learner.residual_norm_grad(torch.from_numpy(h).float().cuda(), c.y, c.dh, c.dz, c.gate, c.after, c.before,
                                     c.scale, EPS)
    rng = np.random.default_rng(4)
    want = backward(h, args["y"], dh, dz, args["gate"], args["after"], args["before"], c.scale)
    for name, grad in got._asdict().items():
        d, step = rng.standard_normal(args[name].shape), 1e-5
        ends = []
        for sign in (1, -1):
            moved = dict(args, **{name: args[name] + sign * step * d})
            a, b = forward(*moved.values(), c.scale)[:2]
            ends.append((a * dh).sum() + (b * dz).sum())
        size = abs(h * dh).sum() + abs(dz).sum()
        # h is rounded to fp32 once before the backward pass: 2 u of every term more
        tol = ((want[name][1] + 4 * U * abs(want[name][0])) * abs(d)).sum() + 1e-8 * size
        assert abs((ref.f64(grad) * d).sum() - (ends[0] - ends[1]) / (2 * step)) <= tol, name


def test_rows_of_zeros_and_not_finite(torch, learner):  # noqa: F811
    x = torch.randn(6, 300, device="cuda")
    y = torch.randn(6, 300, device="cuda")
    w = torch.rand(300, device="cuda") + 0.5
    x[0], y[0] = 0, 0            # padding
    y[1] = 0
    y[2, 5] = float("nan")
    x[3, 299] = float("inf")
    h, z = learner.residual_norm(x, y, after=w, before=w)
    assert bool((h[0] == 0).all() and (z[0] == 0).all()) and torch.equal(h[1], x[1])
    assert bool(h[2].isnan().all() and z[2].isnan().all())
    assert bool(h[3, :299].isfinite().all()) and float(h[3, 299]) == float("inf") and bool(z[3, 299].isnan())
    # other rows are what they are without these
    h2, z2 = learner.residual_norm(x[4:], y[4:], after=w, before=w)
    assert torch.equal(h[4:], h2) and torch.equal(z[4:], z2)
    x[2:4], y[2:4] = 0, 0
    h = learner.residual_norm(x, y, after=w)[0]
    g = learner.residual_norm_grad(h, y, torch.ones_like(h), torch.ones_like(h), after=w, before=w)
    assert all(t is None or bool(t.isfinite().all()) for t in g)
    assert bool((g.y[1] != 0).any())   # a row of zeros has a gradient
    alone = learner.residual_norm_grad(h[4:], y[4:], torch.ones_like(h[4:]), torch.ones_like(h[4:]), after=w, before=w)
    assert torch.equal(g.x[4:], alone.x) and torch.equal(g.y[4:], alone.y)
    # a NaN in a row: its own gradients, and the vectors'
    y[3, 0] = float("nan")
    g = learner.residual_norm_grad(h, y, torch.ones_like(h), torch.ones_like(h), after=w, before=w)
    assert bool(g.y[3].isnan().all() and g.after.isnan().all() and g.before.isfinite().all())
    assert bool(g.x.isfinite().all()) and torch.equal(g.y[4:], alone.y)


@pytest.mark.parametrize("cols", [5, 300, 301, 9000])
def test_infinities_that_no_gradient_depends_on(torch, learner, cols):  # noqa: F811
    """Without a norm before the next block the stream's gradient does not depend on the stream, without one after
    this block its output's not on the output."""
    g = gen(torch, cols)
    h, y, dh, dz = (randn(torch, g, 7, cols) for _ in range(4))
    gate, w = randn(torch, g, cols), randn(torch, g, cols)
    h[1, 2] = h[2, 0] = float("inf")
    h[3, cols - 1] = float("nan")
    got = learner.residual_norm_grad(h, y, dh, gate=gate, after=w)
    clean = learner.residual_norm_grad(torch.zeros_like(h), y, dh, gate=gate, after=w)
    assert torch.equal(got.x, dh)
    assert all(torch.equal(a, b) for a, b in zip(got[1:4], clean[1:4]))
    y[1, 1], y[4, 3] = float("nan"), float("-inf")
    for next_norm in ({}, {"normed_grad": dz, "before": w}):
        finite = torch.ones_like(h)
        got = learner.residual_norm_grad(finite, y, dh, gate=gate, **next_norm)
        clean = learner.residual_norm_grad(finite, torch.zeros_like(y), dh, gate=gate, **next_norm)
        assert torch.equal(got.x, clean.x) and torch.equal(got.y, clean.y)


def test_no_rows_and_no_columns(torch, learner):  # noqa: F811
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.ones(0, 40, device="cuda", dtype=dtype)
        w = torch.ones(40, device="cuda")
        h, z = learner.residual_norm(x, x, w, w, w)
        assert h.shape == z.shape == (0, 40) and learner.rms_norm(x, w).shape == (0, 40)
        gate = torch.ones(3, 40, device="cuda")
        g = learner.residual_norm_grad(x, x, x, x, gate, w, w)
        assert g.x.shape == (0, 40) and all(bool((t == 0).all()) for t in (g.gate, g.after, g.before))
        old = [torch.full_like(t, 3.0) for t in (gate, w, w)]
        learner.residual_norm_grad(x, x, x, x, gate, w, w, gate_out=old[0], after_out=old[1], before_out=old[2],
                                   accumulate=True)
        assert all(bool((t == 3).all()) for t in old)
        x = torch.ones(5, 0, device="cuda", dtype=dtype)
        w = torch.ones(0, device="cuda")
        h, z = learner.residual_norm(x, x, None, w, w)
        assert h.shape == z.shape == (5, 0) and learner.rms_norm_grad(x, w, x)[1].shape == (0,)


def test_many_rows_of_few_columns(torch, learner):  # noqa: F811
    """More rows than workers have at once, gates that end inside them; whole numbers are summed exactly."""
    rows, cols = 70_001 * 3, 8
    g = gen(torch, 8)
    y = torch.randint(-2, 3, (rows, cols), generator=g, device="cuda").float()
    dh = torch.randint(-2, 3, (rows, cols), generator=g, device="cuda").float()
    for gates in (1, 3, 70_001, rows):
        gate = torch.randint(1, 3, (gates, cols), generator=g, device="cuda").float()
        got = learner.residual_norm_grad(y, y, dh, None, gate)
        assert torch.equal(got.gate, (dh * y).view(gates, -1, cols).sum(1))
        assert torch.equal(got.y, dh * gate.repeat_interleave(rows // gates, 0)) and torch.equal(got.x, dh)


def test_types_of_gate_and_gradients(torch, learner):  # noqa: F811
    """A gate of another type than the norms' weights, gradients of another than either."""
    for gate_type, weight_type, out_type in (("bf16", "f32", "f32"), ("f32", "bf16", "bf16"), ("bf16", "f32", "bf16")):
        c = Case(torch, 30, 77, 6, True, True, "bf16", "bf16", weight_type)
        c.gate = c.gate.to(dt(torch, gate_type))
        h, z = learner.residual_norm(c.x, c.y, c.gate, c.after, c.before, 1.0, EPS)
        wh, wz, th, tz = forward(*(c.ref(k) for k in ("x", "y", "gate", "after", "before")), 1.0)
        close(h, wh, th, B16)
        close(z, wz, tz, B16)
        got = learner.residual_norm_grad(c.h, c.y, c.dh, c.dz, c.gate, c.after, c.before, 1.0, EPS,
                                         weight_dtype=dt(torch, out_type))
        want = backward(c.ref("h"), c.ref("y"), c.ref("dh"), c.ref("dz"), c.ref("gate"), c.ref("after"),
                        c.ref("before"), 1.0)
        for name, t in got._asdict().items():
            close(t, *want[name], rounding(t))


def test_offsets_past_32_bits(torch, learner):  # noqa: F811
    """Matrices of more than 2^32 elements: the last rows as by themselves, sums over all rows of whole numbers
    exactly."""
    cols = 8192
    rows = (1 << 32) // cols + 1029
    x = torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16)
    y = torch.zeros_like(x)
    last = slice(rows - 1024, rows)
    g = gen(torch, 1)
    x[last], y[last] = randn(torch, g, 1024, cols), randn(torch, g, 1024, cols)
    w = torch.ones(cols, device="cuda")
    h, z = learner.residual_norm(x, y, after=w, before=w)
    h1, z1 = learner.residual_norm(x[last], y[last], after=w, before=w)
    assert torch.equal(h[last], h1) and torch.equal(z[last], z1) and bool((h[:5] == 0).all())
    del h, z
    y.fill_(1.0)
    got = learner.residual_norm_grad(x, y, y, None, w)
    assert bool((got.gate == rows).all()) and bool((got.y[last] == 1).all()) and bool((got.x[last] == 1).all())


def test_streams_and_graphs(torch, learner):  # noqa: F811
    """Captured once, replayed on new inputs, with eager work between; two graphs that run at once share nothing."""
    c = Case(torch, 130, 700, 13, True, True, "bf16", "bf16", "f32")
    seeds = (1, 2, 3)

    def fill(s):
        for i, t in enumerate((c.x, c.y, c.dh, c.dz)):
            t.copy_(randn(torch, gen(torch, 10 * s + i), c.rows, c.cols))

    def run():
        h, z = learner.residual_norm(c.x, c.y, c.gate, c.after, c.before)
        return (h, z, *learner.residual_norm_grad(h, c.y, c.dh, c.dz, c.gate, c.after, c.before))

    want = {}
    for s in seeds:
        fill(s)
        want[s] = [t.clone() for t in run()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for a, b in zip(run(), want[seeds[-1]]):
            assert torch.equal(a, b)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        graphs.append((graph, out))
    for s in seeds + seeds:
        fill(s)
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        graphs[0][0].replay()
        with torch.cuda.stream(other):
            graphs[1][0].replay()
        eager = run()
        torch.cuda.synchronize()
        for got in (*(g[1] for g in graphs), eager):
            assert all(torch.equal(a, b) for a, b in zip(got, want[s]))


def test_refusals(torch, learner):  # noqa: F811
    x = torch.zeros(6, 20, device="cuda")
    w = torch.ones(20, device="cuda")
    bad = [
        (TypeError, lambda: learner.rms_norm(x.half(), w)),
        (TypeError, lambda: learner.rms_norm(x, w.half())),
        (TypeError, lambda: learner.rms_norm(x, w, dtype=torch.float16)),
        (TypeError, lambda: learner.rms_norm(x, w, dtype=torch.bfloat16, out=x.clone())),
        (ValueError, lambda: learner.rms_norm(x, w[1:])),
        (ValueError, lambda: learner.rms_norm(x.t(), w[:6])),
        (ValueError, lambda: learner.rms_norm(x[0], w)),
        (ValueError, lambda: learner.rms_norm(x.cpu(), w)),
        (ps_error(), lambda: learner.rms_norm(x, w, out=x)),
        (ps_error(), lambda: learner.rms_norm(x, w, eps=0.0)),
        (ps_error(), lambda: learner.rms_norm(x, w, eps=float("nan"))),
        (ps_error(), lambda: learner.rms_norm(torch.ones(1, 20, device="cuda").expand(6, 20), w)),
        (ValueError, lambda: learner.residual_norm(x, x[1:].clone())),
        (TypeError, lambda: learner.residual_norm(x, x.clone(), after=w, before=w.bfloat16())),
        (ValueError, lambda: learner.residual_norm(x, x.clone(), normed_out=x.clone())),
        (ps_error(), lambda: learner.residual_norm(x, x.clone(), gate=torch.ones(4, 20, device="cuda"))),
        (ValueError, lambda: learner.residual_norm(x, x.clone(), gate=torch.ones(6, 19, device="cuda"))),
        (ps_error(), lambda: learner.residual_norm(x, x.clone(), out=x)),
        (TypeError, lambda: learner.residual_norm(x, x.clone(), out=x.bfloat16())),
        (ps_error(), lambda: learner.residual_norm_grad(x, x.clone(), None)),
        (TypeError, lambda: learner.residual_norm_grad(x, None, x)),
        (TypeError, lambda: learner.residual_norm_grad(x, x.clone(), x.bfloat16())),
        (TypeError, lambda: learner.residual_norm_grad(x, x.clone(), x, x.bfloat16(), before=w)),
        (ValueError, lambda: learner.residual_norm_grad(x, x.clone(), x, before=w)),
        (ValueError, lambda: learner.residual_norm_grad(x, x.clone(), x, after_out=w.clone())),
        (ValueError, lambda: learner.residual_norm_grad(x, x.clone(), x, after=w, accumulate=True)),
        (ValueError, lambda: learner.residual_norm_grad(x, x.clone(), x, after=w, after_out=w[1:])),
        (TypeError, lambda: learner.residual_norm_grad(x, x.clone(), x, x.clone(), after=w, before=w,
                                                       after_out=w.clone(), before_out=w.bfloat16())),
        (ps_error(), lambda: learner.residual_norm_grad(x, x.clone(), x, after=w, after_out=w)),
        (ps_error(), lambda: learner.residual_norm_grad(x, x.clone(), x, x_out=x)),
    ]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()


def ps_error():
    from paper_1611_06213_amd import ps
    return ps.PSError


def test_gates_without_rows_or_columns(torch, learner):  # noqa: F811
    """A gate of no rows is none at all only where the stream has none either; one of no columns has nothing to say."""
    x, y = torch.ones(6, 20, device="cuda"), torch.ones(6, 20, device="cuda")
    none = torch.ones(0, 20, device="cuda")
    for call in (lambda: learner.residual_norm(x, y, none),
                 lambda: learner.residual_norm(x, y, none, before=torch.ones(20, device="cuda")),
                 lambda: learner.residual_norm_grad(x, y, x, gate=none),
                 lambda: learner.residual_norm_grad(x, y, x, gate=none, gate_out=none.clone())):
        with pytest.raises(ps_error(), match="0 rows"):
            call()
    for dtype in (torch.float32, torch.bfloat16):
        e = torch.ones(0, 20, device="cuda", dtype=dtype)
        h, z = learner.residual_norm(e, e, none)
        assert h.shape == (0, 20) and z is None
        assert learner.residual_norm_grad(e, e, e, gate=none).gate.shape == (0, 20)
        e = torch.ones(6, 0, device="cuda", dtype=dtype)
        for gate in (torch.ones(0, device="cuda"), torch.ones(3, 0, device="cuda")):
            h, z = learner.residual_norm(e, e, gate)
            assert h.shape == (6, 0) and z is None
            assert learner.residual_norm_grad(e, e, e, gate=gate).gate.shape == gate.shape


@pytest.mark.parametrize("cols", [5, 300, 301, 9000])
@pytest.mark.parametrize("eps", [2.0 ** -126, 1e-40, 2.0 ** -149])
def test_rows_of_zeros_with_a_small_eps(torch, learner, monkeypatch, cols, eps):  # noqa: F811
    """Whose norm's factor is up to 2^74.5, and its square past fp32's range."""
    eps = float(np.float32(eps))
    monkeypatch.setitem(globals(), "EPS", eps)
    c = Case(torch, 6, cols, 3, True, True, "f32", "f32", "f32", 1.25)
    c.h[0], c.h[3], c.y[1], c.y[5] = 0, 0, 0, 0
    want = backward(c.ref("h"), c.ref("y"), c.ref("dh"), c.ref("dz"), c.ref("gate"), c.ref("after"), c.ref("before"),
                    c.scale)
    got = learner.residual_norm_grad(c.h, c.y, c.dh, c.dz, c.gate, c.after, c.before, c.scale, eps)
    for name, t in got._asdict().items():
        close(t, *want[name], rounding(t))
    z = learner.rms_norm(c.h, c.before, eps)
    assert bool((z[0] == 0).all()) and bool(z.isfinite().all())

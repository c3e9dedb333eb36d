"""The text classifier with residual blocks, AdamW learners and answers in 8-bit integers: every part against the
formulas in 64 bits, stage by stage, each from the device's own results of the stage before (which equal calls give
again to the bit). Tolerances are those of the operators (test_gpu_learner, test_gpu_norms, test_gpu_int8, adamw_ref)."""
import numpy as np
import pytest

from tests import adamw_ref
from tests import learner_ref as ref
from tests import test_gpu_int8 as int8
from tests import test_gpu_norms as norms
from tests.test_gpu_learner import B16, U, torch  # noqa: F401
from tests.test_gpu_train_text import product

pytestmark = pytest.mark.gpu


def vectors(v, i):
    """(gate, after, the next block's before) of block i in 64 bits."""
    return (ref.f64(v[f"block{i}.gate"])[None], ref.f64(v[f"block{i}.after"]),
            ref.f64(v[f"block{i + 1}.before"]) if f"block{i + 1}.before" in v else None)


@pytest.fixture()
def eps(monkeypatch):
    monkeypatch.setattr(norms, "EPS", 1e-6)   # the operators' own


def shape_of(tt):
    return tt.Shape(vocab=301, words=5, dim=37, hidden=132, classes=11, drop=0.25, blocks=2)


def test_gradient_row_through_blocks(torch, eps):  # noqa: F811
    from paper_1611_06213_amd import learner
    from paper_1611_06213_amd import train_text as tt
    shape = shape_of(tt)
    n, b = shape.params(), 64
    w = tt.initial_weights(shape, 3)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    for name, v in shape.views(w).items():   # vectors that tell gradients apart
        if v.dim() == 1:
            v += 0.3 * torch.randn(v.shape, generator=gen, device="cuda")
    pad = torch.full((n + 7,), 9.0, device="cuda")
    row = pad[3:3 + n]   # it starts at an odd element
    t = tt.TextLearner(shape, w, row, seed=5)
    t.refresh()
    tokens, labels = tt.Texts(shape, 3).batch(b)
    drops = t.drops()
    t.calls = 0
    t.gradient(tokens, labels)
    assert bool((pad[:3] == 9).all() and (pad[3 + n:] == 9).all())

    kept = []
    x, h, d, logits = t.forward(tokens, drops, kept)
    v, g = shape.views(w), shape.views(row)
    s, z = d, None
    for i, (si, zi, yi) in enumerate(kept[:-1]):
        assert torch.equal(si, s)
        if i == 0:   # the first norm has no block before it
            _, want, _, tol = norms.forward(ref.f64(s), None, None, None, ref.f64(v["block0.before"]), 1.0)
            norms.close(zi, want, tol, B16)
        else:
            assert torch.equal(zi, z)
        wq = ref.values(v[f"block{i}.weight"], True)
        y = ref.values(zi) @ wq.T + ref.f64(v[f"block{i}.bias"])
        size = np.abs(ref.values(zi)) @ np.abs(wq).T
        assert (np.abs(ref.f64(yi) - np.maximum(y, 0)) <= 2.0 ** -15 * size + np.abs(y) * 2.0 ** -8).all()
        gate, after, before = vectors(v, i)
        wh, wz, th, tz = norms.forward(ref.f64(s), ref.f64(yi), gate, after, before, 1.0)
        s, z = learner.residual_norm(s, yi, **t.vectors(i))
        norms.close(s, wh, th, B16)
        if before is not None:
            norms.close(z, wz, tz, B16)
    assert torch.equal(kept[-1], s) and z is None
    product(logits - v["fc2.bias"], ref.values(s), ref.values(v["fc2.weight"], True))

    dz = torch.log_softmax(logits, 1).exp()
    dz[torch.arange(b), labels] -= 1
    dz /= b
    product(g["fc2.weight"], ref.values(dz.t()), ref.values(s.t()))
    ds, _ = learner.linear_fp8_grad(s, dz, t.fc2_t)
    dn = None
    for i in (1, 0):
        si, zi, yi = kept[i]
        gate, after, before = vectors(v, i)
        want = norms.backward(ref.f64(kept[i + 1][0] if i == 0 else kept[-1]), ref.f64(yi), ref.f64(ds),
                              None if dn is None else ref.f64(dn), gate, after, before, 1.0)
        got = learner.residual_norm_grad(kept[i + 1][0] if i == 0 else kept[-1], yi, ds, dn, **t.vectors(i))
        norms.close(got.x, *want["x"], B16)
        norms.close(got.y, *want["y"], B16)
        norms.close(g[f"block{i}.gate"], want["gate"][0][0], want["gate"][1][0], U)
        norms.close(g[f"block{i}.after"], *want["after"], U)
        if before is not None:
            norms.close(g[f"block{i + 1}.before"], *want["before"], U)
        dy = got.y * (yi > 0)
        assert torch.equal(g[f"block{i}.bias"], dy.float().sum(0))
        product(g[f"block{i}.weight"], ref.values(dy.t()), ref.values(zi.t()))
        dn, _ = learner.linear_fp8_grad(zi, dy, t.blocks[i][1])
        ds = got.x
    want = norms.backward(ref.f64(d), None, ref.f64(ds), ref.f64(dn), None, None, ref.f64(v["block0.before"]), 1.0)
    norms.close(g["block0.before"], *want["before"], U)
    dd, _ = learner.rms_norm_grad(d, v["block0.before"], dn, stream_grad=ds)
    norms.close(dd, *want["x"], B16)
    dh = learner.dropout(dd, drops[1]) * (h > 0)
    product(g["fc1.weight"], ref.values(dh.t()), ref.values(x.t()))


@pytest.mark.parametrize("bits", [8, 32])
def test_pushed_steps(torch, bits):  # noqa: F811
    """A learner's row after `step` is the AdamW step of its gradient, decay on matrices only."""
    from paper_1611_06213_amd import train_text as tt
    shape = shape_of(tt)
    w, row = tt.initial_weights(shape, 3), torch.zeros(shape.params(), device="cuda")
    t = tt.TextLearner(shape, w, row, seed=5)
    t.refresh()
    t.use_adamw(bits, 0.1)
    texts = tt.Texts(shape, 3)
    v = list(shape.views(w).values())
    want = adamw_ref.Reference([x.numel() for x in v], [0.1 if x.dim() == 2 else 0.0 for x in v], (0.9, 0.999), 1e-8,
                               bits, 5)
    for _ in range(2):
        t.gradient(*texts.batch(32))
        g = [ref.f64(x).reshape(-1) for x in shape.views(row).values()]
        t.step(0.01)
        steps = want.step([ref.f64(x).reshape(-1) for x in v], g, float(np.float32(0.01)))
        for x, (step, tol) in zip(shape.views(row).values(), steps):
            assert (np.abs(ref.f64(x).reshape(-1) - step) <= tol + U * (np.abs(step) + tol) + 1e-45).all()
    assert t.adamw.steps == 2


def test_answers(torch, eps):  # noqa: F811
    """Each layer against exact sums of its integers; a text's answer is the same alone and in any batch."""
    from paper_1611_06213_amd import learner
    from paper_1611_06213_amd import train_text as tt
    shape = shape_of(tt)
    w = tt.initial_weights(shape, 3)
    t = tt.Answers(shape, w)
    t.refresh()
    tokens, _ = tt.Texts(shape, 3).batch(200)
    logits = t.logits(tokens)
    for rows in (slice(0, 1), slice(7, 12), slice(150, 200)):
        assert torch.equal(t.logits(tokens[rows].contiguous()), logits[rows])
    v = shape.views(w)

    def layer(x, name, relu, got):
        want, tol = int8.product(*int8.integers(x), *int8.integers(v[name + ".weight"]), ref.f64(v[name + ".bias"]), relu)
        int8.close(got, want, tol)

    x = learner.embedding(tokens.view(-1), v["embedding"], dtype=torch.bfloat16).view(200, -1)
    d = learner.linear_int8(x, t.fc1, bias=v["fc1.bias"], relu=True)
    layer(x, "fc1", True, d)
    s, kept = t.stack(d, lambda i, z: learner.linear_int8(z, t.blocks[i], bias=v[f"block{i}.bias"], relu=True))
    for i, (_, z, y) in enumerate(kept):
        layer(z, f"block{i}", True, y)
    layer(s, "fc2", False, logits)


@pytest.mark.parametrize("adamw,lr", [(0, 0.02), (8, 0.001), (32, 0.001)])
def test_run(torch, adamw, lr):  # noqa: F811
    """It runs, and equal runs give equal bits."""
    from paper_1611_06213_amd import train_text as tt
    shape = tt.Shape(vocab=300, hidden=136, classes=10, blocks=2)
    a = tt.train(shape, learners=3, steps=12, batch=32, lr=lr, adamw=adamw, answers=64)
    assert bool(a[0].isfinite().all()) and 0 <= a[1] <= 1
    b = tt.train(shape, learners=3, steps=12, batch=32, lr=lr, adamw=adamw, answers=64)
    assert torch.equal(a[0], b[0]) and a[1] == b[1]

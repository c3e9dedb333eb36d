"""The text classifier: every part of a learner's gradient row against the formulas in 64 bits, and
a run.

The formulas are those of the 8-bit form (values rounded as tests/learner_ref.py rounds them), stage by
stage: each takes the device's own results of the stage before, which equal calls give again to the
bit. Tolerances are those of the operators (tests/test_gpu_learner.py)."""
import math

import numpy as np
import pytest

from tests import learner_ref as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    return torch


def product(got, a, b):
    """got = a b^T of 8-bit values a and b, summed in fp32."""
    tol = 4 * (a.shape[1] / 128 + 16) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)
    assert (np.abs(ref.f64(got) - a @ b.T) <= tol).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_gradient_row(torch, dtype):
    from paper_1611_06213_amd import learner
    from paper_1611_06213_amd import train_text as tt
    shape = tt.Shape(vocab=301, words=5, dim=37, hidden=130, classes=11, drop=0.25)
    n, b = shape.params(), 64
    w = tt.initial_weights(shape, 3).to(getattr(torch, dtype))
    pad = torch.full((n + 7,), 9.0, device="cuda")
    row = pad[3:3 + n]   # it starts at an odd element
    t = tt.TextLearner(shape, w, row, seed=5)
    t.refresh()
    tokens, labels = tt.Texts(shape, 3).batch(b)
    tokens[0, 0] = -1   # padding
    drops = t.drops()
    t.calls = 0
    loss = t.gradient(tokens, labels)
    assert bool((pad[:3] == 9).all() and (pad[3 + n:] == 9).all())

    x, h, d, logits = t.forward(tokens, drops)
    v = shape.views(w)
    want = ref.embedding(tokens, v["embedding"], 1.0, drops[0]).reshape(b, -1)
    assert (np.abs(ref.f64(x) - want) <= np.abs(want) * (3 * U + 2.0 ** -8)).all()
    z = ref.values(x) @ ref.values(v["fc1.weight"], True).T + ref.f64(v["fc1.bias"])
    size = np.abs(ref.values(x)) @ np.abs(ref.values(v["fc1.weight"], True)).T
    # bf16: the 8-bit instructions' sums (2^-15 of the magnitudes at most), then one rounding
    assert (np.abs(ref.f64(h) - np.maximum(z, 0)) <= 2.0 ** -15 * size + np.abs(z) * 2.0 ** -8).all()
    want = ref.drop(ref.f64(h), drops[1])
    assert (np.abs(ref.f64(d) - want) <= np.abs(want) * (3 * U + 2.0 ** -8)).all()
    product(logits - v["fc2.bias"].float(), ref.values(d), ref.values(v["fc2.weight"], True))
    assert abs(float(loss) - float(torch.nn.functional.cross_entropy(logits.double(), labels))) < 1e-5

    g = shape.views(row)
    dz = torch.log_softmax(logits, 1).exp()
    dz[torch.arange(b), labels] -= 1
    dz /= b
    product(g["fc2.weight"], ref.values(dz.t()), ref.values(d.t()))
    assert torch.equal(g["fc2.bias"], dz.sum(0))
    dd, _ = learner.linear_fp8_grad(d, dz, t.fc2_t)
    dh = learner.dropout(dd, drops[1]) * (h > 0)
    product(g["fc1.weight"], ref.values(dh.t()), ref.values(x.t()))
    assert torch.equal(g["fc1.bias"], dh.float().sum(0))
    dx, _ = learner.linear_fp8_grad(x, dh, t.fc1_t)
    want, size, count = ref.embedding_grad(tokens, dx.view(-1, shape.dim), shape.vocab, 1.0, drops[0])
    assert (np.abs(ref.f64(g["embedding"]) - want) <= (count[:, None] + 3) * U * size + 1e-44).all()


def test_run_learns(torch):
    """The loss falls below that of a guess, and equal runs give equal bits."""
    from paper_1611_06213_amd import train_text as tt
    shape = tt.Shape(vocab=500, hidden=200, classes=10)
    a = tt.train(shape, learners=3, steps=150, batch=64)
    assert bool(a.isfinite().all())
    assert float(a[-15:].mean()) < math.log(10) < float(a[:3].mean())
    assert torch.equal(a, tt.train(shape, learners=3, steps=150, batch=64))

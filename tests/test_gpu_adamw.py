"""AdamW on the GPU: states and what 8 bits keep of them to the bit, steps within their roundings (adamw_ref)."""
import numpy as np
import pytest

from tests import adamw_ref
from tests import learner_ref as ref
from tests.test_gpu_learner import B16, U, dt, gen, learner, randn, torch  # noqa: F401

pytestmark = pytest.mark.gpu




class Tensors:
    """Tensors one after another in a flat vector that begins at an odd element, sentinels around."""

    def __init__(self, torch, sizes, weights, grads, seed=1, gap=0):  # noqa: F811
        self.sizes = sizes
        total = sum(sizes) + gap * len(sizes)
        self.flat = [torch.full((total + 64,), 7.0, device="cuda", dtype=dt(torch, t)) for t in (weights, grads)]
        self.w, self.g, at = [], [], 3
        for i, n in enumerate(sizes):
            for views, flat, std in ((self.w, self.flat[0], 0.1), (self.g, self.flat[1], 1e-2)):
                views.append(flat[at:at + n])
                views[-1].copy_(randn(torch, gen(torch, 100 * seed + 2 * i), n, std=std))
            at += n + gap

    def around(self):
        for views, flat in ((self.w, self.flat[0]), (self.g, self.flat[1])):
            copy = flat.clone()
            at = 3
            for v in views:
                start = v.storage_offset()
                copy[start:start + v.numel()] = 7.0
                at += v.numel()
            assert bool((copy == 7.0).all())


def states(opt):
    return {k: v.cpu().numpy() for k, v in opt.state().items() if k != "steps"}


def same_states(opt, want):
    got = states(opt)
    if opt.bits == 32:
        pairs = ((got["m"], want.m), (got["v"], want.v))
    else:
        # a block that is NaN has any codes
        bad = [np.repeat(s == 255, 128) for s in (want.ms, want.vs)]
        pairs = ((np.where(bad[0], 0, got["m"]), np.where(bad[0], 0, want.m)),
                 (np.where(bad[1], 0, got["v"]), np.where(bad[1], 0, want.v)),
                 (got["m_scales"], want.ms), (got["v_scales"], want.vs))
    for a, b in pairs:
        assert np.array_equal(a, b, equal_nan=a.dtype == np.float32), (np.argwhere(a != b)[:4], a[a != b][:4], b[a != b][:4])


SIZES = [[1], [127], [128], [129, 1, 3], [1000, 10, 4097, 5], [2048, 2049, 4096], [300] * 70, [8193, 20001]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("weights,grads,push", [("f32", "f32", False), ("f32", "bf16", False), ("f32", "f32", True),
                                                ("bf16", "bf16", True), ("bf16", "f32", True),
                                                ("f32", "bf16", True)])
def test_steps(torch, learner, sizes, bits, weights, grads, push):  # noqa: F811
    t = Tensors(torch, sizes, weights, grads, gap=2)
    decay = [0.1 if i % 3 else 0.0 for i in range(len(sizes))]
    seed, betas, eps = (0xFEDCBA9876543210, (0.9, 0.999), 1e-8)
    opt = learner.AdamW(t.w, t.g, decay, betas, eps, bits, push, seed)
    want = adamw_ref.Reference(sizes, decay, betas, eps, bits, seed)
    lr, factor = 0.01, 0.75
    for k in range(4):
        for i, g in enumerate(t.g):   # gradients of different sizes, some zeros
            fresh = randn(torch, gen(torch, 1000 * k + i), g.numel(), std=10.0 ** (k - 2))
            g.copy_(torch.where(fresh.abs() < fresh.abs().mean() * 0.2, 0.0, fresh))
        w, g = [ref.f64(x) for x in t.w], [ref.f64(x) for x in t.g]
        opt.step(lr, factor)
        steps = want.step(w, g, float(np.float32(lr)), factor)
        same_states(opt, want)
        for i, (step, tol) in enumerate(steps):
            got = ref.f64((t.g if push else t.w)[i])
            value = step if push else w[i] - step
            unit = B16 if push and grads == "bf16" else U
            ok = abs(got - value) <= tol + unit * (abs(value) + tol) + 1e-45
            assert ok.all(), (k, i, np.argwhere(~ok)[:3], got[~ok][:3], value[~ok][:3])
            assert push or np.array_equal(ref.f64(t.g[i]), g[i])
            assert not push or np.array_equal(ref.f64(t.w[i]), w[i])
        t.around()
    assert opt.steps == 4
    # the values that the states stand for, tensor by tensor
    for dtype in (torch.float32, torch.bfloat16):
        m, v = opt.moments(dtype)
        if bits == 8:
            wm, wv = (adamw_ref.decode(want.m, want.ms, True), adamw_ref.decode(want.v, want.vs, False))
            assert np.array_equal(ref.f64(m), wm) and np.array_equal(ref.f64(v), wv)
        elif dtype == torch.float32:
            assert m is opt.m and v is opt.v
        for i, (a, b) in enumerate(zip(opt.views(m), t.w)):
            assert a.shape == b.shape and torch.equal(a, m[want.at[i]:want.at[i] + sizes[i]])


def test_large_parts(torch, learner):  # noqa: F811
    """A list large enough for the longer parts, in both forms: each tensor's states as in a list of its own."""
    sizes = [9_000_001, 100, 8_000_000]
    for bits in (8, 32):
        t = Tensors(torch, sizes, "f32", "bf16")
        before = [w.clone() for w in t.w]
        opt = learner.AdamW(t.w, t.g, 0.01, bits=bits, seed=5)
        opt.step(0.01)
        m, v = (opt.views(x) for x in opt.moments())
        for i, n in enumerate(sizes):
            w, g = before[i].clone(), t.g[i].clone()
            one = learner.AdamW([w], [g], 0.01, bits=32)
            one.step(0.01)
            assert torch.equal(w, t.w[i])
            a, b = one.moments()
            if bits == 32:
                assert torch.equal(m[i], a[:n]) and torch.equal(v[i], b[:n])
            else:   # within a code's spacing, 2^-3 of a value, or the least of the block
                blocks = torch.nn.functional.pad(a[:n], (0, -n % 128)).view(-1, 128).abs().amax(1)
                least = (blocks * 2.0 ** -17).repeat_interleave(128)[:n]
                assert bool(((m[i] - a[:n]).abs() <= a[:n].abs() / 8 + least).all())
                assert bool(((v[i] > 0) == (b[:n] > 0)).all())


def test_offsets_past_32_bits(torch, learner):  # noqa: F811
    """More than 2^32 elements: a tensor at the end as in a list of its own but for its random numbers, which go by
    its place."""
    if learner._native is False:
        pytest.skip("the same library calls")
    big, n = (1 << 32) + 5, 2900
    flat_w = torch.zeros(big + n, device="cuda", dtype=torch.bfloat16)
    flat_g = torch.zeros(big + n, device="cuda", dtype=torch.bfloat16)
    flat_w[big:] = randn(torch, gen(torch, 1), n)
    flat_g[big:] = randn(torch, gen(torch, 2), n)
    w, g = flat_w[big:].clone(), flat_g[big:].clone()
    opt = learner.AdamW([flat_w[:big], flat_w[big:]], [flat_g[:big], flat_g[big:]], 0.01, bits=8, push=True, seed=3)
    one = learner.AdamW([w], [g], 0.01, bits=8, push=True, seed=3)
    opt.step(0.01)
    one.step(0.01)
    assert torch.equal(flat_g[big:], g) and bool((flat_g[:1000] == 0).all()) and opt.steps == 1
    at = -(-big // 128) * 128
    assert torch.equal(opt.m_scales[at // 128:], one.m_scales)
    assert [adamw_word(j, 1, 3) for j in range(8)] == adamw_ref.random_words(8, 1, 3).tolist()
    padded = np.zeros(2944, np.float32)
    padded[:n] = np.float32(1 - 0.9) * ref.f64(randn(torch, gen(torch, 2), n).bfloat16()).astype(np.float32)
    codes, scales = adamw_ref.encode(padded, np.array([adamw_word(at + j, 1, 3) & 0xFFFF for j in range(2944)]), True)
    assert np.array_equal(opt.m[at:].cpu().numpy(), codes) and np.array_equal(one.m_scales.cpu().numpy(), scales)


def adamw_word(j, t, seed):
    """Word j & 3 of Philox4x32-7 of (j >> 2, t) and the seed, in Python's whole numbers."""
    c, k = [j >> 2 & 0xFFFFFFFF, j >> 34, t & 0xFFFFFFFF, t >> 32], [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(7):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [p1 >> 32 ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, p0 >> 32 ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c[j & 3]


def test_rounding_is_right_on_average(torch, learner):  # noqa: F811
    """m of a constant gradient after one step is 0.1 g; the mean of many roundings differs from it by five standard
    errors at most: a rounding's variance is at most a quarter of the spacing squared, the spacing 2^-3 of the value
    at most (numbers below the block's largest by less than 2^14)."""
    n = 1 << 20
    g = torch.full((n,), 0.0123, device="cuda")
    g[::128] = 1.0
    w = torch.zeros(n, device="cuda")
    opt = learner.AdamW([w], [g], 0.0, bits=8, seed=3)
    opt.step(0.0)
    m, v = opt.moments()
    for got, value in ((m, 0.1 * 0.0123), (v, 0.001 * 0.0123 ** 2)):
        x = got.view(-1, 128)[:, 1:].double()
        assert x.unique().numel() == 2   # its two neighbours
        assert abs(float(x.mean()) - value) <= 5 * (value / 8 / 2) / x.numel() ** 0.5 + 2.0 ** -16 * value
    # other steps and other seeds round otherwise
    again = learner.AdamW([w], [g], 0.0, bits=8, seed=4)
    again.step(0.0)
    assert not torch.equal(again.m, opt.m)


def test_not_finite(torch, learner):  # noqa: F811
    for bits in (8, 32):
        w, g = torch.ones(500, device="cuda"), torch.full((500,), 0.01, device="cuda")
        g[130], g[300] = float("nan"), float("inf")
        want = adamw_ref.Reference([500], [0.0], (0.9, 0.999), 1e-8, bits, 0)
        opt = learner.AdamW([w], [g], 0.0, bits=bits)
        opt.step(0.1)
        want.step([np.ones(500)], [ref.f64(g)], 0.1)
        same_states(opt, want)
        assert bool(w[130].isnan()) and bool(w[300].isnan()) and int(w.isnan().sum()) == 2   # inf / inf
        m, v = opt.moments()
        if bits == 8:   # the block's values are lost
            assert m[128:384].isnan().all() and v[128:384].isnan().all() and m[:128].isfinite().all()
            g.fill_(0.01)
            opt.step(0.1)
            assert bool(w[128:384].isnan().all()) and bool(w[:128].isfinite().all()) and bool(w[384:].isfinite().all())
        else:
            assert int(m.isnan().sum()) == 1 and int(m.isinf().sum()) == 1


def test_zero_gradients_and_small_numbers(torch, learner):  # noqa: F811
    """Elements far below their block's largest: a positive v stays positive, so no step is unbounded."""
    for bits in (8, 32):
        g = torch.full((256,), 1e-12, device="cuda")
        g[0], g[5], g[200:] = 1.0, 0.0, 0.0
        w = torch.zeros(256, device="cuda")
        opt = learner.AdamW([w], [g], 0.0, bits=bits, eps=1e-30, seed=9)
        want = adamw_ref.Reference([256], [0.0], (0.9, 0.999), 1e-30, bits, 9)
        for _ in range(6):
            opt.step(1.0)
            want.step([np.zeros(256)], [ref.f64(g)], 1.0)
        same_states(opt, want)
        v = opt.moments()[1]
        assert bool((v[1:5] > 0).all()) and float(v[5]) == 0
        assert bool(w.isfinite().all()) and float(w.abs().max()) < 60 and float(w[5]) == 0 and bool((w[200:] == 0).all())


@pytest.mark.parametrize("eps", [2.0 ** -30, 2.0 ** -31])
@pytest.mark.parametrize("beta2", [1 - 2.0 ** -18, 1 - 2.0 ** -28])
def test_second_moments_below_normal_numbers(torch, learner, beta2, eps):  # noqa: F811
    """v of 2^-127 to 2^-126 and less, multiplied by 2^18 and 2^28 in the first step: of a denominator with this eps
    more than a step's tolerance where the factor is large."""
    size = 1.9 * 2.0 ** -(50 if beta2 > 1 - 2.0 ** -20 else 55)
    g = size * torch.cat([torch.ones(64), 0.7 * torch.ones(64), 1e-3 * torch.ones(64)]).cuda()
    w = torch.zeros(192, device="cuda")
    opt = learner.AdamW([w], [g], 0.0, (0.0, beta2), eps)
    want = adamw_ref.Reference([192], [0.0], (0.0, beta2), eps, 32, 0)
    for _ in range(2):
        before = ref.f64(w)
        opt.step(1.0)
        (step, tol), = want.step([before], [ref.f64(g)], 1.0)
        same_states(opt, want)
        value = before - step
        assert (abs(ref.f64(w) - value) <= tol + U * (abs(value) + tol)).all()


def test_numbers_on_the_device_and_graphs(torch, learner):  # noqa: F811
    """lr and factor from device memory; a captured step counts on when it is replayed; two optimizers' graphs at
    once; a saved state goes on."""
    for bits in (8, 32):
        sizes = [1000, 257]
        lr, factor = torch.tensor([0.01], device="cuda"), torch.tensor(0.5, device="cuda")
        sides = [Tensors(torch, sizes, "f32", "f32", seed=2) for _ in range(3)]
        opts = [learner.AdamW(t.w, t.g, 0.01, bits=bits, seed=1) for t in sides]
        graphs = []
        for opt in opts[1:]:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                opt.step(lr, factor)
            graphs.append(graph)
        assert opts[1].steps == 0   # recorded, not made
        for k in range(5):
            lr.fill_(0.01 / (k + 1))
            for t in sides:
                for i, g in enumerate(t.g):
                    g.copy_(randn(torch, gen(torch, 10 * k + i), g.numel()))
            other = torch.cuda.Stream()
            other.wait_stream(torch.cuda.current_stream())
            graphs[0].replay()
            with torch.cuda.stream(other):
                graphs[1].replay()
            opts[0].step(float(lr), 0.5)
            torch.cuda.synchronize()
            for t in sides[1:]:
                assert torch.equal(t.flat[0], sides[0].flat[0])
        assert [o.steps for o in opts] == [5, 5, 5]
        fresh = Tensors(torch, sizes, "f32", "f32", seed=2)
        fresh.flat[0].copy_(sides[0].flat[0])
        fresh.flat[1].copy_(sides[0].flat[1])
        opt = learner.AdamW(fresh.w, fresh.g, 0.01, bits=bits, seed=1)
        opt.load(opts[0].state())
        opt.step(0.01)
        opts[0].step(0.01)
        assert torch.equal(fresh.flat[0], sides[0].flat[0]) and opt.steps == 6
        assert all(np.array_equal(a, b) for a, b in zip(states(opt).values(), states(opts[0]).values()))


def test_a_server_makes_pushed_steps(torch, learner):  # noqa: F811
    """A learner that pushes its steps to a server with lr 1 has its weights, to the bit, where another changes its own."""
    from paper_1611_06213_amd import ps
    n = 5000
    w0 = randn(torch, gen(torch, 1), n, std=0.1)
    own, og = w0.clone(), torch.zeros(n, device="cuda")
    direct = learner.AdamW([own[:3000], own[3000:]], [og[:3000], og[3000:]], 0.05, bits=8, seed=2)
    srv = ps.ParameterServer(n, 1.0, 0.0, queue_depth=1, stream=torch.cuda.current_stream())
    try:
        srv.set_weights(w0)
        row, replica = srv.alloc_rows(2)
        srv.pull_many([0], [replica])
        pushing = learner.AdamW([replica[:3000], replica[3000:]], [row[:3000], row[3000:]], 0.05, bits=8, push=True,
                                seed=2)
        for k in range(4):
            g = randn(torch, gen(torch, 50 + k), n)
            og.copy_(g)
            direct.step(0.01)
            row.copy_(g)
            pushing.step(0.01)
            srv.push(0, row)
            srv.apply_pull([0], [replica])
            srv.sync()
            assert torch.equal(replica, own)
    finally:
        srv.close()


def test_refusals(torch, learner):  # noqa: F811
    from paper_1611_06213_amd import ps
    w, g = torch.ones(100, device="cuda"), torch.ones(100, device="cuda")
    A = learner.AdamW

    def exchanged(bits, **parts):
        opt = A([w], [g], bits=bits)
        for k, t in parts.items():
            setattr(opt, k, t)
        return opt

    bad = [
        (ValueError, lambda: A([], [])),
        (ValueError, lambda: A([w], [])),
        (ValueError, lambda: A([w], [g[:99]])),
        (ValueError, lambda: A([w[::2]], [g[:50]])),
        (ValueError, lambda: A([w], [g], bits=16)),
        (ValueError, lambda: A([w], [g], seed=1 << 64)),
        (ValueError, lambda: A([w], [g], [0.1, 0.2])),
        (ValueError, lambda: A([w.cpu()], [g])),
        (TypeError, lambda: A([w.half()], [g])),
        (TypeError, lambda: A([w[:50], w[50:].bfloat16()], [g[:50], g[50:]], push=True)),
        (ps.PSError, lambda: A([w.bfloat16()], [g])),   # weights in bf16 would lose small steps
        (ps.PSError, lambda: A([w], [w])),
        (ps.PSError, lambda: A([w, w], [g, g.clone()])),
        (ps.PSError, lambda: A([w[:60], w[50:]], [g[:60], g[50:]])),
        (ps.PSError, lambda: A([w, w.clone()], [g, g], push=True)),
        (ps.PSError, lambda: A([w], [g], betas=(1.0, 0.9)).step(0.1)),
        (ps.PSError, lambda: A([w], [g], betas=(0.9, -0.1)).step(0.1)),
        (ps.PSError, lambda: A([w], [g], eps=float("nan")).step(0.1)),
        (TypeError, lambda: A([w], [g]).step(torch.tensor([0.1, 0.2], device="cuda"))),
        (TypeError, lambda: A([w], [g]).step(0.1, torch.tensor(1.0, device="cuda", dtype=torch.float64))),
        (ValueError, lambda: A([w], [g]).step(torch.tensor([0.1]))),
        (ValueError, lambda: A([w], [g]).load({"steps": 1})),
        (ValueError, lambda: A([w], [g]).load(A([w[:10]], [g[:10]]).state() | {"m": torch.zeros(1, device="cuda")})),
        (ValueError, lambda: A([w], [g], bits=8).load(A([w], [g]).state())),
        (TypeError, lambda: A([w], [g], bits=8).moments(torch.float16)),
        (ValueError, lambda: exchanged(8, m=torch.zeros(127, device="cuda", dtype=torch.uint8)).step(0.1)),
        (ValueError, lambda: exchanged(8, v_scales=torch.zeros(1, device="cuda")).step(0.1)),
        (ValueError, lambda: exchanged(32, v=torch.zeros(128, device="cuda", dtype=torch.bfloat16)).step(0.1)),
        (ValueError, lambda: exchanged(32, m=torch.zeros(128)).step(0.1)),
        (ValueError, lambda: exchanged(8, v=torch.zeros(256, device="cuda", dtype=torch.uint8)[::2]).moments()),
        (ValueError, lambda: exchanged(8, plan=torch.zeros(40, dtype=torch.uint8)).step(0.1)),
        (ValueError, lambda: exchanged(8, plan=torch.zeros(39, device="cuda", dtype=torch.uint8)).step(0.1)),
    ]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()
    assert bool((w == 1).all())
    # weights that share memory are only read with push; empty tensors take no part
    a, b = g.clone(), g.clone()
    A([w, w], [a, b], push=True).step(0.1)
    assert torch.equal(a, b)
    empty = A([w[:0]], [g[:0]])
    empty.step(0.1)
    assert empty.steps == 0 and empty.moments()[0].numel() == 0


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("grads,patterns", [
    ("f32", (0xFFFFFFFF, 0xFFF00001, 0xFFC00000, 0x7FFFFFFF, 0x7FC00000, 0xFF800000)),
    ("bf16", (0xFFFF, 0xFFF1, 0xFFC0, 0x7FFF, 0xFF80))])
@pytest.mark.parametrize("push", [False, True])
def test_not_finite_of_any_bits(torch, learner, bits, grads, patterns, push):  # noqa: F811
    """A NaN of any sign and payload, of memory filled with ones, say, and the lower infinity: products and sums keep
    a NaN's bits, so that they come to where a block's largest is found. The block of 8 bits is NaN, no other is."""
    kind = torch.int32 if grads == "f32" else torch.int16
    half = 1 << (31 if grads == "f32" else 15)
    for pattern in patterns:
        bad = pattern - 2 * half if pattern >= half else pattern
        for where in (slice(130, 131), slice(128, 256)):
            w, g = torch.ones(500, device="cuda"), torch.full((500,), 0.01, device="cuda", dtype=dt(torch, grads))
            g.view(kind)[where] = bad
            want = adamw_ref.Reference([500], [0.0], (0.9, 0.999), 1e-8, bits, 0)
            opt = learner.AdamW([w], [g], 0.0, bits=bits, push=push)
            before = ref.f64(g)
            opt.step(0.1)
            want.step([np.ones(500)], [before], 0.1)
            got = g if push else w
            assert bool(got[where].isnan().all()) and int(got.isnan().sum()) == where.stop - where.start, hex(pattern)
            m, v = opt.moments()
            if bits == 8:
                assert opt.v_scales.tolist()[1] == 255 and opt.m_scales.tolist()[1] == 255, hex(pattern)
                for x in (m, v):
                    assert bool(x[128:256].isnan().all()) and int(x.isnan().sum()) == 128, hex(pattern)
            same_states(opt, want)
            if push:
                g.fill_(0.01)
                opt.step(0.1)
                want.step([np.ones(500)], [ref.f64(torch.full_like(g, 0.01))], 0.1)
                same_states(opt, want)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("grads,push", [("f32", False), ("bf16", False), ("f32", True)])
def test_weights_past_the_caches(torch, learner, bits, grads, push):  # noqa: F811
    """Weights in 32 bits that do not fit in the last level (256 MB): the list's first elements as in a shorter list,
    whose weights do, states and codes to the bit over several steps, as random numbers go by an element's place; its
    last ones, of which the random numbers of 8 bits differ, for one step."""
    if learner._native is False:
        pytest.skip("the same library calls")
    big, first, last = 70_000_001, 128 * 20_003, 5003
    w = torch.randn(big + 129, generator=gen(torch, 1), device="cuda") * 0.1
    g = (torch.randn(big + 129, generator=gen(torch, 2), device="cuda") * 1e-2).to(dt(torch, grads))
    parts = [(slice(0, big), slice(big, big + 129)), (slice(0, first),),
             (slice(big - last, big), slice(big, big + 129))]
    flats = [(w.clone(), g.clone()) for _ in parts]
    opts = [learner.AdamW([a[s] for s in where], [b[s] for s in where], 0.05, bits=bits, push=push, seed=7)
            for (a, b), where in zip(flats, parts)]
    for k in range(3):
        if push:
            for _, b in flats:
                b.copy_(g).mul_(0.5 ** k)
        for opt in opts:
            opt.step(0.01, 0.5)
        (a, b), (a1, b1), (a2, b2) = flats
        out, out1, out2 = (b, b1, b2) if push else (a, a1, a2)
        assert torch.equal(out[:first], out1[:first]) and not torch.equal(out[:first], (g if push else w)[:first])
        if k == 0 or bits == 32:
            assert torch.equal(out[big - last:], out2[big - last:])
        room = first // 128
        for name, n in (("m", first), ("v", first), ("m_scales", room), ("v_scales", room))[:4 if bits == 8 else 2]:
            assert torch.equal(getattr(opts[0], name)[:n], getattr(opts[1], name)[:n]), name
        # what is only read
        assert torch.equal(a, w) if push else torch.equal(b, g)


@pytest.mark.parametrize("eps", [2.0 ** 100, 2.0 ** 101, 2.0 ** 126, 1e38, 3e38])
@pytest.mark.parametrize("bits", [8, 32])
def test_large_eps(torch, learner, eps, bits):  # noqa: F811
    """Denominators whose reciprocals are below 2^-126."""
    eps = float(np.float32(eps))
    g = randn(torch, gen(torch, 3), 300, std=1e17)
    w = torch.zeros(300, device="cuda")
    opt = learner.AdamW([w], [g], 0.0, (0.9, 0.99), eps, bits)
    want = adamw_ref.Reference([300], [0.0], (0.9, 0.99), eps, bits, 0)
    for _ in range(2):
        before = ref.f64(w)
        opt.step(1.0)
        (step, tol), = want.step([before], [ref.f64(g)], 1.0)
        same_states(opt, want)
        value, got = before - step, ref.f64(w)
        ok = abs(got - value) <= tol + U * (abs(value) + tol) + 1e-45
        assert ok.all(), (got[~ok][:3], value[~ok][:3])

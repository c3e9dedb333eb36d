"""Timed cases of more of a learner's operators: what a residual stack of fully
connected layers takes between a pull and a push, and when it answers.

The operators (`op` of a case):

  norm        the norms after and before a block: from the stream x and the block's
              output y,  h = scale x + gate * after * N(y),  z = before * N(h);
              without a block z = before * N(x) alone
  norm_grad   the gradients for x, y, gate, after and before from those of h and z
  linear      relu(x W^T + bias) in 8-bit integers, a scale per token (row of x) and
              per channel (row of W)
  adamw       one AdamW step over many tensors, states in 32 bits or in 8

Fields of a case:

  rows, cols          norm, norm_grad
  block               whether there is a y; after: whether it is normed
  gates               0: no gate; else the rows of the gate, each for rows / gates
                      neighbouring rows (1: one gate for all)
  scale               of x
  stream, branch      element types of x, h and of y, z: "f32" or "bf16"
  weights             type of gate, after, before
  m, n, k             linear: x is m x k, W n x k; x, out: element types
  sizes               adamw: elements of the tensors, which lie one after another in
                      the weights' and the gradients' vectors
  bits                of a state's element: 32 or 8
  push                the step is written in the gradient's place (for a server that
                      subtracts it) and the weights are only read
  weights, grad       adamw: element types

Definitions, exact up to the rounding of sums:

  N(v)      v / sqrt(mean(v^2) + EPS) over a row
  integers  a row's scale is max(|row|, 2^-100) / 127; its elements times 127 over
            that maximum are rounded to nearest even
  adamw     t = steps made + 1; m = B1 m + (1-B1) g; v = B2 v + (1-B2) g^2;
            step = LR (m / (1-B1^t) / (sqrt(v / (1-B2^t)) + EPS) + decay w); w -= step
            States lie tensor after tensor, each from a multiple of 128 elements on;
            what lies between is zeros.
  8 bits    for each 128 elements of m (v) a byte s: the exponent field of the block's
            largest magnitude as an fp32 number, plus 1 if its fraction is above 7/8.
            An element's code is that of |x| 2^(15-s) (v: 2^(31-s)) as an fp32
            number's bits, of which the upper 12 are kept (the upper 4 of those are
            zeros; m has a sign in the 8 bits' first): bits + 16 r, shifted by 20, where r is a
            16-bit random number. A positive v's code is 1 at least. Element j's
            r: word j & 3 of Philox4x32-7 (Salmon, Moraes, Dror, Shaw, 2011) with
            the counter (j >> 2 low, high, t low, high) and the key (seed low, high),
            its low half for m, its high half for v.

Sizes are those of the models in workloads.py and generic ones.
"""
import random

import torch

own = False

NORM_EPS = 1e-6
LR, B1, B2, EPS, DECAY, SEED = 1e-3, 0.9, 0.999, 1e-8, 0.01, 0x9E3779B97F4A7C15
# a drawn case: at most the work of the large listed ones
MAX_ROWS, MAX_COLS, MAX_ELEMENTS = 32768, 16384, 1 << 27
MAX_FLOPS, MAX_BYTES, MAX_WEIGHTS = 1.1e12, 1.6e9, 25088 * 4096
MAX_TENSORS, MAX_PARAMS = 256, 1 << 27
_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}


def _norm(op, rows, cols, block=True, after=True, gates=1, scale=1.0, stream="bf16", branch="bf16",
          weights="f32"):
    return {"op": op, "rows": rows, "cols": cols, "block": block, "after": after, "gates": gates,
            "scale": scale, "stream": stream, "branch": branch, "weights": weights}


def _linear(m, n, k, x="bf16", out="bf16"):
    return {"op": "linear", "m": m, "n": n, "k": k, "x": x, "out": out}


def _adamw(sizes, bits, push, weights="f32", grad="f32"):
    return {"op": "adamw", "sizes": ",".join(map(str, sizes)), "bits": bits, "push": push,
            "weights": weights, "grad": grad}


def _alexnet():
    convs = [(64, 3, 11), (192, 64, 5), (384, 192, 3), (256, 384, 3), (256, 256, 3)]
    full = [(4096, 9216), (4096, 4096), (1000, 4096)]
    return [n for o, i, k in convs for n in (o * i * k * k, o)] + [n for o, i in full for n in (o * i, o)]


def _vgg16():
    chans = [3, 64, 64, 128, 128, 256, 256, 256, 512, 512, 512, 512, 512, 512]
    full = [(4096, 25088), (4096, 4096), (1000, 4096)]
    return ([n for i, o in zip(chans, chans[1:]) for n in (9 * i * o, o)]
            + [n for o, i in full for n in (o * i, o)])


def listed():
    # train_text's classifier: embedding, two layers with biases
    classifier = [500000, 900000, 1000, 50000, 50]
    cases = {
        # one request's hidden units of the Text-CNN: the smallest call
        "norm_one": _norm("norm", 1, 1000, stream="f32", branch="f32"),
        # a batch of 57 of them, odd, fp32
        "norm_text": _norm("norm_grad", 57, 1000, stream="f32", branch="f32"),
        # behind fc7 of AlexNet or VGG-16 over a long batch: an fp32 stream past bf16 layers
        "norm_fc7": _norm("norm", 4096, 4096, gates=0, scale=1.4142135, stream="f32"),
        # a long batch, every part, gates of 32 sequences
        "norm_long": _norm("norm", 16384, 8192, gates=32, weights="bf16"),
        # and backward through the blocks of a 4096-wide stack
        "norm_grad_long": _norm("norm_grad", 16384, 4096, gates=32),
        # VGG-16 fc6 answering a single request
        "int8_one": _linear(1, 4096, 25088),
        # Text-CNN fc1 answering an odd batch of fp32 activations
        "int8_text": _linear(57, 1000, 900, x="f32", out="f32"),
        # AlexNet fc6 over a batch of 128
        "int8_batch": _linear(128, 4096, 9216),
        # the product at its largest
        "int8_large": _linear(8192, 8192, 8192),
        # the text classifier's learner, which pushes its steps
        "adamw_text": _adamw(classifier, 8, True),
        # AlexNet's tensors in 32 bits, fp32 throughout
        "adamw_alexnet": _adamw(_alexnet(), 32, False),
        # VGG-16's with states in 8 bits and bf16 gradients
        "adamw_vgg16": _adamw(_vgg16(), 8, False, grad="bf16"),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "linear", "adamw"])
    if op in ("norm", "norm_grad"):
        rows, cols = _log_int(rng, 1, MAX_ROWS), _log_int(rng, 8, MAX_COLS)
        while rows * cols > MAX_ELEMENTS // (2 if op == "norm_grad" else 1):
            rows = max(1, rows * 2 // 3)
        gates = rng.choice([0, 1, rows, rng.choice([d for d in range(1, rows + 1) if rows % d == 0])])
        block = rng.random() < 0.8
        stream = rng.choice(["f32", "bf16"])
        return _norm(op, rows, cols, block, block and rng.random() < 0.7, gates if block else 0,
                     rng.choice([1.0, 1.5]) if block else 1.0, stream, rng.choice([stream, "bf16"]),
                     rng.choice(["f32", "bf16"]))
    if op == "linear":
        wide = rng.choice(["f32", "bf16"])
        case = _linear(_log_int(rng, 1, 16384), _log_int(rng, 64, 25088), _log_int(rng, 64, 25088), wide,
                       rng.choice(["f32", "bf16"]))
        while (work(case)["flops"] > MAX_FLOPS or work(case)["bytes"] > MAX_BYTES
               or case["n"] * case["k"] > MAX_WEIGHTS):
            longest = max(("m", "n", "k"), key=case.get)
            case[longest] = case[longest] * 2 // 3
        return case
    count, params = _log_int(rng, 1, MAX_TENSORS), _log_int(rng, 1000, MAX_PARAMS)
    shares = [rng.random() ** 6 + 1e-6 for _ in range(count)]
    sizes = [max(1, int(params * s / sum(shares))) for s in shares]
    push = rng.random() < 0.5
    return _adamw(sizes, rng.choice([8, 32]), push, rng.choice(["f32", "bf16"]) if push else "f32",
                  rng.choice(["f32", "bf16"]))


def _sizes(case):
    return [int(n) for n in case["sizes"].split(",")]


def work(case):
    op = case["op"]
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k * _SIZE[case["x"]] + n * k + 8 * n + m * n * _SIZE[case["out"]],
                "flops": 2 * m * n * k}
    if op == "adamw":
        n = sum(_sizes(case))
        w, g = _SIZE[case["weights"]], _SIZE[case["grad"]]
        # weights, gradients; m and v read and written; in 8 bits their values too
        each = w + g + (g if case["push"] else w) + (16 if case["bits"] == 32 else 4 + 4 / 128 + 4)
        return {"bytes": n * each, "flops": 16 * n}
    rows, cols = case["rows"], case["cols"]
    x, y, w = _SIZE[case["stream"]], _SIZE[case["branch"]], _SIZE[case["weights"]]
    vectors = cols * (1 + case["after"] + case["gates"])
    if op == "norm":
        each = 2 * x + 2 * y if case["block"] else x + y
        return {"bytes": rows * cols * each + vectors * w, "flops": (14 if case["block"] else 5) * rows * cols}
    # h, dz, dx; with a block dh, y, dy too
    each = 3 * x + 3 * y if case["block"] else 2 * x + y
    return {"bytes": rows * cols * each + vectors * (w + 4), "flops": (30 if case["block"] else 10) * rows * cols}


# ----------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g)


def _matrix(g, rows, cols, std):
    """Columns of different sizes, as features are."""
    spread = torch.exp(_normal(g, cols, std=0.5))
    return _normal(g, rows, cols, std=std).mul_(spread)


def _layout(case, device="cuda"):
    """(elements of all tensors, elements of a state, where each tensor begins in the
    weights and in a state)."""
    sizes = torch.tensor(_sizes(case), dtype=torch.int64, device=device)
    room = (sizes + 127) // 128 * 128
    return int(sizes.sum()), int(room.sum()), sizes, sizes.cumsum(0) - sizes, room.cumsum(0) - room


def _places(case):
    """Where each element of the weights' vector is in a state, and its decay."""
    _, _, sizes, flat, padded = _layout(case)
    at = torch.arange(int(sizes.sum()), device="cuda") + (padded - flat).repeat_interleave(sizes)
    decay = torch.zeros(len(sizes), device="cuda")
    decay[::2] = DECAY   # weights have it, the biases behind them do not
    return at, decay.repeat_interleave(sizes)


def _inputs(case, seed):
    g = _gen(seed)
    op = case["op"]
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"x": _matrix(g, m, k, 1.0).to(_DT[case["x"]]),
                "w": _matrix(g, n, k, (2.0 / k) ** 0.5).to(torch.bfloat16),
                "bias": _normal(g, n, std=0.1)}
    if op == "adamw":
        n, room = _layout(case)[:2]
        s = {"w": _normal(g, n, std=0.05).to(_DT[case["weights"]]),
             "g": (_normal(g, n) * torch.exp(_normal(g, n)) * 1e-3).to(_DT[case["grad"]]),
             "steps": 100 + seed % 900}
        # what earlier gradients left: the states of steps made before
        at = _places(case)[0]
        spread = torch.exp(_normal(g, n)) * 1e-3
        m, v = torch.zeros(room, device="cuda"), torch.zeros(room, device="cuda")
        m[at] = _normal(g, n) * spread * 0.3
        v[at] = spread * spread * torch.exp(_normal(g, n, std=0.3))
        s["m"], s["v"] = m, v
        if case["bits"] == 8:
            half = torch.full((room,), 0x8000, dtype=torch.int32, device="cuda")
            s["m"], s["m_scales"] = _encode(m, half, True)
            s["v"], s["v_scales"] = _encode(v, half, False)
        return s
    rows, cols, x, y, w = (case[i] for i in ("rows", "cols", "stream", "branch", "weights"))
    s = {"x": _matrix(g, rows, cols, 2.0).to(_DT[x]), "before": (1 + _normal(g, cols, std=0.1)).to(_DT[w])}
    if case["block"]:
        s["y"] = _matrix(g, rows, cols, 0.5).to(_DT[y])
    if case["after"]:
        s["after"] = (1 + _normal(g, cols, std=0.1)).to(_DT[w])
    if case["gates"]:
        s["gate"] = _normal(g, case["gates"], cols, std=0.5).to(_DT[w])
    if op == "norm_grad":
        # x stands for h, the stream behind the block
        s["dz"] = _matrix(g, rows, cols, 1e-3).to(_DT[y])
        if case["block"]:
            s["dh"] = _matrix(g, rows, cols, 1e-3).to(_DT[x])
    return s


def prepare(case, seed):
    """The inputs, with a layer's weights as integers, as they are after a pull, and an
    optimizer's handle."""
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "linear":
        w = s.pop("w")
        if own:
            from paper_1611_06213_amd import learner
            s["w"] = learner.quantize_int8(w)
        else:
            s["w"] = _integers(w)
    if case["op"] == "adamw":
        if own:
            from paper_1611_06213_amd import learner
            sizes = _sizes(case)
            names = ("m", "v") if case["bits"] == 32 else ("m", "v", "m_scales", "v_scales")
            s["adamw"] = learner.AdamW(
                s["w"].split(sizes), s["g"].split(sizes),
                decay=[0.0 if i % 2 else DECAY for i in range(len(sizes))], betas=(B1, B2), eps=EPS,
                bits=case["bits"], push=case["push"], seed=SEED)
            s["adamw"].load({"steps": s.pop("steps"), **{k: s.pop(k) for k in names}})
        else:
            s["at"], s["decay"] = _places(case)
    return s


# ------------------------------------------------------------ plain forms

def _integers(x):
    """(integers, scale of each row)."""
    x = x.float()
    most = x.abs().amax(dim=1, keepdim=True).clamp(min=2.0 ** -100)
    return torch.round(x * (127 / most)).to(torch.int8), most / 127


def _plain_linear(s):
    q, scale = _integers(s["x"])
    w, w_scale = s["w"]
    y = (q.float() @ w.float().t()) * scale * w_scale.t() + s["bias"]
    return torch.clamp(y, min=0.0).to(_DT[s["case"]["out"]])


def _mulhilo(a, b):
    """High and low 32 bits of a * b for a constant a and a tensor b of 32-bit
    numbers held in 64."""
    low = a * (b & 0xFFFF)
    high = a * (b >> 16) + (low >> 16)
    return high >> 16, ((high & 0xFFFF) << 16) | (low & 0xFFFF)


def _random(count, t):
    """A 32-bit number for each of `count` elements (a multiple of 4), in 64 bits."""
    j = torch.arange(count // 4, device="cuda")
    c0, c1, c2, c3 = j & 0xFFFFFFFF, j >> 32, torch.full_like(j, t & 0xFFFFFFFF), torch.full_like(j, t >> 32)
    k0, k1 = SEED & 0xFFFFFFFF, SEED >> 32
    for _ in range(7):
        h0, l0 = _mulhilo(0xD2511F53, c0)
        h1, l1 = _mulhilo(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return torch.stack([c0, c1, c2, c3], dim=1).view(-1)


def _power(e):
    """2^e, exactly, in 64 bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _encode(x, r, signed):
    """(codes, a byte for each block) of x, a multiple of 128 elements in 32 bits."""
    x = x.view(-1, 128)
    most = x.abs().amax(dim=1).view(torch.int32)
    byte = (most + 0xFFFFF) >> 23
    scaled = (x.abs().double() * _power((15 if signed else 31) - byte)[:, None]).float()
    code = (scaled.view(torch.int32) + 16 * r.view(-1, 128)) >> 20
    code = code | ((x < 0) << 7) if signed else torch.maximum(code, (x > 0).int())
    return code.to(torch.uint8).view(-1), byte.to(torch.uint8)


def _decode(codes, scales, signed):
    c = codes.view(-1, 128).int()
    value = ((c & (127 if signed else 255)) << 20).view(torch.float32).double()
    value = (value * _power(scales.int() - (15 if signed else 31))[:, None]).float()
    return (torch.where(c > 127, -value, value) if signed else value).view(-1)


def _plain_adamw(s):
    case = s["case"]
    small = case["bits"] == 8
    t = s["steps"] = s["steps"] + 1
    at, w, g = s["at"], s["w"].float(), s["g"].float()
    m_all = _decode(s["m"], s["m_scales"], True) if small else s["m"]
    v_all = _decode(s["v"], s["v_scales"], False) if small else s["v"]
    m = B1 * m_all[at] + (1 - B1) * g
    v = B2 * v_all[at] + (1 - B2) * (g * g)
    up, root = 1 / (1 - B1 ** t), (1 / (1 - B2 ** t)) ** 0.5
    step = LR * (m * up / (torch.sqrt(v) * root + EPS) + s["decay"] * w)
    m_all[at], v_all[at] = m, v
    if case["push"]:
        s["g"].copy_(step)
    else:
        s["w"].copy_(w - step)
    if small:
        r = _random(m_all.numel(), t).int()
        s["m"], s["m_scales"] = _encode(m_all, r & 0xFFFF, True)
        s["v"], s["v_scales"] = _encode(v_all, r >> 16 & 0xFFFF, False)
        # a value has 4 bits of precision: exact in bf16
        m_all = _decode(s["m"], s["m_scales"], True).to(torch.bfloat16)
        v_all = _decode(s["v"], s["v_scales"], False).to(torch.bfloat16)
    return {"updated": s["g"] if case["push"] else s["w"], "m": m_all, "v": v_all}


def _normed(v):
    return v * torch.rsqrt((v * v).mean(dim=1, keepdim=True) + NORM_EPS)


def _gates(s, rows):
    gate = s["gate"].to(torch.float32)
    return gate if len(gate) in (1, rows) else gate.repeat_interleave(rows // len(gate), dim=0)


def _plain_norm(s):
    case = s["case"]
    h = s["x"].float()
    if case["block"]:
        b = s["y"].float()
        if case["after"]:
            b = _normed(b) * s["after"].float()
        if case["gates"]:
            b = b * _gates(s, case["rows"])
        h = case["scale"] * h + b
    z = (_normed(h) * s["before"].float()).to(_DT[case["branch"]])
    return {"h": h.to(s["x"].dtype), "z": z} if case["block"] else {"z": z}


def _norm_back(v, dn):
    """The gradient for v from that of N(v)."""
    r = torch.rsqrt((v * v).mean(dim=1, keepdim=True) + NORM_EPS)
    return r * (dn - v * (r * r * (dn * v).mean(dim=1, keepdim=True)))


def _plain_norm_grad(s):
    case = s["case"]
    h, dz = s["x"].float(), s["dz"].float()
    total = _norm_back(h, dz * s["before"].float())
    out = {"before": (dz * _normed(h)).sum(dim=0)}
    if case["block"]:
        total = total + s["dh"].float()
        y = s["y"].float()
        b = _normed(y) if case["after"] else y
        d = total
        if case["gates"]:
            whole = total * (b * s["after"].float() if case["after"] else b)
            out["gate"] = whole.view(case["gates"], -1, case["cols"]).sum(dim=1)
            d = total * _gates(s, case["rows"])
        if case["after"]:
            out["after"] = (d * b).sum(dim=0)
            d = _norm_back(y, d * s["after"].float())
        out["y"] = d.to(s["y"].dtype)
    out["x"] = (case["scale"] * total).to(s["x"].dtype)
    return out


_PLAIN = {"linear": _plain_linear, "adamw": _plain_adamw, "norm": _plain_norm, "norm_grad": _plain_norm_grad}


# ------------------------------------------------------------- own calls

def _run_own(s):
    from paper_1611_06213_amd import learner
    case = s["case"]
    op = case["op"]
    if op == "linear":
        return learner.linear_int8(s["x"], s["w"], bias=s["bias"], relu=True, dtype=_DT[case["out"]])
    if op == "adamw":
        s["adamw"].step(LR)
        m, v = s["adamw"].moments(torch.bfloat16 if case["bits"] == 8 else torch.float32)
        return {"updated": s["g"] if case["push"] else s["w"], "m": m, "v": v}
    parts = {"gate": s.get("gate"), "after": s.get("after"), "before": s["before"], "eps": NORM_EPS}
    if op == "norm":
        if not case["block"]:
            return {"z": learner.rms_norm(s["x"], s["before"], eps=NORM_EPS, dtype=_DT[case["branch"]])}
        h, z = learner.residual_norm(s["x"], s["y"], scale=case["scale"], **parts)
        return {"h": h, "z": z}
    if not case["block"]:
        dx, before = learner.rms_norm_grad(s["x"], s["before"], s["dz"], eps=NORM_EPS)
        return {"x": dx, "before": before}
    got = learner.residual_norm_grad(s["x"], s["y"], s["dh"], s["dz"], scale=case["scale"], **parts)
    return {k: v for k, v in got._asdict().items() if v is not None}


def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["op"]](state)


# ------------------------------------------------- definitions in 64 bits

def _exact_random(j, t):
    """As the definition has it, with products that wrap at 64 bits: the word of each j."""
    f = 0xFFFFFFFF
    a, b = (j >> 2) & f, j >> 34
    c, d = torch.full_like(j, t & f), torch.full_like(j, t >> 32)
    for i in range(7):
        x, y = a * 0xD2511F53, c * 0xCD9E8D57
        k0, k1 = (SEED + i * 0x9E3779B9) & f, ((SEED >> 32) + i * 0xBB67AE85) & f
        a, b, c, d = ((y >> 32) & f) ^ b ^ k0, y & f, ((x >> 32) & f) ^ d ^ k1, x & f
    which = j & 3
    return torch.where(which == 0, a, torch.where(which == 1, b, torch.where(which == 2, c, d)))


def _exact_8bit(x, r, exponents):
    """x in 64 bits, a block's numbers 2^-3 of their power of two apart, over `exponents`
    exponents below the block's largest; rounded up where the rest and r make one."""
    b = x.view(-1, 128)
    mantissa, e = torch.frexp(b.abs().amax(dim=1))   # in [0.5, 1)
    top = e + (mantissa > 15 / 16)
    _, e = torch.frexp(b)
    e = torch.maximum(e, (top - exponents + 2)[:, None])
    unit = _power(e - 4)
    n = torch.floor(b.abs() / unit + r.view(-1, 128).double() / 65536)
    if exponents == 32:
        n = torch.maximum(n, (b > 0).double())
    return (torch.sign(b) * n * unit).view(-1)


def _exact_adamw(case, s):
    t = s["steps"] + 1
    sizes = _sizes(case)
    room = s["m"].numel()
    at = torch.cat([torch.arange(n, device="cuda") + p for n, p in
                    zip(sizes, _layout(case, "cpu")[4].tolist())])
    decay = torch.cat([torch.full((n,), 0.0 if i % 2 else DECAY, device="cuda", dtype=torch.float64)
                       for i, n in enumerate(sizes)])
    if case["bits"] == 8:
        m, v = (_decode(s[k], s[k + "_scales"], k == "m").double() for k in ("m", "v"))
    else:
        m, v = s["m"].double(), s["v"].double()
    w, g = s["w"].double(), s["g"].double()
    m[at] = B1 * m[at] + (1 - B1) * g
    v[at] = B2 * v[at] + (1 - B2) * g ** 2
    step = LR * ((m[at] / (1 - B1 ** t)) / (torch.sqrt(v[at] / (1 - B2 ** t)) + EPS) + decay * w)
    if case["bits"] == 8:
        word = _exact_random(torch.arange(room, device="cuda"), t)
        m, v = _exact_8bit(m, word & 0xFFFF, 16), _exact_8bit(v, word >> 16, 32)
    return {"updated": step if case["push"] else w - step, "m": m, "v": v}


def _exact_norm(case, s):
    def n(v):
        return v / torch.sqrt(torch.mean(v ** 2, 1, True) + NORM_EPS)

    s = {k: v.double().requires_grad_(k not in ("dz", "dh")) for k, v in s.items()}
    h = s["x"]
    if case["op"] == "norm":
        if case["block"]:
            h = case["scale"] * h + _exact_branch(case, s, n)
            return {"h": h.detach(), "z": (n(h) * s["before"]).detach()}
        return {"z": (n(h) * s["before"]).detach()}
    names = ["x", "before"]
    total, before = torch.autograd.grad((n(h) * s["before"] * s["dz"]).sum(), [s[k] for k in names])
    out = {"x": total, "before": before}
    if case["block"]:
        total = total + s["dh"]
        out["x"] = case["scale"] * total
        names = [k for k in ("y", "gate", "after") if k in s]
        out.update(zip(names, torch.autograd.grad((_exact_branch(case, s, n) * total).sum(),
                                                  [s[k] for k in names])))
    return out


def _exact_branch(case, s, n):
    b = n(s["y"]) * s["after"] if case["after"] else s["y"]
    if not case["gates"]:
        return b
    return (b.view(case["gates"], -1, case["cols"]) * s["gate"][:, None, :]).view(b.shape)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(case, s)
    if case["op"] != "linear":
        return _exact_norm(case, s)

    def whole(x):
        # the integers are those of the definition in 32 bits, which a border decides
        x = x.float()
        most = torch.maximum(x.abs().max(dim=1).values, torch.tensor(2.0 ** -100, device=x.device))
        return torch.round(x * (127 / most)[:, None]).double(), most.double() / 127

    (q, a), (w, b) = whole(s["x"]), whole(s["w"])
    y = (q @ w.t()) * a[:, None] * b + s["bias"].double()
    return y * (y > 0)

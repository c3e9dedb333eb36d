"""The norms, the products of 8-bit integers and AdamW on a machine without a GPU: what the host can see to be wrong
is refused before any device work; plans are laid out as declared; the waits for copies to LDS as compiled."""
import ctypes
import os
import random
import re
import subprocess

import pytest
import torch

from paper_1611_06213_amd import build as B
from paper_1611_06213_amd import learner, ps
from tests.test_learner_abi import P, lib, refused  # noqa: F401


def test_norm_refuses(lib):  # noqa: F811
    def call(x=P, xdt=0, xld=40, y=2 * P, ydt=1, yld=40, rows=6, cols=40, gate=None, gdt=0, gates=0, gld=40,
             after=None, before=4 * P, wdt=0, scale=1.0, eps=1e-6, out=5 * P, old=40, normed=6 * P, nld=40):
        return lib.pl_norm(x, xdt, xld, y, ydt, yld, rows, cols, gate, gdt, gates, gld, after, before, wdt, scale, eps,
                           out, old, normed, nld, None)
    refused(lib, call(rows=1 << 31), "rows")
    refused(lib, call(rows=-1), "rows")
    refused(lib, call(cols=(1 << 31) + 1), "cols")
    # more columns than one launch joins the gradients' sums of
    refused(lib, call(cols=(1 << 29) + 1, xld=1 << 30, yld=1 << 30, old=1 << 30, nld=1 << 30), "cols")
    assert lib.pl_norm_grad_workspace(1, 1 << 29) > 0 and lib.pl_norm_grad_workspace(1, (1 << 29) + 1) == 0
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        refused(lib, call(eps=eps), "eps")
    refused(lib, call(x=None), "x: null")
    refused(lib, call(xdt=2), "dtype")
    refused(lib, call(ydt=-1), "dtype")
    refused(lib, call(wdt=5), "dtype")
    refused(lib, call(xld=39), "row stride")
    refused(lib, call(yld=0), "row stride")
    refused(lib, call(y=2 * P + 1), "aligned")
    refused(lib, call(out=None), "out: null")
    refused(lib, call(out=P + 4), "overlaps x")
    refused(lib, call(normed=2 * P), "overlaps y")
    refused(lib, call(normed=5 * P + 8), "overlaps")
    refused(lib, call(normed=4 * P), "overlaps before")
    refused(lib, call(normed=None), "before without normed")
    refused(lib, call(gate=3 * P), "gate: 0 rows")
    refused(lib, call(gates=2), "gate: 2 rows")
    refused(lib, call(gate=3 * P, gates=4), "6 rows for 4 gates")
    refused(lib, call(gate=3 * P, gates=-2), "gates")
    refused(lib, call(gate=3 * P, gates=3, gld=39), "row stride")
    refused(lib, call(gate=5 * P, gates=3), "overlaps gate")
    refused(lib, call(after=5 * P), "overlaps after")
    # without a block
    refused(lib, call(y=None), "out without y")
    refused(lib, call(y=None, out=None, after=3 * P), "without y")
    refused(lib, call(y=None, out=None, scale=2.0), "scale without y")
    refused(lib, call(y=None, out=None, normed=None), "normed: null")
    assert call(rows=0) == 0 and call(cols=0) == 0


def test_norm_grad_refuses(lib):  # noqa: F811
    need = lib.pl_norm_grad_workspace(600, 40)
    assert need > 0 and lib.pl_norm_grad_workspace(600, 4000) > need
    assert lib.pl_norm_grad_workspace(0, 40) == 0 and lib.pl_norm_grad_workspace(1 << 31, 4) == 0
    # rows that no worker holds in registers need room for their sums
    assert lib.pl_norm_grad_workspace(1 << 20, 100_000) >= 16 << 20

    def call(h=P, xdt=0, hld=40, y=2 * P, ydt=0, yld=40, dh=3 * P, dhld=40, dz=4 * P, dzld=40, rows=600, cols=40,
             gate=5 * P, gates=6, gld=40, after=6 * P, before=7 * P, scale=1.0, eps=1e-6, dx=8 * P, dxld=40, dy=9 * P,
             dyld=40, dgate=10 * P, dgld=40, dafter=11 * P, dbefore=12 * P, odt=0, acc=0, ws=13 * P, size=need):
        return lib.pl_norm_grad(h, xdt, hld, y, ydt, yld, dh, dhld, dz, dzld, rows, cols, gate, 0, gates, gld, after,
                                before, 0, scale, eps, dx, dxld, dy, dyld, dgate, dgld, dafter, dbefore, odt, acc, ws,
                                size, None)
    refused(lib, call(dh=None, dz=None), "no gradient")
    refused(lib, call(dz=None), "before without normed_grad")
    refused(lib, call(dz=None, before=None), "before without normed_grad")   # before_out
    refused(lib, call(y=None), "without y")
    refused(lib, call(y=None, gate=None, gates=0, after=None), "y_out without y")
    refused(lib, call(gate=None, gates=0), "gate_out without a gate")
    refused(lib, call(after=None), "after_out without after")
    refused(lib, call(before=None), "before_out without before")
    for name in ("h", "y", "dx", "dy", "ws"):
        refused(lib, call(**{name: None}), "y" if name == "y" else "null")
    refused(lib, call(odt=3), "dtype")
    refused(lib, call(dgld=39), "row stride")
    refused(lib, call(gates=7), "600 rows for 7 gates")
    refused(lib, call(size=need - 1), "needed", ps.PS_ENOMEM)
    refused(lib, call(ws=13 * P + 8), "16-byte")
    for name, at, text in (("dx", P, "h"), ("dy", 3 * P, "grad"), ("dgate", 4 * P, "normed_grad"),
                           ("dafter", 6 * P, "after"), ("dbefore", 8 * P, "overlaps"), ("dx", 9 * P, "y_out"),
                           ("ws", 2 * P, "y"), ("dbefore", 13 * P, "workspace")):
        refused(lib, call(**{name: at}), text)
    assert call(cols=0) == 0


def int8(values, scales):
    return ctypes.byref(learner.pl_int8(values, scales))


def test_int8_refuses(lib):  # noqa: F811
    assert lib.pl_int8_ld(0) == 0 and lib.pl_int8_ld(1) == 128 and lib.pl_int8_ld(129) == 256
    assert lib.pl_int8_values_bytes(3, 129) == 768 and lib.pl_int8_values_bytes(-1, 5) == 0

    def quantize(x=P, dt=0, rows=300, cols=200, ld=200, out=int8(2 * P, 3 * P)):
        return lib.pl_quantize_int8(x, dt, rows, cols, ld, out, None)
    refused(lib, quantize(x=None), "x: null")
    refused(lib, quantize(dt=2), "dtype")
    refused(lib, quantize(ld=199), "row stride")
    refused(lib, quantize(rows=(1 << 28) + 1), "rows")
    refused(lib, quantize(cols=(1 << 17) + 1, ld=1 << 18), "cols")
    refused(lib, quantize(out=None), "out: null")
    refused(lib, quantize(out=int8(None, 3 * P)), "null")
    refused(lib, quantize(out=int8(2 * P, 3 * P + 4)), "16-byte")
    refused(lib, quantize(out=int8(P, 3 * P)), "overlaps x")
    refused(lib, quantize(out=int8(2 * P, 2 * P + 128)), "overlaps")
    assert quantize(rows=0) == 0

    a, b = int8(P, 2 * P), int8(3 * P, 4 * P)

    def matmul(m=8, n=8, k=300, a=a, b=b, bias=None, bdt=0, out=5 * P, odt=1, ld=8, ws=6 * P, size=1 << 24):
        return lib.pl_matmul_int8(m, n, k, a, b, bias, bdt, 0, out, odt, ld, ws, size, None)
    refused(lib, matmul(m=-1), "m:")
    refused(lib, matmul(n=(1 << 28) + 1), "n:")
    refused(lib, matmul(k=(1 << 17) + 1), "k:")
    refused(lib, matmul(a=None), "a: null")
    refused(lib, matmul(b=int8(3 * P, None)), "b: null")
    refused(lib, matmul(odt=3), "dtype")
    refused(lib, matmul(bias=7 * P, bdt=9), "dtype")
    refused(lib, matmul(ld=7), "row stride")
    for at, name in ((P, "a"), (2 * P, "a"), (3 * P + 64, "b"), (4 * P, "b")):
        refused(lib, matmul(out=at), f"overlaps {name}")
    need = lib.pl_matmul_int8_workspace(100, 8, 100_000)
    assert need > 0   # few tiles: k is split
    big = {"m": 100, "k": 100_000, "a": int8(8 * P, 24 * P), "b": int8(32 * P, 48 * P)}
    refused(lib, matmul(**big, size=need - 1), "needed", ps.PS_ENOMEM)
    refused(lib, matmul(**big, ws=None), "workspace: null")
    refused(lib, matmul(**big, ws=8 * P), "overlaps a")
    assert lib.pl_matmul_int8_workspace(8192, 8192, 8192) == 0
    assert lib.pl_matmul_int8_workspace(8, 8, (1 << 17) + 1) == 0
    assert matmul(m=0) == 0 and matmul(n=0) == 0

    def linear(x=P, dt=0, m=8, k=300, ld=300, n=16, w=int8(2 * P, 3 * P), bias=None, out=5 * P, odt=1, old=16,
               ws=6 * P, size=1 << 24):
        return lib.pl_linear_int8(x, dt, m, k, ld, n, w, bias, 0, 0, out, odt, old, ws, size, None)
    refused(lib, linear(m=-1), "m:")
    refused(lib, linear(k=(1 << 17) + 1, ld=1 << 18), "k:")
    refused(lib, linear(x=None), "x: null")
    refused(lib, linear(ld=299), "row stride")
    refused(lib, linear(w=int8(2 * P + 4, 3 * P)), "16-byte")
    refused(lib, linear(out=P + 64), "overlaps x")
    refused(lib, linear(bias=5 * P), "overlaps bias")
    need = lib.pl_linear_int8_workspace(100, 16, 300)
    assert need > 0 and lib.pl_linear_int8_workspace(1, 16, 300) == 0   # a few rows: one launch
    refused(lib, linear(m=100, size=need - 1), "needed", ps.PS_ENOMEM)
    refused(lib, linear(m=100, ws=P), "overlaps x")
    assert linear(m=0) == 0 and linear(n=0) == 0


def tensors(*rows):
    return (learner.pl_adamw_tensor * len(rows))(*(learner.pl_adamw_tensor(*r) for r in rows))


def test_adamw_plan(lib):  # noqa: F811
    t = tensors((P, 2 * P, 1000, 0.1), (3 * P, 4 * P, 0, 0.2), (5 * P + 4, 6 * P + 4, 5000, 0.3))
    assert lib.pl_adamw_room(t, 3) == 1024 + 5120
    parts = lib.pl_adamw_parts(t, 3)
    size = lib.pl_adamw_plan_bytes(parts)
    plan = torch.zeros(size, dtype=torch.uint8)

    def make(t=t, n=3, wdt=0, gdt=0, push=0, steps=7, plan=plan.data_ptr(), size=size):
        return lib.pl_adamw_plan(t, n, wdt, gdt, push, steps, plan, size)
    assert make() == 0 and lib.pl_adamw_steps(plan.data_ptr()) == 7
    # every element is in one part, at its place in the states
    entry = size // parts
    seen = []
    for i in range(parts):
        raw = bytes(plan[i * entry:(i + 1) * entry].tolist())
        w, g, at, steps = (int.from_bytes(raw[8 * j:8 * j + 8], "little") for j in range(4))
        count = int.from_bytes(raw[32:36], "little")
        assert steps == 7 and count > 0 and at % 128 == 0
        seen.append((w, g, at, count))
    first = [p for p in seen if p[0] < 3 * P]
    second = [p for p in seen if p[0] >= 3 * P]
    for part, base, start, total in ((first, (P, 2 * P), 0, 1000), (second, (5 * P + 4, 6 * P + 4), 1024, 5000)):
        done = 0
        for w, g, at, count in part:
            assert (w, g, at) == (base[0] + 4 * done, base[1] + 4 * done, start + done)
            done += count
        assert done == total
    refused(lib, make(plan=None), "plan: null")
    refused(lib, make(size=size - 1), "needed", ps.PS_ENOMEM)
    refused(lib, make(wdt=1), "weight: dtype")
    refused(lib, make(gdt=2), "grad: dtype")
    refused(lib, make(steps=-1), "steps")
    for bad, text in (((None, 2 * P, 9, 0), "weight: null"), ((P, None, 9, 0), "grad: null"),
                      ((P + 2, 2 * P, 9, 0), "4-byte"), ((P, 2 * P + 1, 9, 0), "4-byte"), ((P, 2 * P, -1, 0), "count")):
        refused(lib, make(t=tensors(bad), n=1), text)
    assert lib.pl_adamw_parts(tensors((P, P, (1 << 40) + 1, 0)), 1) == -1
    assert lib.pl_adamw_room(tensors((P, P, 1 << 40, 0), (P, P, 1, 0)), 2) == -1
    assert lib.pl_adamw_room(None, 1) == -1 and lib.pl_adamw_room(None, 0) == 0
    assert lib.pl_adamw_plan(None, 0, 0, 0, 0, 0, None, 0) == 0


def test_adamw_overlaps(lib):  # noqa: F811
    """Against every pair, on random lists."""
    rng = random.Random(5)
    plan = torch.zeros(1 << 16, dtype=torch.uint8)
    kinds = set()
    for _ in range(600):
        n = rng.randint(1, 5)
        rows = [(P + 4 * rng.randint(0, 90), P + 4 * rng.randint(0, 90) + rng.choice([0, 4000]), rng.randint(0, 12), 0.0)
                for _ in range(n)]
        for push in (0, 1):
            spans = [[(r[k], r[k] + 4 * r[2]) for r in rows if r[2]] for k in (0, 1)]
            written, read = (spans[1], spans[0]) if push else spans

            def meet(a, b):
                return a[0] < b[1] and b[0] < a[1]
            bad = any(meet(a, b) for i, a in enumerate(written) for b in written[:i]) or \
                any(meet(a, b) for a in written for b in read)
            rc = lib.pl_adamw_plan(tensors(*rows), n, 0, 0, push, 0, plan.data_ptr(), plan.numel())
            assert rc == (ps.PS_EINVAL if bad else 0), (rows, push)
            kinds.add((bad, push))
    assert len(kinds) == 4


def test_adamw_step_refuses(lib):  # noqa: F811
    def call(plan=P, parts=3, wdt=0, gdt=0, push=0, bits=8, room=1024, m=2 * P, v=3 * P, ms=4 * P, vs=5 * P, b1=0.9,
             b2=0.99, eps=1e-8, lr_at=None, factor_at=None):
        return lib.pl_adamw_step(plan, parts, wdt, gdt, push, bits, room, m, v, ms, vs, b1, b2, eps, 0.1, lr_at, 1.0,
                                 factor_at, 0, None)
    refused(lib, call(parts=-1), "parts")
    refused(lib, call(room=100), "multiple of 128")
    refused(lib, call(room=-128), "room")
    refused(lib, call(wdt=1), "weight")
    refused(lib, call(gdt=7), "grad")
    refused(lib, call(bits=16), "16 bits")
    for b in (1.0, -0.5, float("nan"), 1 - 2.0 ** -29):
        refused(lib, call(b1=b), "beta")
        refused(lib, call(b2=b), "beta")
    refused(lib, call(eps=-1.0), "eps")
    refused(lib, call(eps=float("inf")), "eps")
    for name in ("plan", "m", "v", "ms", "vs"):
        refused(lib, call(**{name: None}), "null")
    refused(lib, call(m=2 * P + 8), "16-byte")
    refused(lib, call(lr_at=6 * P + 2), "4-byte")
    refused(lib, call(v=2 * P + 512), "overlaps")
    refused(lib, call(vs=P), "plan overlaps")
    refused(lib, call(lr_at=2 * P), "overlaps lr_at")
    assert call(parts=0) == 0

    def moments(room=1024, m=P, v=2 * P, ms=3 * P, vs=4 * P, mo=5 * P, vo=6 * P, dt=0):
        return lib.pl_adamw_moments(room, m, v, ms, vs, mo, vo, dt, None)
    refused(lib, moments(room=130), "multiple")
    refused(lib, moments(dt=2), "dtype")
    refused(lib, moments(mo=None), "null")
    refused(lib, moments(vo=6 * P + 2), "4-byte")
    refused(lib, moments(mo=P + 512), "overlaps m")
    refused(lib, moments(vo=5 * P), "overlaps")
    assert moments(room=0) == 0


def test_binding_refuses_host_tensors():
    x = torch.ones(4, 4)
    for call in (lambda: learner.rms_norm(x), lambda: learner.residual_norm(x, x),
                 lambda: learner.residual_norm_grad(x, x, x), lambda: learner.rms_norm_grad(x, None, x),
                 lambda: learner.quantize_int8(x), lambda: learner.AdamW([x], [x])):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(TypeError, match="Int8Matrix"):
        learner.linear_int8(x, x)


def test_waits_for_copies(tmp_path):
    """The tiled products of integers wait for their copies to LDS by counting what was issued after them: before
    every barrier of the main loop, all copies but those of the last two steps have arrived, as compiled."""
    src = os.path.join(B.CSRC, "pl_matmul_int8.hip")
    out = str(tmp_path / "int8.s")
    flags = [f for f in B.LEARNER_FLAGS if f != "-fPIC"]
    subprocess.run([B.HIPCC, *flags, "--cuda-device-only", "-S", src, "-o", out], check=True,
                   stderr=subprocess.DEVNULL)
    text, checked = open(out).read(), 0
    for name in re.findall(r"^(\S*tilesILi\S*):", text, re.M):
        n = 2 * int(re.search(r"tilesILi(\d)E", name).group(1))   # copies of a step
        body = text[text.index("\n" + name + ":"):]
        body = body[:body.index(".Lfunc_end")].split("; the first unit's copies")[1]
        ops = []
        for line in body.splitlines():
            line = line.split(";")[0].strip()
            if line.startswith("buffer_load_dwordx4") and line.endswith(" lds"):
                ops.append("copy")
            elif re.match(r"(buffer|global|flat|scratch)_(load|store)", line):
                ops.append("other")
            elif line.startswith("s_waitcnt") and "vmcnt" in line:
                ops.append(int(re.search(r"vmcnt\((\d+)\)", line).group(1)))
            elif line.startswith("s_barrier"):
                ops.append("barrier")
        # up to the barrier that ends the loop: two before it, then two a block for two blocks
        barriers = [i for i, op in enumerate(ops) if op == "barrier"]
        ops = ops[:barriers[5] + 1]
        first = ops.index("copy")
        assert "other" not in ops[first:], name   # before them: the scales' copies
        queue, copies, ended = [], 0, 0
        for op in ops:
            if op == "copy":
                queue.append(copies // n)   # the step that it belongs to
                copies += 1
            elif op == "other":
                queue.append(-1)
            elif op == "barrier":
                # before step s (0, 1, ..) steps 0 .. s + 1 are there; the first two barriers are before step 0
                before = max(0, ended - 1)
                assert all(step > before + 1 for step in queue), (name, ended)
                ended += 1
            else:
                del queue[:max(0, len(queue) - op)]
        assert copies == 8 * n, name
        checked += 1
    assert checked == 6


REGS = re.compile(r"\b([av])(?:(\d+)|\[(\d+):(\d+)\])")


def registers(text):
    return {f"{kind}{i}" for kind, one, first, last in REGS.findall(text)
            for i in (range(int(first), int(last) + 1) if first else (int(one),))}


def too_near(lines):
    """Where a matrix instruction comes fewer than two wait states after a vector instruction that writes what it reads,
    or another instruction than these fewer than 19 after one whose sums it names (16 passes, the longest, and 3)."""
    time, wrote, product, found = 0, {}, {}, []
    for line in lines:
        op, _, rest = line.partition(" ")
        if op == "s_nop":
            time += int(rest) + 1
            continue
        if op.startswith("v_mfma"):
            out = registers(rest.split(",")[0])
            found += [line for r in registers(rest) if time - wrote.get(r, -99) <= 2]
            product.update((r, time) for r in out)
        elif re.match(r"(v|ds|buffer|global|flat|scratch)_", op):
            found += [line for r in registers(rest) if time - product.get(r, -99) <= 19]
            if op.startswith("v_"):
                named = rest.split(",")
                wrote.update((r, time) for r in registers(",".join(named[:2] if "swap" in op else named[:1])))
        time += 1
    return found


@pytest.mark.parametrize("between,near", [
    (["s_nop 0"], True), (["s_nop 1"], False), (["s_nop 0", "s_mov_b32 s0, 0"], False),
    (["v_mov_b32_e32 v9, 0", "v_mov_b32_e32 v3, 0", "s_nop 0"], True)])
def test_too_near(between, near):
    product = "v_mfma_i32_16x16x64_i8 a[0:3], v[0:3], v[4:7], a[0:3]"
    assert (too_near(["v_accvgpr_write_b32 a3, v8", *between, product]) != []) == near
    for waits, early in ((["s_nop 15", "s_nop 1"], True), (["s_nop 15", "s_nop 2"], False)):
        for use in ("v_accvgpr_read_b32 v8, a2", "global_store_dwordx4 v[8:9], a[0:3], off", "v_accvgpr_mov_b32 a0, a9"):
            assert (too_near([product, *waits, use]) != []) == early
    assert too_near([product, product, "v_mov_b32_e32 v8, 0"]) == []


def test_products_wait_for_what_they_read(tmp_path):
    """The tiled products' matrix instructions are inline assembly, of whose time the compiler knows nothing: as
    compiled, no operand is written right before one, and no sum is read or written before it is there. Each loop
    follows itself, too."""
    src = os.path.join(B.CSRC, "pl_matmul_int8.hip")
    out = str(tmp_path / "int8.s")
    flags = [f for f in B.LEARNER_FLAGS if f != "-fPIC"]
    subprocess.run([B.HIPCC, *flags, "--cuda-device-only", "-S", src, "-o", out], check=True,
                   stderr=subprocess.DEVNULL)
    text, checked = open(out).read(), 0
    for name in re.findall(r"^(\S*tilesILi\S*):", text, re.M):
        body = text[text.index("\n" + name + ":") + 1:]
        lines = [line.split(";")[0].strip() for line in body[:body.index(".Lfunc_end")].splitlines()[1:]]
        lines = [line for line in lines if line and (not line.startswith(".") or line.endswith(":"))]
        labels = {line[:-1]: i for i, line in enumerate(lines) if line.endswith(":")}
        products = [i for i, line in enumerate(lines) if line.startswith("v_mfma")]
        # four blocks of k's halves, each with 4 F F products
        tile = int(re.search(r"tilesILi(\d)E", name).group(1))
        assert len(products) == 4 * 4 * tile * tile, name
        assert not any(line.startswith("v_cmpx") for line in lines[products[0] - 8:products[-1]])
        assert too_near(lines) == [], name
        loops = 0
        for i, line in enumerate(lines):
            target = labels.get(line.split()[-1], i) if line.startswith(("s_cbranch", "s_branch")) else i
            if target < i and any(target < p < i for p in products):
                loops += 1
                assert too_near(lines[target:i] + lines[target:i]) == [], name
        assert loops >= 1, name
        checked += 1
    assert checked == 6

"""The learner's operators on a machine without a GPU: the library loads, exports what
include/ps_learner.h declares, and refuses what the host can see to be wrong before any
device work; its kernels' code keeps to the rules that the others' keeps to."""
import ctypes
import os
import re
import subprocess
import sys

import pytest
import torch

from paper_1611_06213_amd import build as B
from paper_1611_06213_amd import learner, ps

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20   # an address: nothing here reaches a kernel


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(learner.LIB_PATH):
        pytest.fail("libgadeilearner.so is not built (run __graft_entry__.build())")
    return learner.load_library()


def test_every_declared_symbol_is_exported(lib):
    text = open(os.path.join(ROOT, "include", "ps_learner.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(pl_[a-z0-9_]+)\s*\(", text))
    assert names == set(learner._SIGS) and len(names) >= 10
    for n in names:
        assert hasattr(lib, n), n
    for name in ("PL_I32", "PL_I64"):
        assert int(re.search(rf"\b{name}\s*=\s*(\d+)", text).group(1)) == getattr(learner, name)


def test_header_is_c(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include "ps_learner.h"\n'
                   "int main(void) { pl_drop d = {0.5f, 1, 2}; pl_fp8 q = {0, 0};"
                   " return d.p > 1 || q.values != 0; }\n")
    r = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-fsyntax-only", "-I",
                        B.INCLUDE, str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_binding_refuses_missing_library(tmp_path):
    with pytest.raises(RuntimeError, match="not built"):
        learner.load_library(str(tmp_path / "missing.so"))


def drop(p=0.5):
    return ctypes.byref(learner.pl_drop(p, 1, 2))


def refused(lib, rc, text, code=ps.PS_EINVAL):
    assert rc == code and text in lib.pl_last_error().decode(), (rc, lib.pl_last_error())


def test_embedding_refuses(lib):
    def call(ids=P, id_type=1, tokens=4, table=2 * P, tdt=0, vocab=9, dim=6, ld=6, d=None, out=3 * P,
             odt=0, old=6):
        return lib.pl_embedding(ids, id_type, tokens, table, tdt, vocab, dim, ld, 1.0, d, out, odt,
                                old, None)
    refused(lib, call(id_type=2), "id type")
    refused(lib, call(ids=None), "ids: null")
    refused(lib, call(ids=P + 4), "8-byte")
    refused(lib, call(table=None), "table: null")
    refused(lib, call(table=2 * P + 2), "aligned")
    refused(lib, call(tdt=2), "dtype")
    refused(lib, call(odt=-1), "dtype")
    refused(lib, call(ld=5), "row stride")
    refused(lib, call(old=5), "row stride")
    refused(lib, call(tokens=-1), "tokens")
    refused(lib, call(tokens=1 << 32), "tokens")
    refused(lib, call(vocab=-1), "vocab")
    refused(lib, call(dim=(1 << 32) + 1, ld=1 << 33, old=1 << 33), "dim")
    refused(lib, call(d=drop(1.01)), "probability")
    refused(lib, call(d=drop(float("nan"))), "probability")
    refused(lib, call(out=2 * P + 4), "overlaps table")
    refused(lib, call(out=P + 8), "overlaps ids")
    assert call(tokens=0) == 0 and call(dim=0) == 0   # nothing to do, nothing launched


def test_embedding_grad_refuses(lib):
    need = lib.pl_embedding_grad_workspace(40, 9, 6)
    assert need > 0
    # it grows with every size
    for bigger in ((4000, 9, 6), (40_000, 9000, 6), (4000, 9, 60)):
        assert lib.pl_embedding_grad_workspace(*bigger) > need
    for bad in ((-1, 9, 6), (40, 0, 6), (40, 9, -2), (1 << 31, 9, 6), (40, (1 << 31) + 1, 6)):
        assert lib.pl_embedding_grad_workspace(*bad) == 0

    def call(ids=P, id_type=0, tokens=40, grad=2 * P, gdt=0, gld=6, dim=6, d=None, out=3 * P, odt=0,
             old=6, vocab=9, ws=4 * P, size=need):
        return lib.pl_embedding_grad(ids, id_type, tokens, grad, gdt, gld, dim, 1.0, d, out, odt, old,
                                     vocab, 0, ws, size, None)
    refused(lib, call(id_type=-1), "id type")
    refused(lib, call(tokens=1 << 31), "tokens")
    refused(lib, call(vocab=(1 << 31) + 1), "vocab")
    refused(lib, call(gld=3), "row stride")
    refused(lib, call(out=None), "out: null")
    refused(lib, call(d=drop(-0.1)), "probability")
    refused(lib, call(size=need - 1), "needed", ps.PS_ENOMEM)
    refused(lib, call(ws=None), "workspace: null")
    refused(lib, call(ws=4 * P + 8), "16-byte")
    refused(lib, call(out=2 * P), "overlaps grad")
    refused(lib, call(out=4 * P), "overlaps workspace")
    refused(lib, call(ws=2 * P), "overlaps grad")
    assert call(vocab=0) == 0 and call(dim=0) == 0


def test_dropout_refuses(lib):
    def call(x=P, dt=0, rows=3, cols=5, ld=5, d=drop(), out=2 * P, old=5):
        return lib.pl_dropout(x, dt, rows, cols, ld, d, out, old, None)
    refused(lib, call(d=None), "null")
    refused(lib, call(x=None), "null")
    refused(lib, call(dt=7), "dtype")
    refused(lib, call(ld=4), "row stride")
    refused(lib, call(rows=1 << 32), "rows")
    refused(lib, call(cols=-1), "cols")
    refused(lib, call(out=P + 4), "overlaps")
    refused(lib, call(out=P, old=6), "overlaps")   # in place with another stride
    refused(lib, call(d=drop(2.0)), "probability")
    assert call(rows=0) == 0


def fp8(values, scales):
    return ctypes.byref(learner.pl_fp8(values, scales))


def test_fp8_refuses(lib):
    assert lib.pl_fp8_ld(1) == 128 and lib.pl_fp8_ld(129) == 256 and lib.pl_fp8_ld(0) == 0
    assert lib.pl_fp8_values_bytes(3, 129) == 768 and lib.pl_fp8_values_bytes(0, 5) == 0
    assert lib.pl_fp8_scales_bytes(3, 512) == 12 and lib.pl_fp8_scales_bytes(3, 513) == 24

    def quantize(x=P, dt=0, rows=300, cols=200, ld=200, out=fp8(2 * P, 3 * P), out_t=None):
        return lib.pl_quantize_fp8(x, dt, rows, cols, ld, 0, out, out_t, None)
    refused(lib, quantize(out=None), "no output")
    refused(lib, quantize(x=None), "null")
    refused(lib, quantize(dt=2), "dtype")
    refused(lib, quantize(ld=199), "row stride")
    refused(lib, quantize(rows=1 << 31), "rows")
    refused(lib, quantize(out=fp8(None, 3 * P)), "null")
    refused(lib, quantize(out=fp8(2 * P + 8, 3 * P)), "16-byte")
    refused(lib, quantize(out=fp8(P, 3 * P)), "overlaps x")
    refused(lib, quantize(out_t=fp8(2 * P, 5 * P)), "overlaps")
    assert quantize(rows=0) == 0

    a, b = fp8(P, 2 * P), fp8(3 * P, 4 * P)

    def matmul(m=8, n=8, k=300, a=a, b=b, bias=None, relu=0, out=5 * P, odt=1, ld=8, acc=0, ws=6 * P,
               size=1 << 24):
        return lib.pl_matmul_fp8(m, n, k, a, b, bias, 0, relu, out, odt, ld, acc, ws, size, None)
    refused(lib, matmul(m=-1), "m:")
    refused(lib, matmul(k=(1 << 22) + 1), "k:")
    refused(lib, matmul(m=(1 << 28) + 1), "m:")
    refused(lib, matmul(n=(1 << 28) + 1), "n:")
    refused(lib, matmul(a=None), "a: null")
    refused(lib, matmul(b=fp8(3 * P, None)), "b: null")
    refused(lib, matmul(odt=3), "dtype")
    refused(lib, matmul(ld=7), "row stride")
    refused(lib, matmul(acc=1, relu=1), "accumulate")
    refused(lib, matmul(acc=1, bias=7 * P), "accumulate")
    refused(lib, matmul(out=P), "overlaps a")
    refused(lib, matmul(out=3 * P + 64), "overlaps b")
    refused(lib, matmul(bias=7 * P, out=7 * P), "overlaps bias")
    need = lib.pl_matmul_fp8_workspace(100, 8, 100_000, 1)
    assert need > 0   # few tiles: k is split
    refused(lib, matmul(m=100, k=100_000, a=fp8(8 * P, 24 * P), b=fp8(32 * P, 48 * P), size=need - 1), "needed", ps.PS_ENOMEM)
    assert lib.pl_matmul_fp8_workspace(8192, 8192, 8192, 1) == 0
    assert matmul(m=0) == 0 and matmul(n=0) == 0


def test_binding_refuses_host_tensors():
    x = torch.ones(4, 4)
    for call in (lambda: learner.dropout(x, learner.Dropout(0.5, 1)),
                 lambda: learner.embedding(torch.zeros(3, dtype=torch.int64), x),
                 lambda: learner.quantize_fp8(x)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(TypeError, match="tensor expected"):
        learner.dropout([1.0], learner.Dropout(0.5, 1))


def waits_of_tiles(text):
    """The tiled products wait for their copies to LDS by counting what was issued after them. Run
    through each kernel's memory instructions as compiled: before every barrier of the main loop, all
    copies but those of the last two steps have arrived."""
    checked = 0
    for name in re.findall(r"^(\S*tilesILi\S*):", text, re.M):
        fm, fn = map(int, re.search(r"tilesILi(\d)ELi(\d)E", name).groups())
        n = fm + fn   # copies of a step, and words of scales that are loaded together
        body = text[text.index("\n" + name + ":"):]
        bodies = body[:body.index(".Lfunc_end")].split("; the first unit's copies")[1:]
        for body in bodies:   # one, or two of a launch with results of two types
            waits_of_units(body, n, name)
            checked += 1
    assert checked == 6


def waits_of_units(body, n, name):
    ops = []
    for line in body.splitlines():
        line = line.split(";")[0].strip()
        if line.startswith("buffer_load_dword"):
            ops.append("copy" if line.endswith(" lds") else "word")
        elif re.match(r"(global|flat|scratch)_(load|store)", line):
            ops.append("other")
        elif line.startswith("s_waitcnt") and "vmcnt" in line:
            ops.append(int(re.search(r"vmcnt\((\d+)\)", line).group(1)))
        elif line.startswith("s_barrier"):
            ops.append("barrier")
    # up to the barrier that ends the loop: two before it, then two a block for two blocks
    barriers = [i for i, op in enumerate(ops) if op == "barrier"]
    ops = ops[:barriers[5] + 1]
    assert "other" not in ops, name
    queue, copies, ended = [], 0, 0
    for op in ops:
        if op == "copy":
            queue.append(copies // n)   # the step that it belongs to
            copies += 1
        elif op == "word":
            queue.append(None)
        elif op == "barrier":
            # before step s (0, 1, ..) steps 0 .. s + 1 are there; the first two barriers are before
            # step 0
            before = max(0, ended - 1)
            assert all(step is None or step > before + 1 for step in queue), (name, ended)
            ended += 1
        else:
            del queue[:max(0, len(queue) - op)]
    assert copies == 8 * n, name


def test_kernels_use_no_scratch_and_no_packed_fp32(tmp_path):
    running = []
    for src in B.LEARNER_SOURCES:
        if src.endswith(".hip"):
            out = str(tmp_path / (os.path.basename(src) + ".s"))
            flags = [f for f in B.LEARNER_FLAGS if f != "-fPIC"]
            running.append((out, subprocess.Popen([B.HIPCC, *flags, "--cuda-device-only", "-S", src, "-o",
                                                   out], stderr=subprocess.DEVNULL)))
    assert running
    for out, p in running:
        assert p.wait(timeout=600) == 0
        text = open(out).read()
        if out.endswith("pl_matmul.hip.s"):
            waits_of_tiles(text)
        sizes = re.findall(r"\.amdhsa_private_segment_fixed_size (\d+)", text)
        assert sizes and set(sizes) == {"0"}, out
        assert not re.search(r"^\s*v_pk_(add|mul|fma)_f32", text, re.M), out


def test_linear_refuses(lib):
    """The layer and its backward pass check everything before the first launch."""
    w = fp8(2 * P, 3 * P)

    def linear(x=P, dt=0, m=8, k=300, ld=300, n=16, w=w, bias=None, out=5 * P, odt=1, old=16, ws=6 * P,
               size=1 << 24):
        return lib.pl_linear_fp8(x, dt, m, k, ld, n, w, bias, 0, 0, out, odt, old, ws, size, None)
    refused(lib, linear(m=-1), "m:")
    refused(lib, linear(k=(1 << 22) + 1, ld=1 << 23), "k:")
    refused(lib, linear(x=None), "x: null")
    refused(lib, linear(dt=4), "dtype")
    refused(lib, linear(ld=299), "row stride")
    refused(lib, linear(w=fp8(2 * P + 4, 3 * P)), "16-byte")
    refused(lib, linear(out=P + 64), "overlaps x")
    refused(lib, linear(out=2 * P), "overlaps w")
    refused(lib, linear(bias=5 * P), "overlaps bias")
    need = lib.pl_linear_fp8_workspace(100, 16, 300, 0, 1)
    assert need > 0 and lib.pl_linear_fp8_workspace(1, 16, 300, 0, 1) == 0   # a few rows: one launch
    refused(lib, linear(m=100, size=need - 1), "needed", ps.PS_ENOMEM)
    refused(lib, linear(m=100, ws=None), "workspace: null")
    refused(lib, linear(m=100, ws=P), "overlaps x")
    assert linear(m=0) == 0 and linear(n=0) == 0

    need = lib.pl_linear_fp8_grad_workspace(8, 16, 300, 1, 0)
    assert need > 0

    def grad(x=P, xdt=0, xld=300, g=4 * P, gdt=1, gld=16, m=8, n=16, k=300, w=w, out=5 * P, odt=1, old=300,
             wout=6 * P, wdt=0, wld=300, ws=8 * P, size=need):
        return lib.pl_linear_fp8_grad(x, xdt, xld, g, gdt, gld, m, n, k, w, out, odt, old, wout, wdt, wld, 0,
                                      ws, size, None)
    refused(lib, grad(m=(1 << 22) + 1), "m:")
    refused(lib, grad(k=(1 << 28) + 1, xld=1 << 29, old=1 << 29, wld=1 << 29), "k:")
    refused(lib, grad(x=None), "x: null")
    refused(lib, grad(g=None), "grad: null")
    refused(lib, grad(gld=15), "row stride")
    refused(lib, grad(w=None), "w_t: null")
    refused(lib, grad(wdt=9), "dtype")
    refused(lib, grad(out=P), "overlaps x")
    refused(lib, grad(wout=5 * P), "overlaps")
    refused(lib, grad(size=need - 1), "needed", ps.PS_ENOMEM)
    refused(lib, grad(ws=4 * P), "overlaps grad")


def test_binding_gives_the_stride_that_a_tensor_has(monkeypatch):
    """Rows that share their memory: 0, whatever their columns, which the library refuses."""
    monkeypatch.setattr(learner, "_on_device", lambda name, t: None)
    one = torch.ones(1, 1)
    assert learner._matrix("x", one.expand(300, 1))[2] == 0
    assert learner._matrix("x", torch.ones(1, 7).expand(300, 7))[2] == 0
    assert learner._matrix("x", torch.ones(300, 4)[:, :1])[2] == 4


def test_native_calls_take_the_lock_back(tmp_path):
    """What throws while a call runs without the interpreter's lock comes out with the lock held."""
    src, out = tmp_path / "throws.cpp", str(tmp_path / "throws.so")
    src.write_text(f'#include "{B.LEARNER_BINDING_SRC}"\n' + r"""
static PyObject *throws(PyObject *, PyObject *) {
    bool thrown = false;
    try {
        unlocked([]() -> int { throw std::runtime_error("a HIP error"); });
    } catch (const std::exception &) { thrown = true; }
    if (!thrown || !PyGILState_Check()) _exit(3);
    return PyLong_FromLong(unlocked([] { return PyGILState_Check() ? 1 : 7; }));
}
static PyMethodDef own[] = {{"throws", throws, METH_NOARGS, ""}, {nullptr, nullptr, 0, nullptr}};
static PyModuleDef mod = {PyModuleDef_HEAD_INIT, "throws", nullptr, -1, own, nullptr, nullptr, nullptr, nullptr};
PyMODINIT_FUNC PyInit_throws(void) { return PyModule_Create(&mod); }
""")
    cmd = B._binding_cmd(str(src), out, ["-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM", "-include", "unistd.h", "-isystem",
                                         os.path.join(B.ROCM, "include")],
                         ["-lc10_hip", "-L", B.HERE, "-lgadeilearner", "-Wl,-rpath," + B.HERE])
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    os.replace(out + ".tmp", out)
    code = "import sys, torch; sys.path.insert(0, sys.argv[1]); import throws; sys.exit(throws.throws())"
    assert subprocess.run([sys.executable, "-c", code, str(tmp_path)]).returncode == 7

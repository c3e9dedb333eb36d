// Host side of a learner's operators: the C ABI declared in include/ps_learner.h.
// Checks every argument that the host can see, then launches. No state; no allocation and nothing
// that throws but in pl_adamw_plan, which is called once and catches it.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <vector>

#include "pl_kernels.h"

namespace {

using namespace gadei::learner;

thread_local char g_error[256];

__attribute__((format(printf, 2, 3))) int fail(int code, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(g_error, sizeof(g_error), fmt, ap);
    va_end(ap);
    return code;
}

int launched(hipError_t e, const char *what) {
    if (e == hipSuccess) return PS_OK;
    if (e == hipErrorInvalidConfiguration)
        return fail(PS_EINVAL, "%s: more elements than one launch takes", what);
    return fail(PS_EHIP, "%s: %s", what, hipGetErrorString(e));
}

bool is_dtype(int d) { return d == PS_F32 || d == PS_BF16; }
size_t dtype_bytes(int d) { return d == PS_F32 ? 4 : 2; }
constexpr int64_t kMax = int64_t(1) << 32;
constexpr int64_t kMostRows = int64_t(1) << 28;   // of a product's operands: 4 bytes a row of scales
constexpr int64_t kMostCols = int64_t(1) << 22;

// A buffer named in a call: bytes from p on, 0 of them for an empty one.
struct Span {
    const char *name;
    uintptr_t p;
    uint64_t bytes;
};

// A matrix's buffer, checked. rows, cols >= 0 and cols <= 2^32 before the call.
int matrix(const char *name, const void *p, int dtype, int64_t rows, int64_t cols, int64_t ld,
           Span *out) {
    *out = Span{name, reinterpret_cast<uintptr_t>(p), 0};
    if (!is_dtype(dtype)) return fail(PS_EINVAL, "%s: dtype %d", name, dtype);
    if (rows == 0 || cols == 0) return PS_OK;
    if (p == nullptr) return fail(PS_EINVAL, "%s: null pointer", name);
    if (out->p % dtype_bytes(dtype)) return fail(PS_EINVAL, "%s: not aligned to its elements", name);
    if (rows == 1) ld = cols;
    if (ld < cols || ld > (int64_t(1) << 40))
        return fail(PS_EINVAL, "%s: row stride %lld for %lld columns", name,
                    static_cast<long long>(ld), static_cast<long long>(cols));
    const unsigned __int128 bytes =
        (static_cast<unsigned __int128>(rows - 1) * static_cast<uint64_t>(ld) + cols) * dtype_bytes(dtype);
    if (bytes >> 62) return fail(PS_EINVAL, "%s: too large", name);
    out->bytes = static_cast<uint64_t>(bytes);
    return PS_OK;
}

int plain(const char *name, const void *p, uint64_t bytes, size_t align, Span *out) {
    *out = Span{name, reinterpret_cast<uintptr_t>(p), bytes};
    if (bytes == 0) return PS_OK;
    if (p == nullptr) return fail(PS_EINVAL, "%s: null pointer", name);
    if (out->p % align) return fail(PS_EINVAL, "%s: not on a %zu-byte boundary", name, align);
    return PS_OK;
}

// No output may overlap another buffer.
int apart(const Span &out, const Span *others, int count) {
    for (int i = 0; i < count; ++i) {
        const Span &o = others[i];
        if (out.bytes && o.bytes && out.p < o.p + o.bytes && o.p < out.p + out.bytes)
            return fail(PS_EINVAL, "%s overlaps %s", out.name, o.name);
    }
    return PS_OK;
}

int size_in(const char *name, int64_t x, int64_t most) {
    if (x < 0 || x > most)
        return fail(PS_EINVAL, "%s: %lld outside [0, %lld]", name, static_cast<long long>(x),
                    static_cast<long long>(most));
    return PS_OK;
}

// The kernels' form of `drop`; *factor is multiplied by what survivors are.
int dropping(const pl_drop *drop, Drop *d, float *factor) {
    *d = Drop{0, 0, 0, 0, 0};
    if (drop == nullptr) return PS_OK;
    if (!(drop->p >= 0.0f && drop->p <= 1.0f))
        return fail(PS_EINVAL, "dropout probability %g outside [0, 1]", static_cast<double>(drop->p));
    d->drop = static_cast<uint32_t>(std::floor(65536.0 * static_cast<double>(drop->p) + 0.5));
    d->k0 = static_cast<uint32_t>(drop->seed);
    d->k1 = static_cast<uint32_t>(drop->seed >> 32);
    d->o0 = static_cast<uint32_t>(drop->offset);
    d->o1 = static_cast<uint32_t>(drop->offset >> 32);
    const double up = d->drop < 65536 ? 65536.0 / (65536.0 - d->drop) : 0.0;
    *factor = static_cast<float>(static_cast<double>(*factor) * up);
    return PS_OK;
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

int64_t blocks_of(int64_t cols) { return (cols + 127) / 128; }

int fp8(const char *name, const pl_fp8 *q, int64_t rows, int64_t cols, Span *values, Span *scales) {
    if (q == nullptr) return fail(PS_EINVAL, "%s: null", name);
    if (int rc = plain(name, q->values, pl_fp8_values_bytes(rows, cols), 16, values)) return rc;
    return plain(name, q->scales, pl_fp8_scales_bytes(rows, cols), 16, scales);
}

}  // namespace

const char *pl_last_error(void) { return g_error; }

int pl_embedding(const void *ids, int id_type, int64_t tokens, const void *table, int table_dtype,
                 int64_t vocab, int64_t dim, int64_t table_ld, float scale, const pl_drop *drop,
                 void *out, int out_dtype, int64_t out_ld, void *stream) {
    if (id_type != PL_I32 && id_type != PL_I64) return fail(PS_EINVAL, "id type %d", id_type);
    if (int rc = size_in("tokens", tokens, kMax - 1)) return rc;
    if (int rc = size_in("vocab", vocab, int64_t(1) << 48)) return rc;
    if (int rc = size_in("dim", dim, kMax)) return rc;
    RowsArgs a{};
    a.factor = scale;
    if (int rc = dropping(drop, &a.drop, &a.factor)) return rc;
    const size_t id_bytes = id_type == PL_I32 ? 4 : 8;
    Span in[2], o;
    if (int rc = plain("ids", ids, dim == 0 ? 0 : id_bytes * static_cast<uint64_t>(tokens), id_bytes, &in[0]))
        return rc;
    if (int rc = matrix("table", table, table_dtype, vocab, dim, table_ld, &in[1])) return rc;
    if (int rc = matrix("out", out, out_dtype, tokens, dim, out_ld, &o)) return rc;
    if (int rc = apart(o, in, 2)) return rc;
    if (tokens == 0 || dim == 0) return PS_OK;
    a.ids = ids;
    a.x = table;
    a.out = out;
    a.vocab = static_cast<uint64_t>(vocab);
    a.x_ld = table_ld;
    a.out_ld = out_ld;
    a.rows = static_cast<uint32_t>(tokens);
    a.cols = static_cast<uint64_t>(dim);
    return launched(launch_rows(a, id_type, table_dtype, out_dtype, static_cast<hipStream_t>(stream)),
                    "pl_embedding");
}

size_t pl_embedding_grad_workspace(int64_t tokens, int64_t vocab, int64_t dim) {
    if (tokens < 0 || tokens >= kMax / 2 || vocab <= 0 || vocab > kMax / 2 || dim <= 0 || dim > kMax)
        return 0;
    return grad_workspace(tokens, vocab, dim);
}

int pl_embedding_grad(const void *ids, int id_type, int64_t tokens, const void *grad,
                      int grad_dtype, int64_t grad_ld, int64_t dim, float scale,
                      const pl_drop *drop, void *out, int out_dtype, int64_t out_ld,
                      int64_t vocab, int accumulate, void *workspace, size_t workspace_bytes,
                      void *stream) {
    if (id_type != PL_I32 && id_type != PL_I64) return fail(PS_EINVAL, "id type %d", id_type);
    if (int rc = size_in("tokens", tokens, kMax / 2 - 1)) return rc;
    if (int rc = size_in("vocab", vocab, kMax / 2)) return rc;
    if (int rc = size_in("dim", dim, kMax)) return rc;
    GradArgs a{};
    a.factor = scale;
    if (int rc = dropping(drop, &a.drop, &a.factor)) return rc;
    const size_t id_bytes = id_type == PL_I32 ? 4 : 8;
    const size_t need = pl_embedding_grad_workspace(tokens, vocab, dim);
    Span in[3], o;
    if (int rc = plain("ids", ids, id_bytes * static_cast<uint64_t>(tokens), id_bytes, &in[0])) return rc;
    if (int rc = matrix("grad", grad, grad_dtype, tokens, dim, grad_ld, &in[1])) return rc;
    if (int rc = matrix("out", out, out_dtype, vocab, dim, out_ld, &o)) return rc;
    if (vocab == 0 || dim == 0) return PS_OK;
    if (workspace_bytes < need)
        return fail(PS_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    if (int rc = plain("workspace", workspace, need, 16, &in[2])) return rc;
    if (int rc = apart(o, in, 3)) return rc;
    if (int rc = apart(in[2], in, 2)) return rc;
    a.ids = ids;
    a.grad = grad;
    a.out = out;
    a.grad_ld = grad_ld;
    a.out_ld = out_ld;
    a.tokens = static_cast<uint32_t>(tokens);
    a.vocab = static_cast<uint32_t>(vocab);
    a.dim = static_cast<uint64_t>(dim);
    a.accumulate = accumulate != 0;
    a.workspace = workspace;
    return launched(launch_grad(a, id_type, grad_dtype, out_dtype, static_cast<hipStream_t>(stream)),
                    "pl_embedding_grad");
}

int pl_dropout(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld,
               const pl_drop *drop, void *out, int64_t out_ld, void *stream) {
    if (drop == nullptr) return fail(PS_EINVAL, "drop: null pointer");
    if (int rc = size_in("rows", rows, kMax - 1)) return rc;
    if (int rc = size_in("cols", cols, kMax)) return rc;
    RowsArgs a{};
    a.factor = 1.0f;
    if (int rc = dropping(drop, &a.drop, &a.factor)) return rc;
    Span in, o;
    if (int rc = matrix("x", x, dtype, rows, cols, ld, &in)) return rc;
    if (int rc = matrix("out", out, dtype, rows, cols, out_ld, &o)) return rc;
    if (x != out || (ld != out_ld && rows > 1))
        if (int rc = apart(o, &in, 1)) return rc;
    if (rows == 0 || cols == 0) return PS_OK;
    a.x = x;
    a.out = out;
    a.x_ld = ld;
    a.out_ld = out_ld;
    a.rows = static_cast<uint32_t>(rows);
    a.cols = static_cast<uint64_t>(cols);
    return launched(launch_rows(a, kNoIds, dtype, dtype, static_cast<hipStream_t>(stream)), "pl_dropout");
}

int64_t pl_fp8_ld(int64_t cols) { return cols <= 0 ? 0 : 128 * blocks_of(cols); }

size_t pl_fp8_values_bytes(int64_t rows, int64_t cols) {
    if (rows <= 0 || cols <= 0) return 0;
    return static_cast<size_t>(rows) * static_cast<size_t>(pl_fp8_ld(cols));
}

size_t pl_fp8_scales_bytes(int64_t rows, int64_t cols) {
    if (rows <= 0 || cols <= 0) return 0;
    return 4 * static_cast<size_t>(rows) * static_cast<size_t>((blocks_of(cols) + 3) / 4);
}

int pl_quantize_fp8(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, int square,
                    const pl_fp8 *out, const pl_fp8 *out_t, void *stream) {
    if (int rc = size_in("rows", rows, kMax / 2 - 1)) return rc;
    if (int rc = size_in("cols", cols, kMax / 2 - 1)) return rc;
    if (out == nullptr && out_t == nullptr) return fail(PS_EINVAL, "no output");
    Span in, o[4] = {};
    if (int rc = matrix("x", x, dtype, rows, cols, ld, &in)) return rc;
    if (out != nullptr)
        if (int rc = fp8("out", out, rows, cols, &o[0], &o[1])) return rc;
    if (out_t != nullptr)
        if (int rc = fp8("out_t", out_t, cols, rows, &o[2], &o[3])) return rc;
    for (int i = 0; i < 4; ++i) {
        if (int rc = apart(o[i], &in, 1)) return rc;
        if (int rc = apart(o[i], o + i + 1, 3 - i)) return rc;
    }
    if (rows == 0 || cols == 0) return PS_OK;
    QuantArgs a{};
    a.x = x;
    a.ld = ld;
    a.rows = rows;
    a.cols = cols;
    if (out != nullptr) {
        a.values = static_cast<uint8_t *>(out->values);
        a.scales = out->scales;
    }
    if (out_t != nullptr) {
        a.values_t = static_cast<uint8_t *>(out_t->values);
        a.scales_t = out_t->scales;
    }
    return launched(launch_quantize(a, dtype, square != 0, static_cast<hipStream_t>(stream)),
                    "pl_quantize_fp8");
}

namespace {

MatmulArgs product(int64_t m, int64_t n, int64_t k, const pl_fp8 *a, const pl_fp8 *b, void *out,
                   int64_t out_ld, void *workspace) {
    MatmulArgs g{};
    g.a = static_cast<const uint8_t *>(a->values);
    g.b = static_cast<const uint8_t *>(b->values);
    g.sa = a->scales;
    g.sb = b->scales;
    g.out = out;
    g.out_ld = out_ld;
    g.m = static_cast<uint32_t>(m);
    g.n = static_cast<uint32_t>(n);
    g.k = static_cast<uint32_t>(k);
    g.partial = static_cast<float *>(workspace);
    return g;
}

}  // namespace

size_t pl_matmul_fp8_workspace(int64_t m, int64_t n, int64_t k, int out_dtype) {
    if (m < 0 || m > kMostRows || n < 0 || n > kMostRows || k < 0 || k > kMostCols || !is_dtype(out_dtype))
        return 0;
    return matmul_workspace(m, n, k, out_dtype);
}

int pl_matmul_fp8(int64_t m, int64_t n, int64_t k, const pl_fp8 *a, const pl_fp8 *b,
                  const void *bias, int bias_dtype, int relu, void *out, int out_dtype,
                  int64_t out_ld, int accumulate, void *workspace, size_t workspace_bytes,
                  void *stream) {
    if (int rc = size_in("m", m, kMostRows)) return rc;
    if (int rc = size_in("n", n, kMostRows)) return rc;
    if (int rc = size_in("k", k, kMostCols)) return rc;
    if (accumulate && (bias != nullptr || relu))
        return fail(PS_EINVAL, "accumulate with a bias or relu");
    Span in[6] = {}, o;
    if (int rc = fp8("a", a, m, k, &in[0], &in[1])) return rc;
    if (int rc = fp8("b", b, n, k, &in[2], &in[3])) return rc;
    if (bias != nullptr)
        if (int rc = matrix("bias", bias, bias_dtype, 1, n, n, &in[4])) return rc;
    if (int rc = matrix("out", out, out_dtype, m, n, out_ld, &o)) return rc;
    if (m == 0 || n == 0) return PS_OK;
    const size_t need = pl_matmul_fp8_workspace(m, n, k, out_dtype);
    if (workspace_bytes < need)
        return fail(PS_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    if (int rc = plain("workspace", workspace, need, 16, &in[5])) return rc;
    if (int rc = apart(o, in, 6)) return rc;
    if (int rc = apart(in[5], in, 5)) return rc;
    MatmulArgs g = product(m, n, k, a, b, out, out_ld, workspace);
    g.bias = bias;
    g.bias_bf16 = bias != nullptr && bias_dtype == PS_BF16;
    g.relu = relu != 0;
    g.accumulate = accumulate != 0;
    return launched(launch_matmul(g, out_dtype, static_cast<hipStream_t>(stream)), "pl_matmul_fp8");
}

size_t pl_linear_fp8_workspace(int64_t m, int64_t n, int64_t k, int dtype, int out_dtype) {
    if (m < 0 || m > kMostRows || n < 0 || n > kMostRows || k < 0 || k > kMostCols || !is_dtype(dtype) ||
        !is_dtype(out_dtype))
        return 0;
    if (converts(m, n, k)) return 0;
    return align256(pl_fp8_values_bytes(m, k)) + align256(pl_fp8_scales_bytes(m, k)) +
           matmul_workspace(m, n, k, out_dtype);
}

int pl_linear_fp8(const void *x, int dtype, int64_t m, int64_t k, int64_t ld, int64_t n,
                  const pl_fp8 *w, const void *bias, int bias_dtype, int relu, void *out,
                  int out_dtype, int64_t out_ld, void *workspace, size_t workspace_bytes,
                  void *stream) {
    // everything is checked before the first launch
    Span in[5] = {}, o;
    if (int rc = size_in("m", m, kMostRows)) return rc;
    if (int rc = size_in("n", n, kMostRows)) return rc;
    if (int rc = size_in("k", k, kMostCols)) return rc;
    if (int rc = matrix("x", x, dtype, m, k, ld, &in[0])) return rc;
    if (int rc = fp8("w", w, n, k, &in[1], &in[2])) return rc;
    if (bias != nullptr)
        if (int rc = matrix("bias", bias, bias_dtype, 1, n, n, &in[3])) return rc;
    if (int rc = matrix("out", out, out_dtype, m, n, out_ld, &o)) return rc;
    if (m == 0 || n == 0) return PS_OK;
    const size_t need = pl_linear_fp8_workspace(m, n, k, dtype, out_dtype);
    if (workspace_bytes < need)
        return fail(PS_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    if (int rc = plain("workspace", workspace, need, 16, &in[4])) return rc;
    if (int rc = apart(o, in, 5)) return rc;
    if (int rc = apart(in[4], in, 4)) return rc;
    if (converts(m, n, k)) {
        const pl_fp8 none = {};
        MatmulArgs g = product(m, n, k, &none, w, out, out_ld, nullptr);
        g.bias = bias;
        g.bias_bf16 = bias != nullptr && bias_dtype == PS_BF16;
        g.relu = relu != 0;
        g.x = x;
        g.x_ld = ld;
        return launched(launch_convert_matmul(g, dtype, out_dtype, static_cast<hipStream_t>(stream)),
                        "pl_linear_fp8");
    }
    char *ws = static_cast<char *>(workspace);
    const size_t values = align256(pl_fp8_values_bytes(m, k)), scales = align256(pl_fp8_scales_bytes(m, k));
    const pl_fp8 q = {ws, reinterpret_cast<uint32_t *>(ws + values)};
    if (int rc = pl_quantize_fp8(x, dtype, m, k, ld, 0, &q, nullptr, stream)) return rc;
    return pl_matmul_fp8(m, n, k, &q, w, bias, bias_dtype, relu, out, out_dtype, out_ld, 0,
                         ws + values + scales, need - values - scales, stream);
}

namespace {

// Where the backward pass has what in its workspace.
struct GradRoom {
    size_t g_values, g_scales, t_values, t_scales, x_values, x_scales;
    size_t out, out_bytes, weight, weight_bytes;   // parts' sums of the two products
    size_t bytes;
};

GradRoom grad_room(int64_t m, int64_t n, int64_t k, int out_dtype, int weight_dtype) {
    GradRoom r{};
    size_t at = 0;
    auto take = [&at](size_t bytes) {
        const size_t was = at;
        at += align256(bytes);
        return was;
    };
    r.g_values = take(pl_fp8_values_bytes(m, n));
    r.g_scales = take(pl_fp8_scales_bytes(m, n));
    r.t_values = take(pl_fp8_values_bytes(n, m));
    r.t_scales = take(pl_fp8_scales_bytes(n, m));
    r.x_values = take(pl_fp8_values_bytes(k, m));
    r.x_scales = take(pl_fp8_scales_bytes(k, m));
    r.out = take(r.out_bytes = matmul_workspace(m, k, n, out_dtype));
    r.weight = take(r.weight_bytes = matmul_workspace(n, k, m, weight_dtype));
    r.bytes = at;
    return r;
}

}  // namespace

size_t pl_linear_fp8_grad_workspace(int64_t m, int64_t n, int64_t k, int out_dtype, int weight_dtype) {
    if (m < 0 || m > kMostCols || n < 0 || n > kMostCols || k < 0 || k > kMostRows ||
        !is_dtype(out_dtype) || !is_dtype(weight_dtype))
        return 0;
    return grad_room(m, n, k, out_dtype, weight_dtype).bytes;
}

int pl_linear_fp8_grad(const void *x, int x_dtype, int64_t x_ld, const void *grad, int grad_dtype,
                       int64_t grad_ld, int64_t m, int64_t n, int64_t k, const pl_fp8 *w_t, void *out,
                       int out_dtype, int64_t out_ld, void *weight_out, int weight_dtype,
                       int64_t weight_ld, int accumulate, void *workspace, size_t workspace_bytes,
                       void *stream) {
    if (int rc = size_in("m", m, kMostCols)) return rc;
    if (int rc = size_in("n", n, kMostCols)) return rc;
    if (int rc = size_in("k", k, kMostRows)) return rc;
    Span in[5] = {}, o[2];
    if (int rc = matrix("x", x, x_dtype, m, k, x_ld, &in[0])) return rc;
    if (int rc = matrix("grad", grad, grad_dtype, m, n, grad_ld, &in[1])) return rc;
    if (int rc = fp8("w_t", w_t, k, n, &in[2], &in[3])) return rc;
    if (int rc = matrix("out", out, out_dtype, m, k, out_ld, &o[0])) return rc;
    if (int rc = matrix("weight_out", weight_out, weight_dtype, n, k, weight_ld, &o[1])) return rc;
    const GradRoom r = grad_room(m, n, k, out_dtype, weight_dtype);
    if (workspace_bytes < r.bytes)
        return fail(PS_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, r.bytes);
    if (int rc = plain("workspace", workspace, r.bytes, 16, &in[4])) return rc;
    if (int rc = apart(o[0], in, 5)) return rc;
    if (int rc = apart(o[1], in, 5)) return rc;
    if (int rc = apart(o[0], &o[1], 1)) return rc;
    if (int rc = apart(in[4], in, 4)) return rc;
    char *ws = static_cast<char *>(workspace);
    auto at = [ws](size_t values, size_t scales) {
        return pl_fp8{ws + values, reinterpret_cast<uint32_t *>(ws + scales)};
    };
    const pl_fp8 g = at(r.g_values, r.g_scales), t = at(r.t_values, r.t_scales);
    const pl_fp8 xt = at(r.x_values, r.x_scales);
    hipStream_t s = static_cast<hipStream_t>(stream);
    QuantArgs qg{}, qx{};
    qg.x = grad;
    qg.ld = grad_ld;
    qg.rows = m;
    qg.cols = n;
    qg.values = static_cast<uint8_t *>(g.values);
    qg.scales = g.scales;
    qg.values_t = static_cast<uint8_t *>(t.values);
    qg.scales_t = t.scales;
    qx.x = x;
    qx.ld = x_ld;
    qx.rows = m;
    qx.cols = k;
    qx.values_t = static_cast<uint8_t *>(xt.values);
    qx.scales_t = xt.scales;
    const char *what = "pl_linear_fp8_grad";
    if (x_dtype == grad_dtype) {
        if (int rc = launched(launch_quantize_two(qg, qx, x_dtype, false, s), what)) return rc;
    } else {
        if (int rc = launched(launch_quantize_two(qg, QuantArgs{}, grad_dtype, false, s), what)) return rc;
        if (int rc = launched(launch_quantize_two(qx, QuantArgs{}, x_dtype, false, s), what)) return rc;
    }
    MatmulArgs p = product(m, k, n, &g, w_t, out, out_ld, r.out_bytes ? ws + r.out : nullptr);
    MatmulArgs pw = product(n, k, m, &t, &xt, weight_out, weight_ld,
                            r.weight_bytes ? ws + r.weight : nullptr);
    pw.accumulate = accumulate != 0;
    if (pairs(p, out_dtype, pw, weight_dtype))
        return launched(launch_matmul_two(p, out_dtype, pw, weight_dtype, s), what);
    if (p.m != 0 && p.n != 0)
        if (int rc = launched(launch_matmul(p, out_dtype, s), what)) return rc;
    if (pw.m == 0 || pw.n == 0) return PS_OK;
    return launched(launch_matmul(pw, weight_dtype, s), what);
}

// ------------------------------------------------------------------ norms

namespace {

constexpr int64_t kMostNormed = int64_t(1) << 29;   // columns: four threads each are one launch

// What the norms and their gradients have in common, checked; *in: spans of gate, after and before.
int norm_vectors(int64_t rows, int64_t cols, bool block, const void *gate, int gate_dtype, int64_t gates,
                 int64_t gate_ld, const void *after, const void *before, int weight_dtype, float scale, float eps,
                 Span *in) {
    if (int rc = size_in("rows", rows, kMax / 2 - 1)) return rc;
    if (int rc = size_in("cols", cols, kMostNormed)) return rc;
    if (!(eps > 0.0f) || std::isinf(eps)) return fail(PS_EINVAL, "eps %g", static_cast<double>(eps));
    if (!block && (gate != nullptr || after != nullptr)) return fail(PS_EINVAL, "a gate or after without y");
    if (!block && scale != 1.0f) return fail(PS_EINVAL, "a scale without y");
    if ((gate == nullptr) != (gates == 0)) return fail(PS_EINVAL, "gate: %lld rows", static_cast<long long>(gates));
    if (gate != nullptr) {
        if (int rc = size_in("gates", gates, std::max<int64_t>(rows, kMax / 2 - 1))) return rc;
        if (rows % gates != 0)
            return fail(PS_EINVAL, "%lld rows for %lld gates", static_cast<long long>(rows),
                        static_cast<long long>(gates));
        if (int rc = matrix("gate", gate, gate_dtype, gates, cols, gate_ld, &in[0])) return rc;
    }
    if (after != nullptr)
        if (int rc = matrix("after", after, weight_dtype, 1, cols, cols, &in[1])) return rc;
    if (before != nullptr)
        if (int rc = matrix("before", before, weight_dtype, 1, cols, cols, &in[2])) return rc;
    return PS_OK;
}

}  // namespace

int pl_norm(const void *x, int x_dtype, int64_t x_ld, const void *y, int y_dtype, int64_t y_ld, int64_t rows,
            int64_t cols, const void *gate, int gate_dtype, int64_t gates, int64_t gate_ld, const void *after,
            const void *before, int weight_dtype, float scale, float eps, void *out, int64_t out_ld, void *normed,
            int64_t normed_ld, void *stream) {
    const bool block = y != nullptr;
    Span in[5] = {}, o[2] = {};
    if (int rc = norm_vectors(rows, cols, block, gate, gate_dtype, gates, gate_ld, after, before, weight_dtype, scale,
                              eps, in))
        return rc;
    if (!is_dtype(y_dtype)) return fail(PS_EINVAL, "y: dtype %d", y_dtype);
    if (int rc = matrix("x", x, x_dtype, rows, cols, x_ld, &in[3])) return rc;
    if (block) {
        if (int rc = matrix("y", y, y_dtype, rows, cols, y_ld, &in[4])) return rc;
        if (int rc = matrix("out", out, x_dtype, rows, cols, out_ld, &o[0])) return rc;
    } else if (out != nullptr) {
        return fail(PS_EINVAL, "out without y");
    }
    if (normed != nullptr) {
        if (int rc = matrix("normed", normed, y_dtype, rows, cols, normed_ld, &o[1])) return rc;
    } else if (!block && rows != 0 && cols != 0) {
        return fail(PS_EINVAL, "normed: null pointer");
    }
    if (before != nullptr && normed == nullptr && rows != 0 && cols != 0)
        return fail(PS_EINVAL, "before without normed");
    for (int i = 0; i < 2; ++i) {
        if (int rc = apart(o[i], in, 5)) return rc;
        if (int rc = apart(o[i], o + i + 1, 1 - i)) return rc;
    }
    if (rows == 0 || cols == 0) return PS_OK;
    NormArgs a{};
    a.x = x;
    a.y = y;
    a.x_ld = x_ld;
    a.y_ld = y_ld;
    a.rows = static_cast<uint32_t>(rows);
    a.per_gate = static_cast<uint32_t>(gates == 0 ? 1 : rows / gates);
    a.cols = static_cast<uint64_t>(cols);
    a.gate = gate;
    a.after = after;
    a.before = before;
    a.gate_ld = gate_ld;
    a.gate_bf16 = gate_dtype == PS_BF16;
    a.weight_bf16 = weight_dtype == PS_BF16;
    a.scale = scale;
    a.eps = eps;
    a.out = out;
    a.normed = normed;
    a.out_ld = out_ld;
    a.normed_ld = normed_ld;
    return launched(launch_norm(a, x_dtype, y_dtype, static_cast<hipStream_t>(stream)), "pl_norm");
}

size_t pl_norm_grad_workspace(int64_t rows, int64_t cols) {
    if (rows <= 0 || rows >= kMax / 2 || cols <= 0 || cols > kMostNormed) return 0;
    return norm_grad_workspace(rows, cols);
}

int pl_norm_grad(const void *h, int x_dtype, int64_t h_ld, const void *y, int y_dtype, int64_t y_ld, const void *grad,
                 int64_t grad_ld, const void *normed_grad, int64_t normed_grad_ld, int64_t rows, int64_t cols,
                 const void *gate, int gate_dtype, int64_t gates, int64_t gate_ld, const void *after,
                 const void *before, int weight_dtype, float scale, float eps, void *x_out, int64_t x_out_ld,
                 void *y_out, int64_t y_out_ld, void *gate_out, int64_t gate_out_ld, void *after_out,
                 void *before_out, int weight_out_dtype, int accumulate, void *workspace, size_t workspace_bytes,
                 void *stream) {
    const bool block = y != nullptr, some = rows != 0 && cols != 0;
    Span in[8] = {}, o[5] = {};
    if (int rc = norm_vectors(rows, cols, block, gate, gate_dtype, gates, gate_ld, after, before, weight_dtype, scale,
                              eps, in))
        return rc;
    if (!is_dtype(y_dtype)) return fail(PS_EINVAL, "y: dtype %d", y_dtype);
    if (grad == nullptr && normed_grad == nullptr && some) return fail(PS_EINVAL, "no gradient");
    if (normed_grad == nullptr && some && (before != nullptr || before_out != nullptr))
        return fail(PS_EINVAL, "before without normed_grad");
    if (!block && y_out != nullptr) return fail(PS_EINVAL, "y_out without y");
    if (gate == nullptr && gate_out != nullptr) return fail(PS_EINVAL, "gate_out without a gate");
    if (after == nullptr && after_out != nullptr) return fail(PS_EINVAL, "after_out without after");
    if (before == nullptr && before_out != nullptr) return fail(PS_EINVAL, "before_out without before");
    if (int rc = matrix("h", h, x_dtype, rows, cols, h_ld, &in[3])) return rc;
    if (block)
        if (int rc = matrix("y", y, y_dtype, rows, cols, y_ld, &in[4])) return rc;
    if (grad != nullptr)
        if (int rc = matrix("grad", grad, x_dtype, rows, cols, grad_ld, &in[5])) return rc;
    if (normed_grad != nullptr)
        if (int rc = matrix("normed_grad", normed_grad, y_dtype, rows, cols, normed_grad_ld, &in[6])) return rc;
    if (int rc = matrix("x_out", x_out, x_dtype, rows, cols, x_out_ld, &o[0])) return rc;
    if (block)
        if (int rc = matrix("y_out", y_out, y_dtype, rows, cols, y_out_ld, &o[1])) return rc;
    if (gate_out != nullptr)
        if (int rc = matrix("gate_out", gate_out, weight_out_dtype, gates, cols, gate_out_ld, &o[2])) return rc;
    if (after_out != nullptr)
        if (int rc = matrix("after_out", after_out, weight_out_dtype, 1, cols, cols, &o[3])) return rc;
    if (before_out != nullptr)
        if (int rc = matrix("before_out", before_out, weight_out_dtype, 1, cols, cols, &o[4])) return rc;
    if (cols == 0) return PS_OK;
    const size_t need = pl_norm_grad_workspace(rows, cols);
    if (workspace_bytes < need)
        return fail(PS_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    if (int rc = plain("workspace", workspace, need, 16, &in[7])) return rc;
    for (int i = 0; i < 5; ++i) {
        if (int rc = apart(o[i], in, 8)) return rc;
        if (int rc = apart(o[i], o + i + 1, 4 - i)) return rc;
    }
    if (int rc = apart(in[7], in, 7)) return rc;
    NormGradArgs a{};
    a.h = h;
    a.y = y;
    a.dh = grad;
    a.dz = normed_grad;
    a.h_ld = h_ld;
    a.y_ld = y_ld;
    a.dh_ld = grad_ld;
    a.dz_ld = normed_grad_ld;
    a.rows = static_cast<uint32_t>(rows);
    a.gates = static_cast<uint32_t>(gates);
    a.per_gate = static_cast<uint32_t>(gates == 0 ? 1 : rows / gates);
    a.cols = static_cast<uint64_t>(cols);
    a.gate = gate;
    a.after = after;
    a.before = before;
    a.gate_ld = gate_ld;
    a.gate_bf16 = gate_dtype == PS_BF16;
    a.weight_bf16 = weight_dtype == PS_BF16;
    a.scale = scale;
    a.eps = eps;
    a.dx = x_out;
    a.dy = y_out;
    a.dx_ld = x_out_ld;
    a.dy_ld = y_out_ld;
    a.dgate = gate_out;
    a.dafter = after_out;
    a.dbefore = before_out;
    a.dgate_ld = gate_out_ld;
    a.out_bf16 = weight_out_dtype == PS_BF16;
    a.accumulate = accumulate != 0;
    a.workspace = workspace;
    return launched(launch_norm_grad(a, x_dtype, y_dtype, static_cast<hipStream_t>(stream)), "pl_norm_grad");
}

// ---------------------------------------------------------- 8-bit integers

namespace {

constexpr int64_t kMostTerms = int64_t(1) << 17;   // 127^2 times it is below 2^31

int int8(const char *name, const pl_int8 *q, int64_t rows, int64_t cols, Span *values, Span *scales) {
    if (q == nullptr) return fail(PS_EINVAL, "%s: null", name);
    if (int rc = plain(name, q->values, pl_int8_values_bytes(rows, cols), 16, values)) return rc;
    return plain(name, q->scales, 4 * static_cast<uint64_t>(rows), 16, scales);
}

Int8Args int8_product(int64_t m, int64_t n, int64_t k, const pl_int8 *a, const pl_int8 *b, const void *bias,
                      int bias_dtype, int relu, void *out, int64_t out_ld, void *workspace) {
    Int8Args g{};
    if (a != nullptr) {
        g.a = a->values;
        g.sa = a->scales;
    }
    g.b = b->values;
    g.sb = b->scales;
    g.bias = bias;
    g.bias_bf16 = bias != nullptr && bias_dtype == PS_BF16;
    g.relu = relu != 0;
    g.out = out;
    g.out_ld = out_ld;
    g.m = static_cast<uint32_t>(m);
    g.n = static_cast<uint32_t>(n);
    g.k = static_cast<uint32_t>(k);
    g.partial = static_cast<int32_t *>(workspace);
    return g;
}

bool int8_sizes(int64_t m, int64_t n, int64_t k) {
    return m >= 0 && m <= kMostRows && n >= 0 && n <= kMostRows && k >= 0 && k <= kMostTerms;
}

}  // namespace

int64_t pl_int8_ld(int64_t cols) { return cols <= 0 ? 0 : 128 * blocks_of(cols); }

size_t pl_int8_values_bytes(int64_t rows, int64_t cols) {
    if (rows <= 0 || cols <= 0) return 0;
    return static_cast<size_t>(rows) * static_cast<size_t>(pl_int8_ld(cols));
}

int pl_quantize_int8(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, const pl_int8 *out,
                     void *stream) {
    if (int rc = size_in("rows", rows, kMostRows)) return rc;
    if (int rc = size_in("cols", cols, kMostTerms)) return rc;
    Span in, o[2] = {};
    if (int rc = matrix("x", x, dtype, rows, cols, ld, &in)) return rc;
    if (int rc = int8("out", out, rows, cols, &o[0], &o[1])) return rc;
    if (int rc = apart(o[0], &in, 1)) return rc;
    if (int rc = apart(o[1], &in, 1)) return rc;
    if (int rc = apart(o[0], &o[1], 1)) return rc;
    if (rows == 0) return PS_OK;
    Int8QuantArgs a{};
    a.x = x;
    a.ld = ld;
    a.rows = rows;
    a.cols = cols;
    a.values = out->values;
    a.scales = out->scales;
    return launched(launch_quantize_int8(a, dtype, static_cast<hipStream_t>(stream)), "pl_quantize_int8");
}

size_t pl_matmul_int8_workspace(int64_t m, int64_t n, int64_t k) {
    return int8_sizes(m, n, k) ? int8_workspace(m, n, k) : 0;
}

int pl_matmul_int8(int64_t m, int64_t n, int64_t k, const pl_int8 *a, const pl_int8 *b, const void *bias,
                   int bias_dtype, int relu, void *out, int out_dtype, int64_t out_ld, void *workspace,
                   size_t workspace_bytes, void *stream) {
    if (int rc = size_in("m", m, kMostRows)) return rc;
    if (int rc = size_in("n", n, kMostRows)) return rc;
    if (int rc = size_in("k", k, kMostTerms)) return rc;
    Span in[6] = {}, o;
    if (int rc = int8("a", a, m, k, &in[0], &in[1])) return rc;
    if (int rc = int8("b", b, n, k, &in[2], &in[3])) return rc;
    if (bias != nullptr)
        if (int rc = matrix("bias", bias, bias_dtype, 1, n, n, &in[4])) return rc;
    if (int rc = matrix("out", out, out_dtype, m, n, out_ld, &o)) return rc;
    if (m == 0 || n == 0) return PS_OK;
    const size_t need = pl_matmul_int8_workspace(m, n, k);
    if (workspace_bytes < need)
        return fail(PS_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    if (int rc = plain("workspace", workspace, need, 16, &in[5])) return rc;
    if (int rc = apart(o, in, 6)) return rc;
    if (int rc = apart(in[5], in, 5)) return rc;
    const Int8Args g = int8_product(m, n, k, a, b, bias, bias_dtype, relu, out, out_ld, workspace);
    return launched(launch_int8(g, out_dtype, static_cast<hipStream_t>(stream)), "pl_matmul_int8");
}

size_t pl_linear_int8_workspace(int64_t m, int64_t n, int64_t k) {
    if (!int8_sizes(m, n, k) || int8_converts(m, n, k)) return 0;
    return align256(pl_int8_values_bytes(m, k)) + align256(4 * static_cast<size_t>(m)) + int8_workspace(m, n, k);
}

int pl_linear_int8(const void *x, int dtype, int64_t m, int64_t k, int64_t ld, int64_t n, const pl_int8 *w,
                   const void *bias, int bias_dtype, int relu, void *out, int out_dtype, int64_t out_ld,
                   void *workspace, size_t workspace_bytes, void *stream) {
    // everything is checked before the first launch
    Span in[5] = {}, o;
    if (int rc = size_in("m", m, kMostRows)) return rc;
    if (int rc = size_in("n", n, kMostRows)) return rc;
    if (int rc = size_in("k", k, kMostTerms)) return rc;
    if (int rc = matrix("x", x, dtype, m, k, ld, &in[0])) return rc;
    if (int rc = int8("w", w, n, k, &in[1], &in[2])) return rc;
    if (bias != nullptr)
        if (int rc = matrix("bias", bias, bias_dtype, 1, n, n, &in[3])) return rc;
    if (int rc = matrix("out", out, out_dtype, m, n, out_ld, &o)) return rc;
    if (m == 0 || n == 0) return PS_OK;
    const size_t need = pl_linear_int8_workspace(m, n, k);
    if (workspace_bytes < need)
        return fail(PS_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    if (int rc = plain("workspace", workspace, need, 16, &in[4])) return rc;
    if (int rc = apart(o, in, 5)) return rc;
    if (int rc = apart(in[4], in, 4)) return rc;
    if (int8_converts(m, n, k)) {
        Int8Args g = int8_product(m, n, k, nullptr, w, bias, bias_dtype, relu, out, out_ld, nullptr);
        g.x = x;
        g.x_ld = ld;
        g.x_bf16 = dtype == PS_BF16;
        return launched(launch_int8(g, out_dtype, static_cast<hipStream_t>(stream)), "pl_linear_int8");
    }
    char *ws = static_cast<char *>(workspace);
    const size_t values = align256(pl_int8_values_bytes(m, k)), scales = align256(4 * static_cast<size_t>(m));
    const pl_int8 q = {reinterpret_cast<int8_t *>(ws), reinterpret_cast<float *>(ws + values)};
    if (int rc = pl_quantize_int8(x, dtype, m, k, ld, &q, stream)) return rc;
    return pl_matmul_int8(m, n, k, &q, w, bias, bias_dtype, relu, out, out_dtype, out_ld, ws + values + scales,
                          need - values - scales, stream);
}

// ------------------------------------------------------------------ AdamW

namespace {

constexpr int64_t kMostParams = int64_t(1) << 40;

// Elements of the states of such tensors, or -1.
int64_t adamw_room(const pl_adamw_tensor *tensors, int64_t n) {
    if (size_in("tensors", n, kMax / 2)) return -1;
    if (n != 0 && tensors == nullptr) return fail(-1, "tensors: null pointer");
    int64_t room = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (size_in("a tensor's count", tensors[i].count, kMostParams)) return -1;
        room += (tensors[i].count + 127) / 128 * 128;
        if (room > kMostParams) return fail(-1, "tensors: more than 2^40 elements");
    }
    return room;
}

// Every output against all that is read or written: of neighbours in memory, one that begins before
// an earlier one of which it may share nothing has ended.
int adamw_apart(std::vector<Span> &written, std::vector<Span> &read) {
    auto before = [](const Span &a, const Span &b) { return a.p < b.p; };
    std::sort(written.begin(), written.end(), before);
    for (size_t i = 1; i < written.size(); ++i)
        if (int rc = apart(written[i], &written[i - 1], 1)) return rc;
    std::sort(read.begin(), read.end(), before);
    // written ones share nothing now: their ends are in their order, too
    size_t w = 0;
    for (const Span &r : read) {
        while (w < written.size() && written[w].p + written[w].bytes <= r.p) ++w;
        if (w < written.size())
            if (int rc = apart(written[w], &r, 1)) return rc;
    }
    return PS_OK;
}

}  // namespace

int64_t pl_adamw_room(const pl_adamw_tensor *tensors, int64_t n) { return adamw_room(tensors, n); }

int64_t pl_adamw_parts(const pl_adamw_tensor *tensors, int64_t n) {
    const int64_t room = adamw_room(tensors, n);
    if (room < 0) return -1;
    const int64_t most = adamw_part();
    int64_t parts = 0;
    for (int64_t i = 0; i < n; ++i) parts += (tensors[i].count + most - 1) / most;
    return parts;
}

size_t pl_adamw_plan_bytes(int64_t parts) { return parts <= 0 ? 0 : sizeof(AdamwPart) * static_cast<size_t>(parts); }

int pl_adamw_plan(const pl_adamw_tensor *tensors, int64_t n, int weight_dtype, int grad_dtype, int push,
                  int64_t steps, void *plan, size_t plan_bytes) {
    const int64_t parts = pl_adamw_parts(tensors, n);
    if (parts < 0) return PS_EINVAL;
    if (!is_dtype(weight_dtype) || (!push && weight_dtype != PS_F32))
        return fail(PS_EINVAL, "weight: dtype %d", weight_dtype);
    if (!is_dtype(grad_dtype)) return fail(PS_EINVAL, "grad: dtype %d", grad_dtype);
    if (int rc = size_in("steps", steps, kMostParams)) return rc;
    if (parts == 0) return PS_OK;
    if (plan == nullptr) return fail(PS_EINVAL, "plan: null pointer");
    if (plan_bytes < pl_adamw_plan_bytes(parts))
        return fail(PS_ENOMEM, "plan of %zu bytes, %zu needed", plan_bytes, pl_adamw_plan_bytes(parts));
    const size_t wb = dtype_bytes(weight_dtype), gb = dtype_bytes(grad_dtype);
    try {
        std::vector<Span> weights, grads;
        for (int64_t i = 0; i < n; ++i) {
            const uint64_t count = static_cast<uint64_t>(tensors[i].count);
            Span s;
            if (int rc = plain("weight", tensors[i].weight, count * wb, wb, &s)) return rc;
            if (count != 0) weights.push_back(s);
            if (int rc = plain("grad", tensors[i].grad, count * gb, gb, &s)) return rc;
            if (count != 0) grads.push_back(s);
        }
        if (int rc = push ? adamw_apart(grads, weights) : adamw_apart(weights, grads)) return rc;
    } catch (...) {
        return fail(PS_ENOMEM, "no memory for the check of %lld tensors", static_cast<long long>(n));
    }
    const int64_t most = adamw_part();
    char *to = static_cast<char *>(plan);
    int64_t at = 0;
    for (int64_t i = 0; i < n; ++i) {
        const pl_adamw_tensor &t = tensors[i];
        for (int64_t first = 0; first < t.count; first += most) {
            AdamwPart p{};
            p.weight = static_cast<char *>(t.weight) + first * wb;
            p.grad = static_cast<char *>(t.grad) + first * gb;
            p.at = at + first;
            p.steps = steps;
            p.count = static_cast<uint32_t>(std::min(most, t.count - first));
            p.decay = t.decay;
            std::memcpy(to, &p, sizeof(p));   // the caller's memory may lie anywhere
            to += sizeof(p);
        }
        at += (t.count + 127) / 128 * 128;
    }
    return PS_OK;
}

int64_t pl_adamw_steps(const void *plan) {
    AdamwPart p;
    std::memcpy(&p, plan, sizeof(p));
    return p.steps;
}

int pl_adamw_step(void *plan, int64_t parts, int weight_dtype, int grad_dtype, int push, int bits, int64_t room,
                  void *m, void *v, uint8_t *m_scales, uint8_t *v_scales, double beta1, double beta2, float eps,
                  float lr, const float *lr_at, float factor, const float *factor_at, uint64_t seed, void *stream) {
    if (int rc = size_in("parts", parts, kMostParams / 128)) return rc;
    if (int rc = size_in("room", room, kMostParams)) return rc;
    if (room % 128) return fail(PS_EINVAL, "room: not a multiple of 128");
    if (!is_dtype(weight_dtype) || (!push && weight_dtype != PS_F32))
        return fail(PS_EINVAL, "weight: dtype %d", weight_dtype);
    if (!is_dtype(grad_dtype)) return fail(PS_EINVAL, "grad: dtype %d", grad_dtype);
    if (bits != 8 && bits != 32) return fail(PS_EINVAL, "states of %d bits", bits);
    for (const double b : {beta1, beta2})
        if (!(b >= 0.0 && b <= 1.0 - 0x1p-28)) return fail(PS_EINVAL, "beta %.10g outside [0, 1 - 2^-28]", b);
    if (!(eps >= 0.0f) || std::isinf(eps)) return fail(PS_EINVAL, "eps %g", static_cast<double>(eps));
    Span s[7] = {};
    const uint64_t n = static_cast<uint64_t>(room);
    if (int rc = plain("plan", plan, pl_adamw_plan_bytes(parts), 16, &s[0])) return rc;
    if (int rc = plain("m", m, bits / 8 * n, 16, &s[1])) return rc;
    if (int rc = plain("v", v, bits / 8 * n, 16, &s[2])) return rc;
    if (bits == 8) {
        if (int rc = plain("m_scales", m_scales, n / 128, 1, &s[3])) return rc;
        if (int rc = plain("v_scales", v_scales, n / 128, 1, &s[4])) return rc;
    }
    if (lr_at != nullptr)
        if (int rc = plain("lr_at", lr_at, 4, 4, &s[5])) return rc;
    if (factor_at != nullptr)
        if (int rc = plain("factor_at", factor_at, 4, 4, &s[6])) return rc;
    for (int i = 0; i < 5; ++i)
        if (int rc = apart(s[i], s + i + 1, 6 - i)) return rc;
    if (parts == 0) return PS_OK;
    AdamwArgs a{};
    a.plan = static_cast<AdamwPart *>(plan);
    a.parts = static_cast<uint64_t>(parts);
    a.m = m;
    a.v = v;
    a.m_scales = m_scales;
    a.v_scales = v_scales;
    a.log2_beta1 = std::log2(beta1);
    a.log2_beta2 = std::log2(beta2);
    a.beta1 = static_cast<float>(beta1);
    a.beta2 = static_cast<float>(beta2);
    a.rest1 = static_cast<float>(1.0 - beta1);
    a.rest2 = static_cast<float>(1.0 - beta2);
    a.eps = eps;
    a.lr = lr;
    a.factor = factor;
    a.lr_at = lr_at;
    a.factor_at = factor_at;
    a.seed = seed;
    a.plain = eps >= 0x1p-30f && eps <= 0x1p100f && 1.0 - beta2 >= 0x1p-18;
    return launched(launch_adamw(a, weight_dtype, grad_dtype, bits, push != 0, static_cast<hipStream_t>(stream)),
                    "pl_adamw_step");
}

int pl_adamw_moments(int64_t room, const void *m, const void *v, const uint8_t *m_scales, const uint8_t *v_scales,
                     void *m_out, void *v_out, int dtype, void *stream) {
    if (int rc = size_in("room", room, kMostParams)) return rc;
    if (room % 128) return fail(PS_EINVAL, "room: not a multiple of 128");
    if (!is_dtype(dtype)) return fail(PS_EINVAL, "dtype %d", dtype);
    const uint64_t n = static_cast<uint64_t>(room);
    Span in[4] = {}, o[2] = {};
    if (int rc = plain("m", m, n, 16, &in[0])) return rc;
    if (int rc = plain("v", v, n, 16, &in[1])) return rc;
    if (int rc = plain("m_scales", m_scales, n / 128, 1, &in[2])) return rc;
    if (int rc = plain("v_scales", v_scales, n / 128, 1, &in[3])) return rc;
    if (int rc = plain("m_out", m_out, n * dtype_bytes(dtype), dtype_bytes(dtype), &o[0])) return rc;
    if (int rc = plain("v_out", v_out, n * dtype_bytes(dtype), dtype_bytes(dtype), &o[1])) return rc;
    if (int rc = apart(o[0], in, 4)) return rc;
    if (int rc = apart(o[1], in, 4)) return rc;
    if (int rc = apart(o[0], &o[1], 1)) return rc;
    if (room == 0) return PS_OK;
    MomentsArgs a{};
    a.m = static_cast<const uint8_t *>(m);
    a.v = static_cast<const uint8_t *>(v);
    a.m_scales = m_scales;
    a.v_scales = v_scales;
    a.m_out = m_out;
    a.v_out = v_out;
    a.room = n;
    return launched(launch_moments(a, dtype, static_cast<hipStream_t>(stream)), "pl_adamw_moments");
}

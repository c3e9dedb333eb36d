// One AdamW step over many tensors.
//
// Mathematics, of each element, t = steps made + 1:
//
//   m = b1 m + (1 - b1) f g        v = b2 v + (1 - b2) (f g)^2
//   step = lr (m up / (sqrt(v) root + eps) + decay w)
//   up = 1 / (1 - b1^t), root = (1 - b2^t)^-1/2
//
// and w - step for w, or the step in g's place. Products and sums of m and v round one by one, so
// that what is kept of them in 8 bits is a function of the arguments alone.
//
// States in 8 bits, for each 128 elements one exponent: magnitudes are numbers of 3 fraction bits
// and 4 exponent bits (m, with a sign) or 5 (v, whose root so spans 2^17: an element far below its
// block's largest keeps a denominator). Scaled so that the format's least normal number is fp32's,
// a number's bits without the last 20 are its code, subnormal ones included: rounding is one
// addition of random bits and a shift. The rounding is random because a mean that moves by (1 -
// b2) of itself a step, 2^-10, would never leave a number of 3 fraction bits if rounded to nearest.
// A positive v is never rounded to 0, below which m / sqrt(v) has no bound.
//
// Bound by memory in 32 bits, by memory and vector instructions in 8: 61M elements in 32 bits 298 us (1.71 GB, 5.7
// TB/s; a copy reaches 5.1), 138M in 8 bits with bf16 gradients 317 us (1.94 GB, 6.1 TB/s; vector instructions
// five sixths of the time).
#include "pl_device.h"

namespace gadei::learner {
namespace {

constexpr int kThreads = 256;
constexpr int kFour = 4;    // neighbouring elements a lane
constexpr int kFours = 2;   // of them: 138M elements in 8 bits 333 us with one, 316 with two, 330 with four
constexpr int kPart = kThreads * kFour * kFours;

typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
typedef u16x4 u16x4_any __attribute__((aligned(2)));

__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
    return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
}

// Philox4x32-7: as pl_device.h's philox with seven rounds, the fewest that its authors found to pass
// their tests; a word an element.
__device__ __forceinline__ u32x4 random4(uint64_t j, uint64_t t, uint64_t seed) {
    uint32_t c0 = static_cast<uint32_t>(j), c1 = static_cast<uint32_t>(j >> 32);
    uint32_t c2 = static_cast<uint32_t>(t), c3 = static_cast<uint32_t>(t >> 32);
    uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
#pragma unroll
    for (int i = 0; i < 7; ++i) {
        const uint64_t p0 = static_cast<uint64_t>(0xD2511F53u) * c0;
        const uint64_t p1 = static_cast<uint64_t>(0xCD9E8D57u) * c2;
        c0 = xor3(static_cast<uint32_t>(p1 >> 32), c1, k0);
        c2 = xor3(static_cast<uint32_t>(p0 >> 32), c3, k1);
        c1 = static_cast<uint32_t>(p1);
        c3 = static_cast<uint32_t>(p0);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
}

// Loads and stores, PAST: past the caches. So go gradients and states, which nothing reads before the next step,
// and weights (with push the steps) where they do not fit in the last level, counted as whole parts of weights:
// in us, none past them, gradients and states, and all: 25M in 32 bits 141, 127 and 128 (again on the same tensors
// 141, 106 and 128), 61M 340, 320 and 317 (340, 252 and 312), 138M 775, 737 and 723; 138M in 8 bits with bf16
// gradients 370, 343 and 331.
constexpr uint64_t kLastLevel = 256ull << 20;
template <bool PAST>
__device__ __forceinline__ f32x4 get(const f32x4_any *p) {
    if constexpr (PAST) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool PAST>
__device__ __forceinline__ u32x2 get(const u32x2_any *p) {
    if constexpr (PAST) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool PAST>
__device__ __forceinline__ void put(f32x4_any *p, f32x4 x) {
    if constexpr (PAST) __builtin_nontemporal_store(x, p);
    else *p = x;
}
template <bool PAST>
__device__ __forceinline__ void put(u32x2_any *p, u32x2 x) {
    if constexpr (PAST) __builtin_nontemporal_store(x, p);
    else *p = x;
}

// Four elements as loaded; those past `count` are 0.
template <int DT, bool PAST>
__device__ __forceinline__ f32x4 load4(const void *p, int64_t i, int count) {
    f32x4 x = {0, 0, 0, 0};
    if (count >= kFour) {
        if constexpr (DT == PS_F32) {
            x = get<PAST>(reinterpret_cast<const f32x4_any *>(static_cast<const float *>(p) + i));
        } else {
            const u32x2 w = get<PAST>(reinterpret_cast<const u32x2_any *>(static_cast<const uint16_t *>(p) + i));
            x = f32x4{lo_bf16(w[0]), hi_bf16(w[0]), lo_bf16(w[1]), hi_bf16(w[1])};
        }
    } else {
#pragma unroll
        for (int e = 0; e < kFour; ++e)
            if (e < count) x[e] = load1<DT>(p, i + e);
    }
    return x;
}

template <int DT, bool PAST>
__device__ __forceinline__ void store4(void *p, int64_t i, f32x4 x, int count) {
    if (count >= kFour) {
        if constexpr (DT == PS_F32)
            put<PAST>(reinterpret_cast<f32x4_any *>(static_cast<float *>(p) + i), x);
        else
            put<PAST>(reinterpret_cast<u32x2_any *>(static_cast<uint16_t *>(p) + i),
                      u32x2{bf16x2_rne(x[0], x[1]), bf16x2_rne(x[2], x[3])});
    } else {
#pragma unroll
        for (int e = 0; e < kFour; ++e)
            if (e < count) store1<DT>(p, i + e, x[e]);
    }
}

// The byte of a block whose largest magnitude has these bits (of NaN, with any sign and payload: without the sign
// the sum does not pass 32 bits): the exponent field, one more above 1.875 times its power of two, which is the
// largest code. 255: not finite, or above 1.875 * 2^127.
__device__ __forceinline__ int block_byte(uint32_t bits) {
    return static_cast<int>(min(((bits & 0x7fffffffu) + 0xfffffu) >> 23, 255u));
}
constexpr int kBad = 255;

// Element e of four codes. A code is the upper bits of a small fp32 number, m's below its sign.
template <bool SIGNED>
__device__ __forceinline__ float decode(uint32_t codes, int e, int byte) {
    if constexpr (SIGNED) {
        const int32_t wide = static_cast<int8_t>(codes >> 8 * e);
        return ldexpf(__uint_as_float(static_cast<uint32_t>(wide) << 20 & 0x87f00000u), byte - 15);
    }
    return ldexpf(__uint_as_float((codes >> 8 * e & 0xffu) << 20), byte - 31);
}

// The code of x is the upper byte; r: 16 random bits.
template <bool SIGNED>
__device__ __forceinline__ uint32_t encode(float x, int byte, uint32_t r) {
    const uint32_t scaled = __float_as_uint(ldexpf(x, (SIGNED ? 15 : 31) - byte));
    const uint32_t sum = scaled + 16 * r;   // the sign stays: magnitudes end 4 bits below it
    if constexpr (SIGNED) return (sum & 0x80000000u) | (sum << 4 & 0x7fffffffu);
    return max(sum, x > 0.0f ? 1u << 20 : 0u) << 4;
}

// The upper bytes of four words.
__device__ __forceinline__ uint32_t upper_bytes(const uint32_t (&x)[kFour]) {
    const uint32_t lo = __builtin_amdgcn_perm(x[1], x[0], 0x0c0c0703);
    const uint32_t hi = __builtin_amdgcn_perm(x[3], x[2], 0x07030c0c);
    return lo | hi;
}

// The largest of the 32 lanes that hold a block: sixteen by rotations, then the two rows of lanes.
__device__ __forceinline__ uint32_t most_of_32(uint32_t m) {
    m = max(m, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(m, 0x128, 0xf, 0xf, true)));
    m = max(m, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(m, 0x124, 0xf, 0xf, true)));
    m = max(m, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(m, 0x122, 0xf, 0xf, true)));
    m = max(m, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(m, 0x121, 0xf, 0xf, true)));
    const auto p = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    return max(p[0], p[1]);
}

struct Factors {
    uint64_t t;
    float up, root, lr, factor;
};

// Four elements of a lane, as loaded.
struct Four {
    f32x4 w, g, m, v;       // m and v in 32 bits
    uint32_t cm, cv;        // in 8
    int bm, bv;
};

// A workgroup makes the step of one part, whose loads are all under way while one wave computes the
// factors that depend on the number of the step. FULL: the part has all its elements.
template <int W, int G, int BITS, bool PUSH, bool WEIGHTS_PAST, bool FULL>
__device__ __forceinline__ void step_part(const AdamwArgs &a, AdamwPart *part, const AdamwPart &p, Factors &shared) {
#pragma clang fp contract(off)
    void *const w = p.weight, *const g = p.grad;
    const int64_t first = p.at;   // of the states
    const int count = FULL ? kPart : static_cast<int>(p.count);
    const float decay = p.decay;
    const int room = (count + 127) & ~127;
    Four x[kFours];
#pragma unroll
    for (int j = 0; j < kFours; ++j) {
        const int i = (threadIdx.x + j * kThreads) * kFour, left = FULL ? kFour : count - i;
        if (!FULL && i >= room) continue;
        x[j].w = load4<W, WEIGHTS_PAST>(w, i, left);
        x[j].g = load4<G, true>(g, i, left);
        if constexpr (BITS == 32) {
            x[j].m = get<true>(reinterpret_cast<const f32x4_any *>(static_cast<const float *>(a.m) + first + i));
            x[j].v = get<true>(reinterpret_cast<const f32x4_any *>(static_cast<const float *>(a.v) + first + i));
        } else {
            const auto *const m = static_cast<const uint8_t *>(a.m) + first + i;
            const auto *const v = static_cast<const uint8_t *>(a.v) + first + i;
            x[j].cm = __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(m));
            x[j].cv = __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(v));
            x[j].bm = a.m_scales[(first + i) >> 7];
            x[j].bv = a.v_scales[(first + i) >> 7];
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (threadIdx.x < 2) {
        // Each part counts the steps for itself: the count of a captured step goes on when it is
        // replayed, and no part waits for another.
        const int64_t t = p.steps + 1;
        const double rest = 1.0 - exp2(static_cast<double>(t) * (threadIdx.x == 0 ? a.log2_beta1 : a.log2_beta2));
        if (threadIdx.x == 0) {
            part->steps = t;
            shared.t = static_cast<uint64_t>(t);
            shared.up = static_cast<float>(1.0 / rest);
            shared.lr = a.lr_at != nullptr ? *a.lr_at : a.lr;
            shared.factor = a.factor_at != nullptr ? *a.factor_at : a.factor;
        } else {
            shared.root = static_cast<float>(1.0 / sqrt(rest));
        }
    }
    __syncthreads();
    const Factors f = shared;
#pragma unroll
    for (int j = 0; j < kFours; ++j) {
        const int i = (threadIdx.x + j * kThreads) * kFour, left = FULL ? kFour : count - i;
        if (!FULL && i >= room) continue;
        const int64_t at = first + i;
        f32x4 m = x[j].m, v = x[j].v, y;
        if constexpr (BITS == 8) {
            const int bm = x[j].bm, bv = x[j].bv;
#pragma unroll
            for (int e = 0; e < kFour; ++e) {
                m[e] = decode<true>(x[j].cm, e, bm);
                v[e] = decode<false>(x[j].cv, e, bv);
            }
            if (max(bm, bv) == kBad) {   // rare
#pragma unroll
                for (int e = 0; e < kFour; ++e) {
                    if (bm == kBad) m[e] = __builtin_nanf("");
                    if (bv == kBad) v[e] = __builtin_nanf("");
                }
            }
        }
#pragma unroll
        for (int e = 0; e < kFour; ++e) {
            const float ge = x[j].g[e] * f.factor;
            m[e] = a.beta1 * m[e] + a.rest1 * ge;
            v[e] = a.beta2 * v[e] + a.rest2 * (ge * ge);
        }
        // The instructions' root and reciprocal err by one unit and take numbers below 2^-126 for zeros, whose
        // roots are below 2^-63: times 2^9, as `root` is at most, they round away next to an eps of 2^-30. Of a
        // denominator up to 2^100 and 2^73 the reciprocal is no such number.
        if (a.plain) {
#pragma unroll
            for (int e = 0; e < kFour; ++e)
                y[e] = m[e] * f.up * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[e]) * f.root + a.eps);
        } else {
#pragma unroll
            for (int e = 0; e < kFour; ++e) y[e] = m[e] * f.up / (sqrtf(v[e]) * f.root + a.eps);
        }
#pragma unroll
        for (int e = 0; e < kFour; ++e) {
            y[e] = f.lr * (y[e] + decay * x[j].w[e]);
            if (!PUSH) y[e] = x[j].w[e] - y[e];
        }
        if constexpr (PUSH) store4<G, WEIGHTS_PAST>(g, i, y, left);
        else store4<W, WEIGHTS_PAST>(w, i, y, left);
        if constexpr (BITS == 32) {
            put<true>(reinterpret_cast<f32x4_any *>(static_cast<float *>(a.m) + at), m);
            put<true>(reinterpret_cast<f32x4_any *>(static_cast<float *>(a.v) + at), v);
        } else {
            uint32_t mm = 0, mv = 0;
#pragma unroll
            for (int e = 0; e < kFour; ++e) {
                mm = max(mm, __float_as_uint(m[e]) & 0x7fffffffu);
                mv = max(mv, __float_as_uint(v[e]));   // not negative, or a NaN, of which one with a sign is largest
            }
            const int bm = block_byte(most_of_32(mm)), bv = block_byte(most_of_32(mv));
            const u32x4 r = random4(static_cast<uint64_t>(at) >> 2, f.t, a.seed);
            uint32_t cm[kFour], cv[kFour];
#pragma unroll
            for (int e = 0; e < kFour; ++e) {
                cm[e] = encode<true>(m[e], bm, r[e] & 0xffffu);
                cv[e] = encode<false>(v[e], bv, r[e] >> 16);
            }
            auto *const to_m = static_cast<uint8_t *>(a.m) + at, *const to_v = static_cast<uint8_t *>(a.v) + at;
            __builtin_nontemporal_store(upper_bytes(cm), reinterpret_cast<uint32_t *>(to_m));
            __builtin_nontemporal_store(upper_bytes(cv), reinterpret_cast<uint32_t *>(to_v));
            if ((threadIdx.x & 31) == 0) {
                a.m_scales[at >> 7] = static_cast<uint8_t>(bm);
                a.v_scales[at >> 7] = static_cast<uint8_t>(bv);
            }
        }
    }
}

template <int W, int G, int BITS, bool PUSH, bool WEIGHTS_PAST>
__global__ __launch_bounds__(kThreads) void adamw(AdamwArgs a) {
    __shared__ Factors shared;
    const uint64_t index = block_index();
    if (index >= a.parts) return;
    AdamwPart *const part = a.plan + index;
    const AdamwPart p = *part;   // with the number of steps: a load of it behind the others would wait for them
    if (p.count == kPart) step_part<W, G, BITS, PUSH, WEIGHTS_PAST, true>(a, part, p, shared);
    else step_part<W, G, BITS, PUSH, WEIGHTS_PAST, false>(a, part, p, shared);
}

// The values of states in 8 bits, sixteen lanes a block.
template <bool SIGNED, int OUT, bool PAST>
__device__ __forceinline__ void values(const uint8_t *codes, const uint8_t *scales, void *out, uint64_t at) {
    const u32x2 c = get<PAST>(reinterpret_cast<const u32x2_any *>(codes + at));
    const int byte = scales[at >> 7];
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        x[e] = decode<SIGNED>(c[e >> 2], e & 3, byte);
        if (byte == kBad) x[e] = __builtin_nanf("");
    }
    store8<OUT, PAST>(out, static_cast<int64_t>(at), x);
}

template <int OUT, bool PAST>
__global__ __launch_bounds__(kThreads) void moments(MomentsArgs a) {
    const uint64_t at = (static_cast<uint64_t>(block_index()) * kThreads + threadIdx.x) * 8;
    if (at >= a.room) return;
    values<true, OUT, PAST>(a.m, a.m_scales, a.m_out, at);
    values<false, OUT, PAST>(a.v, a.v_scales, a.v_out, at);
}

template <int W, int G, int BITS, bool PUSH>
hipError_t launch(const AdamwArgs &a, hipStream_t s) {
    dim3 grid;
    if (!grid_of(a.parts, kThreads, &grid)) return hipErrorInvalidConfiguration;
    if (a.parts * kPart * kBytes<W> > kLastLevel) adamw<W, G, BITS, PUSH, true><<<grid, kThreads, 0, s>>>(a);
    else adamw<W, G, BITS, PUSH, false><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

template <int W, int G, bool PUSH>
hipError_t launch_bits(const AdamwArgs &a, int bits, hipStream_t s) {
    return bits == 8 ? launch<W, G, 8, PUSH>(a, s) : launch<W, G, 32, PUSH>(a, s);
}

}  // namespace

uint32_t adamw_part() { return kPart; }

hipError_t launch_adamw(const AdamwArgs &a, int weight_dtype, int grad_dtype, int bits, bool push, hipStream_t s) {
    if (!push)
        return grad_dtype == PS_F32 ? launch_bits<PS_F32, PS_F32, false>(a, bits, s)
                                    : launch_bits<PS_F32, PS_BF16, false>(a, bits, s);
    if (weight_dtype == PS_F32)
        return grad_dtype == PS_F32 ? launch_bits<PS_F32, PS_F32, true>(a, bits, s)
                                    : launch_bits<PS_F32, PS_BF16, true>(a, bits, s);
    return grad_dtype == PS_F32 ? launch_bits<PS_BF16, PS_F32, true>(a, bits, s)
                                : launch_bits<PS_BF16, PS_BF16, true>(a, bits, s);
}

hipError_t launch_moments(const MomentsArgs &a, int dtype, hipStream_t s) {
    dim3 grid;
    if (!grid_of((a.room / 8 + kThreads - 1) / kThreads, kThreads, &grid)) return hipErrorInvalidConfiguration;
    // Results of which more than half of the last level's size is written, past the caches: in us in fp32 and bf16,
    // 138M 299 and 140, not so 347 and 146, 61M 133 and 63, 153 and 66; but 12M 28 and 14.6, 27 and 12.9.
    const bool past = 2 * a.room * (dtype == PS_F32 ? 4 : 2) > kLastLevel / 2;
    if (dtype == PS_F32 && past) moments<PS_F32, true><<<grid, kThreads, 0, s>>>(a);
    else if (dtype == PS_F32) moments<PS_F32, false><<<grid, kThreads, 0, s>>>(a);
    else if (past) moments<PS_BF16, true><<<grid, kThreads, 0, s>>>(a);
    else moments<PS_BF16, false><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace gadei::learner

// AdamW over many tensors in one launch, with first and second moments in f32
// or in 8 bits, and the norm of all gradients with its clip.
//
// Every tensor is cut into chunks of VMOE_ADAMW_CHUNK elements; an entry of the
// plan holds a chunk's own addresses, so a block makes one dependent load (its
// entry) before its operands, however many tensors there are. The kernels are
// streams, bound by HBM: 28 bytes an element with f32 states, weights and
// gradients, 30 with bf16 weights and their master copy, 18 with 8-bit states as
// well. 37.8 million parameters with f32 states take 192 us (5.9 TB/s), 268
// million with 8-bit ones 773 us (6.4 TB/s; a copy reads and writes 4.8 to 5.4),
// the norm of the former's gradients 24 us beside a launch that adds up.
//
// Built without contraction: each product and sum of the moments is rounded by
// itself, which fixes the 8-bit states bit for bit.
#include <math.h>
#include <string.h>

#include "common_train.h"

namespace vmoe {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 4;  // consecutive elements of a lane: 16 bytes of f32, one word of codes
constexpr int kSpan = kThreads * kPer;
constexpr int kStepThreads = 128;  // of a block of the update
constexpr int kStepSpan = kStepThreads * kPer;
constexpr int kStateBlock = 128;  // elements of a scale byte, on 32 lanes
constexpr int kNormBlocks = 1024;

enum : uint32_t { kParamBf16 = 1, kGradBf16 = 2, kState8 = 4 };

struct Entry {
    void* param;
    float* master;
    const void* grad;
    void* m;
    void* v;
    uint8_t* m_scale;
    uint8_t* v_scale;
    uint64_t index0;
    int32_t count;
    uint32_t flags;
    float lr_mult, weight_decay;
};
static_assert(sizeof(Entry) == VMOE_ADAMW_PLAN_ENTRY_BYTES, "plan entry size");

struct Scalars {
    float b1, b1c, b2, b2c, c1, c2, eps, lr, grad_scale;
    uint32_t key;
};

// 32 bits to 32 bits, each output bit on every input bit: xor-shifts between
// products with odd numbers (the leading fraction bits of sqrt 2 and sqrt 3).
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    x ^= x >> 16;
    return x;
}
constexpr uint32_t kGolden = 0x9E3779B1u;  // spreads consecutive numbers over 32 bits

// The 32 random bits of element number i: 16 for m, 16 for v.
__device__ __forceinline__ uint32_t random_bits(uint64_t i, uint32_t key) {
    const uint32_t hi = static_cast<uint32_t>(i >> 32);
    if (hi != 0) key = mix32(key ^ hi);
    return mix32((static_cast<uint32_t>(i) * kGolden) ^ key);
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct Four {
    float x[kPer];
};

// Elements [i, i + 4) of a chunk of n; those at or past n read as 0.
template <bool TAIL, bool BF16>
__device__ __forceinline__ Four load4(const void* p, int i, int n) {
    Four r;
    if constexpr (BF16) {
        const uint16_t* q = static_cast<const uint16_t*>(p) + i;
        if (!TAIL || i + kPer <= n) {
            const u32x2 w = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(q));
            r.x[0] = __uint_as_float(w[0] << 16);
            r.x[1] = __uint_as_float(w[0] & 0xFFFF0000u);
            r.x[2] = __uint_as_float(w[1] << 16);
            r.x[3] = __uint_as_float(w[1] & 0xFFFF0000u);
        } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j) r.x[j] = i + j < n ? bf16_to_f32(q[j]) : 0.0f;
        }
    } else {
        const float* q = static_cast<const float*>(p) + i;
        if (!TAIL || i + kPer <= n) {
            const f32x4 w = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(q));
#pragma unroll
            for (int j = 0; j < kPer; ++j) r.x[j] = w[j];
        } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j) r.x[j] = i + j < n ? q[j] : 0.0f;
        }
    }
    return r;
}

template <bool TAIL, bool BF16>
__device__ __forceinline__ void store4(void* p, int i, int n, const Four& v) {
    if constexpr (BF16) {
        uint16_t* q = static_cast<uint16_t*>(p) + i;
        if (!TAIL || i + kPer <= n) {
            const u32x2 w = {pack_bf16x2(v.x[0], v.x[1]), pack_bf16x2(v.x[2], v.x[3])};
            __builtin_nontemporal_store(w, reinterpret_cast<u32x2*>(q));
        } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if (i + j < n) q[j] = f32_to_bf16(v.x[j]);
        }
    } else {
        float* q = static_cast<float*>(p) + i;
        if (!TAIL || i + kPer <= n) {
            const f32x4 w = {v.x[0], v.x[1], v.x[2], v.x[3]};
            __builtin_nontemporal_store(w, reinterpret_cast<f32x4*>(q));
        } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if (i + j < n) q[j] = v.x[j];
        }
    }
}

// Four codes as one word, those past n as 0.
template <bool TAIL>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int i, int n) {
    if (!TAIL || i + kPer <= n)
        return __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p + i));
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (i + j < n) w |= static_cast<uint32_t>(p[i + j]) << (8 * j);
    return w;
}

template <bool TAIL>
__device__ __forceinline__ void store_codes(uint8_t* p, int i, int n, uint32_t w) {
    if (!TAIL || i + kPer <= n) {
        __builtin_nontemporal_store(w, reinterpret_cast<uint32_t*>(p + i));
        return;
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (i + j < n) p[i + j] = static_cast<uint8_t>(w >> (8 * j));
}

// A code's exponent and mantissa bits, put where an f32 has them, are the
// value at the lowest exponents of f32, its linear range falling on f32's own:
// u 2^-112 for m and u 2^-96 for v. One exponent shift then gives 2^(s-127) u;
// a scale of 255 shifts the all-ones code to infinity.
template <bool SIGNED>
__device__ __forceinline__ float decode(uint32_t code, int s) {
    const uint32_t bits = (SIGNED ? code & 0x7Fu : code & 0xFFu) << 20;
    const float u = __builtin_ldexpf(__uint_as_float(bits), s - (SIGNED ? 15 : 31));
    return SIGNED ? __uint_as_float(__float_as_uint(u) | ((code & 0x80u) << 24)) : u;
}

// The inverse on a magnitude's bits: shift the exponent, add the random bits
// (their middle, so that no fraction rounds up for certain) below the 3
// mantissa bits that stay, and cut. r: 16 random bits at bit 4.
template <bool SIGNED>
__device__ __forceinline__ uint32_t encode(float x, int s, uint32_t r) {
    const float u = __builtin_ldexpf(SIGNED ? fabsf(x) : x, (SIGNED ? 15 : 31) - s);
    uint32_t code = (__float_as_uint(u) + (r | 8u)) >> 20;
    if (SIGNED) return code | ((__float_as_uint(x) >> 24) & 0x80u);
    return code == 0 && x > 0.0f ? 1u : code;
}

__device__ __forceinline__ uint32_t max_u32(uint32_t a, uint32_t b) { return a > b ? a : b; }

template <int ROR>
__device__ __forceinline__ uint32_t rotate_in_row(uint32_t v) {
    return __builtin_amdgcn_update_dpp(v, v, 0x120 + ROR, 0xF, 0xF, false);
}

// Scale byte of a state block: 32 lanes' four magnitudes (as bits, which order
// like the values, with infinities and NaN above every number).
__device__ __forceinline__ int block_scale(const Four& v) {
    uint32_t t = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) t = max_u32(t, __float_as_uint(v.x[j]) & 0x7FFFFFFFu);
    t = max_u32(t, rotate_in_row<8>(t));
    t = max_u32(t, rotate_in_row<4>(t));
    t = max_u32(t, rotate_in_row<2>(t));
    t = max_u32(t, rotate_in_row<1>(t));
    t = max_u32(t, __builtin_amdgcn_ds_swizzle(t, 0x401F));  // lane ^ 16
    const uint32_t s = (t + 0xFFFFFu) >> 23;
    return s > 255u ? 255 : static_cast<int>(s);
}

// The span of a block from element `base` of a chunk.
template <bool PB, bool GB, bool S8, bool TAIL>
__device__ __forceinline__ void adamw_span(const Entry& e, const Scalars& h, float scale, float lr,
                                           float decay, int base) {
    const int n = e.count, tid = threadIdx.x, i = base + tid * kPer;
    float* weights = PB ? e.master : static_cast<float*>(e.param);
    const Four g = load4<TAIL, GB>(e.grad, i, n);
    Four p = load4<TAIL, false>(weights, i, n), m, v;
    uint32_t mc = 0, vc = 0;
    int ms = 0, vs = 0;
    if constexpr (S8) {
        mc = load_codes<TAIL>(static_cast<const uint8_t*>(e.m), i, n);
        vc = load_codes<TAIL>(static_cast<const uint8_t*>(e.v), i, n);
        if (!TAIL || i < n) {
            ms = e.m_scale[i / kStateBlock];
            vs = e.v_scale[i / kStateBlock];
        }
    } else {
        m = load4<TAIL, false>(e.m, i, n);
        v = load4<TAIL, false>(e.v, i, n);
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const float gj = g.x[j] * scale;
        const float m0 = S8 ? decode<true>(mc >> (8 * j), ms) : m.x[j];
        const float v0 = S8 ? decode<false>(vc >> (8 * j), vs) : v.x[j];
        const float mj = m0 * h.b1 + gj * h.b1c;
        const float vj = v0 * h.b2 + (gj * gj) * h.b2c;
        m.x[j] = mj;
        v.x[j] = vj;
        // the square root and the quotient to an ulp or two: their errors
        // reach p below its own rounding, by a factor of lr. The instruction
        // takes numbers below 2^-126 as 0: it gets them 2^32 times as large
        const bool tiny = vj < 0x1p-126f;
        const float root = __builtin_amdgcn_sqrtf(tiny ? vj * 0x1p32f : vj);
        const float den = __builtin_fmaf(root, tiny ? h.c2 * 0x1p-16f : h.c2, h.eps);
        const float step = __builtin_fmaf(decay, p.x[j], (mj * h.c1) * __builtin_amdgcn_rcpf(den));
        p.x[j] = __builtin_fmaf(-lr, step, p.x[j]);
    }
    store4<TAIL, false>(weights, i, n, p);
    if constexpr (PB) store4<TAIL, true>(e.param, i, n, p);
    if constexpr (S8) {
        const int sm = block_scale(m), sv = block_scale(v);
        uint32_t wm = 0, wv = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const uint32_t r = random_bits(e.index0 + static_cast<uint32_t>(i + j), h.key);
            wm |= encode<true>(m.x[j], sm, (r & 0xFFFFu) << 4) << (8 * j);
            wv |= encode<false>(v.x[j], sv, (r >> 16) << 4) << (8 * j);
        }
        // a block that is not finite: codes that read as infinity
        if (sm == 255) wm = 0x7F7F7F7Fu;
        if (sv == 255) wv = 0xFFFFFFFFu;
        store_codes<TAIL>(static_cast<uint8_t*>(e.m), i, n, wm);
        store_codes<TAIL>(static_cast<uint8_t*>(e.v), i, n, wv);
        if ((tid & 31) == 0 && (!TAIL || i < n)) {
            e.m_scale[i / kStateBlock] = static_cast<uint8_t>(sm);
            e.v_scale[i / kStateBlock] = static_cast<uint8_t>(sv);
        }
    } else {
        store4<TAIL, false>(e.m, i, n, m);
        store4<TAIL, false>(e.v, i, n, v);
    }
}

// A block's part of a chunk: one span. Blocks that take their spans one after
// another run the memory pipes dry between them, fresh blocks do not (268 million
// parameters, 8-bit states: 760 us with 1024 elements a block, 782 with 2048, 908
// with 8192). Two waves a block rather than four: 40 million parameters with f32
// states take 197 us instead of 220, with 8-bit states 114 either way.
constexpr int kParts = VMOE_ADAMW_CHUNK / kStepSpan;

template <bool PB, bool GB, bool S8>
__device__ __forceinline__ void adamw_part(const Entry& e, const Scalars& h, float scale, int base) {
    const float lr = h.lr * e.lr_mult, decay = e.weight_decay;
    if (base + kStepSpan <= e.count) adamw_span<PB, GB, S8, false>(e, h, scale, lr, decay, base);
    else adamw_span<PB, GB, S8, true>(e, h, scale, lr, decay, base);
}

__global__ __launch_bounds__(kStepThreads) void adamw_kernel(const Entry* __restrict__ plan, Scalars h,
                                                         const float* __restrict__ clip) {
    const Entry e = plan[blockIdx.x / kParts];
    const int base = static_cast<int>(blockIdx.x % kParts) * kStepSpan;
    if (base >= e.count) return;
    float scale = h.grad_scale;
    if (clip != nullptr) {
        const float c = clip[1];
        if (c != c) return;  // the gradients' norm is not finite: no step
        scale *= c;
    }
    switch (e.flags) {
        case 0: adamw_part<false, false, false>(e, h, scale, base); break;
        case kParamBf16: adamw_part<true, false, false>(e, h, scale, base); break;
        case kGradBf16: adamw_part<false, true, false>(e, h, scale, base); break;
        case kParamBf16 | kGradBf16: adamw_part<true, true, false>(e, h, scale, base); break;
        case kState8: adamw_part<false, false, true>(e, h, scale, base); break;
        case kState8 | kParamBf16: adamw_part<true, false, true>(e, h, scale, base); break;
        case kState8 | kGradBf16: adamw_part<false, true, true>(e, h, scale, base); break;
        default: adamw_part<true, true, true>(e, h, scale, base); break;
    }
}

__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) s += lds[w];
    return s;
}

template <bool BF16>
__device__ __forceinline__ float chunk_squares(const Entry& e) {
    const int n = e.count, tid = threadIdx.x;
    float s = 0.0f;
    constexpr int U = 4;
    int base = 0;
    for (; base + U * kSpan <= n; base += U * kSpan) {
        Four g[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            g[u] = load4<false, BF16>(e.grad, base + u * kSpan + tid * kPer, n);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < kPer; ++j) s = __builtin_fmaf(g[u].x[j], g[u].x[j], s);
    }
    for (; base < n; base += kSpan) {
        const Four g = load4<true, BF16>(e.grad, base + tid * kPer, n);
#pragma unroll
        for (int j = 0; j < kPer; ++j) s = __builtin_fmaf(g.x[j], g.x[j], s);
    }
    return s;
}

__global__ __launch_bounds__(kThreads) void norm_partial_kernel(const Entry* __restrict__ plan,
                                                                long long n_chunks,
                                                                double* __restrict__ partial) {
    __shared__ double lds[kThreads / 64];
    double s = 0.0;
    for (long long c = blockIdx.x; c < n_chunks; c += gridDim.x) {
        const Entry& e = plan[c];
        s += (e.flags & kGradBf16) ? chunk_squares<true>(e) : chunk_squares<false>(e);
    }
    const double t = block_sum(s, lds);
    if (threadIdx.x == 0) partial[blockIdx.x] = t;
}

__global__ __launch_bounds__(kThreads) void norm_final_kernel(const double* __restrict__ partial,
                                                              int n, float grad_scale,
                                                              float max_norm,
                                                              float* __restrict__ clip) {
    __shared__ double lds[kThreads / 64];
    constexpr int U = kNormBlocks / kThreads;
    double v[U], s = 0.0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = u * kThreads + threadIdx.x;
        v[u] = i < n ? partial[i] : 0.0;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) s += v[u];
    s = block_sum(s, lds);
    if (threadIdx.x == 0) {
        const float norm = static_cast<float>(sqrt(s)) * fabsf(grad_scale);
        const float c = max_norm / (norm + 1e-6f);
        clip[0] = norm;
        clip[1] = !(norm < INFINITY) ? NAN : c < 1.0f ? c : 1.0f;
    }
}

// Codes to values: 8 consecutive ones a lane and step (a store of 16 bytes of
// bf16), all of a block's codes requested before any is used (61.6 million to
// bf16: 33 us, 5.5 TB/s; 35 with twice or half as many a block).
constexpr int kValues = 4096;

template <typename T, bool SIGNED>
__global__ __launch_bounds__(kThreads) void state_values_kernel(const uint8_t* __restrict__ codes,
                                                                const uint8_t* __restrict__ scale,
                                                                long long n, T* __restrict__ out) {
    const long long base = static_cast<long long>(blockIdx.x) * kValues;
    const int count = n - base < kValues ? static_cast<int>(n - base) : kValues;
    const uint8_t* c = codes + base;
    const uint8_t* s = scale + base / kStateBlock;
    T* o = out + base;
    constexpr bool BF16 = sizeof(T) == 2;
    constexpr int U = kValues / (2 * kSpan);
    uint32_t w[U][2];
    int e[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = (u * kThreads + threadIdx.x) * 2 * kPer;
        w[u][0] = load_codes<true>(c, i, count);
        w[u][1] = load_codes<true>(c, i + kPer, count);
        e[u] = i < count ? s[i / kStateBlock] : 0;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = (u * kThreads + threadIdx.x) * 2 * kPer;
        Four v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[h].x[j] = decode<SIGNED>(w[u][h] >> (8 * j), e[u]);
        if (BF16 && i + 2 * kPer <= count) {
            typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
            const u32x4 q = {pack_bf16x2(v[0].x[0], v[0].x[1]), pack_bf16x2(v[0].x[2], v[0].x[3]),
                             pack_bf16x2(v[1].x[0], v[1].x[1]), pack_bf16x2(v[1].x[2], v[1].x[3])};
            __builtin_nontemporal_store(q, reinterpret_cast<u32x4*>(o + i));
        } else {
            store4<true, BF16>(o, i, count, v[0]);
            store4<true, BF16>(o, i + kPer, count, v[1]);
        }
    }
}

bool valid_tensor(const vmoe_adamw_tensor& t) {
    if (t.n < 0 || t.reserved != 0) return false;
    if (t.param_dtype != VMOE_F32 && t.param_dtype != VMOE_BF16) return false;
    if (t.grad_dtype != VMOE_F32 && t.grad_dtype != VMOE_BF16) return false;
    if (t.state != VMOE_STATE_F32 && t.state != VMOE_STATE_8BIT) return false;
    if (!(t.lr_mult >= 0.0) || !isfinite(t.lr_mult)) return false;
    if (!(t.weight_decay >= 0.0) || !isfinite(t.weight_decay)) return false;
    if (t.index0 % kStateBlock != 0) return false;
    if (t.n == 0) return true;
    if (!t.param || !aligned16(t.param) || !t.grad || !aligned16(t.grad) || !t.m || !t.v)
        return false;
    if ((t.param_dtype == VMOE_BF16) != (t.master != nullptr) || !aligned16(t.master)) return false;
    const uintptr_t mv = reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v);
    if (t.state == VMOE_STATE_8BIT) return (mv & 3u) == 0 && t.m_scale && t.v_scale;
    return (mv & 15u) == 0 && !t.m_scale && !t.v_scale;
}

long long chunks_of(long long n) {
    return n / VMOE_ADAMW_CHUNK + (n % VMOE_ADAMW_CHUNK != 0);
}

template <typename T>
T* at(T* p, long long bytes) {
    return p ? reinterpret_cast<T*>(reinterpret_cast<uintptr_t>(p) + bytes) : nullptr;
}

}  // namespace

long long adamw_plan_chunks(const vmoe_adamw_tensor* tensors, int n_tensors) {
    long long total = 0;
    for (int i = 0; i < n_tensors; ++i) {
        if (!valid_tensor(tensors[i])) return -1;
        const long long c = chunks_of(tensors[i].n);
        if (c > (1LL << 40)) return -2;
        total += c;
        if (total > 0x7FFFFFFFLL) return -2;
    }
    return total;
}

void adamw_plan_write(const vmoe_adamw_tensor* tensors, int n_tensors, void* plan) {
    Entry* out = static_cast<Entry*>(plan);
    for (int i = 0; i < n_tensors; ++i) {
        const vmoe_adamw_tensor& t = tensors[i];
        const long long pb = t.param_dtype == VMOE_BF16 ? 2 : 4;
        const long long gb = t.grad_dtype == VMOE_BF16 ? 2 : 4;
        const long long sb = t.state == VMOE_STATE_8BIT ? 1 : 4;
        for (long long o = 0; o < t.n; o += VMOE_ADAMW_CHUNK) {
            Entry e;
            e.param = at(t.param, o * pb);
            e.master = at(t.master, o * 4);
            e.grad = at(t.grad, o * gb);
            e.m = at(t.m, o * sb);
            e.v = at(t.v, o * sb);
            e.m_scale = at(t.m_scale, o / kStateBlock);
            e.v_scale = at(t.v_scale, o / kStateBlock);
            e.index0 = t.index0 + static_cast<uint64_t>(o);
            e.count = static_cast<int32_t>(t.n - o < VMOE_ADAMW_CHUNK ? t.n - o : VMOE_ADAMW_CHUNK);
            e.flags = (pb == 2 ? kParamBf16 : 0u) | (gb == 2 ? kGradBf16 : 0u) |
                      (sb == 1 ? kState8 : 0u);
            e.lr_mult = static_cast<float>(t.lr_mult);
            e.weight_decay = static_cast<float>(t.weight_decay);
            memcpy(out++, &e, sizeof e);
        }
    }
}

size_t grad_norm_workspace_bytes(long long n_chunks) {
    const long long blocks = n_chunks < kNormBlocks ? n_chunks : kNormBlocks;
    return sizeof(double) * static_cast<size_t>(blocks > 1 ? blocks : 1);
}

vmoe_status grad_norm_launch(const void* plan, long long n_chunks, double grad_scale,
                             double max_norm, float* clip, void* ws, hipStream_t st) {
    const int blocks = static_cast<int>(n_chunks < kNormBlocks ? n_chunks : kNormBlocks);
    double* partial = static_cast<double*>(ws);
    if (blocks > 0)
        norm_partial_kernel<<<blocks, kThreads, 0, st>>>(static_cast<const Entry*>(plan), n_chunks,
                                                         partial);
    norm_final_kernel<<<1, kThreads, 0, st>>>(partial, blocks, static_cast<float>(grad_scale),
                                              static_cast<float>(max_norm), clip);
    return launch_status();
}

vmoe_status adamw_launch(const void* plan, long long n_chunks, const vmoe_adamw_hyper& hy,
                         const float* clip, hipStream_t st) {
    if (n_chunks == 0) return VMOE_OK;
    Scalars h;
    h.b1 = static_cast<float>(hy.beta1);
    h.b1c = static_cast<float>(1.0 - hy.beta1);
    h.b2 = static_cast<float>(hy.beta2);
    h.b2c = static_cast<float>(1.0 - hy.beta2);
    const double t = static_cast<double>(hy.step);
    // m c1 / (sqrt(v) c2 + eps) with a large eps: both sides 2^-64 times as large,
    // since the reciprocal of a number above 2^126 would be lost below the normal
    // range (the root's side stays below 2^91, c2 being at most 2^27)
    const double side = hy.eps >= 0x1p64 ? 0x1p-64 : 1.0;
    h.c1 = static_cast<float>(side / (1.0 - pow(hy.beta1, t)));
    h.c2 = static_cast<float>(side / sqrt(1.0 - pow(hy.beta2, t)));
    h.eps = static_cast<float>(side * hy.eps);
    h.lr = static_cast<float>(hy.lr);
    h.grad_scale = static_cast<float>(hy.grad_scale);
    h.key = mix32(hy.seed ^ mix32(static_cast<uint32_t>(hy.step) * kGolden));
    const Entry* entries = static_cast<const Entry*>(plan);
    constexpr long long kMost = 1LL << 20;  // a launch has fewer than 2^32 threads
    for (long long at = 0; at < n_chunks; at += kMost) {
        const long long n = n_chunks - at < kMost ? n_chunks - at : kMost;
        adamw_kernel<<<static_cast<unsigned>(n * kParts), kStepThreads, 0, st>>>(entries + at, h, clip);
    }
    return launch_status();
}

vmoe_status state_values_launch(const uint8_t* codes, const uint8_t* scale, bool is_signed,
                                long long n, void* out, int out_dtype, hipStream_t st) {
    if (n == 0) return VMOE_OK;
    constexpr long long kMost = kValues * (1LL << 20);  // a launch has fewer than 2^32 threads
    for (long long at = 0; at < n; at += kMost) {
        const long long left = n - at < kMost ? n - at : kMost;
        const unsigned grid = cdiv(left, kValues);
        const uint8_t *c = codes + at, *s = scale + at / kStateBlock;
        if (out_dtype == VMOE_BF16) {
            uint16_t* o = static_cast<uint16_t*>(out) + at;
            if (is_signed)
                state_values_kernel<uint16_t, true><<<grid, kThreads, 0, st>>>(c, s, left, o);
            else
                state_values_kernel<uint16_t, false><<<grid, kThreads, 0, st>>>(c, s, left, o);
        } else {
            float* o = static_cast<float*>(out) + at;
            if (is_signed)
                state_values_kernel<float, true><<<grid, kThreads, 0, st>>>(c, s, left, o);
            else
                state_values_kernel<float, false><<<grid, kThreads, 0, st>>>(c, s, left, o);
        }
    }
    return launch_status();
}

}  // namespace vmoe

// The experts' demand and the load-balance and z losses of a gate, with their
// gradient with respect to the router logits:
//   L_balance = E sum_e f_e P_e, f_e = demand_e / (k n), P_e = mean of probs;
//   L_z       = mean of lse^2, lse = log sum_e exp z;
//   dlogits   = p (w_balance E (f - <f, p>) + 2 w_z lse) / n.
// The gradient needs f of the whole group, so there are two launches. The first
// reads logits, noise, probs and choices once: a chunk's counts, sums of probs
// and of lse^2, and each token's lse, for which the softmax's largest term is
// enough (lse = max z - log max p: no second exponential). The second adds the
// group's counts in every block (integers, a few hundred short rows from L2)
// and forms the rows of dlogits from probs and lse; the group's first block
// also adds the other sums, in double and in chunk order, and writes the losses.
// Both are bound by latency up to some ten thousand tokens, by HBM beyond.
#include <type_traits>

#include "common_train.h"

namespace vmoe {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kBlocks = 512;  // about so many chunks over all groups
constexpr int kSteps = 4;     // token steps whose loads are in flight together

// EMAX lanes (a power of two >= E) hold a token's row.
template <int EMAX>
struct Rows {
    static constexpr int kTokens = 64 / EMAX;               // tokens a wave takes in a step
    static constexpr int kBlockTokens = kTokens * kWaves;   // and a block
};

struct LossArgs {
    const float *logits, *bias, *noise, *probs;
    const int32_t* idx;
    const uint8_t* mask;
    float *lse, *sum_p, *sum_z;      // workspace: [N], [G, chunks, EMAX], [G, chunks]
    int32_t *counts, *live;          // workspace: [G, chunks, EMAX], [G, chunks]
    float *losses, *mean_probs, *dlogits;
    int32_t* demand;
    int Ng, E, k, chunks, chunk_tokens;
    float w_balance, w_z;
};

template <int EMAX>
__device__ __forceinline__ float row_max(float v) {
#pragma unroll
    for (int o = EMAX / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}
template <int EMAX>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = EMAX / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

template <int EMAX>
__global__ __launch_bounds__(kThreads) void gate_sums_kernel(LossArgs a) {
    using R = Rows<EMAX>;
    __shared__ int hist[kWaves][EMAX];
    __shared__ float wave_p[kWaves][EMAX];
    __shared__ float wave_z[kWaves];
    __shared__ int wave_n[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int e = lane % EMAX, sub = lane / EMAX;
    const int g = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const int t0 = chunk * a.chunk_tokens, t1 = min(t0 + a.chunk_tokens, a.Ng);
    const size_t first = static_cast<size_t>(g) * a.Ng;
    const bool real = e < a.E;
    const float be = a.bias && real ? a.bias[e] : 0.0f;
    float acc_p = 0.0f, acc_z = 0.0f;
    int acc_n = 0;
    for (int b = t0; b < t1; b += kSteps * R::kBlockTokens) {
        float l[kSteps], nz[kSteps], p[kSteps];
        bool on[kSteps];
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int t = b + (u * kWaves + wave) * R::kTokens + sub;
            on[u] = t < t1 && (a.mask == nullptr || a.mask[first + t] != 0);
            const bool need = on[u] && real;
            const size_t q = (first + t) * a.E + e;
            l[u] = need ? a.logits[q] : 0.0f;
            nz[u] = need && a.noise ? a.noise[q] : 0.0f;
            p[u] = need ? a.probs[q] : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int t = b + (u * kWaves + wave) * R::kTokens + sub;
            float z = a.bias ? l[u] + be : l[u];
            if (a.noise) z += nz[u];
            const float top = row_max<EMAX>(real ? z : -INFINITY);
            const float lse = top - logf(row_max<EMAX>(p[u]));
            if (on[u]) {
                acc_p += p[u];
                if (e == 0) {
                    acc_z = __builtin_fmaf(lse, lse, acc_z);
                    acc_n += 1;
                    a.lse[first + t] = lse;
                }
            }
        }
    }
#pragma unroll
    for (int o = EMAX; o < 64; o <<= 1) acc_p += __shfl_xor(acc_p, o);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        acc_z += __shfl_xor(acc_z, o);
        acc_n += __shfl_xor(acc_n, o);
    }
    if (sub == 0) {
        wave_p[wave][e] = acc_p;
        hist[wave][e] = 0;
    }
    if (lane == 0) {
        wave_z[wave] = acc_z;
        wave_n[wave] = acc_n;
    }
    __syncthreads();
    // choices in rows of consecutive words; integer LDS atomics, one set of
    // counts a wave
    const int words = (t1 - t0) * a.k;
    const int32_t* idx = a.idx + (first + t0) * a.k;
    for (int b = tid; b < words; b += kSteps * kThreads) {
        int x[kSteps];
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int w = b + u * kThreads;
            const bool on = w < words && (a.mask == nullptr || a.mask[first + t0 + w / a.k] != 0);
            x[u] = on ? idx[w] : -1;
        }
#pragma unroll
        for (int u = 0; u < kSteps; ++u)
            if (x[u] >= 0 && x[u] < a.E) atomicAdd(&hist[wave][x[u]], 1);
    }
    __syncthreads();
    const size_t row = static_cast<size_t>(g) * a.chunks + chunk;
    if (tid < EMAX) {
        float s = 0.0f;
        int n = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            s += wave_p[w][tid];
            n += hist[w][tid];
        }
        a.sum_p[row * EMAX + tid] = s;
        a.counts[row * EMAX + tid] = n;
    }
    if (tid == 64) {
        float s = 0.0f;
        int n = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            s += wave_z[w];
            n += wave_n[w];
        }
        a.sum_z[row] = s;
        a.live[row] = n;
    }
}

// The group's counts and its number of tokens, in every block: rows of EMAX
// counts as a flat run of 16-byte words, of which a thread always meets the
// same four experts (4 kThreads is a multiple of EMAX).
template <int EMAX>
__device__ __forceinline__ void group_counts(const LossArgs& a, int g, int* total, int& n_live) {
    constexpr int kQuads = EMAX / 4;
    __shared__ int part[kWaves][EMAX];
    __shared__ int part_n[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int4* rows = reinterpret_cast<const int4*>(a.counts +
                                                     static_cast<size_t>(g) * a.chunks * EMAX);
    const int words = a.chunks * kQuads;
    int4 s = make_int4(0, 0, 0, 0);
    for (int b = tid; b < words; b += 8 * kThreads) {
        int4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int w = b + u * kThreads;
            v[u] = w < words ? rows[w] : make_int4(0, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            s.x += v[u].x;
            s.y += v[u].y;
            s.z += v[u].z;
            s.w += v[u].w;
        }
    }
    int n = 0;
    for (int c = tid; c < a.chunks; c += kThreads) n += a.live[static_cast<size_t>(g) * a.chunks + c];
#pragma unroll
    for (int o = kQuads; o < 64; o <<= 1) {
        s.x += __shfl_xor(s.x, o);
        s.y += __shfl_xor(s.y, o);
        s.z += __shfl_xor(s.z, o);
        s.w += __shfl_xor(s.w, o);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
    if (lane < kQuads) *reinterpret_cast<int4*>(&part[wave][lane * 4]) = s;
    if (lane == 0) part_n[wave] = n;
    __syncthreads();
    n_live = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) n_live += part_n[w];
    if (tid < EMAX) {
        int t = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) t += part[w][tid];
        total[tid] = t;
    }
    __syncthreads();
}

// Losses, demand and mean probabilities of a group, by one block.
template <int EMAX>
__device__ __forceinline__ void group_losses(const LossArgs& a, int g, const int* total, int n_live) {
    __shared__ double part[kThreads];
    __shared__ double mean_p[EMAX];
    __shared__ double part_z[kWaves];
    constexpr int kSlices = kThreads / EMAX;
    const int tid = threadIdx.x, e = tid % EMAX, q = tid / EMAX;
    const size_t first = static_cast<size_t>(g) * a.chunks;
    double s = 0.0, z = 0.0;
    for (int c = q; c < a.chunks; c += kSlices) s += a.sum_p[(first + c) * EMAX + e];
    for (int c = tid; c < a.chunks; c += kThreads) z += a.sum_z[first + c];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o);
    part[tid] = s;
    if ((tid & 63) == 0) part_z[tid >> 6] = z;
    __syncthreads();
    const double per = n_live > 0 ? 1.0 / n_live : 0.0;
    if (tid < EMAX) {
        double t = 0.0;
        for (int r = 0; r < kSlices; ++r) t += part[r * EMAX + tid];
        t *= per;
        mean_p[tid] = t;
        if (tid < a.E) {
            a.demand[static_cast<size_t>(g) * a.E + tid] = total[tid];
            if (a.mean_probs) a.mean_probs[static_cast<size_t>(g) * a.E + tid] = static_cast<float>(t);
        }
    }
    __syncthreads();
    if (tid == 0) {
        double loss = 0.0, lz = 0.0;
        for (int x = 0; x < a.E; ++x) loss += total[x] * per / a.k * mean_p[x];
        for (int w = 0; w < kWaves; ++w) lz += part_z[w];
        a.losses[static_cast<size_t>(g) * 2] = static_cast<float>(loss * a.E);
        a.losses[static_cast<size_t>(g) * 2 + 1] = static_cast<float>(lz * per);
    }
}

template <int EMAX>
__global__ __launch_bounds__(kThreads) void gate_grad_kernel(LossArgs a) {
    using R = Rows<EMAX>;
    __shared__ int total[EMAX];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int e = lane % EMAX, sub = lane / EMAX;
    const int g = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const int t0 = chunk * a.chunk_tokens, t1 = min(t0 + a.chunk_tokens, a.Ng);
    const size_t first = static_cast<size_t>(g) * a.Ng;
    const bool real = e < a.E;
    int n_live;
    group_counts<EMAX>(a, g, total, n_live);
    const float per = n_live > 0 ? 1.0f / static_cast<float>(n_live) : 0.0f;
    const float f = real ? static_cast<float>(total[e]) / static_cast<float>(a.k) * per : 0.0f;
    const float cb = a.w_balance * static_cast<float>(a.E) * per, cz = 2.0f * a.w_z * per;
    for (int b = t0; b < t1; b += kSteps * R::kBlockTokens) {
        float p[kSteps], lse[kSteps];
        bool on[kSteps];
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int t = b + (u * kWaves + wave) * R::kTokens + sub;
            on[u] = t < t1 && (a.mask == nullptr || a.mask[first + t] != 0);
            p[u] = on[u] && real ? a.probs[(first + t) * a.E + e] : 0.0f;
            lse[u] = on[u] ? a.lse[first + t] : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int t = b + (u * kWaves + wave) * R::kTokens + sub;
            const float inner = row_sum<EMAX>(f * p[u]);
            const float d = p[u] * __builtin_fmaf(cb, f - inner, cz * lse[u]);
            if (t < t1 && real) a.dlogits[(first + t) * a.E + e] = d;
        }
    }
    if (chunk == 0) group_losses<EMAX>(a, g, total, n_live);
}

template <typename F>
void by_experts(int E, F f) {
    if (E <= 4) f(std::integral_constant<int, 4>{});
    else if (E <= 8) f(std::integral_constant<int, 8>{});
    else if (E <= 16) f(std::integral_constant<int, 16>{});
    else if (E <= 32) f(std::integral_constant<int, 32>{});
    else f(std::integral_constant<int, 64>{});
}

struct Chunks {
    int count, tokens, emax;
};

// Chunks of a group: about kBlocks over all groups, none shorter than a block's
// step. More would cost every block of the second launch more rows of counts.
Chunks chunks_of(const Dims& D) {
    Chunks c = {1, 1, 4};
    by_experts(D.E, [&](auto tag) {
        constexpr int EMAX = decltype(tag)::value;
        c.emax = EMAX;
        const int most = static_cast<int>(cdiv(D.Ng, Rows<EMAX>::kBlockTokens));
        int n = kBlocks / D.G;
        if (n > most) n = most;
        if (n < 1) n = 1;
        c.tokens = D.Ng > 0 ? static_cast<int>(cdiv(D.Ng, n)) : 1;
        c.count = D.Ng > 0 ? static_cast<int>(cdiv(D.Ng, c.tokens)) : 1;
    });
    return c;
}

size_t pad16(size_t n) { return (n + 15) & ~static_cast<size_t>(15); }

}  // namespace

// Workspace: lse [N], sums of probs and counts [G, chunks, EMAX], sums of lse^2
// and numbers of tokens [G, chunks], each at a multiple of 16 bytes.
size_t gate_loss_workspace_bytes(const Dims& D) {
    const Chunks c = chunks_of(D);
    const size_t rows = static_cast<size_t>(D.G) * c.count;
    return pad16(sizeof(float) * static_cast<size_t>(D.N)) + 2 * sizeof(float) * rows * c.emax +
           2 * pad16(sizeof(float) * rows);
}

vmoe_status gate_loss_launch(const Dims& D, const float* logits, const float* bias,
                             const float* noise, const float* probs, const int32_t* idx,
                             const uint8_t* mask, float w_balance, float w_z, float* losses,
                             int32_t* demand, float* mean_probs, float* dlogits, void* ws,
                             hipStream_t st) {
    const Chunks c = chunks_of(D);
    const size_t rows = static_cast<size_t>(D.G) * c.count;
    unsigned char* w = static_cast<unsigned char*>(ws);
    const auto take = [&w](size_t bytes) {
        unsigned char* p = w;
        w += pad16(bytes);
        return p;
    };
    LossArgs a;
    a.logits = logits;
    a.bias = bias;
    a.noise = noise;
    a.probs = probs;
    a.idx = idx;
    a.mask = mask;
    a.lse = reinterpret_cast<float*>(take(sizeof(float) * static_cast<size_t>(D.N)));
    a.sum_p = reinterpret_cast<float*>(take(sizeof(float) * rows * c.emax));
    a.counts = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * rows * c.emax));
    a.sum_z = reinterpret_cast<float*>(take(sizeof(float) * rows));
    a.live = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * rows));
    a.losses = losses;
    a.mean_probs = mean_probs;
    a.dlogits = dlogits;
    a.demand = demand;
    a.Ng = D.Ng;
    a.E = D.E;
    a.k = D.k;
    a.chunks = c.count;
    a.chunk_tokens = c.tokens;
    a.w_balance = w_balance;
    a.w_z = w_z;
    const unsigned grid = static_cast<unsigned>(rows);  // at most N or G
    by_experts(D.E, [&](auto tag) {
        constexpr int EMAX = decltype(tag)::value;
        gate_sums_kernel<EMAX><<<grid, kThreads, 0, st>>>(a);
        gate_grad_kernel<EMAX><<<grid, kThreads, 0, st>>>(a);
    });
    return launch_status();
}

}  // namespace vmoe

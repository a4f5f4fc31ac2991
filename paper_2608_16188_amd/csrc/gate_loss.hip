// The experts' demand and the load-balance and z losses of a gate, with their
// gradient with respect to the router logits:
//   L_balance = E sum_e f_e P_e, f_e = demand_e / (k n), P_e = mean of probs;
//   L_z       = mean of lse^2, lse = log sum_e exp z;
//   dlogits   = p (w_balance E (f - <f, p>) + 2 w_z lse) / n.
// The gradient needs f of the whole group, and f needs the choices alone. Three
// ways, by size:
// - a group of few tokens: one block does everything, in one launch;
// - rows of up to 16 MB: a first launch takes a chunk's counts, sums of probs and
//   of lse^2 and each token's lse, a second adds the group's counts in every
//   block and writes dlogits from probs (read again) and lse, with one more
//   block a group for the losses beside them;
// - more: a first launch counts the choices (a small part of the bytes), a second
//   reads logits, noise and probs once, writes dlogits and leaves sums, and a
//   third writes the losses. Reading probs again would cost more than a launch
//   (61 x 4093 tokens of 64 experts: 51 us, 62 in two launches; 36928 of 32: 17
//   against 12).
// Sums over chunks are in double and in a fixed order. The softmax's largest term
// is enough for lse = max z - log max p: no second exponential. A lane holds four
// consecutive experts of a token (one 16-byte access where E is a multiple of 4),
// so a token takes at most 16 lanes and its maxima and sums are moves within a
// row of lanes, without LDS. Bound by latency up to some ten thousand tokens (197
// of 8 experts 5.4 us, 36928 of 32 11.5 us in two launches of 6), by HBM beyond
// (the rows of 61 x 4093 tokens of 64 experts: 168 MB in 39 us, 4.3 TB/s).
#include <type_traits>

#include "common_train.h"

namespace vmoe {
namespace {

constexpr int kSteps = 4;          // token steps whose loads are in flight together
constexpr int kChunkWaves = 8;     // waves of a block that takes a chunk
constexpr int kGroupWaves = 16;    // of a block that takes a whole group
constexpr int kBlocks = 512;      // most chunks over all groups (but one a group)
constexpr int kGroupChunks = 256;  // most of one group whose counts other blocks add
constexpr int kCountTokens = 512;  // fewest tokens of a part that is only counted
constexpr long long kRereadBytes = 16LL << 20;  // most bytes of probs that are read twice

// EMAX (a power of two >= E) / 4 lanes hold a token's row.
template <int EMAX, int WAVES>
struct Rows {
    static constexpr int kLanes = EMAX / 4;
    static constexpr int kTokens = 64 / kLanes;             // tokens a wave takes in a step
    static constexpr int kBlockTokens = kTokens * WAVES;    // and a block
    static constexpr int kThreads = 64 * WAVES;
    // most tokens of a one-block group (its rows requested at once)
    static constexpr int kGroupTokens = kSteps * kBlockTokens < 2048 ? kSteps * kBlockTokens : 2048;
};

struct LossArgs {
    const float *logits, *bias, *noise, *probs;
    const int32_t* idx;
    const uint8_t* mask;
    float *sum_p, *sum_z;      // workspace: [G, chunks, EMAX], [G, chunks]
    float* lse;                // workspace: [N] where probs are read twice
    int32_t *counts, *live;    // workspace: [G, parts, EMAX], [G, parts]
    float *losses, *mean_probs, *dlogits;
    int32_t* demand;
    int Ng, E, k, chunks, chunk_tokens, parts, part_tokens;
    int first_group;           // of a launch of whole groups
    float w_balance, w_z;
};

template <int CTRL>
__device__ __forceinline__ float lane_move(float v) {
    const int x = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(x, x, CTRL, 0xF, 0xF, false));
}

// Over a token's lanes, for all of them: neighbours, pairs, then halves and
// whole rows mirrored (whose lanes by then agree within 4 and 8).
template <int LANES, typename F>
__device__ __forceinline__ float over_token(float v, F f) {
    if constexpr (LANES > 1) v = f(v, lane_move<0xB1>(v));    // lane ^ 1
    if constexpr (LANES > 2) v = f(v, lane_move<0x4E>(v));    // lane ^ 2
    if constexpr (LANES > 4) v = f(v, lane_move<0x141>(v));   // mirrored in 8
    if constexpr (LANES > 8) v = f(v, lane_move<0x140>(v));   // mirrored in 16
    return v;
}
struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Add {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};

// Experts e0 .. e0 + 3 of a row; 0 past E and for rows that are off.
__device__ __forceinline__ float4 load_row(const float* row, int e0, int E, bool on) {
    float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
    if (!on || e0 >= E) return r;
    if (E % 4 == 0) return *reinterpret_cast<const float4*>(row + e0);
    r.x = row[e0];
    if (e0 + 1 < E) r.y = row[e0 + 1];
    if (e0 + 2 < E) r.z = row[e0 + 2];
    if (e0 + 3 < E) r.w = row[e0 + 3];
    return r;
}

__device__ __forceinline__ bool kept(const LossArgs& a, size_t t) {
    return a.mask == nullptr || a.mask[t] != 0;
}

// Choices and tokens of [t0, t1) of a group that starts at token `first`, by a
// block: choices in rows of consecutive words, counted by integer LDS atomics
// on counts of the wave's own.
template <int EMAX, int WAVES>
struct Counts {
    int hist[WAVES][EMAX];
    int n[WAVES];
    __device__ __forceinline__ int choices(int e) const {
        int t = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) t += hist[w][e];
        return t;
    }
    __device__ __forceinline__ int tokens() const {
        int t = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) t += n[w];
        return t;
    }
};

template <int EMAX, int WAVES>
__device__ __forceinline__ void count(const LossArgs& a, size_t first, int t0, int t1,
                                      Counts<EMAX, WAVES>& c) {
    constexpr int kThreads = 64 * WAVES;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int i = lane; i < EMAX; i += 64) c.hist[wave][i] = 0;
    const int words = (t1 - t0) * a.k;
    const int32_t* idx = a.idx + (first + t0) * a.k;
    for (int b = tid; b < words; b += kSteps * kThreads) {
        int x[kSteps];
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int w = b + u * kThreads;
            x[u] = w < words && kept(a, first + t0 + w / a.k) ? idx[w] : -1;
        }
#pragma unroll
        for (int u = 0; u < kSteps; ++u)
            if (x[u] >= 0 && x[u] < a.E) atomicAdd(&c.hist[wave][x[u]], 1);
    }
    int n = t1 - t0;
    if (a.mask != nullptr) {
        n = 0;
        for (int t = t0 + tid; t < t1; t += kThreads) n += kept(a, first + t) ? 1 : 0;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
    } else if (wave != 0) {
        n = 0;
    }
    if (lane == 0) c.n[wave] = n;
    __syncthreads();
}

// A block's sums of probs and lse^2.
template <int EMAX, int WAVES>
struct Sums {
    float p[WAVES][EMAX];
    float z[WAVES];
    __device__ __forceinline__ float prob(int e) const {
        float t = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) t += p[w][e];
        return t;
    }
    __device__ __forceinline__ float square() const {
        float t = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) t += z[w];
        return t;
    }
};

// What a pass over rows does: the block's sums and lse, dlogits from lse, or both
// at once (lse is not stored).
enum Pass { kSums, kGradient, kBoth };

// Rows [t0, t1). `ready` runs between the first rows' loads and their use and
// sets 1 / n and the lane's four f (not for kSums). Ends with a barrier, unless
// kGradient.
template <int EMAX, int WAVES, Pass PASS, typename F>
__device__ __forceinline__ void do_rows(const LossArgs& a, size_t first, int t0, int t1,
                                        Sums<EMAX, WAVES>* sums, F ready) {
    using R = Rows<EMAX, WAVES>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int e0 = (lane % R::kLanes) * 4, sub = lane / R::kLanes;
    const float4 be = a.bias ? load_row(a.bias, e0, a.E, true) : make_float4(0.f, 0.f, 0.f, 0.f);
    const float bv[4] = {be.x, be.y, be.z, be.w};
    float f4[4] = {0.0f, 0.0f, 0.0f, 0.0f}, cb = 0.0f, cz = 0.0f;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f}, acc_z = 0.0f;
    for (int b = t0; b < t1; b += kSteps * R::kBlockTokens) {
        float4 l[kSteps], nz[kSteps], p[kSteps];
        float ls[kSteps];
        bool on[kSteps];
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int t = b + (u * WAVES + wave) * R::kTokens + sub;
            on[u] = t < t1 && kept(a, first + t);
            const size_t q = (first + t) * a.E;
            p[u] = load_row(a.probs + q, e0, a.E, on[u]);
            if constexpr (PASS == kGradient) {
                ls[u] = on[u] ? a.lse[first + t] : 0.0f;
            } else {
                l[u] = load_row(a.logits + q, e0, a.E, on[u]);
                nz[u] = a.noise ? load_row(a.noise + q, e0, a.E, on[u])
                                : make_float4(0.f, 0.f, 0.f, 0.f);
            }
        }
        if (PASS != kSums && b == t0) {
            float per;
            ready(e0, f4, per);
            cb = a.w_balance * static_cast<float>(a.E) * per;
            cz = 2.0f * a.w_z * per;
        }
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int t = b + (u * WAVES + wave) * R::kTokens + sub;
            const float pv[4] = {p[u].x, p[u].y, p[u].z, p[u].w};
            float lse = 0.0f;
            if constexpr (PASS == kGradient) {
                lse = ls[u];
            } else {
                const float lv[4] = {l[u].x, l[u].y, l[u].z, l[u].w};
                const float nv[4] = {nz[u].x, nz[u].y, nz[u].z, nz[u].w};
                float top = -INFINITY, most = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float z = a.bias ? lv[j] + bv[j] : lv[j];
                    if (a.noise) z += nv[j];
                    if (e0 + j < a.E) top = fmaxf(top, z);
                    most = fmaxf(most, pv[j]);
                    acc[j] += pv[j];
                }
                top = over_token<R::kLanes>(top, Max{});
                most = over_token<R::kLanes>(most, Max{});
                if (on[u]) lse = top - logf(most);
                if (e0 == 0) {
                    acc_z = __builtin_fmaf(lse, lse, acc_z);
                    if (PASS == kSums && on[u]) a.lse[first + t] = lse;
                }
            }
            if constexpr (PASS == kSums) continue;
            float inner = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) inner = __builtin_fmaf(f4[j], pv[j], inner);
            inner = over_token<R::kLanes>(inner, Add{});
            float d[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                d[j] = pv[j] * __builtin_fmaf(cb, f4[j] - inner, cz * lse);
            if (t < t1 && e0 < a.E) {
                float* out = a.dlogits + (first + t) * a.E + e0;
                if (a.E % 4 == 0) {
                    *reinterpret_cast<float4*>(out) = make_float4(d[0], d[1], d[2], d[3]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (e0 + j < a.E) out[j] = d[j];
                }
            }
        }
    }
    if constexpr (PASS == kGradient) return;
#pragma unroll
    for (int o = 32; o >= R::kLanes; o >>= 1)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += __shfl_xor(acc[j], o);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) acc_z += __shfl_xor(acc_z, o);
    if (sub == 0)
#pragma unroll
        for (int j = 0; j < 4; ++j) sums->p[wave][e0 + j] = acc[j];
    if (lane == 0) sums->z[wave] = acc_z;
    __syncthreads();
}

// The lane's four f and 1 / n from a group's totals in LDS.
__device__ __forceinline__ void shares(const LossArgs& a, const int* total, int n_live, int e0,
                                       float (&f4)[4], float& per) {
    per = n_live > 0 ? 1.0f / static_cast<float>(n_live) : 0.0f;
    const float fk = per / static_cast<float>(a.k);
#pragma unroll
    for (int j = 0; j < 4; ++j) f4[j] = static_cast<float>(total[e0 + j]) * fk;
}

// Demand, mean probabilities and losses of a group, by a whole block.
__device__ __forceinline__ void write_losses(const LossArgs& a, int g, const int* total,
                                             const double* sum_p, double sum_z, int n_live) {
    const int tid = threadIdx.x;
    const double per = n_live > 0 ? 1.0 / n_live : 0.0;
    double loss = 0.0;
    if (tid < a.E) {
        const size_t at = static_cast<size_t>(g) * a.E + tid;
        const double mean = sum_p[tid] * per;
        loss = total[tid] * mean;
        a.demand[at] = total[tid];
        if (a.mean_probs) a.mean_probs[at] = static_cast<float>(mean);
    }
    if (tid < 64) {  // E <= 64: one wave
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) loss += __shfl_xor(loss, o);
    }
    if (tid == 0) {
        a.losses[static_cast<size_t>(g) * 2] = static_cast<float>(loss * (a.E * per / a.k));
        a.losses[static_cast<size_t>(g) * 2 + 1] = static_cast<float>(sum_z * per);
    }
}

// A whole group in one block.
template <int EMAX>
__global__ __launch_bounds__(64 * kGroupWaves) void gate_group_kernel(LossArgs a) {
    __shared__ Counts<EMAX, kGroupWaves> counts;
    __shared__ Sums<EMAX, kGroupWaves> sums;
    __shared__ int total[EMAX];
    __shared__ double sum_p[EMAX];
    const int g = a.first_group + blockIdx.x, tid = threadIdx.x;
    const size_t first = static_cast<size_t>(g) * a.Ng;
    int n_live = 0;
    const auto totals = [&] {
        count<EMAX, kGroupWaves>(a, first, 0, a.Ng, counts);
        n_live = counts.tokens();
        if (tid < EMAX) total[tid] = counts.choices(tid);
        __syncthreads();
    };
    if (a.Ng == 0) totals();  // no rows to call it
    do_rows<EMAX, kGroupWaves, kBoth>(a, first, 0, a.Ng, &sums,
                                      [&](int e0, float (&f4)[4], float& per) {
                                          totals();
                                          shares(a, total, n_live, e0, f4, per);
                                      });
    if (tid < EMAX) sum_p[tid] = sums.prob(tid);
    __syncthreads();
    write_losses(a, g, total, sum_p, sums.square(), n_live);
}

// Counts of one part of a group's choices; with them, where probs are read twice,
// the part's sums and lse.
template <int EMAX, bool SUMS>
__global__ __launch_bounds__(64 * kChunkWaves) void gate_count_kernel(LossArgs a) {
    __shared__ Counts<EMAX, kChunkWaves> counts;
    __shared__ Sums<EMAX, kChunkWaves> sums;
    const int g = blockIdx.x / a.parts, part = blockIdx.x % a.parts, tid = threadIdx.x;
    const int t0 = part * a.part_tokens, t1 = min(t0 + a.part_tokens, a.Ng);
    const size_t first = static_cast<size_t>(g) * a.Ng, row = blockIdx.x;
    if constexpr (SUMS)
        do_rows<EMAX, kChunkWaves, kSums>(a, first, t0, t1, &sums,
                                          [](int, float (&)[4], float&) {});
    count<EMAX, kChunkWaves>(a, first, t0, t1, counts);
    if (tid < EMAX) {
        a.counts[row * EMAX + tid] = counts.choices(tid);
        if constexpr (SUMS) a.sum_p[row * EMAX + tid] = sums.prob(tid);
    }
    if (tid == 64) {
        a.live[row] = counts.tokens();
        if constexpr (SUMS) a.sum_z[row] = sums.square();
    }
}

// A group's counts and its number of tokens: rows of EMAX counts as a flat run
// of 16-byte words, of which a thread always meets the same four experts (four
// times a block's threads is a multiple of EMAX). Ends with a barrier.
template <int EMAX>
__device__ __forceinline__ void group_counts(const LossArgs& a, int g, int* total, int& n_live) {
    constexpr int kQuads = EMAX / 4, kThreads = 64 * kChunkWaves, kFlight = 4;
    static_assert(kGroupChunks <= kThreads, "a thread takes one part's tokens");
    __shared__ int part[kChunkWaves][EMAX];
    __shared__ int part_n[kChunkWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int4* rows = reinterpret_cast<const int4*>(a.counts +
                                                     static_cast<size_t>(g) * a.parts * EMAX);
    const int words = a.parts * kQuads;
    int n = tid < a.parts ? a.live[static_cast<size_t>(g) * a.parts + tid] : 0;
    int4 s = make_int4(0, 0, 0, 0);
    for (int b = tid; b < words; b += kFlight * kThreads) {
        int4 v[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            const int w = b + u * kThreads;
            v[u] = w < words ? rows[w] : make_int4(0, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            s.x += v[u].x;
            s.y += v[u].y;
            s.z += v[u].z;
            s.w += v[u].w;
        }
    }
#pragma unroll
    for (int o = kQuads; o < 64; o <<= 1) {
        s.x += __shfl_xor(s.x, o);
        s.y += __shfl_xor(s.y, o);
        s.z += __shfl_xor(s.z, o);
        s.w += __shfl_xor(s.w, o);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
    if (lane == 0) part_n[wave] = n;
    if (lane < kQuads) *reinterpret_cast<int4*>(&part[wave][lane * 4]) = s;
    __syncthreads();
    n_live = 0;
#pragma unroll
    for (int w = 0; w < kChunkWaves; ++w) n_live += part_n[w];
    if (tid < EMAX) {
        int t = 0;
#pragma unroll
        for (int w = 0; w < kChunkWaves; ++w) t += part[w][tid];
        total[tid] = t;
    }
    __syncthreads();
}

// A chunk's rows; where probs are read once, its sums.
template <int EMAX, Pass PASS>
__device__ __forceinline__ void chunk_rows(const LossArgs& a, int g, int chunk) {
    __shared__ Sums<EMAX, kChunkWaves> sums;
    __shared__ int total[EMAX];
    const int tid = threadIdx.x;
    const int t0 = chunk * a.chunk_tokens, t1 = min(t0 + a.chunk_tokens, a.Ng);
    do_rows<EMAX, kChunkWaves, PASS>(a, static_cast<size_t>(g) * a.Ng, t0, t1, &sums,
                                     [&](int e0, float (&f4)[4], float& per) {
                                         int n_live;
                                         group_counts<EMAX>(a, g, total, n_live);
                                         shares(a, total, n_live, e0, f4, per);
                                     });
    if constexpr (PASS == kBoth) {
        const size_t row = static_cast<size_t>(g) * a.chunks + chunk;
        if (tid < EMAX) a.sum_p[row * EMAX + tid] = sums.prob(tid);
        if (tid == 64) a.sum_z[row] = sums.square();
    }
}

// A group's losses from its chunks' sums, by a block: four experts a lane,
// kFlight rows of sums in flight.
template <int EMAX, int kFlight>
__device__ __forceinline__ void group_losses(const LossArgs& a, int g) {
    constexpr int kThreads = 64 * kChunkWaves, kQuads = EMAX / 4, kSlices = kThreads / kQuads;
    __shared__ int total[EMAX];
    __shared__ double part[kChunkWaves][EMAX];
    __shared__ double sum_p[EMAX];
    __shared__ double part_z[kChunkWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, q = tid / kQuads;
    const float4* sp = reinterpret_cast<const float4*>(
                           a.sum_p + static_cast<size_t>(g) * a.chunks * EMAX) + tid % kQuads;
    const float* sz = a.sum_z + static_cast<size_t>(g) * a.chunks;
    double s[4] = {0.0, 0.0, 0.0, 0.0}, z = 0.0;
    for (int c = q; c < a.chunks; c += kFlight * kSlices) {
        float4 v[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
            v[u] = c + u * kSlices < a.chunks ? sp[static_cast<size_t>(c + u * kSlices) * kQuads]
                                              : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            s[0] += v[u].x;
            s[1] += v[u].y;
            s[2] += v[u].z;
            s[3] += v[u].w;
        }
    }
    for (int i = tid; i < a.chunks; i += kThreads) z += sz[i];
    int n_live;
    group_counts<EMAX>(a, g, total, n_live);
#pragma unroll
    for (int o = kQuads; o < 64; o <<= 1)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] += __shfl_xor(s[j], o);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o);
    if (lane < kQuads)
#pragma unroll
        for (int j = 0; j < 4; ++j) part[wave][lane * 4 + j] = s[j];
    if (lane == 0) part_z[wave] = z;
    __syncthreads();
    if (tid < EMAX) {
        double t = 0.0;
#pragma unroll
        for (int w = 0; w < kChunkWaves; ++w) t += part[w][tid];
        sum_p[tid] = t;
    }
    z = 0.0;
#pragma unroll
    for (int w = 0; w < kChunkWaves; ++w) z += part_z[w];
    __syncthreads();
    write_losses(a, g, total, sum_p, z, n_live);
}

template <int EMAX>
__global__ __launch_bounds__(64 * kChunkWaves) void gate_rows_kernel(LossArgs a) {
    chunk_rows<EMAX, kBoth>(a, blockIdx.x / a.chunks, blockIdx.x % a.chunks);
}

template <int EMAX>
__global__ __launch_bounds__(64 * kChunkWaves) void gate_losses_kernel(LossArgs a) {
    group_losses<EMAX, 16>(a, blockIdx.x);
}

// Second launch of two: the block after a group's chunks writes its losses (with
// few enough rows in flight not to cost the other blocks registers).
template <int EMAX>
__global__ __launch_bounds__(64 * kChunkWaves) void gate_gradient_kernel(LossArgs a) {
    const int g = blockIdx.x / (a.chunks + 1), chunk = blockIdx.x % (a.chunks + 1);
    if (chunk < a.chunks) chunk_rows<EMAX, kGradient>(a, g, chunk);
    else group_losses<EMAX, 4>(a, g);
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
    int count, tokens;            // chunks of a group's rows
    int parts, part_tokens;       // parts of its choices
    int emax;
    bool whole;                   // a group in one block
    bool twice;                   // probs are read twice: parts are chunks
};

Chunks chunks_of(const Dims& D) {
    Chunks c = {1, 1, 1, 1, 4, false, false};
    const auto split = [&](int most, int least_tokens, int& count, int& tokens) {
        const int n = static_cast<int>(cdiv(D.Ng, least_tokens));
        const int want = n < most ? n : most;
        tokens = static_cast<int>(cdiv(D.Ng, want < 1 ? 1 : want));
        if (tokens < 1) tokens = 1;
        count = static_cast<int>(cdiv(D.Ng, tokens));
        if (count < 1) count = 1;
    };
    by_experts(D.E, [&](auto tag) {
        constexpr int EMAX = decltype(tag)::value;
        c.emax = EMAX;
        c.whole = D.Ng <= Rows<EMAX, kGroupWaves>::kGroupTokens;
        c.twice = static_cast<long long>(D.N) * D.E * 4 <= kRereadBytes;
        int most = kBlocks / D.G;
        if (c.twice && most > kGroupChunks) most = kGroupChunks;
        split(most, Rows<EMAX, kChunkWaves>::kBlockTokens, c.count, c.tokens);
        split(kGroupChunks, kCountTokens, c.parts, c.part_tokens);
        if (c.twice) {
            c.parts = c.count;
            c.part_tokens = c.tokens;
        }
    });
    return c;
}

size_t pad16(size_t n) { return (n + 15) & ~static_cast<size_t>(15); }

}  // namespace

// Workspace: sums of probs [G, chunks, EMAX], counts [G, parts, EMAX], sums of
// lse^2 [G, chunks], numbers of tokens [G, parts] and, where probs are read
// twice, lse [N], each at a multiple of 16 bytes.
size_t gate_loss_workspace_bytes(const Dims& D) {
    const Chunks c = chunks_of(D);
    const size_t rows = static_cast<size_t>(D.G) * c.count, parts = static_cast<size_t>(D.G) * c.parts;
    return 4 * (rows + parts) * c.emax + pad16(4 * rows) + pad16(4 * parts) +
           (c.twice ? pad16(4 * static_cast<size_t>(D.N)) : 0);
}

vmoe_status gate_loss_launch(const Dims& D, const float* logits, const float* bias,
                             const float* noise, const float* probs, const int32_t* idx,
                             const uint8_t* mask, float w_balance, float w_z, float* losses,
                             int32_t* demand, float* mean_probs, float* dlogits, void* ws,
                             hipStream_t st) {
    const Chunks c = chunks_of(D);
    const size_t rows = static_cast<size_t>(D.G) * c.count, parts = static_cast<size_t>(D.G) * c.parts;
    unsigned char* w = static_cast<unsigned char*>(ws);
    const auto take = [&w](size_t words) {
        unsigned char* p = w;
        w += pad16(4 * words);
        return p;
    };
    LossArgs a;
    a.logits = logits;
    a.bias = bias;
    a.noise = noise;
    a.probs = probs;
    a.idx = idx;
    a.mask = mask;
    a.sum_p = reinterpret_cast<float*>(take(rows * c.emax));
    a.counts = reinterpret_cast<int32_t*>(take(parts * c.emax));
    a.sum_z = reinterpret_cast<float*>(take(rows));
    a.live = reinterpret_cast<int32_t*>(take(parts));
    a.lse = c.twice ? reinterpret_cast<float*>(take(static_cast<size_t>(D.N))) : nullptr;
    a.losses = losses;
    a.mean_probs = mean_probs;
    a.dlogits = dlogits;
    a.demand = demand;
    a.Ng = D.Ng;
    a.E = D.E;
    a.k = D.k;
    a.chunks = c.count;
    a.chunk_tokens = c.tokens;
    a.parts = c.parts;
    a.part_tokens = c.part_tokens;
    a.w_balance = w_balance;
    a.w_z = w_z;
    a.first_group = 0;
    by_experts(D.E, [&](auto tag) {
        constexpr int EMAX = decltype(tag)::value, kThreads = 64 * kChunkWaves;
        if (c.whole) {
            // a launch has fewer than 2^32 threads (groups too long for a block are
            // never so many)
            constexpr int kMost = 1 << 21;
            for (a.first_group = 0; a.first_group < D.G; a.first_group += kMost) {
                const int n = D.G - a.first_group < kMost ? D.G - a.first_group : kMost;
                gate_group_kernel<EMAX><<<n, 64 * kGroupWaves, 0, st>>>(a);
            }
            return;
        }
        const unsigned blocks = static_cast<unsigned>(rows);  // at most N or G
        if (c.twice) {
            gate_count_kernel<EMAX, true><<<blocks, kThreads, 0, st>>>(a);
            gate_gradient_kernel<EMAX><<<blocks + D.G, kThreads, 0, st>>>(a);
            return;
        }
        gate_count_kernel<EMAX, false><<<static_cast<unsigned>(parts), kThreads, 0, st>>>(a);
        gate_rows_kernel<EMAX><<<blocks, kThreads, 0, st>>>(a);
        gate_losses_kernel<EMAX><<<D.G, kThreads, 0, st>>>(a);
    });
    return launch_status();
}

}  // namespace vmoe

// The experts' demand and the load-balance and z losses of a gate, with their
// gradient with respect to the router logits:
//   L_balance = E sum_e f_e P_e, f_e = demand_e / (k n), P_e = mean of probs;
//   L_z       = mean of lse^2, lse = log sum_e exp z;
//   dlogits   = p (w_balance E (f - <f, p>) + 2 w_z lse) / n.
// The gradient needs f of the whole group, so there are two passes. The first
// reads logits, noise, probs and choices once: a chunk's counts, sums of probs
// and of lse^2, and each token's lse, for which the softmax's largest term is
// enough (lse = max z - log max p: no second exponential). The second adds the
// group's counts (integers, a few hundred short rows from L2) in every block
// and forms the rows of dlogits from probs and lse; one more block a group adds
// the other sums, in double and in chunk order, and writes the losses. A group
// of few tokens runs both passes in one block of one launch.
// A lane holds four consecutive experts of a token (one 16-byte access where E
// is a multiple of 4), so a token takes at most 16 lanes and its maxima and sums
// are moves within a row of lanes, without LDS. Both passes are bound by latency
// up to some ten thousand tokens, by HBM beyond.
#include <type_traits>

#include "common_train.h"

namespace vmoe {
namespace {

constexpr int kSteps = 4;        // token steps whose loads are in flight together
constexpr int kChunkWaves = 8;   // waves of a block that takes a chunk
constexpr int kGroupWaves = 16;  // of a block that takes a whole group
constexpr int kBlocks = 1024;    // most chunks over all groups (but one a group)
constexpr int kGroupChunks = 256;  // and of one group

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
    float *lse, *sum_p, *sum_z;      // workspace: [N], [G, chunks, EMAX], [G, chunks]
    int32_t *counts, *live;          // workspace: [G, chunks, EMAX], [G, chunks]
    float *losses, *mean_probs, *dlogits;
    int32_t* demand;
    int Ng, E, k, chunks, chunk_tokens;
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

// A block's sums over tokens [t0, t1) of its group.
template <int EMAX, int WAVES>
struct BlockSums {
    int hist[WAVES][EMAX];
    float p[WAVES][EMAX];
    float z[WAVES];
    int n[WAVES];
    __device__ __forceinline__ int count(int e) const {
        int t = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) t += hist[w][e];
        return t;
    }
    __device__ __forceinline__ float prob(int e) const {
        float t = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) t += p[w][e];
        return t;
    }
    __device__ __forceinline__ float square(float s = 0.0f) const {
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += z[w];
        return s;
    }
    __device__ __forceinline__ int tokens(int s = 0) const {
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += n[w];
        return s;
    }
};

// lse of token t to lse[t - t0]. Ends with a barrier.
template <int EMAX, int WAVES>
__device__ __forceinline__ void sum_tokens(const LossArgs& a, size_t first, int t0, int t1,
                                           BlockSums<EMAX, WAVES>& sums, float* lse) {
    using R = Rows<EMAX, WAVES>;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int e0 = (lane % R::kLanes) * 4, sub = lane / R::kLanes;
    // the first choices are requested before the rows
    const int words = (t1 - t0) * a.k;
    const int32_t* idx = a.idx + (first + t0) * a.k;
    int x[kSteps];
    const auto choices = [&](int b) {
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int w = b + u * R::kThreads;
            x[u] = w < words && kept(a, first + t0 + w / a.k) ? idx[w] : -1;
        }
    };
    choices(tid);
    for (int i = lane; i < EMAX; i += 64) sums.hist[wave][i] = 0;
    const float4 be = a.bias ? load_row(a.bias, e0, a.E, true) : make_float4(0.f, 0.f, 0.f, 0.f);
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f}, acc_z = 0.0f;
    int acc_n = 0;
    for (int b = t0; b < t1; b += kSteps * R::kBlockTokens) {
        float4 l[kSteps], nz[kSteps], p[kSteps];
        bool on[kSteps];
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int t = b + (u * WAVES + wave) * R::kTokens + sub;
            on[u] = t < t1 && kept(a, first + t);
            const size_t q = (first + t) * a.E;
            l[u] = load_row(a.logits + q, e0, a.E, on[u]);
            p[u] = load_row(a.probs + q, e0, a.E, on[u]);
            nz[u] = load_row(a.noise + q, e0, a.E, on[u] && a.noise != nullptr);
        }
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int t = b + (u * WAVES + wave) * R::kTokens + sub;
            const float lv[4] = {l[u].x, l[u].y, l[u].z, l[u].w};
            const float nv[4] = {nz[u].x, nz[u].y, nz[u].z, nz[u].w};
            const float pv[4] = {p[u].x, p[u].y, p[u].z, p[u].w};
            const float bv[4] = {be.x, be.y, be.z, be.w};
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
            if (on[u] && e0 == 0) {
                const float v = top - logf(most);
                acc_z = __builtin_fmaf(v, v, acc_z);
                acc_n += 1;
                lse[t - t0] = v;
            }
        }
    }
#pragma unroll
    for (int o = 32; o >= R::kLanes; o >>= 1)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += __shfl_xor(acc[j], o);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        acc_z += __shfl_xor(acc_z, o);
        acc_n += __shfl_xor(acc_n, o);
    }
    if (sub == 0)
#pragma unroll
        for (int j = 0; j < 4; ++j) sums.p[wave][e0 + j] = acc[j];
    if (lane == 0) {
        sums.z[wave] = acc_z;
        sums.n[wave] = acc_n;
    }
    // choices in rows of consecutive words; integer LDS atomics on the wave's
    // own counts
    for (int b = tid; b < words; b += kSteps * R::kThreads) {
        if (b != tid) choices(b);
#pragma unroll
        for (int u = 0; u < kSteps; ++u)
            if (x[u] >= 0 && x[u] < a.E) atomicAdd(&sums.hist[wave][x[u]], 1);
    }
    __syncthreads();
}

// Rows [t0, t1) of dlogits; f4: the lane's four f, per: 1 / n. `ready` runs
// between the first rows' loads and their use, and sets f4 and per.
template <int EMAX, int WAVES, typename F>
__device__ __forceinline__ void write_rows(const LossArgs& a, size_t first, int t0, int t1,
                                           const float* lse, F ready) {
    using R = Rows<EMAX, WAVES>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int e0 = (lane % R::kLanes) * 4, sub = lane / R::kLanes;
    float f4[4], per = 0.0f, cb = 0.0f, cz = 0.0f;
    for (int b = t0; b < t1; b += kSteps * R::kBlockTokens) {
        float4 p[kSteps];
        float ls[kSteps];
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int t = b + (u * WAVES + wave) * R::kTokens + sub;
            const bool on = t < t1 && kept(a, first + t);
            p[u] = load_row(a.probs + (first + t) * a.E, e0, a.E, on);
            ls[u] = on ? lse[t - t0] : 0.0f;
        }
        if (b == t0) {
            ready(f4, per);
            cb = a.w_balance * static_cast<float>(a.E) * per;
            cz = 2.0f * a.w_z * per;
        }
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int t = b + (u * WAVES + wave) * R::kTokens + sub;
            const float pv[4] = {p[u].x, p[u].y, p[u].z, p[u].w};
            float inner = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) inner = __builtin_fmaf(f4[j], pv[j], inner);
            inner = over_token<R::kLanes>(inner, Add{});
            float d[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                d[j] = pv[j] * __builtin_fmaf(cb, f4[j] - inner, cz * ls[u]);
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
}

// Demand, mean probabilities and losses of a group from its totals in LDS, by a
// whole block.
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

__device__ __forceinline__ void shares(const LossArgs& a, const int* total, int n_live, int e0,
                                       float (&f4)[4], float& per) {
    per = n_live > 0 ? 1.0f / static_cast<float>(n_live) : 0.0f;
    const float fk = per / static_cast<float>(a.k);
#pragma unroll
    for (int j = 0; j < 4; ++j) f4[j] = static_cast<float>(total[e0 + j]) * fk;
}

// A whole group in one block.
template <int EMAX>
__global__ __launch_bounds__(64 * kGroupWaves) void gate_group_kernel(LossArgs a) {
    using R = Rows<EMAX, kGroupWaves>;
    __shared__ BlockSums<EMAX, kGroupWaves> sums;
    __shared__ float lse[R::kGroupTokens];
    __shared__ int total[EMAX];
    __shared__ double sum_p[EMAX];
    const int g = blockIdx.x, tid = threadIdx.x;
    const size_t first = static_cast<size_t>(g) * a.Ng;
    sum_tokens<EMAX, kGroupWaves>(a, first, 0, a.Ng, sums, lse);
    const int n_live = sums.tokens();
    if (tid < EMAX) {
        total[tid] = sums.count(tid);
        sum_p[tid] = sums.prob(tid);
    }
    __syncthreads();
    write_rows<EMAX, kGroupWaves>(a, first, 0, a.Ng, lse, [&](float (&f4)[4], float& per) {
        shares(a, total, n_live, ((tid & 63) % R::kLanes) * 4, f4, per);
    });
    write_losses(a, g, total, sum_p, sums.square(), n_live);
}

// First pass over a chunk.
template <int EMAX>
__global__ __launch_bounds__(64 * kChunkWaves) void gate_sums_kernel(LossArgs a) {
    __shared__ BlockSums<EMAX, kChunkWaves> sums;
    const int g = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks, tid = threadIdx.x;
    const int t0 = chunk * a.chunk_tokens, t1 = min(t0 + a.chunk_tokens, a.Ng);
    const size_t first = static_cast<size_t>(g) * a.Ng;
    sum_tokens<EMAX, kChunkWaves>(a, first, t0, t1, sums, a.lse + first + t0);
    if (tid < EMAX) {
        a.sum_p[static_cast<size_t>(blockIdx.x) * EMAX + tid] = sums.prob(tid);
        a.counts[static_cast<size_t>(blockIdx.x) * EMAX + tid] = sums.count(tid);
    }
    if (tid == 64) {
        a.sum_z[blockIdx.x] = sums.square();
        a.live[blockIdx.x] = sums.tokens();
    }
}

// The group's counts and its number of tokens: rows of EMAX counts as a flat run
// of 16-byte words, of which a thread always meets the same four experts (4
// threads' worth of a block is a multiple of EMAX). Ends with a barrier.
template <int EMAX>
__device__ __forceinline__ void group_counts(const LossArgs& a, int g, int* total, int& n_live) {
    constexpr int kQuads = EMAX / 4, kThreads = 64 * kChunkWaves, kFlight = 16;
    __shared__ int part[kChunkWaves][EMAX];
    __shared__ int part_n[kChunkWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int4* rows = reinterpret_cast<const int4*>(a.counts +
                                                     static_cast<size_t>(g) * a.chunks * EMAX);
    const int words = a.chunks * kQuads;
    int n = 0;
    for (int c = tid; c < a.chunks; c += kThreads) n += a.live[static_cast<size_t>(g) * a.chunks + c];
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
    if (lane < kQuads) *reinterpret_cast<int4*>(&part[wave][lane * 4]) = s;
    if (lane == 0) part_n[wave] = n;
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

// Second pass: a chunk's rows, or (the block after a group's chunks) its losses.
template <int EMAX>
__global__ __launch_bounds__(64 * kChunkWaves) void gate_grad_kernel(LossArgs a) {
    using R = Rows<EMAX, kChunkWaves>;
    constexpr int kSlices = R::kThreads / EMAX;
    __shared__ __align__(16) int total[EMAX];
    __shared__ double part[R::kThreads];
    __shared__ double sum_p[EMAX];
    __shared__ double part_z[kChunkWaves];
    const int g = blockIdx.x / (a.chunks + 1), chunk = blockIdx.x % (a.chunks + 1);
    const int tid = threadIdx.x;
    int n_live;
    if (chunk < a.chunks) {
        const int t0 = chunk * a.chunk_tokens, t1 = min(t0 + a.chunk_tokens, a.Ng);
        const size_t first = static_cast<size_t>(g) * a.Ng;
        write_rows<EMAX, kChunkWaves>(
            a, first, t0, t1, a.lse + first + t0, [&](float (&f4)[4], float& per) {
                group_counts<EMAX>(a, g, total, n_live);
                shares(a, total, n_live, ((tid & 63) % R::kLanes) * 4, f4, per);
            });
        return;
    }
    group_counts<EMAX>(a, g, total, n_live);
    const int e = tid % EMAX, q = tid / EMAX;
    const float* sp = a.sum_p + static_cast<size_t>(g) * a.chunks * EMAX + e;
    const float* sz = a.sum_z + static_cast<size_t>(g) * a.chunks;
    double s = 0.0, z = 0.0;
    int c = q;
    for (; c + 15 * kSlices < a.chunks; c += 16 * kSlices) {  // sixteen in flight, added in order
        float v[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) v[u] = sp[static_cast<size_t>(c + u * kSlices) * EMAX];
#pragma unroll
        for (int u = 0; u < 16; ++u) s += v[u];
    }
    for (; c < a.chunks; c += kSlices) s += sp[static_cast<size_t>(c) * EMAX];
    for (int i = tid; i < a.chunks; i += R::kThreads) z += sz[i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o);
    part[tid] = s;
    if ((tid & 63) == 0) part_z[tid >> 6] = z;
    __syncthreads();
    if (tid < EMAX) {
        double t = 0.0;
#pragma unroll
        for (int r = 0; r < kSlices; ++r) t += part[r * EMAX + tid];
        sum_p[tid] = t;
    }
    z = 0.0;
#pragma unroll
    for (int w = 0; w < kChunkWaves; ++w) z += part_z[w];
    __syncthreads();
    write_losses(a, g, total, sum_p, z, n_live);
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
    bool whole;  // a group in one block
};

// Chunks of a group: about kBlocks over all groups, none shorter than a block's
// step. More would cost every block of the second launch more rows of counts.
Chunks chunks_of(const Dims& D) {
    Chunks c = {1, 1, 4, false};
    by_experts(D.E, [&](auto tag) {
        constexpr int EMAX = decltype(tag)::value;
        c.emax = EMAX;
        c.whole = D.Ng <= Rows<EMAX, kGroupWaves>::kGroupTokens;
        const int most = static_cast<int>(cdiv(D.Ng, Rows<EMAX, kChunkWaves>::kBlockTokens));
        int n = kBlocks / D.G;
        if (n > kGroupChunks) n = kGroupChunks;
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
        if (c.whole) {
            gate_group_kernel<EMAX><<<D.G, 64 * kGroupWaves, 0, st>>>(a);
            return;
        }
        gate_sums_kernel<EMAX><<<grid, 64 * kChunkWaves, 0, st>>>(a);
        gate_grad_kernel<EMAX><<<grid + D.G, 64 * kChunkWaves, 0, st>>>(a);
    });
    return launch_status();
}

}  // namespace vmoe

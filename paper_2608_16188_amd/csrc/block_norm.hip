// Norm after a block, gate, residual add and norm before the next block in one
// pass over the tokens, and its backward.
//
// A team of waves holds a token's whole row in registers, 8 consecutive columns
// a lane and step, so every tensor is read once and written once whatever the
// norms need: means and deviations are sums over the team (lane moves within a
// wave, LDS across waves). Both directions are streams of rows, bound by HBM.
//
// The backward also sums over tokens for each column (the gradients of weights,
// biases and gate). A team keeps those sums in registers over all of its rows;
// a block's rows lie in one group, its sums leave as one row of partials, and a
// second kernel adds the partials of a column in a fixed order. Post-norm sums
// are kept without the gate and the weight, S = sum a G m and T = sum a G (G the
// gradient at x_out, m the unit output): with one gate row a group, dgate =
// w S + b T, dw = sum_g gate S and db = sum_g gate T follow from two sums.
#include <type_traits>

#include "common_train.h"

namespace vmoe {
namespace {

constexpr int kLanes = 64;

// Eight consecutive elements as they lie in memory.
template <typename T> struct Raw8;
template <> struct Raw8<uint16_t> {
    uint4 q;
    __device__ __forceinline__ void load(const uint16_t* p) {
        q = *reinterpret_cast<const uint4*>(p);
    }
    __device__ __forceinline__ void zero() { q = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ float get(int j) const {
        const uint32_t w = j < 2 ? q.x : j < 4 ? q.y : j < 6 ? q.z : q.w;
        return __uint_as_float((j & 1) ? w & 0xFFFF0000u : w << 16);
    }
};
template <> struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = reinterpret_cast<const float4*>(p)[0];
        b = reinterpret_cast<const float4*>(p)[1];
    }
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ float get(int j) const {
        return j == 0 ? a.x : j == 1 ? a.y : j == 2 ? a.z : j == 3 ? a.w
             : j == 4 ? b.x : j == 5 ? b.y : j == 6 ? b.z : b.w;
    }
};

__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                              pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// W waves a row, V steps of 8 columns a lane: columns (i W 64 + lane of team) 8.
template <int W, int V>
struct Team {
    static constexpr int kBlock = W == 1 ? 256 : W * kLanes;
    static constexpr int kRows = kBlock / (W * kLanes);  // rows a block works on at a time
    static __device__ __forceinline__ int lane() {
        return W == 1 ? threadIdx.x & (kLanes - 1) : threadIdx.x;
    }
    static __device__ __forceinline__ int row() { return W == 1 ? threadIdx.x / kLanes : 0; }
    static __device__ __forceinline__ int column(int i) { return (i * W * kLanes + lane()) * 8; }
};

// Sums over a team, for every lane. The two halves of `lds` take turns, so one
// barrier a call is enough: a half is written again only after the barrier of
// the call between, which every wave passes after its reads.
template <int W, int K>
__device__ __forceinline__ void team_sum(float (&s)[K], float* lds, int& turn) {
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = wave_total(s[k]);
    if constexpr (W > 1) {
        float* half = lds + turn * 2 * W;
        turn ^= 1;
        if ((threadIdx.x & (kLanes - 1)) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) half[(threadIdx.x / kLanes) * 2 + k] = s[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float t = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) t += half[w * 2 + k];
            s[k] = t;
        }
    }
}

struct FwdArgs {
    const void *x, *y, *post_w, *post_b, *gate;
    const float* row_scale;
    const void *pre_w, *pre_b;
    void *x_out, *h;
    float *post_stats, *pre_stats;
    int N, Ng, G, d, pre, post;
    float eps, residual, branch;
};

// mean and 1/deviation of a row in registers. Columns past d hold 0 and are
// left out of the sum about the mean.
template <int W, int V>
__device__ __forceinline__ float2 row_stats(const float (&v)[V][8], int kind, int d, float eps,
                                            float inv_d, float* lds, int& turn) {
    using T = Team<W, V>;
    float mean = 0.0f, s[1];
    if (kind == VMOE_NORM_LAYER) {
        s[0] = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] += v[i][j];
        team_sum<W, 1>(s, lds, turn);
        mean = s[0] * inv_d;
    }
    s[0] = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (T::column(i) < d)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float c = v[i][j] - mean;
                s[0] = __builtin_fmaf(c, c, s[0]);
            }
    }
    team_sum<W, 1>(s, lds, turn);
    return make_float2(mean, 1.0f / sqrtf(__builtin_fmaf(s[0], inv_d, eps)));
}

template <typename TA, int V>
__device__ __forceinline__ void load_weights(Raw8<TA> (&w)[V], const void* p, int d, const int (&col)[V]) {
    const TA* q = static_cast<const TA*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (q != nullptr && col[i] < d) w[i].load(q + col[i]);
        else w[i].zero();
    }
}

template <typename TS, typename TA, int W, int V>
__global__ __launch_bounds__((Team<W, V>::kBlock)) void block_norm_fwd_kernel(FwdArgs a) {
    using T = Team<W, V>;
    __shared__ float lds[4 * W];
    int turn = 0;
    int col[V];
#pragma unroll
    for (int i = 0; i < V; ++i) col[i] = T::column(i);
    const float inv_d = 1.0f / static_cast<float>(a.d);
    Raw8<TA> pre_w[V], pre_b[V], post_w[V], post_b[V];
    load_weights<TA, V>(pre_w, a.pre_w, a.d, col);
    load_weights<TA, V>(pre_b, a.pre_b, a.d, col);
    load_weights<TA, V>(post_w, a.post_w, a.d, col);
    load_weights<TA, V>(post_b, a.post_b, a.d, col);
    const int step = gridDim.x * T::kRows;
    for (int t = blockIdx.x * T::kRows + T::row(); t < a.N; t += step) {
        const size_t at = static_cast<size_t>(t) * a.d;
        const TS* x = static_cast<const TS*>(a.x) + at;
        Raw8<TS> xr[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (col[i] < a.d) xr[i].load(x + col[i]);
            else xr[i].zero();
        }
        float v[V][8];
        if (a.y != nullptr) {
            const float rs = a.row_scale ? a.row_scale[t] : 1.0f;
            const float scale = a.branch * rs;
            const bool on = rs != 0.0f;  // the same for the whole team
            Raw8<TA> yr[V], gr[V];
            if (on) {
                const TA* y = static_cast<const TA*>(a.y) + at;
                const TA* gate = a.gate ? static_cast<const TA*>(a.gate) +
                                              static_cast<size_t>(a.G == 1 ? 0 : t / a.Ng) * a.d
                                        : nullptr;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if (col[i] < a.d) {
                        yr[i].load(y + col[i]);
                        if (gate) gr[i].load(gate + col[i]);
                    } else {
                        yr[i].zero();
                        gr[i].zero();
                    }
                }
#pragma unroll
                for (int i = 0; i < V; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[i][j] = yr[i].get(j);
            }
            if (a.post != VMOE_NORM_NONE) {
                float2 st = make_float2(0.0f, 0.0f);
                if (on) {
                    st = row_stats<W, V>(v, a.post, a.d, a.eps, inv_d, lds, turn);
#pragma unroll
                    for (int i = 0; i < V; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            float n = (v[i][j] - st.x) * st.y;
                            if (a.post_w) n *= post_w[i].get(j);
                            if (a.post_b) n += post_b[i].get(j);
                            v[i][j] = n;
                        }
                }
                if (T::lane() == 0) reinterpret_cast<float2*>(a.post_stats)[t] = st;
            }
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float b = 0.0f;
                    if (on) b = scale * (a.gate ? v[i][j] * gr[i].get(j) : v[i][j]);
                    v[i][j] = __builtin_fmaf(a.residual, xr[i].get(j), b);
                }
            TS* xo = static_cast<TS*>(a.x_out) + at;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (col[i] < a.d) store8(xo + col[i], v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = xr[i].get(j);
        }
        if (a.pre != VMOE_NORM_NONE) {
            // columns past d hold what the branch left there: take them out
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (col[i] >= a.d)
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
            const float2 st = row_stats<W, V>(v, a.pre, a.d, a.eps, inv_d, lds, turn);
            if (T::lane() == 0) reinterpret_cast<float2*>(a.pre_stats)[t] = st;
            TA* h = static_cast<TA*>(a.h) + at;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    o[j] = (v[i][j] - st.x) * st.y;
                    if (a.pre_w) o[j] *= pre_w[i].get(j);
                    if (a.pre_b) o[j] += pre_b[i].get(j);
                }
                if (col[i] < a.d) store8(h + col[i], o);
            }
        }
    }
}

struct BwdArgs {
    const void *dx_out, *dh, *x_out, *y, *post_w, *gate;
    const float* row_scale;
    const void* pre_w;
    const float *post_stats, *pre_stats;
    void *dx, *dy;
    float* partial;                  // [blocks, slots, d]
    int slot_w, slot_b, slot_s, slot_t, slots;  // -1: not asked for
    int N, Ng, G, d, pre, post;
    int blocks_per_group, rows_per_block;
    float residual, branch;
};

// One block's sums of one kind into its row of partials.
template <int W, int V>
__device__ __forceinline__ void leave_sums(const float (&acc)[V][8], float* out, int d,
                                           const int (&col)[V], float* lds) {
    using T = Team<W, V>;
    if constexpr (W > 1) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (col[i] < d) store8(out + col[i], acc[i]);
    } else {
        constexpr int kCols = V * kLanes * 8;
        __syncthreads();  // the last use of lds
#pragma unroll
        for (int i = 0; i < V; ++i) store8(lds + T::row() * kCols + col[i], acc[i]);
        __syncthreads();
        for (int c = threadIdx.x; c < d; c += T::kBlock) {
            float s = 0.0f;
#pragma unroll
            for (int r = 0; r < T::kRows; ++r) s += lds[r * kCols + c];
            out[c] = s;
        }
    }
}

template <typename TS, typename TA, typename TH, int W, int V>
__global__ __launch_bounds__((Team<W, V>::kBlock)) void block_norm_bwd_kernel(BwdArgs a) {
    using T = Team<W, V>;
    __shared__ __align__(16) float lds[W == 1 ? T::kRows * V * kLanes * 8 : 4 * W];
    int turn = 0;
    int col[V];
#pragma unroll
    for (int i = 0; i < V; ++i) col[i] = T::column(i);
    const float inv_d = 1.0f / static_cast<float>(a.d);
    const int g = blockIdx.x / a.blocks_per_group;
    const int part = blockIdx.x % a.blocks_per_group;
    const int t0 = g * a.Ng + part * a.rows_per_block;
    const int t1 = min(t0 + a.rows_per_block, (g + 1) * a.Ng);
    Raw8<TA> pre_w[V], post_w[V], gate[V];
    load_weights<TA, V>(pre_w, a.pre_w, a.d, col);
    load_weights<TA, V>(post_w, a.post_w, a.d, col);
    load_weights<TA, V>(gate, a.gate ? static_cast<const TA*>(a.gate) + static_cast<size_t>(g) * a.d
                                     : nullptr, a.d, col);
    float acc_w[V][8], acc_b[V][8], acc_s[V][8], acc_t[V][8];
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc_w[i][j] = acc_b[i][j] = acc_s[i][j] = acc_t[i][j] = 0.0f;

    for (int t = t0 + T::row(); t < t1; t += T::kRows) {
        const size_t at = static_cast<size_t>(t) * a.d;
        const float rs = a.row_scale ? a.row_scale[t] : 1.0f;
        const bool on = a.y != nullptr && rs != 0.0f;  // the same for the whole team
        Raw8<TH> hr[V];
        Raw8<TS> xr[V], ur[V];
        Raw8<TA> yr[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const bool live = col[i] < a.d;
            if (live && a.pre != VMOE_NORM_NONE) {
                hr[i].load(static_cast<const TH*>(a.dh) + at + col[i]);
                xr[i].load(static_cast<const TS*>(a.x_out) + at + col[i]);
            } else {
                hr[i].zero();
                xr[i].zero();
            }
            if (live && a.dx_out) ur[i].load(static_cast<const TS*>(a.dx_out) + at + col[i]);
            else ur[i].zero();
            if (live && on) yr[i].load(static_cast<const TA*>(a.y) + at + col[i]);
            else yr[i].zero();
        }
        float G[V][8];
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) G[i][j] = ur[i].get(j);
        if (a.pre != VMOE_NORM_NONE) {
            const float2 st = reinterpret_cast<const float2*>(a.pre_stats)[t];
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float dh = hr[i].get(j), n = (xr[i].get(j) - st.x) * st.y;
                    const float dn = a.pre_w ? dh * pre_w[i].get(j) : dh;
                    acc_w[i][j] = __builtin_fmaf(dh, n, acc_w[i][j]);
                    acc_b[i][j] += dh;
                    s[0] += dn;
                    s[1] = __builtin_fmaf(dn, n, s[1]);
                }
            team_sum<W, 2>(s, lds, turn);
            const float c0 = a.pre == VMOE_NORM_LAYER ? s[0] * inv_d : 0.0f, c1 = s[1] * inv_d;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const bool live = col[i] < a.d;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float dh = hr[i].get(j), n = (xr[i].get(j) - st.x) * st.y;
                    const float dn = a.pre_w ? dh * pre_w[i].get(j) : dh;
                    const float v = __builtin_fmaf(st.y, dn - c0 - n * c1, G[i][j]);
                    G[i][j] = live ? v : 0.0f;
                }
            }
        }
        const float residual = a.y != nullptr ? a.residual : 1.0f;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (col[i] < a.d) {
                float o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = residual * G[i][j];
                store8(static_cast<TS*>(a.dx) + at + col[i], o);
            }
        if (a.y == nullptr) continue;
        if (on) {
            const float scale = a.branch * rs;
            const bool normed = a.post != VMOE_NORM_NONE;
            float2 st = make_float2(0.0f, 1.0f);
            if (normed) st = reinterpret_cast<const float2*>(a.post_stats)[t];
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float ag = scale * G[i][j], m = (yr[i].get(j) - st.x) * st.y;
                    acc_s[i][j] = __builtin_fmaf(ag, m, acc_s[i][j]);
                    acc_t[i][j] += ag;
                    float dn = a.gate ? ag * gate[i].get(j) : ag;
                    if (a.post_w) dn *= post_w[i].get(j);
                    G[i][j] = dn;
                    s[0] += dn;
                    s[1] = __builtin_fmaf(dn, m, s[1]);
                }
            if (normed) {
                team_sum<W, 2>(s, lds, turn);
                const float c0 = a.post == VMOE_NORM_LAYER ? s[0] * inv_d : 0.0f, c1 = s[1] * inv_d;
#pragma unroll
                for (int i = 0; i < V; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float m = (yr[i].get(j) - st.x) * st.y;
                        G[i][j] = st.y * (G[i][j] - c0 - m * c1);
                    }
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) G[i][j] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (col[i] < a.d) store8(static_cast<TA*>(a.dy) + at + col[i], G[i]);
    }

    if (a.slots == 0) return;
    float* out = a.partial + static_cast<size_t>(blockIdx.x) * a.slots * a.d;
    if (a.slot_w >= 0) leave_sums<W, V>(acc_w, out + static_cast<size_t>(a.slot_w) * a.d, a.d, col, lds);
    if (a.slot_b >= 0) leave_sums<W, V>(acc_b, out + static_cast<size_t>(a.slot_b) * a.d, a.d, col, lds);
    if (a.slot_s >= 0) leave_sums<W, V>(acc_s, out + static_cast<size_t>(a.slot_s) * a.d, a.d, col, lds);
    if (a.slot_t >= 0) leave_sums<W, V>(acc_t, out + static_cast<size_t>(a.slot_t) * a.d, a.d, col, lds);
}

struct ReduceArgs {
    const float* partial;
    const void *post_w, *post_b, *gate;
    float *dpre_w, *dpre_b, *dpost_w, *dpost_b, *dgate;
    int slot_w, slot_b, slot_s, slot_t, slots;
    int G, d, blocks_per_group, blocks;
};

constexpr int kReduceCols = 64, kSlices = 16;

// Sum of one column of partial rows first, first + stride, ... below end.
__device__ __forceinline__ float column_sum(const float* p, size_t row, int first, int end,
                                            int stride) {
    float s = 0.0f;
    int r = first;
    for (; r + 7 * stride < end; r += 8 * stride) {  // eight rows in flight, added in order
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = p[(r + u * stride) * row];
#pragma unroll
        for (int u = 0; u < 8; ++u) s += v[u];
    }
    for (; r < end; r += stride) s += p[r * row];
    return s;
}

// Adds the slices of a column in order, for the threads of slice 0.
__device__ __forceinline__ float over_slices(float v, float (*lds)[kReduceCols]) {
    __syncthreads();
    lds[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    float s = 0.0f;
    if (threadIdx.y == 0)
#pragma unroll
        for (int q = 0; q < kSlices; ++q) s += lds[q][threadIdx.x];
    return s;
}

// Blocks of 64 columns x 16 slices; blockIdx.y 0: the pre-norm's sums, 1: the
// post-norm's and the gate's. With 16 groups and more a slice adds whole
// groups, else all slices share a group's partial rows.
template <typename TA>
__global__ __launch_bounds__(kReduceCols* kSlices) void block_norm_reduce_kernel(ReduceArgs a) {
    __shared__ float lds[kSlices][kReduceCols];
    const int c = blockIdx.x * kReduceCols + threadIdx.x, q = threadIdx.y;
    const bool live = c < a.d;
    const size_t row = static_cast<size_t>(a.slots) * a.d;
    const float* p = a.partial + (live ? c : 0);
    if (blockIdx.y == 0) {
        if (a.slot_w >= 0) {
            const float s = over_slices(column_sum(p + static_cast<size_t>(a.slot_w) * a.d, row, q,
                                                   a.blocks, kSlices), lds);
            if (q == 0 && live) a.dpre_w[c] = s;
        }
        if (a.slot_b >= 0) {
            const float s = over_slices(column_sum(p + static_cast<size_t>(a.slot_b) * a.d, row, q,
                                                   a.blocks, kSlices), lds);
            if (q == 0 && live) a.dpre_b[c] = s;
        }
        return;
    }
    const float w = a.post_w && live ? Elem<TA>::load(static_cast<const TA*>(a.post_w), c) : 1.0f;
    const float b = a.post_b && live ? Elem<TA>::load(static_cast<const TA*>(a.post_b), c) : 0.0f;
    const float* ps = p + static_cast<size_t>(a.slot_s < 0 ? 0 : a.slot_s) * a.d;
    const float* pt = p + static_cast<size_t>(a.slot_t < 0 ? 0 : a.slot_t) * a.d;
    const bool whole = a.G >= kSlices;
    float sum_w = 0.0f, sum_b = 0.0f;
    for (int g = whole ? q : 0; g < a.G; g += whole ? kSlices : 1) {
        const int first = g * a.blocks_per_group, end = min(first + a.blocks_per_group, a.blocks);
        float S = 0.0f, T = 0.0f;
        if (whole) {
            if (a.slot_s >= 0) S = column_sum(ps, row, first, end, 1);
            if (a.slot_t >= 0) T = column_sum(pt, row, first, end, 1);
        } else {
            if (a.slot_s >= 0) S = over_slices(column_sum(ps, row, first + q, end, kSlices), lds);
            if (a.slot_t >= 0) T = over_slices(column_sum(pt, row, first + q, end, kSlices), lds);
        }
        if (live && (whole || q == 0)) {
            const size_t at = static_cast<size_t>(g) * a.d + c;
            const float gate = a.gate ? Elem<TA>::load(static_cast<const TA*>(a.gate), at) : 1.0f;
            if (a.dgate) a.dgate[at] = __builtin_fmaf(w, S, b * T);
            sum_w = __builtin_fmaf(gate, S, sum_w);
            sum_b = __builtin_fmaf(gate, T, sum_b);
        }
    }
    if (whole) {
        sum_w = over_slices(sum_w, lds);
        sum_b = over_slices(sum_b, lds);
    }
    if (q == 0 && live) {
        if (a.dpost_w) a.dpost_w[c] = sum_w;
        if (a.dpost_b) a.dpost_b[c] = sum_b;
    }
}

// Waves a row and steps a lane by width: one wave up to 1024 columns (no
// barrier in a row), more waves beyond, so that the backward's four sums and
// its row stay in registers.
template <typename F>
void by_width(int d, F f) {
    if (d <= 512) f(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{});
    else if (d <= 1024) f(std::integral_constant<int, 1>{}, std::integral_constant<int, 2>{});
    else if (d <= 2048) f(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
    else if (d <= 4096) f(std::integral_constant<int, 4>{}, std::integral_constant<int, 2>{});
    else if (d <= 8192) f(std::integral_constant<int, 8>{}, std::integral_constant<int, 2>{});
    else f(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
}

struct BwdGrid {
    int blocks_per_group, rows_per_block;
    long long blocks;
};

// About kBwdBlocks blocks over all groups, none across two groups, a row or
// more for every wave of one.
constexpr int kBwdBlocks = 768;
BwdGrid bwd_grid(const vmoe_norm_shape& s) {
    const int Ng = s.n_tokens / s.n_groups;
    if (Ng == 0) return {1, 1, 0};
    const int least = s.d_model <= 1024 ? 4 : 1;
    int per_group = kBwdBlocks / s.n_groups;
    const int most = (Ng + least - 1) / least;
    if (per_group > most) per_group = most;
    if (per_group < 1) per_group = 1;
    BwdGrid b;
    b.rows_per_block = (Ng + per_group - 1) / per_group;
    b.blocks_per_group = (Ng + b.rows_per_block - 1) / b.rows_per_block;
    b.blocks = static_cast<long long>(b.blocks_per_group) * s.n_groups;
    return b;
}

}  // namespace

size_t block_norm_bwd_workspace_bytes(const vmoe_norm_shape& s) {
    return sizeof(float) * 4 * static_cast<size_t>(bwd_grid(s).blocks) * s.d_model;
}

vmoe_status block_norm_fwd_launch(const vmoe_norm_shape& s, const void* x, const void* y,
                                  const void* post_w, const void* post_b, const void* gate,
                                  const float* row_scale, const void* pre_w, const void* pre_b,
                                  void* x_out, void* h, float* post_stats, float* pre_stats,
                                  hipStream_t st) {
    if (s.n_tokens == 0) return VMOE_OK;
    const FwdArgs a = {x, y, post_w, post_b, gate, row_scale, pre_w, pre_b, x_out, h, post_stats,
                       pre_stats, s.n_tokens, s.n_tokens / s.n_groups, s.n_groups, s.d_model,
                       s.pre_norm, s.post_norm, s.eps, s.residual_scale, s.branch_scale};
    by_width(s.d_model, [&](auto wt, auto vt) {
        constexpr int W = decltype(wt)::value, V = decltype(vt)::value;
        using T = Team<W, V>;
        // as many waves as stay resident, each on several rows
        const unsigned rows = cdiv(s.n_tokens, T::kRows), most = 4096 * kLanes / T::kBlock;
        const unsigned grid = rows < most ? rows : most;
        if (s.dtype == VMOE_F32)
            block_norm_fwd_kernel<float, float, W, V><<<grid, T::kBlock, 0, st>>>(a);
        else if (s.stream_dtype == VMOE_F32)
            block_norm_fwd_kernel<float, uint16_t, W, V><<<grid, T::kBlock, 0, st>>>(a);
        else
            block_norm_fwd_kernel<uint16_t, uint16_t, W, V><<<grid, T::kBlock, 0, st>>>(a);
    });
    return launch_status();
}

vmoe_status block_norm_bwd_launch(const vmoe_norm_shape& s, const void* dx_out, const void* dh,
                                  const void* x_out, const void* y, const void* post_w,
                                  const void* post_b, const void* gate, const float* row_scale,
                                  const void* pre_w, const float* post_stats,
                                  const float* pre_stats, void* dx, void* dy, float* dpost_w,
                                  float* dpost_b, float* dgate, float* dpre_w, float* dpre_b,
                                  void* ws, hipStream_t st) {
    const BwdGrid b = bwd_grid(s);
    int slots = 0;
    const int slot_w = dpre_w ? slots++ : -1, slot_b = dpre_b ? slots++ : -1;
    const int slot_s = dpost_w || dgate ? slots++ : -1;
    const int slot_t = dpost_b || (dgate && post_b) ? slots++ : -1;
    const BwdArgs a = {dx_out, dh, x_out, y, post_w, gate, row_scale, pre_w, post_stats, pre_stats,
                       dx, dy, static_cast<float*>(ws), slot_w, slot_b, slot_s, slot_t, slots,
                       s.n_tokens, s.n_tokens / s.n_groups, s.n_groups, s.d_model, s.pre_norm,
                       s.post_norm, b.blocks_per_group, b.rows_per_block, s.residual_scale,
                       s.branch_scale};
    if (b.blocks > 0) {
        const unsigned grid = static_cast<unsigned>(b.blocks);
        by_width(s.d_model, [&](auto wt, auto vt) {
            constexpr int W = decltype(wt)::value, V = decltype(vt)::value;
            constexpr int B = Team<W, V>::kBlock;
            const bool h32 = s.dh_dtype == VMOE_F32;
            if (s.dtype == VMOE_F32)
                block_norm_bwd_kernel<float, float, float, W, V><<<grid, B, 0, st>>>(a);
            else if (s.stream_dtype == VMOE_F32 && h32)
                block_norm_bwd_kernel<float, uint16_t, float, W, V><<<grid, B, 0, st>>>(a);
            else if (s.stream_dtype == VMOE_F32)
                block_norm_bwd_kernel<float, uint16_t, uint16_t, W, V><<<grid, B, 0, st>>>(a);
            else if (h32)
                block_norm_bwd_kernel<uint16_t, uint16_t, float, W, V><<<grid, B, 0, st>>>(a);
            else
                block_norm_bwd_kernel<uint16_t, uint16_t, uint16_t, W, V><<<grid, B, 0, st>>>(a);
        });
    }
    if (slots > 0) {
        const ReduceArgs r = {static_cast<float*>(ws), post_w, post_b, gate, dpre_w, dpre_b,
                              dpost_w, dpost_b, dgate, slot_w, slot_b, slot_s, slot_t, slots,
                              s.n_groups, s.d_model, b.blocks_per_group,
                              static_cast<int>(b.blocks)};
        const dim3 grid(cdiv(s.d_model, kReduceCols), slot_s >= 0 || slot_t >= 0 ? 2 : 1);
        const dim3 block(kReduceCols, kSlices);
        if (s.dtype == VMOE_F32) block_norm_reduce_kernel<float><<<grid, block, 0, st>>>(r);
        else block_norm_reduce_kernel<uint16_t><<<grid, block, 0, st>>>(r);
    }
    return launch_status();
}

}  // namespace vmoe

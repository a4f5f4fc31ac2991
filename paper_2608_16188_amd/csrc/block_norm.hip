// Norm after a block, gate, residual add and norm before the next block in one
// pass over the tokens, and its backward.
//
// A team of waves holds a token's whole row in registers, 8 consecutive columns
// a lane and step, so every tensor is read once and written once whatever the
// norms need: means and deviations are sums over the team (lane moves within a
// wave, LDS across waves). Both directions are streams of rows, bound by HBM:
// 36928 rows of 1024 in bf16 take 53 us forward (297 MB, 5.6 TB/s) and 105 us
// backward (529 MB, 5.1 TB/s); all in f32 119 us and, with the column sums'
// launch, 187 (605 and 908 MB). A copy of 256 MiB runs at 5.4 TB/s, AdamW's update
// at 6.4. The rows' stores stay in the caches for the call that reads them next:
// stores past them make the backward alone 2 to 20 % faster, and it with its
// reader 3 to 5 % slower.
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
constexpr long long kMostThreads = 1LL << 31;  // of a launch, which takes fewer than 2^32

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Eight consecutive elements as they lie in memory. `stream`: of a row that
// this kernel reads once, past what the caches should keep (25216 rows of 768
// forward: 27 us, 32 with plain loads; 36928 of 1024 backward: 109 us, 112).
template <typename T> struct Raw8;
template <> struct Raw8<uint16_t> {
    u32x4 q;
    __device__ __forceinline__ void load(const uint16_t* p) {
        q = *reinterpret_cast<const u32x4*>(p);
    }
    __device__ __forceinline__ void stream(const uint16_t* p) {
        q = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    }
    __device__ __forceinline__ void zero() { q = 0; }
    __device__ __forceinline__ float get(int j) const {
        const uint32_t w = q[j / 2];
        return __uint_as_float((j & 1) ? w & 0xFFFF0000u : w << 16);
    }
};
template <> struct Raw8<float> {
    f32x4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = reinterpret_cast<const f32x4*>(p)[0];
        b = reinterpret_cast<const f32x4*>(p)[1];
    }
    // two accesses meet in every cache line: it has to stay for the second
    __device__ __forceinline__ void stream(const float* p) { load(p); }
    __device__ __forceinline__ void zero() { a = b = 0.0f; }
    __device__ __forceinline__ float get(int j) const { return j < 4 ? a[j] : b[j - 4]; }
};

__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
    *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                         pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    reinterpret_cast<f32x4*>(p)[0] = f32x4{v[0], v[1], v[2], v[3]};
    reinterpret_cast<f32x4*>(p)[1] = f32x4{v[4], v[5], v[6], v[7]};
}

// A row's team: W waves, or L lanes of one; V steps of 8 columns a lane, columns
// (i W L + lane of team) 8.
template <int L, int W, int V>
struct Team {
    static_assert(L == kLanes || W == 1, "part of a wave, or whole waves");
    static constexpr int kL = L, kW = W, kV = V;
    static constexpr int kBlock = W == 1 ? 256 : W * kLanes;
    static constexpr int kRows = kBlock / (W * L);  // rows a block works on at a time
    static constexpr int kCols = W * L * V * 8;
    // whether a row is requested while the one before it is worked on (8197 rows
    // of 4096 backward: 126 us, 131 without): a block of 16 waves has no
    // registers left for it
    static constexpr bool kAhead = W < 16;
    static __device__ __forceinline__ int lane() {
        return W == 1 ? threadIdx.x & (L - 1) : threadIdx.x;
    }
    // of a whole wave: the same in all lanes, and known to be, so that row
    // addresses stay scalar
    static __device__ __forceinline__ int row() {
        if (W > 1) return 0;
        return L == kLanes ? __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes)
                           : threadIdx.x / L;
    }
    static __device__ __forceinline__ int column(int i) { return (i * W * L + lane()) * 8; }
};

template <int CTRL>
__device__ __forceinline__ float add_rotated(float v) {
    const int x = __builtin_bit_cast(int, v);
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(x, x, CTRL, 0xF, 0xF, false));
}

// Sum over L lanes for all of them; lanes of one team are active together.
template <int L>
__device__ __forceinline__ float lanes_total(float v) {
    if constexpr (L == kLanes) return wave_total(v);
    v = add_rotated<0x128>(v);  // rotations within 16 lanes by 8, 4, 2, 1
    v = add_rotated<0x124>(v);
    v = add_rotated<0x122>(v);
    v = add_rotated<0x121>(v);
    if constexpr (L == 32)      // lane ^ 16
        v += __builtin_bit_cast(
            float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), 0x401F));
    return v;
}

// Sums over a team, for every lane. The two halves of `lds` take turns, so one
// barrier a call is enough: a half is written again only after the barrier of
// the call between, which every wave passes after its reads.
template <int L, int W, int K>
__device__ __forceinline__ void team_sum(float (&s)[K], float* lds, int& turn) {
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = lanes_total<L>(s[k]);
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
template <int L, int W, int V>
__device__ __forceinline__ float2 row_stats(const float (&v)[V][8], int kind, int d, float eps,
                                            float inv_d, float* lds, int& turn) {
    using T = Team<L, W, V>;
    float mean = 0.0f, s[1];
    if (kind == VMOE_NORM_LAYER) {
        s[0] = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] += v[i][j];
        team_sum<L, W, 1>(s, lds, turn);
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
    team_sum<L, W, 1>(s, lds, turn);
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

// A row on its way: requested while the row before it is worked on.
template <typename TS, typename TA, int V>
struct FwdRow {
    Raw8<TS> x[V];
    Raw8<TA> y[V], gate[V];
    float scale;  // branch_scale row_scale, 0 where the block is left out
    __device__ __forceinline__ void load(const FwdArgs& a, int t, float row_scale,
                                         const int (&col)[V]) {
        const size_t at = static_cast<size_t>(t) * a.d;
        const TS* xp = static_cast<const TS*>(a.x) + at;
        const TA* yp = static_cast<const TA*>(a.y) + at;
        const TA* gp = static_cast<const TA*>(a.gate) +
                       (a.G == 1 ? 0 : static_cast<size_t>(t / a.Ng) * a.d);
        const bool on = a.y != nullptr && row_scale != 0.0f;
        scale = a.branch * row_scale;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const bool live = col[i] < a.d;
            if (live) x[i].stream(xp + col[i]);
            else x[i].zero();
            if (live && on) y[i].stream(yp + col[i]);
            else y[i].zero();
            if (live && on && a.gate) gate[i].load(gp + col[i]);
            else gate[i].zero();
        }
    }
};

// POST: whether the block's output has a norm.
template <typename TS, typename TA, int L, int W, int V, bool POST>
__global__ __launch_bounds__((Team<L, W, V>::kBlock)) void block_norm_fwd_kernel(FwdArgs a) {
    using T = Team<L, W, V>;
    __shared__ float lds[4 * W];
    int turn = 0;
    int col[V];
#pragma unroll
    for (int i = 0; i < V; ++i) col[i] = T::column(i);
    const float inv_d = 1.0f / static_cast<float>(a.d);
    Raw8<TA> pre_w[V], pre_b[V], post_w[V], post_b[V];
    load_weights<TA, V>(pre_w, a.pre_w, a.d, col);
    load_weights<TA, V>(pre_b, a.pre_b, a.d, col);
    if constexpr (POST) {
        load_weights<TA, V>(post_w, a.post_w, a.d, col);
        load_weights<TA, V>(post_b, a.post_b, a.d, col);
    }
    const int step = gridDim.x * T::kRows;
    int t = blockIdx.x * T::kRows + T::row();
    if (t >= a.N) return;  // whole waves; with W > 1 the grid has no more blocks than rows
    const auto scale_of = [&](int r) { return a.row_scale && r < a.N ? a.row_scale[r] : 1.0f; };
    FwdRow<TS, TA, V> next;
    float rs = scale_of(t), rs_next = scale_of(t + step);
    if (T::kAhead) next.load(a, t, rs, col);
    for (; t < a.N; t += step) {
        if (!T::kAhead) next.load(a, t, rs, col);
        const FwdRow<TS, TA, V> r = next;
        const bool on = rs != 0.0f;
        rs = rs_next;
        if (t + step < a.N) {
            rs_next = scale_of(t + 2 * step);
            if (T::kAhead) next.load(a, t + step, rs, col);
        }
        const size_t at = static_cast<size_t>(t) * a.d;
        float v[V][8];
        if (a.y != nullptr) {
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = r.y[i].get(j);
            if constexpr (POST) {
                float2 st = make_float2(0.0f, 0.0f);
                if (on) {
                    st = row_stats<L, W, V>(v, a.post, a.d, a.eps, inv_d, lds, turn);
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
                    if (on) b = r.scale * (a.gate ? v[i][j] * r.gate[i].get(j) : v[i][j]);
                    v[i][j] = __builtin_fmaf(a.residual, r.x[i].get(j), b);
                }
            TS* xo = static_cast<TS*>(a.x_out) + at;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (col[i] < a.d) store8(xo + col[i], v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = r.x[i].get(j);
        }
        if (a.pre != VMOE_NORM_NONE) {
            if constexpr (POST) {
                // columns past d hold what the norm of y left there: take them out
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (col[i] >= a.d)
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
            }
            const float2 st = row_stats<L, W, V>(v, a.pre, a.d, a.eps, inv_d, lds, turn);
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
    int first_block;                 // of this launch
};

// One sum of a block into its row of partials: a team of several waves writes its
// columns, teams of one wave meet in LDS first.
template <int L, int W, int V>
__device__ __forceinline__ void leave_sum(const float (&acc)[V][8], float* out, int d,
                                          const int (&col)[V], float* lds) {
    using T = Team<L, W, V>;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (W > 1) {
            if (col[i] < d) store8(out + col[i], acc[i]);
        } else {
            store8(lds + T::row() * T::kCols + col[i], acc[i]);
        }
    }
}

template <typename TS, typename TA, typename TH, int V>
struct BwdRow {
    Raw8<TH> dh[V];
    Raw8<TS> x[V], dx[V];
    Raw8<TA> y[V];
    float2 pre, post;
    __device__ __forceinline__ void load(const BwdArgs& a, int t, bool on, const int (&col)[V]) {
        const size_t at = static_cast<size_t>(t) * a.d;
        const bool normed = a.pre != VMOE_NORM_NONE;
        pre = normed ? reinterpret_cast<const float2*>(a.pre_stats)[t] : make_float2(0.0f, 0.0f);
        post = a.post != VMOE_NORM_NONE && on ? reinterpret_cast<const float2*>(a.post_stats)[t]
                                              : make_float2(0.0f, 1.0f);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const bool live = col[i] < a.d;
            if (live && normed) {
                dh[i].stream(static_cast<const TH*>(a.dh) + at + col[i]);
                x[i].stream(static_cast<const TS*>(a.x_out) + at + col[i]);
            } else {
                dh[i].zero();
                x[i].zero();
            }
            if (live && a.dx_out) dx[i].stream(static_cast<const TS*>(a.dx_out) + at + col[i]);
            else dx[i].zero();
            if (live && on) y[i].stream(static_cast<const TA*>(a.y) + at + col[i]);
            else y[i].zero();
        }
    }
};

// POST: whether the block's output has a norm. Without one there is no T to sum
// (no bias) and no sum over the row on y's side.
template <typename TS, typename TA, typename TH, int L, int W, int V, bool POST>
__global__ __launch_bounds__((Team<L, W, V>::kBlock)) void block_norm_bwd_kernel(BwdArgs a) {
    using T = Team<L, W, V>;
    // teams of one wave: their sums at the end, up to four kinds at once
    constexpr int kSums = T::kRows * T::kCols;
    __shared__ __align__(16) float lds[W == 1 ? (POST ? 4 : 3) * kSums : 4 * W];
    int turn = 0;
    int col[V];
#pragma unroll
    for (int i = 0; i < V; ++i) col[i] = T::column(i);
    const float inv_d = 1.0f / static_cast<float>(a.d);
    const int block = a.first_block + blockIdx.x;
    const int g = block / a.blocks_per_group, part = block % a.blocks_per_group;
    const int t0 = g * a.Ng + part * a.rows_per_block;
    const int t1 = min(t0 + a.rows_per_block, (g + 1) * a.Ng);
    Raw8<TA> pre_w[V], post_w[V], gate[V];
    load_weights<TA, V>(pre_w, a.pre_w, a.d, col);
    if constexpr (POST) load_weights<TA, V>(post_w, a.post_w, a.d, col);
    load_weights<TA, V>(gate, a.gate ? static_cast<const TA*>(a.gate) + static_cast<size_t>(g) * a.d
                                     : nullptr, a.d, col);
    float acc_w[V][8], acc_b[V][8], acc_s[V][8], acc_t[V][8];
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc_w[i][j] = acc_b[i][j] = acc_s[i][j] = acc_t[i][j] = 0.0f;

    const auto scale_of = [&](int t) { return a.row_scale && t < t1 ? a.row_scale[t] : 1.0f; };
    int t = t0 + T::row();
    float rs = scale_of(t), rs_next = scale_of(t + T::kRows);
    BwdRow<TS, TA, TH, V> next;
    if (T::kAhead && t < t1) next.load(a, t, a.y != nullptr && rs != 0.0f, col);
    for (; t < t1; t += T::kRows) {
        if (!T::kAhead) next.load(a, t, a.y != nullptr && rs != 0.0f, col);
        const BwdRow<TS, TA, TH, V> r = next;
        const bool on = a.y != nullptr && rs != 0.0f;  // the same for the whole team
        const float scale = a.branch * rs;
        rs = rs_next;
        if (t + T::kRows < t1) {
            rs_next = scale_of(t + 2 * T::kRows);
            if (T::kAhead) next.load(a, t + T::kRows, a.y != nullptr && rs != 0.0f, col);
        }
        const size_t at = static_cast<size_t>(t) * a.d;
        float G[V][8];
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) G[i][j] = r.dx[i].get(j);
        if (a.pre != VMOE_NORM_NONE) {
            const float2 st = r.pre;
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float dh = r.dh[i].get(j), n = (r.x[i].get(j) - st.x) * st.y;
                    const float dn = a.pre_w ? dh * pre_w[i].get(j) : dh;
                    acc_w[i][j] = __builtin_fmaf(dh, n, acc_w[i][j]);
                    acc_b[i][j] += dh;
                    s[0] += dn;
                    s[1] = __builtin_fmaf(dn, n, s[1]);
                }
            team_sum<L, W, 2>(s, lds, turn);
            const float c0 = a.pre == VMOE_NORM_LAYER ? s[0] * inv_d : 0.0f, c1 = s[1] * inv_d;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const bool live = col[i] < a.d;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float dh = r.dh[i].get(j), n = (r.x[i].get(j) - st.x) * st.y;
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
            const float2 st = r.post;
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float ag = scale * G[i][j];
                    const float m = POST ? (r.y[i].get(j) - st.x) * st.y : r.y[i].get(j);
                    acc_s[i][j] = __builtin_fmaf(ag, m, acc_s[i][j]);
                    float dn = a.gate ? ag * gate[i].get(j) : ag;
                    if constexpr (POST) {
                        acc_t[i][j] += ag;
                        if (a.post_w) dn *= post_w[i].get(j);
                        s[0] += dn;
                        s[1] = __builtin_fmaf(dn, m, s[1]);
                    }
                    G[i][j] = dn;
                }
            if constexpr (POST) {
                team_sum<L, W, 2>(s, lds, turn);
                const float c0 = a.post == VMOE_NORM_LAYER ? s[0] * inv_d : 0.0f, c1 = s[1] * inv_d;
#pragma unroll
                for (int i = 0; i < V; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float m = (r.y[i].get(j) - st.x) * st.y;
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
    float* out = a.partial + static_cast<size_t>(block) * a.slots * a.d;
    const auto slot = [&](int k) { return out + static_cast<size_t>(k) * a.d; };
    const auto shared = [&](int k) { return lds + (W == 1 ? k * kSums : 0); };
    if (a.slot_w >= 0) leave_sum<L, W, V>(acc_w, slot(a.slot_w), a.d, col, shared(a.slot_w));
    if (a.slot_b >= 0) leave_sum<L, W, V>(acc_b, slot(a.slot_b), a.d, col, shared(a.slot_b));
    if (a.slot_s >= 0) leave_sum<L, W, V>(acc_s, slot(a.slot_s), a.d, col, shared(a.slot_s));
    if constexpr (POST)
        if (a.slot_t >= 0) leave_sum<L, W, V>(acc_t, slot(a.slot_t), a.d, col, shared(a.slot_t));
    if constexpr (W == 1) {
        __syncthreads();
        for (int k = 0; k < a.slots; ++k)
            for (int c = threadIdx.x * 4; c < a.d; c += T::kBlock * 4) {
                f32x4 s = 0.0f;
#pragma unroll
                for (int r = 0; r < T::kRows; ++r)
                    s += *reinterpret_cast<const f32x4*>(shared(k) + r * T::kCols + c);
                *reinterpret_cast<f32x4*>(slot(k) + c) = s;
            }
    }
}

struct ReduceArgs {
    const float* partial;
    const void *post_w, *post_b, *gate;
    float *dpre_w, *dpre_b, *dpost_w, *dpost_b, *dgate;
    int slot_w, slot_b, slot_s, slot_t, slots;
    int G, d, blocks_per_group, blocks;
    int tiles, jobs;  // column tiles; sums over all rows (the gate's blocks come after)
    int slices;       // that share a group's rows
    bool merged;      // dgate's blocks write dpost_weight and dpost_bias
    int first_job;    // of this launch
};

// Blocks of 32 columns (a cache line of a partial row) x 32 slices of the rows,
// one block a sum and column tile, so that even a narrow model's sums fill some
// of the chip.
constexpr int kReduceCols = 32, kSlices = 32;

// Slices that share a group's partial rows in dgate's blocks.
int group_slices(int rows) { return rows <= 8 ? 1 : rows <= 64 ? 8 : kSlices; }

// Sum over rows first, first + stride, ... below end of a column, each times
// its group's gate where there is one; eight rows in flight, added in order.
template <typename TA>
__device__ __forceinline__ float column_sum(const float* p, size_t row, int first, int end,
                                            int stride, const TA* gate, int d, int per_group) {
    float s = 0.0f;
    for (int r = first; r < end; r += 8 * stride) {
        float v[8], w[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int q = r + u * stride;
            v[u] = q < end ? p[q * row] : 0.0f;
            w[u] = gate && q < end
                       ? Elem<TA>::load(gate, static_cast<size_t>(q / per_group) * d) : 1.0f;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) s = __builtin_fmaf(w[u], v[u], s);
    }
    return s;
}

// Adds `slices` neighbouring slices of each column in order, for the threads of
// the first of them.
__device__ __forceinline__ float over_slices(float v, int slices, float (*lds)[kReduceCols]) {
    const int c = threadIdx.x % kReduceCols, q = threadIdx.x / kReduceCols;
    __syncthreads();
    lds[q][c] = v;
    __syncthreads();
    float s = 0.0f;
    if (q % slices == 0)
        for (int k = 0; k < slices; ++k) s += lds[q + k][c];
    return s;
}

// Jobs: dpre_weight, dpre_bias, dpost_weight, dpost_bias (those asked for; the
// last two weigh each partial row with its group's gate), then dgate, a block
// as many groups and a column tile as its slices serve. The sums of an only
// group give dpost_weight and dpost_bias too, without jobs of their own (and
// with their bits: gate times the same sum).
template <typename TA>
__global__ __launch_bounds__(kReduceCols* kSlices) void block_norm_reduce_kernel(ReduceArgs a) {
    __shared__ float lds[kSlices][kReduceCols];
    const int job = a.first_job + blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles;
    const int c = tile * kReduceCols + threadIdx.x % kReduceCols, q = threadIdx.x / kReduceCols;
    const bool live = c < a.d;
    const int cc = live ? c : 0;
    const size_t row = static_cast<size_t>(a.slots) * a.d;
    const auto column = [&](int slot) { return a.partial + static_cast<size_t>(slot) * a.d + cc; };
    const TA* gate = a.gate ? static_cast<const TA*>(a.gate) + cc : nullptr;
    if (job < a.jobs) {
        // the job-th of the sums that are asked for
        float* const outs[4] = {a.dpre_w, a.dpre_b, a.merged ? nullptr : a.dpost_w,
                                a.merged ? nullptr : a.dpost_b};
        const int slots[4] = {a.slot_w, a.slot_b, a.slot_s, a.slot_t};
        int k = 0;
        for (int left = job; k < 4; ++k)
            if (outs[k] && left-- == 0) break;
        const bool weighted = k >= 2 && gate != nullptr;
        float s = over_slices(column_sum<TA>(column(slots[k]), row, q, a.blocks, kSlices,
                                             weighted && a.G > 1 ? gate : nullptr, a.d,
                                             a.blocks_per_group), kSlices, lds);
        if (weighted && a.G == 1) s *= Elem<TA>::load(gate, 0);
        if (q == 0 && live) outs[k][c] = s;
        return;
    }
    const float w = a.post_w ? Elem<TA>::load(static_cast<const TA*>(a.post_w), cc) : 1.0f;
    const float b = a.post_b ? Elem<TA>::load(static_cast<const TA*>(a.post_b), cc) : 0.0f;
    const int g = (job - a.jobs) * (kSlices / a.slices) + q / a.slices, slice = q % a.slices;
    const bool on = g < a.G && a.blocks > 0;
    const int first = g * a.blocks_per_group, end = on ? first + a.blocks_per_group : first;
    float S = column_sum<TA>(column(a.slot_s), row, first + slice, end, a.slices, nullptr, 0, 1);
    float T = 0.0f;
    if (a.slot_t >= 0)
        T = column_sum<TA>(column(a.slot_t), row, first + slice, end, a.slices, nullptr, 0, 1);
    if (a.slices > 1) {
        S = over_slices(S, a.slices, lds);
        T = over_slices(T, a.slices, lds);
    }
    if (!live || slice != 0 || g >= a.G) return;
    a.dgate[static_cast<size_t>(g) * a.d + c] = __builtin_fmaf(w, S, b * T);
    if (a.merged) {
        const float gc = gate ? Elem<TA>::load(gate, 0) : 1.0f;
        if (a.dpost_w) a.dpost_w[c] = gc * S;
        if (a.dpost_b) a.dpost_b[c] = gc * T;
    }
}

// Lanes or waves a row and steps a lane by width: as few lanes as hold it up to
// 512 columns (39603 rows of 72 take 16 us backward, 29 with a wave a row), one
// wave up to 1024 (no barrier in a row: 25216 rows of 768 take 61 us backward, 67
// with two waves a row), more waves beyond, so that the backward's sums and two
// rows stay in registers (8197 rows of 4096: 74 us forward with eight waves, 77
// with four; 4000 of 8192: 107 us backward with eight, 111 with sixteen).
template <typename F>
void by_width(int d, F f) {
    if (d <= 128) f(Team<16, 1, 1>{});
    else if (d <= 256) f(Team<32, 1, 1>{});
    else if (d <= 512) f(Team<64, 1, 1>{});
    else if (d <= 1024) f(Team<64, 1, 2>{});
    else if (d <= 2048) f(Team<64, 4, 1>{});
    else if (d <= 4096) f(Team<64, 8, 1>{});
    else if (d <= 8192) f(Team<64, 8, 2>{});
    else f(Team<64, 16, 2>{});
}

template <typename F>
void by_flag(bool on, F f) {
    if (on) f(std::true_type{});
    else f(std::false_type{});
}

unsigned at_most(long long n, long long most) {
    return static_cast<unsigned>(n < most ? n : most);
}

struct BwdGrid {
    int blocks_per_group, rows_per_block;
    long long blocks;
};

// As many blocks as are resident (two of four waves on a CU, one of more), no
// block across two groups, a row or more for every wave of one. More blocks
// would only leave more partial rows. Groups of a few rows take a block each all the
// same, with idle waves and four partial rows a group (36864 x 1024: 111 us with 1024
// groups, 170 with 9216; 36928 with a group a row 523).
BwdGrid bwd_grid(const vmoe_norm_shape& s) {
    const int Ng = s.n_tokens / s.n_groups;
    if (Ng == 0) return {1, 1, 0};
    int least = 1;
    by_width(s.d_model, [&](auto team) { least = decltype(team)::kRows; });
    int per_group = (s.d_model <= 2048 ? 512 : 256) / s.n_groups;
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
    by_width(s.d_model, [&](auto team) {
        using T = decltype(team);
        constexpr int L = T::kL, W = T::kW, V = T::kV;
        // As many waves as stay resident, each on several rows; four times as many
        // where each still has two, since fresh waves keep more loads on their
        // way (36928 rows of 1024: 53 against 56 us, with a post-norm 56 against
        // 63; 25216 of 768: 27.3 against 26.8, 6304 of 768: 10.1 against 9.4).
        const unsigned rows = cdiv(s.n_tokens, T::kRows);
        const long long waves = static_cast<long long>(s.n_tokens) * W;
        const unsigned most = (L == kLanes && waves >= 32768 ? 16384 : 4096) * kLanes / T::kBlock;
        const unsigned grid = rows < most ? rows : most;
        by_flag(s.post_norm != VMOE_NORM_NONE, [&](auto post) {
            constexpr bool P = decltype(post)::value;
            if (s.dtype == VMOE_F32)
                block_norm_fwd_kernel<float, float, L, W, V, P><<<grid, T::kBlock, 0, st>>>(a);
            else if (s.stream_dtype == VMOE_F32)
                block_norm_fwd_kernel<float, uint16_t, L, W, V, P><<<grid, T::kBlock, 0, st>>>(a);
            else
                block_norm_fwd_kernel<uint16_t, uint16_t, L, W, V, P><<<grid, T::kBlock, 0, st>>>(a);
        });
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
    BwdArgs a = {dx_out, dh, x_out, y, post_w, gate, row_scale, pre_w, post_stats, pre_stats,
                 dx, dy, static_cast<float*>(ws), slot_w, slot_b, slot_s, slot_t, slots,
                 s.n_tokens, s.n_tokens / s.n_groups, s.n_groups, s.d_model, s.pre_norm,
                 s.post_norm, b.blocks_per_group, b.rows_per_block, s.residual_scale,
                 s.branch_scale, 0};
    by_width(s.d_model, [&](auto team) {
        using T = decltype(team);
        constexpr int L = T::kL, W = T::kW, V = T::kV, B = T::kBlock;
        const bool h32 = s.dh_dtype == VMOE_F32;
        for (long long at = 0; at < b.blocks; at += kMostThreads / B) {
            const unsigned grid = at_most(b.blocks - at, kMostThreads / B);
            a.first_block = static_cast<int>(at);
            by_flag(s.post_norm != VMOE_NORM_NONE, [&](auto post) {
                constexpr bool P = decltype(post)::value;
                using B16 = uint16_t;
                if (s.dtype == VMOE_F32)
                    block_norm_bwd_kernel<float, float, float, L, W, V, P><<<grid, B, 0, st>>>(a);
                else if (s.stream_dtype == VMOE_F32 && h32)
                    block_norm_bwd_kernel<float, B16, float, L, W, V, P><<<grid, B, 0, st>>>(a);
                else if (s.stream_dtype == VMOE_F32)
                    block_norm_bwd_kernel<float, B16, B16, L, W, V, P><<<grid, B, 0, st>>>(a);
                else if (h32)
                    block_norm_bwd_kernel<B16, B16, float, L, W, V, P><<<grid, B, 0, st>>>(a);
                else
                    block_norm_bwd_kernel<B16, B16, B16, L, W, V, P><<<grid, B, 0, st>>>(a);
            });
        }
    });
    if (slots > 0) {
        const int tiles = static_cast<int>(cdiv(s.d_model, kReduceCols));
        const bool merged = dgate && s.n_groups == 1;
        const int jobs = (dpre_w != nullptr) + (dpre_b != nullptr) +
                         (merged ? 0 : (dpost_w != nullptr) + (dpost_b != nullptr));
        const int slices = s.n_groups == 1 ? kSlices : group_slices(b.blocks_per_group);
        const int gates = dgate ? static_cast<int>(cdiv(s.n_groups, kSlices / slices)) : 0;
        ReduceArgs r = {static_cast<float*>(ws), post_w, post_b, gate, dpre_w, dpre_b,
                        dpost_w, dpost_b, dgate, slot_w, slot_b, slot_s, slot_t, slots,
                        s.n_groups, s.d_model, b.blocks_per_group,
                        static_cast<int>(b.blocks), tiles, jobs, slices, merged, 0};
        constexpr int B = kReduceCols * kSlices;
        const int most = static_cast<int>(kMostThreads / B) / tiles, all = jobs + gates;
        for (; r.first_job < all; r.first_job += most) {
            const unsigned grid = at_most(all - r.first_job, most) * tiles;
            if (s.dtype == VMOE_F32)
                block_norm_reduce_kernel<float><<<grid, B, 0, st>>>(r);
            else
                block_norm_reduce_kernel<uint16_t><<<grid, B, 0, st>>>(r);
        }
    }
    return launch_status();
}

}  // namespace vmoe

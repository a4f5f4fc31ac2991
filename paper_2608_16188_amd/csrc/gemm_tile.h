// The matrix-core tile shared by the grouped products of the expert MLP and the
// products with a head's weight (gfx950, bf16): operand stages in LDS, fragments,
// and the phased main loop. What becomes of the accumulators is the including file's.
#pragma once

#include <type_traits>

#include "common.h"

namespace vmoe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

enum Epi { EPI_FWD1 = 0, EPI_BIAS = 1, EPI_GELU_GRAD = 2, EPI_STORE = 3, EPI_F32 = 4 };

// Operand: element (mn, k) of expert e is
//   k-major : base[e*estride + mn*ld + k]
//   mn-major: base[e*estride + k*ld + mn]
struct Operand {
    const void* base;
    long long estride;
    int ld;
};

struct GemmArgs {
    Operand a, b;
    int M, N, K;            // static sizes; M or K is replaced by n_e (see var_k)
    int var_k;              // 0: M = n_e, 1: K = n_e
    const int32_t* counts;  // [G, E]
    int G, E;
    void* out;              // primary output (EPI_FWD1: gelu(H))
    void* out2;             // EPI_FWD1: gelu'(H)
    long long out_estride;
    int ldo;
    const void* bias;       // EPI_FWD1 / EPI_BIAS
    long long bias_estride;
    const void* aux;        // EPI_GELU_GRAD: saved gelu'(H)
    float* bsum;            // EPI_F32: row sums of A per expert, or null
    // Gathered operand (kernels built with GATHER != 0): the operand's rows
    // are token rows of x, row r of expert e being x[tok[e * tok_estride + r]];
    // its base is x itself (estride 0) and gather_bytes the size of x.
    const int32_t* tok;     // null: this problem's operand is not gathered
    long long tok_estride;
    long long gather_bytes;
};

// ------------------------------------------------------------------ bf16 MFMA

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// The wave's index in its block, as a scalar.
__device__ __forceinline__ int wave_id() {
    return __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
}

// Operand stages of KB k values (32 or 64) in LDS, filled by buffer_load ... lds:
// lane L of a wave instruction fills bytes [16 L, 16 L + 16) of a 1 KB block, so
// rows are unpadded and 16-byte chunks are XOR-swizzled instead (k-major: chunk ^
// ((row / P) mod Q) with P rows per 256 bytes and Q chunks per row; mn-major: chunk
// ^ s (k mod 4) with s = 4, or 2 when a row's chunk count is a multiple of 8 but
// not 16, so the XOR stays inside the row), which keeps fragment and transpose
// reads free of bank conflicts.

// XOR applied to the 16-byte chunk index of k-row k of an mn-major DMA stage.
template <int ROWS>
__device__ __forceinline__ int mn_swizzle(int k) {
    static_assert((ROWS / 8) % 8 == 0, "mn-major rows must hold a multiple of 8 chunks");
    constexpr int SHIFT = (ROWS / 8) % 16 == 0 ? 2 : 1;
    return (k & 3) << SHIFT;
}

// Element offset (in bf16) of (mn, k) inside one operand stage.
template <int ROWS, bool KMAJOR, int KB>
__device__ __forceinline__ int lds_off(int mn, int k) {
    if constexpr (KMAJOR) {
        constexpr int Q = KB / 8, P = 16 / Q;  // chunks per row, rows per 256 bytes
        return mn * KB + (((k >> 3) ^ ((mn / P) % Q)) << 3) + (k & 7);
    } else {
        return k * ROWS + (((mn >> 3) ^ mn_swizzle<ROWS>(k)) << 3) + (mn & 7);
    }
}

// Byte offset in HBM of the 16-byte vector holding (mn, k..k+7) [k-major] or
// (k, mn..mn+7) [mn-major], or kOutOfRange when it lies outside the operand.
template <bool KMAJOR>
__device__ __forceinline__ uint32_t vec_off(int ld, int mn, int mn_lim, int k, int k_lim) {
    const bool ok = (mn < mn_lim) && (k < k_lim);
    const int e = KMAJOR ? mn * ld + k : k * ld + mn;
    return ok ? static_cast<uint32_t>(e) * 2u : kOutOfRange;
}

// An operand stage is ROWS * KB / 512 blocks of 1 KB; wave w
// issues blocks [w * PER, (w + 1) * PER). Lane L of a block holds physical
// bytes [16 L, 16 L + 16), whose logical (swizzled) position decides what it
// fetches.
template <int ROWS, bool KMAJOR, int KB, int NT>
struct DmaStage {
    static constexpr int BLOCKS = ROWS * KB * 2 / 1024;
    static constexpr int PER = BLOCKS / (NT / 64);  // wave instructions per stage
    static_assert(PER >= 1 && PER * (NT / 64) == BLOCKS, "1 KB blocks must split evenly over waves");
    static __device__ __forceinline__ void issue(__amdgpu_buffer_rsrc_t rs, int ld, int mn0,
                                                 int mn_lim, int k0, int k_lim, uint16_t* s) {
        const int lane = threadIdx.x & 63, wave = wave_id();
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            const int blk = wave * PER + q;
            const int byte = blk * 1024 + 16 * lane;
            uint32_t off;
            if (KMAJOR) {
                constexpr int RB = KB * 2, Q = KB / 8, P = 16 / Q;
                const int r = byte / RB;
                const int c = ((byte % RB) >> 4) ^ ((r / P) % Q);
                off = vec_off<true>(ld, mn0 + r, mn_lim, k0 + 8 * c, k_lim);
            } else {
                constexpr int RB = ROWS * 2;  // bytes per k row
                const int r = byte / RB;
                const int c = ((byte % RB) >> 4) ^ mn_swizzle<ROWS>(r);
                off = vec_off<false>(ld, mn0 + 8 * c, mn_lim, k0 + r, k_lim);
            }
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rs, (__attribute__((address_space(3))) void*)(s + blk * 512), 16, off, 0, 0, 0);
        }
    }
    // Stages that lie inside K: the lane's byte offset of wave instruction q at
    // k = 0 (kOutOfRange outside the operand) holds for every stage, whose k
    // goes into the scalar offset, so a stage costs its PER instructions and
    // no per-lane arithmetic.
    static __device__ __forceinline__ void lane_offs(int ld, int mn0, int mn_lim,
                                                     uint32_t (&off)[PER]) {
        const int lane = threadIdx.x & 63, wave = wave_id();
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            const int byte = (wave * PER + q) * 1024 + 16 * lane;
            if (KMAJOR) {
                constexpr int RB = KB * 2, Q = KB / 8, P = 16 / Q;
                const int r = byte / RB;
                const int c = ((byte % RB) >> 4) ^ ((r / P) % Q);
                off[q] = vec_off<true>(ld, mn0 + r, mn_lim, 8 * c, KB);
            } else {
                constexpr int RB = ROWS * 2;
                const int r = byte / RB;
                const int c = ((byte % RB) >> 4) ^ mn_swizzle<ROWS>(r);
                off[q] = vec_off<false>(ld, mn0 + 8 * c, mn_lim, r, KB);
            }
        }
    }
    // (k-major, gathered rows: rowoff as in issue_rows)
    static __device__ __forceinline__ void lane_offs_rows(const int (&rowoff)[PER],
                                                          uint32_t (&off)[PER]) {
        static_assert(KMAJOR, "row gather: k-major operand");
        const int lane = threadIdx.x & 63, wave = wave_id();
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            const int byte = (wave * PER + q) * 1024 + 16 * lane;
            constexpr int RB = KB * 2, Q = KB / 8, P = 16 / Q;
            const int c = ((byte % RB) >> 4) ^ ((byte / RB / P) % Q);
            off[q] = rowoff[q] >= 0 ? static_cast<uint32_t>(rowoff[q] + 8 * c) * 2u : kOutOfRange;
        }
    }
    static __device__ __forceinline__ void issue_inside(__amdgpu_buffer_rsrc_t rs,
                                                        const uint32_t (&off)[PER],
                                                        uint32_t k_bytes, uint16_t* s) {
        const int wave = wave_id();
#pragma unroll
        for (int q = 0; q < PER; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rs, (__attribute__((address_space(3))) void*)(s + (wave * PER + q) * 512), 16,
                off[q], k_bytes, 0, 0);
    }
    // Gathered operands (rows of x): the stage row lane L fetches in wave
    // instruction q (k-major: an mn row of the tile; mn-major: a k row).
    static __device__ __forceinline__ int lane_row(int q) {
        const int lane = threadIdx.x & 63, wave = wave_id();
        const int byte = (wave * PER + q) * 1024 + 16 * lane;
        return byte / (KMAJOR ? KB * 2 : ROWS * 2);
    }
    // k-major, gathered rows: rowoff[q] = element offset in x of the start of
    // the row lane_row(q) stands for (-1 past the rows).
    static __device__ __forceinline__ void issue_rows(__amdgpu_buffer_rsrc_t rs,
                                                      const int (&rowoff)[PER], int k0,
                                                      int k_lim, uint16_t* s) {
        static_assert(KMAJOR, "row gather: k-major operand");
        const int lane = threadIdx.x & 63, wave = wave_id();
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            const int blk = wave * PER + q;
            const int byte = blk * 1024 + 16 * lane;
            constexpr int RB = KB * 2, Q = KB / 8, P = 16 / Q;
            const int r = byte / RB;
            const int c = ((byte % RB) >> 4) ^ ((r / P) % Q);
            const int kk = k0 + 8 * c;
            const uint32_t off = (rowoff[q] >= 0 && kk < k_lim)
                                     ? static_cast<uint32_t>(rowoff[q] + kk) * 2u
                                     : kOutOfRange;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rs, (__attribute__((address_space(3))) void*)(s + blk * 512), 16, off, 0, 0, 0);
        }
    }
    // mn-major, gathered k rows: rowoff[q] = byte offset in x of the k row
    // lane_row(q) stands for in this stage, col[q] = byte offset of the lane's
    // 8 columns in it (krow_cols); either is kGatherSentinel outside the
    // operand, which puts the sum past the end of x.
    static __device__ __forceinline__ void krow_cols(int mn0, int mn_lim, uint32_t (&col)[PER]) {
        static_assert(!KMAJOR, "k-row gather: mn-major operand");
        const int lane = threadIdx.x & 63, wave = wave_id();
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            const int byte = (wave * PER + q) * 1024 + 16 * lane;
            constexpr int RB = ROWS * 2;
            const int r = byte / RB;
            const int mn = mn0 + 8 * (((byte % RB) >> 4) ^ mn_swizzle<ROWS>(r));
            col[q] = mn < mn_lim ? static_cast<uint32_t>(mn) * 2u : kGatherSentinel;
        }
    }
    static __device__ __forceinline__ void issue_krows(__amdgpu_buffer_rsrc_t rs,
                                                       const uint32_t (&rowoff)[PER],
                                                       const uint32_t (&col)[PER], uint16_t* s) {
        const int wave = wave_id();
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            const int blk = wave * PER + q;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rs, (__attribute__((address_space(3))) void*)(s + blk * 512), 16,
                rowoff[q] + col[q], 0, 0, 0);
        }
    }
};

// s_waitcnt immediate for vmcnt(n) and lgkmcnt(0) (expcnt left alone).
template <int N>
struct VmWait {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    static constexpr int imm = (N & 15) | ((N >> 4) << 14) | (7 << 4);
};

// Workgroup barrier for the operand stages. __syncthreads() fences all memory at
// workgroup scope, which waits for every LDS DMA in flight (vmcnt(0)) and
// would cap the prefetch at one stage, so the callers see to two things
// themselves: the DMA of what is read next has landed (their s_waitcnt on vmcnt),
// and this wave's reads of what is refilled next are done. The ring of whole
// stages waits for the latter too (lgkmcnt(0) in VmWait). phase_tile does not: it
// refills a panel, or a stage's A, one phase after the phase whose products
// consumed the fragments read from it, and consuming them waited for those reads.
// The signal fences keep the compiler from moving memory accesses across it.
__device__ __forceinline__ void ring_barrier() {
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

// A barrier that waits for this wave's LDS accesses only: its stores stay in
// flight across it.
__device__ __forceinline__ void lds_barrier() {
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

// ds_read_b64_tr_b16: within each 16-lane group, lane j reads 4 bf16 at its
// address and lane i receives element i % 4 of lanes i/4, i/4+4, i/4+8, i/4+12.
// With lane j pointing at row j/4, column 4*(j%4) of a 4 x 16 block, lane i
// gets column i: four consecutive k values of one mn index.
__device__ __forceinline__ s16x4 lds_read_tr(const uint16_t* p) {
    typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p));
}

// Operand fragment of v_mfma_f32_32x32x16_bf16 for 32 mn values (lane & 31)
// x 8 k values (k = 16 * kstep + 8 * (lane >> 5) + 0..7).
template <int ROWS, bool KMAJOR, int KB>
__device__ __forceinline__ bf16x8 read_frag(const uint16_t* s, int blk, int kstep, int lane) {
    if (KMAJOR) {
        const int mn = blk * 32 + (lane & 31), k = kstep * 16 + (lane >> 5) * 8;
        return *reinterpret_cast<const bf16x8*>(s + lds_off<ROWS, true, KB>(mn, k));
    } else {
        // 16-lane group g covers mn [16 (g & 1), +16) and k [8 (g >> 1), +8)
        const int g = lane >> 4, j = lane & 15;
        const int k = kstep * 16 + 8 * (g >> 1) + (j >> 2);
        const int mn = blk * 32 + 16 * (g & 1) + 4 * (j & 3);
        const s16x4 lo = lds_read_tr(s + lds_off<ROWS, false, KB>(mn, k));
        const s16x4 hi = lds_read_tr(s + lds_off<ROWS, false, KB>(mn, k + 4));
        const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(bf16x8, v);
    }
}

// A 256-row tile whose 64-deep stages are worked through in PB phases, one per
// 64-column panel of B (phase_tile below): eight waves as 4 x 2, a wave's 64
// rows against 32 columns of the phase's panel.
template <int PB_>
struct PhaseTile {
    static constexpr int PB = PB_;
    static constexpr int BM = 256, BN = 64 * PB, WGN = 2, KB = 64, NS = 2;
    static constexpr bool PHASED = true;
    static constexpr int NW = 8, NT = 512, WAVES_PER_EU = 2;
    static constexpr int WM = 64, FM = 2;
    // LDS: two A stages, two stages of PB panels of B (panels 0, 1 and the rest
    // in arrays of their own, so that the compiler can tell a read of one from
    // the loads in flight into another), the epilogue's 4 KB a wave
    static constexpr int A_EL = BM * KB, P_EL = 64 * KB, S_EL = NW * 2048;
    static constexpr int BL_EL = 2 * P_EL, BH_EL = (PB - 2) * P_EL;
};

// LDS-typed views of a tile's arrays (a pointer selected
// among the arrays at run time would otherwise become a flat pointer, whose
// accesses wait on the vector-memory counter too)
typedef __attribute__((address_space(3))) uint16_t lds_u16;
typedef __attribute__((address_space(3))) v4i32 lds_v4;
typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
typedef __attribute__((address_space(3))) float lds_f32;

// A phased tile's LDS arrays, and their eight 16 KB pieces (a select over values:
// a closure or array of the arrays' addresses would sit in scratch memory)
struct LdsArrays {
    uint16_t *b0, *b1, *b2, *b3, *b4, *b5, *b6;
};
__device__ __forceinline__ lds_u16* pick_lds(int i, const LdsArrays& a) {
    uint16_t* b = a.b0;
    if (i == 1) b = a.b0 + 8192;
    if (i == 2) b = a.b1;
    if (i == 3) b = a.b1 + 8192;
    if (i == 4) b = a.b6;
    if (i == 5) b = a.b6 + 8192;
    if (i == 6) b = a.b2;
    if (i == 7) b = a.b4;
    return (lds_u16*)(b);
}

// One tile of a PhaseTile<PB>: wave w = (wm, wn) accumulates rows 64 wm .. + 63
// and, of every 64-column panel b, columns 32 wn .. + 31 (acc[i][b]: 32-row
// block i). A stage is 64 deep; its phase b multiplies the wave's A fragments
// (read once per stage) by panel b and meanwhile reads the next panel's
// fragments, in the last phase also the next stage's A fragments, each right
// after the last product that uses the old one.
//
// Every phase opens with a barrier, and a panel's LDS slot is refilled one
// phase after its fragments were used, so the loads of a stage go out a few
// at a time and early: with PB = 4, six phases (1.5 stages) before they
// are read, where a ring of two whole stages issued all eight of a wave's
// loads in one burst behind the barrier, ahead of the products, and needed
// them back within the stage. 4 x 2 waves and 64-column panels keep every
// row segment a whole 128-byte line in either layout (a ring of 32-deep
// stages fetches half lines and measured 10-20% slower). Measured against
// that ring, whose tiles were the same size: down-projection 306 -> 260 us,
// gelu'-product 396 -> 347 at 49 000 rows over 32 experts, d = 768, f = 3072
// (256 x 256); down-projection 140 -> 109, dxe beside the weight gradients
// 345 -> 291 on the 17-task batch (256 x 192). Matrix products alone (no
// loads, no LDS reads) take 156 of the 260, the rate the card holds on random
// data; waiting for all but half of the loads in flight costs 6%, so neither
// depth nor latency binds. Per phase a wave issues
//   phase 0: panel PB - 1 of stage kt + 1     phase 1: panel 0, A of stage kt + 2
//   phase b: panel b - 1 of stage kt + 2
// and waits before phase b for what phase b reads, counting what was issued
// after it. Every fragment read in a phase is used by the next phase's products
// (the last phase's A fragments by all of them in the next stage's phase 0), which
// the scheduling barriers keep ahead of the barrier that opens the phase after
// that: there alone may their LDS be refilled, without a wait for LDS reads.
// Only the last stage's read of a stage past K goes unused; nothing is requested
// after it. (A wave without live rows reads no fragments and only requests.)
//
// The accumulators go to finish_tile(tag of T and EPI, p, acc, ...), which the
// including file defines for its own arguments, with the sums of A's rows (where
// row_sum) and the number of the wave's 32-row blocks inside M; the operand arrays
// are free then.
template <int PB>
struct PhaseWaits {
    static constexpr int issued(int b) { return b == 1 ? 5 : 1; }  // wave instructions, phase b
    static constexpr int stage() { return PB + 4; }
    static constexpr int upto(int b) {  // of phases 0 .. b - 1
        int n = 0;
        for (int q = 0; q < b; ++q) n += issued(q);
        return n;
    }
    // Instructions that may be in flight when phase b opens. Phase b < PB - 1
    // reads panel b + 1 of its stage: issued in phase b + 2 of two stages
    // before (first of that phase's instructions), or, panel PB - 1, in phase 0
    // of the stage before. The last phase reads panel 0 and A of the next
    // stage, issued in phase 1 of the stage before.
    static constexpr int flight(int b) {
        if (b == PB - 1) return stage() - upto(2) + upto(b);
        if (b == PB - 2) return stage() - upto(1) + upto(b);
        return (stage() - upto(b + 2) - 1) + stage() + upto(b);
    }
};

template <class T, int EPI>
struct TileKind {
    using Tile = T;
    static constexpr int epi = EPI;
};

template <class T, bool A_KMAJOR, bool B_KMAJOR, int EPI, int GS, class ARGS>
__device__ __forceinline__ void phase_tile(const ARGS& p, __amdgpu_buffer_rsrc_t ra_rs,
                                           __amdgpu_buffer_rsrc_t rb_rs, int e, int M, int N,
                                           int K, int m0, int n0, int tn, uint16_t* a0,
                                           uint16_t* a1, uint16_t* bl0, uint16_t* bh0,
                                           uint16_t* bl1, uint16_t* bh1, uint16_t* stg) {
    constexpr int PB = T::PB, KB = T::KB, FM = T::FM, P_EL = T::P_EL;
    using DA = DmaStage<T::BM, A_KMAJOR, KB, T::NT>;  // four wave instructions a stage
    using DB = DmaStage<64, B_KMAJOR, KB, T::NT>;     // one a panel
    static_assert(DA::PER == 4 && DB::PER == 1, "stage split");
    using W = PhaseWaits<PB>;
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
    const int wm = wave / T::WGN, wn = wave % T::WGN;
    // 32-row blocks of the wave's rows that lie inside M
    const int fm_live = min(FM, max(0, (M - m0 - wm * T::WM + 31) / 32));

    int arow[GS == 1 ? DA::PER : 1];
    uint32_t aoff[DA::PER], boff[PB];
    uint32_t* const tok_s = reinterpret_cast<uint32_t*>(stg);  // k-row gather's row table
    uint32_t bk = 0;
    if constexpr (GS == 1) {
#pragma unroll
        for (int q = 0; q < DA::PER; ++q) {
            const int r = DA::lane_row(q);
            arow[q] = m0 + r < M ? p.tok[e * p.tok_estride + m0 + r] * p.a.ld : -1;
        }
        DA::lane_offs_rows(arow, aoff);
    } else {
        DA::lane_offs(p.a.ld, m0, M, aoff);
    }
    if constexpr (GS == 2) {
        // the expert's k rows as byte offsets of their rows of x, and the
        // sentinel past K up to the last stage that is requested
        const int kfill = ((K + 2 * KB - 1) / (2 * KB) + 1) * 2 * KB;
        for (int i = tid; i < kfill; i += T::NT)
            tok_s[i] = i < K ? static_cast<uint32_t>(p.tok[e * p.tok_estride + i]) *
                                   (2u * static_cast<uint32_t>(p.b.ld))
                             : kGatherSentinel;
        __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < PB; ++b) {
        uint32_t o[1];
        if constexpr (GS == 2) DB::krow_cols(n0 + 64 * b, N, o);
        else DB::lane_offs(p.b.ld, n0 + 64 * b, N, o);
        boff[b] = o[0];
    }
    const uint32_t a_step = (A_KMAJOR ? KB : KB * p.a.ld) * 2;
    const uint32_t b_step = (B_KMAJOR ? KB : KB * p.b.ld) * 2;
    const int nk = (K + KB - 1) / KB;
    const int n_inside = K / KB;  // stages that lie inside K

    // requests of stage kt (inside K, or any: zeros past K)
    auto issue_a = [&](int kt, uint16_t* dst, auto inside) {
        if constexpr (decltype(inside)::value) DA::issue_inside(ra_rs, aoff, kt * a_step, dst);
        else if constexpr (GS == 1) DA::issue_rows(ra_rs, arow, kt * KB, K, dst);
        else DA::issue(ra_rs, p.a.ld, m0, M, kt * KB, K, dst);
    };
    // panel b of stage buffer S
    auto panel = [&](auto parity, int b) {
        constexpr int S = decltype(parity)::value;
        return b < 2 ? (S ? bl1 : bl0) + b * P_EL : (S ? bh1 : bh0) + (b - 2) * P_EL;
    };
    auto issue_b = [&](int kt, int b, auto parity, auto inside) {
        uint32_t o[1] = {boff[b]};
        uint16_t* const dst = panel(parity, b);
        if constexpr (GS == 2) {
            // panels of a stage are requested in order: its rows with panel 0
            if (b == 0) bk = tok_s[kt * KB + DB::lane_row(0)];
            const uint32_t ro[1] = {bk};
            DB::issue_krows(rb_rs, ro, o, dst);
        } else if constexpr (decltype(inside)::value) {
            DB::issue_inside(rb_rs, o, kt * b_step, dst);
        } else {
            DB::issue(rb_rs, p.b.ld, n0 + 64 * b, N, kt * KB, K, dst);
        }
    };
    using YES = std::true_type;
    using NO = std::false_type;

    // The bias of the wave's columns 64 b + 32 wn + 8 q + 4 (lane / 32) + 0..3
    // starts the accumulators.
    constexpr bool BIAS = EPI == EPI_FWD1 || EPI == EPI_BIAS;
    uint2 bias[BIAS ? PB * 4 : 1];
    if constexpr (BIAS) {
#pragma unroll
        for (int b = 0; b < PB; ++b)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = n0 + 64 * b + 32 * wn + 8 * q + 4 * (lane >> 5);
                bias[b * 4 + q] = n < N ? *reinterpret_cast<const uint2*>(
                                              static_cast<const uint16_t*>(p.bias) +
                                              e * p.bias_estride + n)
                                        : make_uint2(0u, 0u);
            }
    }

    // the loop's first two stages, in the order the phases would have issued them
    using P0 = std::integral_constant<int, 0>;
    using P1 = std::integral_constant<int, 1>;
    issue_b(0, 0, P0{}, NO{});
    issue_a(0, a0, NO{});
#pragma unroll
    for (int b = 1; b < PB; ++b) issue_b(0, b, P0{}, NO{});
    issue_b(1, 0, P1{}, NO{});
    issue_a(1, a1, NO{});
#pragma unroll
    for (int b = 1; b < PB - 1; ++b) issue_b(1, b, P1{}, NO{});

    f32x16 acc[FM][PB];
#pragma unroll
    for (int b = 0; b < PB; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float b4[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if constexpr (BIAS) {
                const uint2 bb = bias[b * 4 + q];
                b4[0] = bf16_to_f32(bb.x & 0xFFFFu);
                b4[1] = bf16_to_f32(bb.x >> 16);
                b4[2] = bf16_to_f32(bb.y & 0xFFFFu);
                b4[3] = bf16_to_f32(bb.y >> 16);
            }
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][b][4 * q + r] = b4[r];
        }

    // bias gradients: the first n-tile's waves of column half 0 also sum
    // their A rows (dot products with ones, from the fragments)
    const bool row_sum = EPI == EPI_F32 && p.bsum != nullptr && tn == 0 && wn == 0;
    float rsum[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) rsum[i] = 0.0f;

    // A and panel 0 of stage 0 have landed
    __builtin_amdgcn_s_waitcnt(VmWait<W::flight(PB - 1) + W::issued(PB - 1)>::imm | (15 << 8));
    ring_barrier();

    auto ring = [&](auto live_blocks) {
        constexpr int FL = decltype(live_blocks)::value;
        bf16x8 fa[FM][4], fb[2][4];
        auto read_a = [&](const uint16_t* as, int ks) {
#pragma unroll
            for (int i = 0; i < FL; ++i)
                fa[i][ks] = read_frag<T::BM, A_KMAJOR, KB>(as, wm * FM + i, ks, lane);
        };
        if constexpr (FL > 0) {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                read_a(a0, ks);
                fb[0][ks] = read_frag<64, B_KMAJOR, KB>(bl0, wn, ks, lane);
            }
        }
        // stage kt: A in ac, the next stage's in an; S = kt mod 2
        auto stage = [&](int kt, uint16_t* ac, uint16_t* an, auto parity, auto inside) {
            constexpr int S = decltype(parity)::value;
            using NX = std::integral_constant<int, 1 - S>;
            auto phase = [&](auto which) {
                constexpr int b = decltype(which)::value;
                constexpr int cur = (S * PB + b) & 1;
                __builtin_amdgcn_s_waitcnt(VmWait<W::flight(b)>::imm | (15 << 8));
                ring_barrier();
                const uint16_t* bs = b < PB - 1 ? panel(parity, b + 1) : panel(NX{}, 0);
                auto products = [&](int ks) {
#pragma unroll
                    for (int i = 0; i < FL; ++i)
                        acc[i][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            fb[cur][ks], fa[i][ks], acc[i][b], 0, 0, 0);
                };
                auto next_b = [&](int ks) {
                    if constexpr (FL > 0)
                        fb[cur ^ 1][ks] =
                            read_frag<64, B_KMAJOR, KB>(bs, wn, ks, lane);
                };
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) {
                    products(ks);
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (b == PB - 1) {
                        if constexpr (EPI == EPI_F32) {
                            if (row_sum) {
#pragma unroll
                                for (int i = 0; i < FL; ++i) {
                                    const bf16x8 v = fa[i][ks];
#pragma unroll
                                    for (int c = 0; c < 8; ++c)
                                        rsum[i] += static_cast<float>(v[c]);
                                }
                            }
                        }
                        read_a(an, ks);
                        next_b(ks);
                    } else if (ks < 2) {
                        next_b(2 * ks);
                        next_b(2 * ks + 1);
                    }
                    // this phase's requests
                    if (ks == 0) {
                        if constexpr (b == 0) issue_b(kt + 1, PB - 1, NX{}, inside);
                        else issue_b(kt + 2, b - 1, parity, inside);
                    }
                    if constexpr (b == 1)
                        if (ks == 1) issue_a(kt + 2, ac, inside);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            phase(std::integral_constant<int, 0>{});
            phase(std::integral_constant<int, 1>{});
            if constexpr (PB > 2) phase(std::integral_constant<int, 2>{});
            if constexpr (PB > 3) phase(std::integral_constant<int, 3>{});
        };
        int kt = 0;
        for (; kt + 3 < n_inside; kt += 2) {
            stage(kt, a0, a1, P0{}, YES{});
            stage(kt + 1, a1, a0, P1{}, YES{});
        }
        // (an odd last stage runs alone: with a stage of zeros after it an expert of
        // at most 64 rows paid for two stages of weight gradients, backward at 64
        // rows, E = 64, d = 1008, f = 2016 358 us against 339)
        for (; kt < nk; kt += 2) {
            stage(kt, a0, a1, P0{}, NO{});
            if (kt + 1 < nk) stage(kt + 1, a1, a0, P1{}, NO{});
        }
    };
    if (fm_live > 1) ring(std::integral_constant<int, 2>{});
    else if (fm_live > 0) ring(std::integral_constant<int, 1>{});
    else ring(std::integral_constant<int, 0>{});
    // the requests past K have landed (here, so that no wait stands behind the stores)
    __builtin_amdgcn_s_waitcnt(VmWait<0>::imm | (15 << 8));
    finish_tile(TileKind<T, EPI>{}, p, acc, rsum, row_sum,
                LdsArrays{a0, a1, bl0, bh0, bl1, bh1, stg}, e, M, N, m0, n0, fm_live);
}

}  // namespace
}  // namespace vmoe

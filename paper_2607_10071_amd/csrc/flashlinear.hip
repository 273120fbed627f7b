// The matrix product with bias, activation and residual in its epilogue, and
// its gradients, for AMD MI355X (gfx950).  C ABI: include/block/flashblock.h.
//
// Three products, one kernel.  With an operand's rows over the reduction axis
// ("along") or its columns ("across"),
//
//   forward      out[m,n]  = sum_k x[m,k] W[n,k]     x along,  W along
//   grad_x       gx[m,k]   = sum_n d[m,n] W[n,k]     d along,  W across
//   grad_weight  gw[n,k]   = sum_m d[m,n] x[m,k]     d across, x across
//
// so each is C[i,j] = sum_r A(i,r) B(j,r) with operands in one of two layouts.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block_common.h"

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// ---------------------------------------------------------------------------
// activations
// ---------------------------------------------------------------------------
// On the hardware's exp2 and reciprocal (one unit in the last place each): an
// output of 40000 x 1024 gelus is 41 M of them, and with the library's erff, expf and
// IEEE division its product took 109 us where it takes 75 with these.
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSqrt2OverPi = 0.79788456080286536f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;

__device__ __forceinline__ float sigmoid(float v)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * v));
}

// v, or the nearest of -m and m: factors of terms that are 0 there, so that an
// infinite v does not make them NaN
__device__ __forceinline__ float within(float v, float m)
{
    return __builtin_fminf(__builtin_fmaxf(v, -m), m);
}

// erfc(|v| / sqrt 2) = t P(t) exp(-v^2 / 2) with t = 1 / (1 + 0.43 |v| / sqrt 2): P is
// the polynomial of degree 7 with the least relative error over |v| <= 17
// (1.8e-7), found by weighted least squares in float64.  `e` gets the exponential.
// From erfc of |v| neither tail of gelu cancels.
__device__ __forceinline__ float erfc_half(float v, float &e)
{
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(v), 0.30405591591021541f, 1.0f));
    e = __builtin_amdgcn_exp2f(v * v * (-0.5f * kLog2e));
    float q = 0.070911642f;
    q = __builtin_fmaf(q, t, -0.299038637f);
    q = __builtin_fmaf(q, t, 0.364747453f);
    q = __builtin_fmaf(q, t, -0.068830498f);
    q = __builtin_fmaf(q, t, 0.238214638f);
    q = __builtin_fmaf(q, t, 0.207467761f);
    q = __builtin_fmaf(q, t, 0.243988763f);
    q = __builtin_fmaf(q, t, 0.242538700f);
    return q * t * e;
}

__device__ __forceinline__ float act_value(int act, float v)
{
    switch (act) {
    case FLASHBLOCK_ACT_RELU: return v > 0.0f ? v : (v == v ? 0.0f : v);
    case FLASHBLOCK_ACT_GELU: {
        float e;
        const float h = 0.5f * __builtin_fminf(__builtin_fabsf(v), 20.0f) * erfc_half(v, e);
        return v > 0.0f ? v - h : -h;   // (erfc is 0 at 20 already)
    }
    case FLASHBLOCK_ACT_GELU_TANH:   // (1 + tanh z) / 2 = 1 / (1 + exp(-2 z))
        return v * sigmoid(2.0f * kSqrt2OverPi * v * __builtin_fmaf(0.044715f, v * v, 1.0f));
    case FLASHBLOCK_ACT_SILU: return v * sigmoid(v);
    default: return v;
    }
}

__device__ __forceinline__ float act_slope(int act, float v)
{
    switch (act) {
    case FLASHBLOCK_ACT_RELU: return v > 0.0f ? 1.0f : 0.0f;
    case FLASHBLOCK_ACT_GELU: {
        float e;
        const float h = 0.5f * erfc_half(v, e);
        return __builtin_fmaf(within(v, 20.0f) * kInvSqrt2Pi, e, v > 0.0f ? 1.0f - h : h);
    }
    case FLASHBLOCK_ACT_GELU_TANH: {
        const float p = sigmoid(2.0f * kSqrt2OverPi * v * __builtin_fmaf(0.044715f, v * v, 1.0f));
        const float w = within(v, 20.0f);
        const float dz = 2.0f * kSqrt2OverPi * __builtin_fmaf(0.134145f, w * w, 1.0f);
        return __builtin_fmaf(w * p * (1.0f - p), dz, p);
    }
    case FLASHBLOCK_ACT_SILU: {
        const float p = sigmoid(v);
        return p * __builtin_fmaf(within(v, 100.0f), 1.0f - p, 1.0f);
    }
    default: return 1.0f;
    }
}

// ---------------------------------------------------------------------------
// epilogue: V sums of one row, columns n..n+V-1
// ---------------------------------------------------------------------------
struct Epilogue {
    void *out;
    void *pre;              // null: not wanted
    const void *bias;       // null: none
    const void *residual;   // null: none
    int64_t ldo, ldp, ldr;  // elements
    float scale;
    int act;
    int out_f32;            // out and residual are float32, else the inputs' type
};

template <int DT, int V>
__device__ __forceinline__ void epilogue(const Epilogue &e, int64_t m, int n, int N, float (&v)[V])
{
    const bool whole = n + V <= N;
    const int es = elem_size(DT);
    if (e.bias) {
        if (whole) {
            float b[V];
            load_elems<DT>(static_cast<const char *>(e.bias) + (int64_t)n * es, b);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += b[i];
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (n + i < N) v[i] += load_elem<DT>(e.bias, n + i);
        }
    }
    if (e.pre) {
        char *p = static_cast<char *>(e.pre) + (m * e.ldp + n) * es;
        if (whole) {
            store_elems<DT>(p, v);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (n + i < N) store_elem<DT>(p, i, v[i]);
        }
    }
    switch (e.act) {   // the switch outside the loop: one activation's code per call
    case FLASHBLOCK_ACT_RELU:
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = act_value(FLASHBLOCK_ACT_RELU, v[i]);
        break;
    case FLASHBLOCK_ACT_GELU:
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = act_value(FLASHBLOCK_ACT_GELU, v[i]);
        break;
    case FLASHBLOCK_ACT_GELU_TANH:
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = act_value(FLASHBLOCK_ACT_GELU_TANH, v[i]);
        break;
    case FLASHBLOCK_ACT_SILU:
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = act_value(FLASHBLOCK_ACT_SILU, v[i]);
        break;
    default: break;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] *= e.scale;
    if (e.out_f32) {
        char *p = static_cast<char *>(e.out) + (m * e.ldo + n) * 4;
        const char *r = static_cast<const char *>(e.residual);
        if (r) r += (m * e.ldr + n) * 4;
        if (whole) {
            if (r) {
                float b[V];
                load_elems<FLASHBEV_F32>(r, b);
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] += b[i];
            }
            store_elems<FLASHBEV_F32>(p, v);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (n + i < N)
                    store_elem<FLASHBEV_F32>(p, i, r ? v[i] + load_elem<FLASHBEV_F32>(r, i) : v[i]);
        }
    } else {
        char *p = static_cast<char *>(e.out) + (m * e.ldo + n) * es;
        const char *r = static_cast<const char *>(e.residual);
        if (r) r += (m * e.ldr + n) * es;
        if (whole) {
            if (r) {
                float b[V];
                load_elems<DT>(r, b);
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] += b[i];
            }
            store_elems<DT>(p, v);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (n + i < N) store_elem<DT>(p, i, r ? v[i] + load_elem<DT>(r, i) : v[i]);
        }
    }
}

// ---------------------------------------------------------------------------
// the tiled product
// ---------------------------------------------------------------------------
// A workgroup computes a BM x BN tile of C in 32 x 32 MFMA blocks, FM x FN of
// them for each of its WM x WN wavefronts, over steps of 128 bytes of the
// reduction axis (64 16-bit or 32 float32 elements).  A granule is 16 bytes: eight
// 16-bit elements, one lane's share of a 32x32x16 MFMA, or four float32, one
// lane's share of four 32x32x2 MFMAs (MFMA q takes element q of both operands'
// granules, so the reduction index runs in the same order on both sides).
//
// LDS layout.  Along: row i holds its 8 granules, granule g at place g ^ (i / 2 & 7),
// so that 16 lanes reading the same granule of 16 rows use all 64 banks (rows are
// 32 banks long).  Across: row r of the reduction axis holds the tile's columns.  16-bit
// columns are read transposed (ds_read_b64_tr_b16: 16 lanes take a 4 x 16 block
// and each ends with one column's 4 rows); the 32-byte column blocks of row r
// stand at places XORed with 2 (r & 3), so that the two blocks of 4 rows that half a
// wavefront reads use different banks.  float32 columns are read as they stand.
struct Gemm {
    const char *a, *b;
    int64_t lda, ldb;          // bytes
    int rows, cols;            // of C
    int red;                   // length of the reduction axis
    int padded;                // A's rows end in zeros up to a multiple of 8 elements
    int tiles_m, tiles_n;
    int split;                 // workgroups that share a tile's reduction axis
    int steps;                 // reduction steps for each of them
    float *partial;            // split > 1: [split][rows][pld] float32 sums
    int64_t pld;
    Epilogue e;
};

template <int DT>
__device__ __forceinline__ void mma(f32x16 &c, const u32x4 &a, const u32x4 &b)
{
    if constexpr (DT == FLASHBEV_BF16) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                    __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else if constexpr (DT == FLASHBEV_F16) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                   __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    } else {
        const f32x4 fa = __builtin_bit_cast(f32x4, a), fb = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[q], fb[q], c, 0, 0, 0);
    }
}

// the place of an "along" row's granules (see above)
__device__ __forceinline__ int along_swizzle(int row) { return row >> 1 & 7; }

// One operand's tile of R rows (or columns) of C on its way from memory to LDS.
template <int DT, bool ACROSS, int R, int NT>
struct Tile {
    static constexpr int ES = elem_size(DT);
    static constexpr int E = 16 / ES;
    static constexpr int KT = 128 / ES;        // reduction elements per step
    static constexpr int BYTES = R * 128;
    static constexpr int G = R * 8 / NT;       // granules per thread
    static constexpr int GPR = ACROSS ? R * ES / 16 : 8;   // granules per LDS row
    static constexpr int PAIRS = R / 16;       // 32-byte column blocks (16-bit, across)
    static_assert(R * 8 % NT == 0, "whole granules per thread");

    // the step's granules, `left` reduction elements from it on (rows of C past
    // the last one repeat it: their sums are not stored)
    template <bool EDGE>
    static __device__ __forceinline__ void load(u32x4 (&v)[G], const char *base, int64_t ld, int c0,
                                                int cend, int r0, int rend, int tid)
    {
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int q = tid + i * NT;
            const int row = q / GPR, g = q % GPR;
            if constexpr (!ACROSS) {
                const int c = min(c0 + row, cend - 1);
                const char *p = base + (int64_t)c * ld;
                if constexpr (EDGE)
                    v[i] = load_granule_edge<DT>(p, r0 + g * E, rend);
                else
                    v[i] = load16(p + (int64_t)(r0 + g * E) * ES);
            } else {
                const char *p = base + (int64_t)(r0 + row) * ld;
                if constexpr (EDGE) {
                    if (r0 + row < rend)
                        v[i] = load_granule_edge<DT>(p, c0 + g * E, cend);
                    else
                        v[i] = u32x4{0, 0, 0, 0};
                } else {
                    v[i] = load16(p + (int64_t)(c0 + g * E) * ES);
                }
            }
        }
    }

    static __device__ __forceinline__ int swizzle(int r)
    {
        return PAIRS >= 8 ? (r & 3) << 1 : r & 2;   // (rows of 4 are half the banks long)
    }

    static __device__ __forceinline__ void store(const u32x4 (&v)[G], char *lds, int tid)
    {
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int q = tid + i * NT;
            const int row = q / GPR, g = q % GPR;
            int place = g;
            if constexpr (!ACROSS) place = g ^ along_swizzle(row);
            else if constexpr (ES == 2) place = g ^ (swizzle(row) << 1);
            *reinterpret_cast<u32x4 *>(lds + (row * GPR + place) * 16) = v[i];
        }
    }

    // the lane's granule g of reduction elements for column (row of C) c0 + lane % 32
    static __device__ __forceinline__ u32x4 fragment(const char *lds, int c0, int kk, int lane)
    {
        const int h = lane >> 5;
        if constexpr (!ACROSS) {
            const int row = c0 + (lane & 31), g = 2 * kk + h;
            return *reinterpret_cast<const u32x4 *>(lds + (row * 8 + (g ^ along_swizzle(row))) * 16);
        } else if constexpr (ES == 2) {
            const int j = lane & 15;
            const int pair = (c0 >> 4) + (lane >> 4 & 1);
            const int r = kk * 16 + h * 8 + (j >> 2);
            u32x4 v;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int rr = r + 4 * q;
                const char *p = lds + rr * (R * 2) + ((pair ^ swizzle(rr)) * 32) + (j & 3) * 8;
                const s16x4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4 *)(p));
                const uint64_t w = __builtin_bit_cast(uint64_t, t);
                v[2 * q] = (uint32_t)w;
                v[2 * q + 1] = (uint32_t)(w >> 32);
            }
            return v;
        } else {
            const int r = (2 * kk + h) * 4;
            u32x4 v;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                v[q] = *reinterpret_cast<const uint32_t *>(lds + ((r + q) * R + c0 + (lane & 31)) * 4);
            return v;
        }
    }
};

template <int DT, bool AX, bool BX, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(WM *WN * 64) linear_tiles(Gemm p)
{
    constexpr int NT = WM * WN * 64;
    constexpr int TM = BM / WM, TN = BN / WN;      // a wavefront's part of the tile
    constexpr int FM = TM / 32, FN = TN / 32;
    using TA = Tile<DT, AX, BM, NT>;
    using TB = Tile<DT, BX, BN, NT>;
    constexpr int KT = TA::KT;
    constexpr int STAGE = TA::BYTES + TB::BYTES;
    constexpr int ESTRIDE = TN + 4;                // floats; epilogue rows, 16-byte aligned
    constexpr int EBYTES = WM * WN * 32 * ESTRIDE * 4;
    __shared__ __attribute__((aligned(16))) char lds[2 * STAGE > EBYTES ? 2 * STAGE : EBYTES];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = wave / WN, wn = wave % WN;
    const int tile = block_index() / p.split, part = block_index() % p.split;
    if (tile >= p.tiles_m * p.tiles_n) return;
    const int m0 = tile / p.tiles_n * BM, n0 = tile % p.tiles_n * BN;

    f32x16 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

    const int total = (p.red + KT - 1) / KT;
    const int s0 = part * p.steps, s1 = min(total, s0 + p.steps);
    // tiles that hang over an "across" operand's columns, and the last step of an
    // axis that is no multiple of a step, take the checked loads
    const bool edge = (AX && m0 + BM > p.rows) || (BX && n0 + BN > p.cols);
    u32x4 va[TA::G], vb[TB::G];
    auto fetch = [&](int s) {
        if (edge || (s + 1) * KT > p.red) {
            TA::template load<true>(va, p.a, p.lda, m0, p.rows, s * KT, p.red, tid);
            TB::template load<true>(vb, p.b, p.ldb, n0, p.cols, s * KT, p.red, tid);
        } else {
            TA::template load<false>(va, p.a, p.lda, m0, p.rows, s * KT, p.red, tid);
            TB::template load<false>(vb, p.b, p.ldb, n0, p.cols, s * KT, p.red, tid);
        }
    };
    if (s0 < s1) fetch(s0);
    for (int s = s0; s < s1; ++s) {
        char *la = lds + (s - s0 & 1) * STAGE, *lb = la + TA::BYTES;
        TA::store(va, la, tid);
        TB::store(vb, lb, tid);
        __syncthreads();
        if (s + 1 < s1) fetch(s + 1);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            u32x4 fa[FM], fb[FN];
#pragma unroll
            for (int i = 0; i < FM; ++i) fa[i] = TA::fragment(la, wm * TM + i * 32, kk, lane);
#pragma unroll
            for (int j = 0; j < FN; ++j) fb[j] = TB::fragment(lb, wn * TN + j * 32, kk, lane);
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) mma<DT>(acc[i][j], fa[i], fb[j]);
        }
    }
    __syncthreads();

    // Epilogue: the MFMA leaves a lane with one column's 16 rows; through LDS,
    // 32 rows at a time, each lane gets a row's consecutive columns, so that
    // bias, residual and output move in 16-byte vectors.
    float *stage = reinterpret_cast<float *>(lds) + wave * 32 * ESTRIDE;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                stage[(8 * (e / 4) + 4 * (lane >> 5) + e % 4) * ESTRIDE + j * 32 + (lane & 31)] =
                    acc[i][j][e];
        wave_lds_sync();
        constexpr int V = 16 / elem_size(DT);
        constexpr int LPR = TN / V, RPP = 64 / LPR;    // lanes per row, rows per pass
#pragma unroll
        for (int q = 0; q < 32 / RPP; ++q) {
            const int r = q * RPP + lane / LPR, c = lane % LPR * V;
            const int m = m0 + wm * TM + i * 32 + r, n = n0 + wn * TN + c;
            float v[V];
#pragma unroll
            for (int e = 0; e < V; e += 4) {
                const f32x4 w = *reinterpret_cast<const f32x4 *>(stage + r * ESTRIDE + c + e);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[e + k] = w[k];
            }
            if (m >= p.rows || n >= p.cols) continue;
            if (p.split > 1)
                store_elems<FLASHBEV_F32>(p.partial + ((int64_t)part * p.rows + m) * p.pld + n, v);
            else
                epilogue<DT>(p.e, m, n, p.cols, v);
        }
        wave_lds_sync();
    }
}

// ---------------------------------------------------------------------------
// the streamed product: rows at 16-byte places, widths of whole granules
// ---------------------------------------------------------------------------
// As linear_tiles, with three differences.  Granules go from memory to LDS
// without passing registers (global_load_lds), into a ring of S stages, S - 1 of
// them in flight.  A workgroup takes tile after tile, and the ring runs on over
// the border: the next tile's first steps load while this one's results are
// written.  And the MFMA's operands are swapped, so that a lane ends with one row's
// columns: two half-wavefront swaps of neighbouring groups of four give it 8
// consecutive ones, which need no pass through LDS.
//
// Granules past the reduction axis's end come from 16 bytes of zeros.
__device__ const __attribute__((aligned(16))) uint32_t kZeros[4] = {0, 0, 0, 0};

// 16 bytes of each lane to LDS at `lds` + 16 lane.  Written in assembly, without
// registers to be written: the compiler would wait for every load in flight before
// the next LDS read, whichever stage it reads.  m0, which holds the place in LDS, is an
// operand, so that the compiler knows it (s_nop: the wait between its write and the load).
__device__ __forceinline__ void to_lds(const void *base, uint32_t off, uint32_t lds)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "{m0}"(lds), "v"(off), "s"(base) : "memory");
}

__device__ __forceinline__ void to_lds(const void *p, uint32_t lds)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :: "{m0}"(lds), "v"(p) : "memory");
}

// Until at most N vector memory operations are in flight: s_waitcnt with vmcnt N
// (bits 3..0 and 15..14) and no other limit.  Not in assembly: the compiler has to
// know that its own loads are back, or it waits for them inside the loop.
template <int N>
__device__ __forceinline__ void wait_loads()
{
    static_assert(N < 64, "vmcnt");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70);
    asm volatile("" ::: "memory");
}

// One operand's granules of a tile: where they are read from and what of a step is there.
template <int DT, bool ACROSS, int R, int NT>
struct Stream {
    using T = Tile<DT, ACROSS, R, NT>;
    static constexpr int G = T::G;
    static constexpr int ES = T::ES, E = T::E, KT = T::KT;
    static constexpr int STEP = NT / T::GPR;     // LDS rows between a lane's granules
    static_assert(STEP % (!ACROSS ? 16 : ES == 2 ? 4 : 1) == 0, "a lane's granules share one swizzle");

    // a lane's byte offsets from its tile's first row (along) or column (across)
    static __device__ __forceinline__ void offsets(uint32_t (&off)[G], int64_t ld, int c0, int cend,
                                                   int tid)
    {
        const int row = tid / T::GPR, place = tid % T::GPR;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int r = row + i * STEP;
            if constexpr (!ACROSS) {
                const int g = place ^ along_swizzle(row);
                off[i] = (uint32_t)(min(c0 + r, cend - 1) - c0) * (uint32_t)ld + g * 16;
            } else {
                const int g = ES == 2 ? place ^ (T::swizzle(row) << 1) : place;
                off[i] = (uint32_t)r * (uint32_t)ld + (uint32_t)(min(c0 + g * E, cend - E) - c0) * ES;
            }
        }
    }

    static __device__ __forceinline__ const char *at(const char *p, int64_t ld, int c0, int r0)
    {
        return ACROSS ? p + (int64_t)r0 * ld + (int64_t)c0 * ES : p + (int64_t)c0 * ld + (int64_t)r0 * ES;
    }

    static __device__ __forceinline__ void load(const char *base, const uint32_t (&off)[G], uint32_t lds)
    {
#pragma unroll
        for (int i = 0; i < G; ++i) to_lds(base, off[i], lds + i * NT * 16);
    }

    // a step that holds `left` < KT elements of the reduction axis
    static __device__ __forceinline__ void load_last(const char *base, const uint32_t (&off)[G],
                                                     uint32_t lds, int left, int tid)
    {
        const int row = tid / T::GPR, place = tid % T::GPR;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const bool there = ACROSS ? row + i * STEP < left : (place ^ along_swizzle(row)) * E < left;
            to_lds(there ? base + off[i] : reinterpret_cast<const char *>(kZeros), lds + i * NT * 16);
        }
    }
};

// The MFMA leaves a lane with four groups of four columns of a row in each block
// (group k: columns 8 k + 4 (lane / 32) ..); swapping halves of the wavefront
// between groups 2 q and 2 q + 1 makes them columns 16 q + 8 (lane / 32) .. + 7.
__device__ __forceinline__ void columns_of(const f32x16 &acc, int q, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float x = acc[8 * q + i], y = acc[8 * q + 4 + i];
        const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x),
                                                        __builtin_bit_cast(unsigned, y), false, false);
        const unsigned a = r[0], b = r[1];
        v[i] = __builtin_bit_cast(float, a);
        v[4 + i] = __builtin_bit_cast(float, b);
    }
}

// A wavefront's epilogue, its blocks' first row and column at (m, n).  Loads and
// stores come back in one order, so a load behind a store waits for it (with each
// vector's bias read before its store, these waits were two thirds of a 256-long
// product's time): the bias and the residual of the first row blocks are read first
// (of all, where there are two), each further one before its predecessor's stores.
// The scheduling barriers keep the compiler from working on all vectors at once, which
// spilled.
template <int DT, int ODT, int ACT, bool FULL, bool ENDS, int FM, int FN>
__device__ __forceinline__ void write_tile(const Gemm &p, int m, int n, int lane,
                                           const f32x16 (&acc)[FM][FN])
{
    constexpr int ES = elem_size(DT), OS = elem_size(ODT);
    constexpr int BW = ES / 2, OW = OS / 2;     // 16-byte words of 8 elements
    constexpr int AHEAD = FM <= 2 ? FM : 1;     // row blocks of residual in registers
    const Epilogue &e = p.e;
    const int m0 = m + (lane & 31), n0 = n + 8 * (lane >> 5);
    u32x4 res[AHEAD][FN][2][OW], bias[FN][2][BW];
    auto fetch = [&](int f) {
        const char *r = static_cast<const char *>(e.residual) + ((int64_t)(m0 + f * 32) * e.ldr + n0) * OS;
        if (m0 + f * 32 < p.rows) {
#pragma unroll
            for (int g = 0; g < FN; ++g)
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    if (n0 + g * 32 + q * 16 + 8 <= p.cols) {
#pragma unroll
                        for (int w = 0; w < OW; ++w)
                            res[f % AHEAD][g][q][w] = load16(r + (g * 32 + q * 16) * OS + w * 16);
                    }
        }
    };
    if (FULL && e.residual) {
#pragma unroll
        for (int f = 0; f < AHEAD; ++f) fetch(f);
    }
    if (FULL && e.bias) {
        const char *b = static_cast<const char *>(e.bias) + (int64_t)n0 * ES;
#pragma unroll
        for (int g = 0; g < FN; ++g)
#pragma unroll
            for (int q = 0; q < 2; ++q)
                if (n0 + g * 32 + q * 16 + 8 <= p.cols) {
#pragma unroll
                    for (int w = 0; w < BW; ++w)
                        bias[g][q][w] = load16(b + (g * 32 + q * 16) * ES + w * 16);
                }
    }
#pragma unroll
    for (int f = 0; f < FM; ++f) {
        const int64_t row = m0 + f * 32;
        float v[FN][2][8];
        [[maybe_unused]] float end[8];
        [[maybe_unused]] int at = -1;   // first column of the vector that holds C's last columns, if here
#pragma unroll
        for (int g = 0; g < FN; ++g)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float b[8];
                columns_of(acc[f][g], q, v[g][q]);
                if constexpr (ENDS) {
                    const int n1 = n0 + g * 32 + q * 16;
                    if (n1 < p.cols && n1 + 8 > p.cols) {
                        at = n1;
#pragma unroll
                        for (int i = 0; i < 8; ++i) end[i] = v[g][q][i];
                    }
                }
                if (FULL && e.bias) {
                    elems_of<DT>(bias[g][q], b);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[g][q][i] += b[i];
                }
                if (FULL && e.pre && row < p.rows && n0 + g * 32 + q * 16 + 8 <= p.cols)
                    store_elems<DT>(static_cast<char *>(e.pre) +
                                        (row * e.ldp + n0 + g * 32 + q * 16) * ES, v[g][q]);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[g][q][i] = act_value(ACT, v[g][q][i]) * e.scale;
                if (FULL && e.residual) {
                    elems_of<ODT>(res[f % AHEAD][g][q], b);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[g][q][i] += b[i];
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        if (FULL && f == FM - 1) {
            // For the compiler, which sees a path on which these loads are not waited
            // for and would wait for everything at the loop over the steps.
#pragma unroll
            for (int g = 0; g < FN; ++g)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
#pragma unroll
                    for (int w = 0; w < BW; ++w) asm volatile("" ::"v"(bias[g][q][w]));
#pragma unroll
                    for (int a = 0; a < AHEAD; ++a)
#pragma unroll
                        for (int w = 0; w < OW; ++w) asm volatile("" ::"v"(res[a][g][q][w]));
                }
        }
        if (FULL && e.residual && f + AHEAD < FM) fetch(f + AHEAD);
        char *o = static_cast<char *>(e.out) + (row * e.ldo + n0) * OS;
#pragma unroll
        for (int g = 0; g < FN; ++g)
#pragma unroll
            for (int q = 0; q < 2; ++q)
                if (row < p.rows && n0 + g * 32 + q * 16 + 8 <= p.cols)
                    store_elems<ODT>(o + (g * 32 + q * 16) * OS, v[g][q]);
        if constexpr (ENDS) {
            if (at >= 0 && row < p.rows) epilogue<DT>(e, row, at, p.cols, end);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The float32 sums of a part of the reduction axis.
template <int FM, int FN>
__device__ __forceinline__ void write_part(const Gemm &p, int part, int m, int n, int lane,
                                           const f32x16 (&acc)[FM][FN])
{
    const int m0 = m + (lane & 31), n0 = n + 8 * (lane >> 5);
    float *o = p.partial + ((int64_t)part * p.rows + m0) * p.pld + n0;
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int g = 0; g < FN; ++g)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float v[8];
                columns_of(acc[f][g], q, v);
                if (m0 + f * 32 < p.rows && n0 + g * 32 + q * 16 < p.cols)
                    store_elems<FLASHBEV_F32>(o + f * 32 * p.pld + g * 32 + q * 16, v);
                __builtin_amdgcn_sched_barrier(0);
            }
}

// FULL: the forward, with every activation and type of output; else a gradient
// in the inputs' type.  ENDS: a forward whose rows end inside a vector of 8 (in
// kernels of their own: its code in the others cost the value projection 15 us of 55).
template <int DT, bool FULL, bool ENDS, int FM, int FN>
__device__ __forceinline__ void write_any(const Gemm &p, int part, int m, int n, int lane,
                                          const f32x16 (&acc)[FM][FN])
{
    // nothing of the epilogue is to be computed ahead of the loop over the steps,
    // whose registers are short
    asm volatile("" : "+v"(lane));
    if (p.split > 1) return write_part(p, part, m, n, lane, acc);
    // One activation's code per call.  (The branches in this order: with the types
    // inside the activations' cases the 256 x 256 forward spilled beside the ring's
    // loads, 536 -> 765 us for the large product.)
#define FLASHBLOCK_WRITE(OUT, ACT) \
    return write_tile<DT, OUT, ACT, FULL, ENDS>(p, m, n, lane, acc)
    if constexpr (!FULL) {
        write_tile<DT, DT, FLASHBLOCK_ACT_NONE, FULL, ENDS>(p, m, n, lane, acc);
    } else if (DT == FLASHBEV_F32 || !p.e.out_f32) {
        switch (p.e.act) {
        case FLASHBLOCK_ACT_RELU: FLASHBLOCK_WRITE(DT, FLASHBLOCK_ACT_RELU);
        case FLASHBLOCK_ACT_GELU: FLASHBLOCK_WRITE(DT, FLASHBLOCK_ACT_GELU);
        case FLASHBLOCK_ACT_GELU_TANH: FLASHBLOCK_WRITE(DT, FLASHBLOCK_ACT_GELU_TANH);
        case FLASHBLOCK_ACT_SILU: FLASHBLOCK_WRITE(DT, FLASHBLOCK_ACT_SILU);
        default: FLASHBLOCK_WRITE(DT, FLASHBLOCK_ACT_NONE);
        }
    } else {
        switch (p.e.act) {
        case FLASHBLOCK_ACT_RELU: FLASHBLOCK_WRITE(FLASHBEV_F32, FLASHBLOCK_ACT_RELU);
        case FLASHBLOCK_ACT_GELU: FLASHBLOCK_WRITE(FLASHBEV_F32, FLASHBLOCK_ACT_GELU);
        case FLASHBLOCK_ACT_GELU_TANH: FLASHBLOCK_WRITE(FLASHBEV_F32, FLASHBLOCK_ACT_GELU_TANH);
        case FLASHBLOCK_ACT_SILU: FLASHBLOCK_WRITE(FLASHBEV_F32, FLASHBLOCK_ACT_SILU);
        default: FLASHBLOCK_WRITE(FLASHBEV_F32, FLASHBLOCK_ACT_NONE);
        }
    }
#undef FLASHBLOCK_WRITE
}

// LDS lets two workgroups of 64 x 64 or 128 x 128 tiles onto a CU, or one of 256 x 256: two
// wavefronts a SIMD.  The compiler's bound of four for 64 x 64 tiles is for its choice of
// registers alone (at most 128): with two 40000 x 256 x 256 float32 takes 62 us, with four 58;
// other products are the same to 2%.
template <int DT, bool AX, bool BX, int BM, int BN, int WM, int WN, int S, bool ENDS>
__global__ void __launch_bounds__(WM *WN * 64, BM == 64 ? 4 : 2) linear_stream(Gemm p)
{
    constexpr int NT = WM * WN * 64;
    constexpr int TM = BM / WM, TN = BN / WN;
    constexpr int FM = TM / 32, FN = TN / 32;
    using SA = Stream<DT, AX, BM, NT>;
    using SB = Stream<DT, BX, BN, NT>;
    using TA = typename SA::T;
    using TB = typename SB::T;
    constexpr int KT = TA::KT;
    constexpr int STAGE = TA::BYTES + TB::BYTES;
    constexpr int LOADS = SA::G + SB::G;
    extern __shared__ __attribute__((aligned(16))) char ring[];   // S stages

    int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const uint32_t lds0 =
        __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)ring +
                                       wave * 1024);
    const int total = (p.red + KT - 1) / KT;
    const int items = p.tiles_m * p.tiles_n * p.split;
    // An XCD's workgroups (one in eight of the grid) take a contiguous share of the
    // items, which runs over blocks of eight tile rows: what is read together
    // meets in one L2.
    const int per = (items + 7) / 8, first = blockIdx.x % 8 * per;
    const int mine = min(per, items - first), stride = gridDim.x / 8;

    struct Item {
        int m0, n0, part, s0, s1;
    };
    auto item_at = [&](int i) {
        Item it;
        const int id = first + i;
        const int tile = id / p.split;
        it.part = id - tile * p.split;
        const int group = tile / (8 * p.tiles_n), rest = tile - group * 8 * p.tiles_n;
        const int rows = min(8, p.tiles_m - 8 * group);
        it.n0 = rest / rows * BN;
        it.m0 = (group * 8 + rest % rows) * BM;
        it.s0 = it.part * p.steps;
        it.s1 = min(total, it.s0 + p.steps);
        return it;
    };

    f32x16 acc[FM][FN];
    auto clear = [&] {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    };

    // the loading end of the ring
    int li = blockIdx.x / 8, ls = 0, slot = 0;
    Item load{};
    uint32_t oa[SA::G], ob[SB::G];
    const char *pa = nullptr, *pb = nullptr;
    bool loading = li < mine;
    auto offsets = [&] {
        SA::offsets(oa, p.lda, load.m0, AX && p.padded ? (p.rows + 7) & ~7 : p.rows, tid);
        SB::offsets(ob, p.ldb, load.n0, p.cols, tid);
    };
    auto open = [&] {
        load = item_at(li);
        offsets();
        ls = load.s0;
        pa = SA::at(p.a, p.lda, load.m0, ls * KT);
        pb = SB::at(p.b, p.ldb, load.n0, ls * KT);
    };
    auto fetch = [&] {
        const uint32_t la = lds0 + slot * STAGE, lb = la + TA::BYTES;
        const int left = p.red - ls * KT;
        if (left >= KT) {
            SA::load(pa, oa, la);
            SB::load(pb, ob, lb);
        } else {
            SA::load_last(pa, oa, la, left, tid);
            SB::load_last(pb, ob, lb, left, tid);
        }
        slot = slot + 1 == S ? 0 : slot + 1;
        pa += AX ? (int64_t)KT * p.lda : (int64_t)128;
        pb += BX ? (int64_t)KT * p.ldb : (int64_t)128;
        if (++ls == load.s1) {
            li += stride;
            loading = li < mine;
            if (loading) open();
        }
    };
    if (loading) open();
#pragma unroll
    for (int i = 0; i < S - 1; ++i)
        if (loading) fetch();

    // Fragments of a quarter step are read while the quarter before it is multiplied
    // (left alone, the compiler reads each one just before its use); the barrier
    // between steps stands before the last quarter's products, whose operands are in
    // registers, so that the matrix cores work on through it.
    u32x4 fa[2][FM], fb[2][FN];
    int read = 0;
    auto quarter = [&](int kk) {
        const char *la = ring + read * STAGE, *lb = la + TA::BYTES;
#pragma unroll
        for (int g = 0; g < FN; ++g) fb[kk & 1][g] = TB::fragment(lb, wn * TN + g * 32, kk, lane);
#pragma unroll
        for (int f = 0; f < FM; ++f) fa[kk & 1][f] = TA::fragment(la, wm * TM + f * 32, kk, lane);
    };
    // to the ring's next stage: it is the oldest in flight, of S - 1 (fewer near the
    // end, where all are waited for); past the barrier every wavefront has read the
    // stage before it, whose place is filled again
    auto advance = [&] {
        if (loading) wait_loads<(S - 2) * LOADS>();
        else wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (loading) fetch();
        quarter(0);
    };
    for (int i = blockIdx.x / 8; i < mine; i += stride) {
        const Item it = item_at(i);
        clear();
        if (it.s0 < it.s1) advance();
        for (int s = it.s0; s < it.s1; ++s) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                if (kk < 3) {
                    quarter(kk + 1);
                } else {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    read = read + 1 == S ? 0 : read + 1;
                    if (s + 1 < it.s1) advance();
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int f = 0; f < FM; ++f)
#pragma unroll
                    for (int g = 0; g < FN; ++g) mma<DT>(acc[f][g], fb[kk & 1][g], fa[kk & 1][f]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        write_any<DT, !BX, ENDS>(p, it.part, it.m0 + wm * TM, it.n0 + wn * TN, lane, acc);
        // what the lanes' addresses are made of is computed again rather than kept
        // in registers through the epilogue (where it spilled, the ring's loads
        // waited for its way back)
        tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        lane = tid & 63;
        if (loading) offsets();
    }
}

// ---------------------------------------------------------------------------
// few rows: one pass over the weight
// ---------------------------------------------------------------------------
// Up to 32 rows (one or two blocks of 16) read every weight once, which is nearly all the
// time they take.  A workgroup owns 16 output channels; its 8 wavefronts take the
// K axis in turns of 16 (for two blocks 8) 64-byte pieces of each of the 16 weight
// rows (a piece: a 16x16x32 MFMA of 16-bit elements, or four 16x16x4 of float32), all
// in flight, from memory straight into the operands; their sums are added through LDS in the
// wavefronts' order.  One launch and no workspace: 1 x 4096 x 4096 bfloat16 takes 8.5 us
// (33.6 MB, 4 TB/s) where parts of 64 x 64 tiles and their join take 11.3.
constexpr int kFewRows = 32;
constexpr int kFewWaves = 8;

struct Few {
    const char *x, *w;
    int64_t ldx, ldw;   // bytes
    int M, N, K;
    Epilogue e;
};

template <int DT>
__device__ __forceinline__ void mma16(f32x4 &c, const u32x4 &a, const u32x4 &b)
{
    if constexpr (DT == FLASHBEV_BF16) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                    __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else if constexpr (DT == FLASHBEV_F16) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                   __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    } else {
        const f32x4 fa = __builtin_bit_cast(f32x4, a), fb = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[q], fb[q], c, 0, 0, 0);
    }
}

template <int DT, int MB>
__global__ void __launch_bounds__(64 * kFewWaves) linear_few(Few p)
{
    constexpr int ES = elem_size(DT), E = 16 / ES, KS = 4 * E;   // elements of a piece
    constexpr int U = MB == 1 ? 16 : 8;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n0 = blockIdx.x * 16, k0 = (lane >> 4) * E;
    // rows and channels past the last repeat it; their sums are not stored
    const char *w = p.w + (int64_t)min(n0 + (lane & 15), p.N - 1) * p.ldw;
    const char *x[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) x[b] = p.x + (int64_t)min(b * 16 + (lane & 15), p.M - 1) * p.ldx;
    f32x4 acc[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int whole = p.K / KS;
    int done = 0;
    for (; done + kFewWaves * U <= whole; done += kFewWaves * U) {
        u32x4 fw[U], fx[U][MB];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = (int64_t)((done + wave * U + u) * KS + k0) * ES;
            fw[u] = load16(w + at);
#pragma unroll
            for (int b = 0; b < MB; ++b) fx[u][b] = load16(x[b] + at);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int b = 0; b < MB; ++b) mma16<DT>(acc[b], fw[u], fx[u][b]);
    }
    int s = done + wave;
    for (; s < whole; s += kFewWaves) {
        const int64_t at = (int64_t)(s * KS + k0) * ES;
        const u32x4 fw = load16(w + at);
#pragma unroll
        for (int b = 0; b < MB; ++b) mma16<DT>(acc[b], fw, load16(x[b] + at));
    }
    if (s == whole && whole * KS < p.K) {   // the axis's end, on its wavefront
        const u32x4 fw = load_granule_edge<DT>(w, s * KS + k0, p.K);
#pragma unroll
        for (int b = 0; b < MB; ++b)
            mma16<DT>(acc[b], fw, load_granule_edge<DT>(x[b], s * KS + k0, p.K));
    }
    // lane: row lane % 16, channels 4 (lane / 16) .. + 3 of each block
    __shared__ float part[kFewWaves][MB * 16][16 + 1], sum[MB * 16][16 + 4];
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            part[wave][b * 16 + (lane & 15)][4 * (lane >> 4) + i] = acc[b][i];
    __syncthreads();
    if (threadIdx.x < MB * 256) {
        const int m = threadIdx.x >> 4, n = threadIdx.x & 15;
        float v = 0.0f;
#pragma unroll
        for (int q = 0; q < kFewWaves; ++q) v += part[q][m][n];
        sum[m][n] = v;
    }
    __syncthreads();
    const int m = threadIdx.x >> 1, n = (threadIdx.x & 1) * 8;
    if (m >= p.M || n0 + n >= p.N) return;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = sum[m][n + i];
    epilogue<DT>(p.e, m, n0 + n, p.N, v);
}

// ---------------------------------------------------------------------------
// sums of the parts of a split reduction axis, in their order
// ---------------------------------------------------------------------------
struct Join {
    const float *partial;   // [split][rows][pld], pld a multiple of 8
    int64_t pld;
    int rows, cols, split;
    Epilogue e;
};

// 64 vectors of columns to a workgroup; its four wavefronts take the parts in turns,
// and their sums are added in the wavefronts' order.
template <int DT>
__global__ void __launch_bounds__(256) linear_join(Join p)
{
    constexpr int V = 8;
    const int per_row = (p.cols + V - 1) / V;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t i = (int64_t)blockIdx.x * 64 + lane;
    const int64_t m = i / per_row;
    const int n = (int)(i % per_row) * V;
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = 0.0f;
    if (m < p.rows) {
        const float *src = p.partial + m * p.pld + n;
#pragma unroll 4
        for (int s = wave; s < p.split; s += 4) {
            float w[V];
            load_elems<FLASHBEV_F32>(src + (int64_t)s * p.rows * p.pld, w);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] += w[e];
        }
    }
    __shared__ float part[3][V][64];
    if (wave > 0) {
#pragma unroll
        for (int e = 0; e < V; ++e) part[wave - 1][e][lane] = v[e];
    }
    __syncthreads();
    if (wave > 0 || m >= p.rows) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] += part[w][e][lane];
    epilogue<DT>(p.e, m, n, p.cols, v);
}

// ---------------------------------------------------------------------------
// d = scale act'(pre) grad_out in the inputs' type, and its column sums
// ---------------------------------------------------------------------------
// A workgroup takes 256 columns of a range of rows; 32 lanes share a row, 8
// columns each, and 8 rows are in flight.  Its column sums (float32, of the
// unrounded values) go to its range's row of `partial`; column_join adds those in
// order.
struct Slope {
    const void *grad;       // [M, N], DT or float32
    const void *pre;        // null without an activation
    void *d;                // null: column sums alone
    float *partial;         // [ranges][pld], null: no column sums
    int64_t ldg, ldp, ldd, pld;   // elements
    int M, N, rows;         // rows of a range
    int col_blocks;
    int act, grad_f32;
    int copy;               // d is grad_out itself: without the scale, which the products take
    float scale;
};

template <int DT>
__global__ void __launch_bounds__(256) linear_slope(Slope p)
{
    const int cb = blockIdx.x % p.col_blocks, range = blockIdx.x / p.col_blocks;
    const int n = cb * 256 + (threadIdx.x & 31) * 8;
    const int64_t r0 = (int64_t)range * p.rows, r1 = min((int64_t)p.M, r0 + p.rows);
    constexpr int es = elem_size(DT);
    float sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
    if (n < p.N) {
        const bool whole = n + 8 <= p.N;
#pragma unroll 2
        for (int64_t m = r0 + (threadIdx.x >> 5); m < r1; m += 8) {
            float g[8], v[8];
            const char *gp = static_cast<const char *>(p.grad) + (m * p.ldg + n) * (p.grad_f32 ? 4 : es);
            const char *vp = static_cast<const char *>(p.pre) + (m * p.ldp + n) * es;
            if (whole) {
                if (p.grad_f32) load_elems<FLASHBEV_F32>(gp, g);
                else load_elems<DT>(gp, g);
                if (p.act) load_elems<DT>(vp, v);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool in = n + e < p.N;
                    g[e] = !in ? 0.0f : p.grad_f32 ? load_elem<FLASHBEV_F32>(gp, e) : load_elem<DT>(gp, e);
                    v[e] = in && p.act ? load_elem<DT>(vp, e) : 0.0f;
                }
            }
            if (p.act) {
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] *= act_slope(p.act, v[e]);
            }
            // d is rounded to the inputs' type, in which the matrix units read it (its column
            // sums are not); pre was rounded to it as the forward wrote it.  On 4000 x 256 x 1024
            // bfloat16 with gelu the products' gradients are 0.00241 off float64 (norms of the
            // difference and the value) where their own rounding alone is 0.00166: 0.00235 for
            // d alone, 0.00175 for pre alone.
            const float scale = p.copy ? 1.0f : p.scale;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                g[e] *= scale;
                sum[e] += g[e];
            }
            // whole vectors, with zeros past N (ldd is a multiple of 8)
            if (p.d) store_elems<DT>(static_cast<char *>(p.d) + (m * p.ldd + n) * es, g);
        }
    }
    if (!p.partial) return;
    __shared__ float part[8][256 + 8];
#pragma unroll
    for (int e = 0; e < 8; ++e) part[threadIdx.x >> 5][(threadIdx.x & 31) * 8 + e] = sum[e];
    __syncthreads();
    const int c = cb * 256 + threadIdx.x;
    float s = 0.0f;
#pragma unroll
    for (int r = 0; r < 8; ++r) s += part[r][threadIdx.x];
    if (c < p.N) p.partial[(int64_t)range * p.pld + c] = p.copy ? s * p.scale : s;
}

// out[n] = sum over ranges of partial[range][n], in `DT`; 16 columns per workgroup
struct ColumnJoin {
    const float *partial;
    int64_t pld;
    int ranges, N;
    void *out;
};

template <int DT>
__global__ void __launch_bounds__(256) column_join(ColumnJoin p)
{
    const int n = blockIdx.x * 16 + (threadIdx.x & 15), r0 = threadIdx.x >> 4;
    float s = 0.0f;
    if (n < p.N)
#pragma unroll 8
        for (int r = r0; r < p.ranges; r += 16) s += p.partial[(int64_t)r * p.pld + n];
    __shared__ float part[16][17];
    part[r0][threadIdx.x & 15] = s;
    __syncthreads();
    if (r0 != 0 || n >= p.N) return;
    s = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) s += part[r][threadIdx.x];
    store_elem<DT>(p.out, n, s);
}

// ---------------------------------------------------------------------------
// host: plans and launches
// ---------------------------------------------------------------------------
constexpr int kCus = 256;

uint64_t round_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

// Tile, and parts of the reduction axis, with the least estimated time.  A tile's
// time is its steps' and a fixed part (filling the ring, writing the results);
// `resident` workgroups run at once.  The constants (us) are fitted to measured
// products: in 256, 128 and 64 tiles, bfloat16, 8192 x 8192 over 4096 takes 461, 536 and
// 937; 184950 x 256 over 256 51, 57 and 86; 40000 x 512 over 256 with a float32 output
// 41, 27 and 38; 1024 x 256 over 40000 (in parts) 57, 57 and 74; float32
// 40000 x 256 over 256 77, 58 and 58.  float32 tiles of 256 and 128 are close where both fill the
// card (8192 cubed 7687 and 7550, 16384 x 4096 over 4096 3879 and 3796, gradient 512 x 512
// over 65536 270 and 278) and up to 18% apart where the estimate takes 256 for a short axis
// (40001 x 520 over 72 71 and 60).  Checked tiles of 128 and 64: half 3331 x 777 over 515 22 and 16,
// bfloat16 40001 x 72 over 129 12.8 and 14.6, 40001 x 520 over 129 46 and 42, 8191 x 4095 over 4095
// 416 and 659, 200 x 72 over 129 10.1 and 5.6.  `estimate` gets the least time.
struct TilePlan {
    int tile, split, steps;
    uint64_t workspace;    // bytes of partial sums
};

struct TileCost {
    int tile, resident;
    float step, fixed;
};
constexpr TileCost kStream16[] = {{256, kCus, 1.72f, 7.5f}, {128, 2 * kCus, 1.02f, 4.0f},
                                  {64, 2 * kCus, 0.5f, 3.0f}};
constexpr TileCost kStream32[] = {{256, kCus, 7.4f, 7.5f}, {128, 2 * kCus, 3.8f, 4.0f},
                                  {64, 2 * kCus, 1.0f, 3.0f}};
// linear_tiles, which widths of other than whole granules take
constexpr TileCost kChecked[] = {{128, 2 * kCus, 3.0f, 4.0f}, {64, 4 * kCus, 1.5f, 3.0f}};

TilePlan plan_tiles(int64_t rows, int64_t cols, int64_t red, int dt, bool checked,
                    float *estimate = nullptr)
{
    const int64_t total = (red + 128 / elem_size(dt) - 1) / (128 / elem_size(dt));
    TilePlan best{64, 1, (int)(total > 0 ? total : 1), 0};
    const TileCost *costs = checked ? kChecked : dt == FLASHBEV_F32 ? kStream32 : kStream16;
    float least = 0.0f;
    for (int k = 0; k < (checked ? 2 : 3); ++k) {
        const TileCost &c = costs[k];
        const int64_t tiles = ((rows + c.tile - 1) / c.tile) * ((cols + c.tile - 1) / c.tile);
        for (int64_t split = 1; split == 1 || (split <= total / 2 && split * tiles <= 2 * c.resident);
             split *= 2) {
            const int64_t steps = total > 0 ? (total + split - 1) / split : 1;
            const int64_t parts = total > 0 ? (total + steps - 1) / steps : 1;
            const int64_t rounds = (tiles * parts + c.resident - 1) / c.resident;
            float us = (float)rounds * (c.fixed + c.step * (float)steps);
            if (parts > 1)   // the sums' way to memory and back, another launch
                us += 3.0f + (float)parts * (float)rows * (float)cols * 2e-6f;
            if (least == 0.0f || us < least) {
                least = us;
                best = {c.tile, (int)parts, (int)steps, 0};
            }
        }
    }
    if (best.split > 1)
        best.workspace = round_up((uint64_t)best.split * rows * round_up(cols, 8) * 4, 256);
    if (estimate) *estimate = least;
    return best;
}

// linear_few's time (us): a workgroup's grows with its weights' row and with the rows of x,
// and 256 workgroups (4096 channels) run at once.  Against tiles (M x K x N, the kernel's
// and the tiles' measured us): bfloat16 1 x 4096 x 4096 8.5 and 11.3, 16 rows 10.7 and 12.2,
// 32 rows 14.5 and 12.6, 16 x 4096 x 64 9.6 and 6.7, 32 x 1024 x 1024 5.5 and 7.2; float32
// 1 x 4096 x 4096 16.6 and 25.4, 32 rows 26.3 and 26.8, 32 x 8192 x 64 44 and 10.5, 16 x 4096 x 1024
// 17.6 and 13.9.  More than 32 rows would take two calls (33 x 4096 x 4096 21.4 and 12.6).
float few_estimate(const flashblock_linear *p)
{
    const float bytes = (float)p->K * elem_size(p->dtype), rounds = (float)p->N / 4096.0f;
    return 3.0f + bytes * (0.0005f + 0.000025f * (float)p->M) * (rounds > 1.0f ? rounds : 1.0f);
}

// What the sizes alone say about linear_stream's layout (linear_stream also needs
// its strides and addresses): widths of whole granules, the reduction axis of an
// operand along it or the columns of one across it, and a gradient's rows of whole
// vectors.
// `padded`: A's rows end in zeros up to a multiple of 8 (B, whose rows run along the
// reduction axis then, is checked against its end).
bool whole_granules(int64_t rows, int64_t cols, int64_t red, int dt, bool ax, bool bx, bool padded)
{
    const int e = 16 / elem_size(dt);
    return (padded || (ax ? rows : red) % e == 0) && (bx ? cols % 8 : red % e) == 0;
}

// Whether the backward makes d a tensor of its own (rows padded with zeros): where
// an activation or a type makes it another one than grad_out, and where grad_out's rows
// alone would keep both products from streaming (a copy: 150278 x 80 -> 333 bfloat16).
bool forms_d(const flashblock_linear *p)
{
    return p->act != FLASHBLOCK_ACT_NONE || p->out_dtype != p->dtype || (p->N % 8 && p->K % 8 == 0);
}

TilePlan plan_forward(const flashblock_linear *p)
{
    float us;
    const TilePlan t = plan_tiles(p->M, p->N, p->K, p->dtype,
                                  !whole_granules(p->M, p->N, p->K, p->dtype, false, false, false), &us);
    if (p->M <= kFewRows && few_estimate(p) <= us) return {0, 1, 0, 0};   // linear_few
    return t;
}

TilePlan plan_grad_x(const flashblock_linear *p)
{
    return plan_tiles(p->M, p->K, p->N, p->dtype,
                      !whole_granules(p->M, p->K, p->N, p->dtype, false, true, forms_d(p)));
}

TilePlan plan_grad_weight(const flashblock_linear *p)
{
    return plan_tiles(p->N, p->K, p->M, p->dtype,
                      !whole_granules(p->N, p->K, p->M, p->dtype, true, true, forms_d(p)));
}

template <int DT, bool AX, bool BX, int BM, int BN, int WM, int WN, int S>
int launch_stream(Gemm &g, hipStream_t st)
{
    const void *fn = (const void *)linear_stream<DT, AX, BX, BM, BN, WM, WN, S, false>;
    if constexpr (!BX) {
        if (g.cols % 8) fn = (const void *)linear_stream<DT, AX, BX, BM, BN, WM, WN, S, true>;
    }
    constexpr size_t lds = (size_t)S * (BM + BN) * 128;
    g.tiles_m = (g.rows + BM - 1) / BM;
    g.tiles_n = (g.cols + BN - 1) / BN;
    const uint64_t items = (uint64_t)g.tiles_m * g.tiles_n * g.split;
    if (items > 0x7fffffffull) return FLASHBEV_ERR_UNSUPPORTED;
    constexpr uint64_t resident = kCus * (163840 / lds);
    const uint64_t blocks = items < resident ? round_up(items, 8) : resident;
    if (lds > 65536 &&
        hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
        return FLASHBEV_ERR_HIP;
    return launch_kernel(fn, blocks, WM * WN * 64, g, lds, st);
}

template <int DT, bool AX, bool BX>
bool streamable(const Gemm &g)
{
    return g.red > 0 && !misaligned(g.a, 16) && !misaligned(g.b, 16) && g.lda % 16 == 0 &&
           g.ldb % 16 == 0 && whole_granules(g.rows, g.cols, g.red, DT, AX, BX, g.padded);
}

template <int DT, bool AX, bool BX, int TILE>
int launch_checked(Gemm &g, hipStream_t st)
{
    g.tiles_m = (g.rows + TILE - 1) / TILE;
    g.tiles_n = (g.cols + TILE - 1) / TILE;
    return launch_rows((const void *)linear_tiles<DT, AX, BX, TILE, TILE, 2, 2>,
                       (uint64_t)g.tiles_m * g.tiles_n * g.split, 256, g, st);
}

template <int DT, bool AX, bool BX>
int launch_tiles(Gemm &g, const TilePlan &t, hipStream_t st)
{
    if (streamable<DT, AX, BX>(g)) {
        if (t.tile == 256) return launch_stream<DT, AX, BX, 256, 256, 2, 4, 2>(g, st);
        if (t.tile == 128) return launch_stream<DT, AX, BX, 128, 128, 2, 2, 2>(g, st);
        return launch_stream<DT, AX, BX, 64, 64, 2, 2, 4>(g, st);
    }
    return t.tile == 64 ? launch_checked<DT, AX, BX, 64>(g, st) : launch_checked<DT, AX, BX, 128>(g, st);
}

// C = A B^T through the epilogue; `workspace` of t.workspace bytes
template <bool AX, bool BX>
int product(const TilePlan &t, int dt, const void *a, int64_t lda, const void *b, int64_t ldb,
            int64_t rows, int64_t cols, int64_t red, bool padded, const Epilogue &e, void *workspace,
            hipStream_t st)
{
    if (rows == 0 || cols == 0) return FLASHBEV_OK;
    const int es = elem_size(dt);
    Gemm g{};
    g.a = static_cast<const char *>(a);
    g.b = static_cast<const char *>(b);
    g.lda = lda * es;
    g.ldb = ldb * es;
    g.rows = (int)rows;
    g.cols = (int)cols;
    g.red = (int)red;
    g.padded = padded;
    g.split = t.split;
    g.steps = t.steps;
    g.partial = static_cast<float *>(workspace);
    g.pld = (int64_t)round_up(cols, 8);
    g.e = e;
    int rc = dt == FLASHBEV_F32   ? launch_tiles<FLASHBEV_F32, AX, BX>(g, t, st)
             : dt == FLASHBEV_F16 ? launch_tiles<FLASHBEV_F16, AX, BX>(g, t, st)
                                  : launch_tiles<FLASHBEV_BF16, AX, BX>(g, t, st);
    if (rc || t.split == 1) return rc;
    Join j{g.partial, g.pld, g.rows, g.cols, t.split, e};
    const uint64_t vecs = (uint64_t)rows * ((cols + 7) / 8);
    const void *fn = dt == FLASHBEV_F32   ? (const void *)linear_join<FLASHBEV_F32>
                     : dt == FLASHBEV_F16 ? (const void *)linear_join<FLASHBEV_F16>
                                          : (const void *)linear_join<FLASHBEV_BF16>;
    return launch_kernel(fn, (vecs + 63) / 64, 256, j, 0, st);
}

template <int DT>
const void *few_kernel(bool two)
{
    return two ? (const void *)linear_few<DT, 2> : (const void *)linear_few<DT, 1>;
}

int check_sizes(const flashblock_linear *p)
{
    if (!p) return FLASHBEV_ERR_NULLPTR;
    if (p->M < 0 || p->K < 0 || p->N < 0) return FLASHBEV_ERR_SHAPE;
    if (!known_dtype(p->dtype) || (p->out_dtype != p->dtype && p->out_dtype != FLASHBEV_F32))
        return FLASHBEV_ERR_DTYPE;
    if (p->act < FLASHBLOCK_ACT_NONE || p->act > FLASHBLOCK_ACT_SILU || !finite_value(p->scale))
        return FLASHBEV_ERR_VALUE;
    if (p->M > FLASHBLOCK_ROWS_MAX || p->K > FLASHBLOCK_WIDTH_MAX || p->N > FLASHBLOCK_WIDTH_MAX)
        return FLASHBEV_ERR_UNSUPPORTED;
    return FLASHBEV_OK;
}

// a tensor of `rows` rows: its stride and pointer
int check_rows(const void *p, int64_t rows, int64_t ld, int64_t width, int es)
{
    if (rows == 0 || width == 0) return FLASHBEV_OK;
    if (!p) return FLASHBEV_ERR_NULLPTR;
    if (ld < width) return FLASHBEV_ERR_SHAPE;
    if (ld > FLASHBLOCK_LD_MAX) return FLASHBEV_ERR_UNSUPPORTED;
    return misaligned(p, es) ? FLASHBEV_ERR_ALIGN : FLASHBEV_OK;
}

int check_workspace(const void *ws, uint64_t have, uint64_t need)
{
    if (need == 0) return FLASHBEV_OK;
    if (!ws) return FLASHBEV_ERR_NULLPTR;
    if (misaligned(ws, 256)) return FLASHBEV_ERR_ALIGN;
    return have < need ? FLASHBEV_ERR_SCRATCH : FLASHBEV_OK;
}

struct Range {
    const void *p;
    uint64_t n;
};

// The backward's workspace: d, then the column sums, then the products' partial
// sums (grad_weight's, and after it grad_x's in the same place).
struct BackwardPlan {
    bool slope;            // d is a tensor of its own
    bool column_sums;
    int ranges, range_rows;
    int64_t ldd;
    uint64_t d_bytes, sum_bytes, partial_bytes, total;
};

BackwardPlan plan_backward(const flashblock_linear *p, bool want_x, bool want_w, bool want_b)
{
    BackwardPlan b{};
    const int es = elem_size(p->dtype);
    b.slope = (want_x || want_w) && forms_d(p);
    b.column_sums = want_b;
    b.ldd = (int64_t)round_up((uint64_t)p->N, 8);
    b.d_bytes = b.slope ? round_up((uint64_t)p->M * b.ldd * es, 256) : 0;
    // ranges: about four workgroups per CU, of 32 rows or more
    const int64_t col_blocks = (p->N + 255) / 256;
    int64_t ranges = col_blocks > 0 ? 4 * kCus / col_blocks : 1;
    if (ranges > 256) ranges = 256;
    if (ranges > p->M / 32) ranges = p->M / 32;
    if (ranges < 1) ranges = 1;
    b.range_rows = (int)((p->M + ranges - 1) / ranges);
    if (b.range_rows < 1) b.range_rows = 1;
    b.ranges = (int)((p->M + b.range_rows - 1) / b.range_rows);
    if (b.ranges < 1) b.ranges = 1;
    b.sum_bytes = want_b ? round_up((uint64_t)b.ranges * b.ldd * 4, 256) : 0;
    if (want_w) b.partial_bytes = plan_grad_weight(p).workspace;
    if (want_x) {
        const uint64_t w = plan_grad_x(p).workspace;
        if (w > b.partial_bytes) b.partial_bytes = w;
    }
    b.total = b.d_bytes + b.sum_bytes + b.partial_bytes;
    return b;
}

}  // namespace

extern "C" {

int flashblock_linear_workspace_size(const flashblock_linear *p, uint64_t *bytes)
{
    if (!bytes) return FLASHBEV_ERR_NULLPTR;
    if (const int rc = check_sizes(p)) return rc;
    *bytes = p->M && p->N ? plan_forward(p).workspace : 0;
    return FLASHBEV_OK;
}

int flashblock_linear_forward(const flashblock_linear *p, const void *x, const void *weight,
                              const void *bias, const void *residual, void *out, void *pre,
                              void *workspace, uint64_t workspace_bytes, void *stream)
{
    int rc = check_sizes(p);
    if (rc) return rc;
    const int es = elem_size(p->dtype), os = elem_size(p->out_dtype);
    if (p->M == 0 || p->N == 0) return FLASHBEV_OK;
    if ((rc = check_rows(x, p->M, p->ldx, p->K, es)) ||
        (rc = check_rows(weight, p->N, p->ldw, p->K, es)) ||
        (rc = check_rows(out, p->M, p->ldo, p->N, os)))
        return rc;
    if (residual && (rc = check_rows(residual, p->M, p->ldr, p->N, os))) return rc;
    if (pre && (rc = check_rows(pre, p->M, p->ldp, p->N, es))) return rc;
    if (misaligned(bias, es)) return FLASHBEV_ERR_ALIGN;
    const TilePlan plan = plan_forward(p);
    const uint64_t need = plan.workspace;
    if ((rc = check_workspace(workspace, workspace_bytes, need))) return rc;
    const bool in_place = residual == out && p->ldr == p->ldo;
    const Range ins[] = {{x, span_bytes(p->M, p->ldx, p->K, es)},
                         {weight, span_bytes(p->N, p->ldw, p->K, es)},
                         {bias, (uint64_t)p->N * es},
                         {residual, span_bytes(p->M, p->ldr, p->N, os)}};
    const Range outs[] = {{out, span_bytes(p->M, p->ldo, p->N, os)},
                          {pre, span_bytes(p->M, p->ldp, p->N, es)},
                          {workspace, need}};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 4; ++i)
            if (!(o == 0 && i == 3 && in_place) &&
                ranges_overlap(outs[o].p, outs[o].n, ins[i].p, ins[i].n))
                return FLASHBEV_ERR_ALIAS;
        for (int q = 0; q < o; ++q)
            if (ranges_overlap(outs[o].p, outs[o].n, outs[q].p, outs[q].n)) return FLASHBEV_ERR_ALIAS;
    }
    Epilogue e{out, pre, bias, residual, p->ldo, p->ldp, p->ldr, p->scale, p->act,
               p->out_dtype == FLASHBEV_F32};
    if (plan.tile == 0) {
        Few f{static_cast<const char *>(x), static_cast<const char *>(weight), p->ldx * es,
              p->ldw * es, (int)p->M, p->N, p->K, e};
        const bool two = p->M > 16;
        const void *fn = p->dtype == FLASHBEV_F32   ? few_kernel<FLASHBEV_F32>(two)
                         : p->dtype == FLASHBEV_F16 ? few_kernel<FLASHBEV_F16>(two)
                                                    : few_kernel<FLASHBEV_BF16>(two);
        return launch_kernel(fn, (uint64_t)(p->N + 15) / 16, 64 * kFewWaves, f, 0,
                             static_cast<hipStream_t>(stream));
    }
    return product<false, false>(plan, p->dtype, x, p->ldx, weight, p->ldw, p->M, p->N, p->K, false, e,
                                 workspace, static_cast<hipStream_t>(stream));
}

int flashblock_linear_backward_workspace_size(const flashblock_linear *p, int32_t want_x,
                                              int32_t want_weight, int32_t want_bias,
                                              uint64_t *bytes)
{
    if (!bytes) return FLASHBEV_ERR_NULLPTR;
    if (const int rc = check_sizes(p)) return rc;
    *bytes = plan_backward(p, want_x, want_weight, want_bias).total;
    return FLASHBEV_OK;
}

int flashblock_linear_backward(const flashblock_linear *p, const void *grad_out, const void *x,
                               const void *weight, const void *pre, void *grad_x, int64_t ldgx,
                               void *grad_weight, int64_t ldgw, void *grad_bias, void *workspace,
                               uint64_t workspace_bytes, void *stream)
{
    int rc = check_sizes(p);
    if (rc) return rc;
    const int es = elem_size(p->dtype), os = elem_size(p->out_dtype);
    // gradients without elements have no address and nothing to write
    const bool has_x = p->M > 0 && p->K > 0, has_w = p->N > 0 && p->K > 0, has_b = p->N > 0;
    if (!grad_x && !grad_weight && !grad_bias && has_x && has_w && has_b)
        return FLASHBEV_ERR_NULLPTR;
    const bool want_x = grad_x && has_x, want_w = grad_weight && has_w, want_b = grad_bias && has_b;
    if (!want_x && !want_w && !want_b) return FLASHBEV_OK;
    if ((rc = check_rows(grad_out, p->M, p->ldo, p->N, os))) return rc;
    if (want_w && (rc = check_rows(x, p->M, p->ldx, p->K, es))) return rc;
    if (want_x && (rc = check_rows(weight, p->N, p->ldw, p->K, es))) return rc;
    if (p->act != FLASHBLOCK_ACT_NONE && (rc = check_rows(pre, p->M, p->ldp, p->N, es))) return rc;
    if (want_x && (rc = check_rows(grad_x, p->M, ldgx, p->K, es))) return rc;
    if (want_w && (rc = check_rows(grad_weight, p->N, ldgw, p->K, es))) return rc;
    if (misaligned(grad_bias, es)) return FLASHBEV_ERR_ALIGN;
    const BackwardPlan b = plan_backward(p, want_x, want_w, want_b);
    if ((rc = check_workspace(workspace, workspace_bytes, b.total))) return rc;
    const Range ins[] = {
        {grad_out, span_bytes(p->M, p->ldo, p->N, os)},
        {want_w ? x : nullptr, span_bytes(p->M, p->ldx, p->K, es)},
        {want_x ? weight : nullptr, span_bytes(p->N, p->ldw, p->K, es)},
        {p->act != FLASHBLOCK_ACT_NONE ? pre : nullptr, span_bytes(p->M, p->ldp, p->N, es)}};
    const Range outs[] = {{want_x ? grad_x : nullptr, span_bytes(p->M, ldgx, p->K, es)},
                          {want_w ? grad_weight : nullptr, span_bytes(p->N, ldgw, p->K, es)},
                          {want_b ? grad_bias : nullptr, (uint64_t)p->N * es},
                          {workspace, b.total}};
    for (int o = 0; o < 4; ++o) {
        for (int i = 0; i < 4; ++i)
            if (ranges_overlap(outs[o].p, outs[o].n, ins[i].p, ins[i].n)) return FLASHBEV_ERR_ALIAS;
        for (int q = 0; q < o; ++q)
            if (ranges_overlap(outs[o].p, outs[o].n, outs[q].p, outs[q].n)) return FLASHBEV_ERR_ALIAS;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    char *ws = static_cast<char *>(workspace);
    const int dt = p->dtype;
    const void *d = grad_out;
    int64_t ldd = p->ldo;
    float alpha = p->scale;
    if (b.slope || b.column_sums) {
        Slope s{};
        s.grad = grad_out;
        s.pre = pre;
        s.ldg = p->ldo;
        s.ldp = p->ldp;
        s.ldd = b.ldd;
        s.pld = b.ldd;
        s.M = (int)p->M;
        s.N = p->N;
        s.rows = b.range_rows;
        s.col_blocks = (p->N + 255) / 256;
        s.act = p->act;
        s.grad_f32 = p->out_dtype == FLASHBEV_F32;
        s.scale = p->scale;
        s.copy = p->act == FLASHBLOCK_ACT_NONE && p->out_dtype == p->dtype;
        s.d = b.slope ? ws : nullptr;
        s.partial = b.column_sums ? reinterpret_cast<float *>(ws + b.d_bytes) : nullptr;
        const void *fn = dt == FLASHBEV_F32   ? (const void *)linear_slope<FLASHBEV_F32>
                         : dt == FLASHBEV_F16 ? (const void *)linear_slope<FLASHBEV_F16>
                                              : (const void *)linear_slope<FLASHBEV_BF16>;
        if ((rc = launch_kernel(fn, (uint64_t)s.col_blocks * b.ranges, 256, s, 0, st))) return rc;
        if (b.slope) {
            d = ws;
            ldd = b.ldd;
            if (!s.copy) alpha = 1.0f;
        }
        if (b.column_sums) {
            ColumnJoin c{s.partial, b.ldd, b.ranges, p->N, grad_bias};
            fn = dt == FLASHBEV_F32   ? (const void *)column_join<FLASHBEV_F32>
                 : dt == FLASHBEV_F16 ? (const void *)column_join<FLASHBEV_F16>
                                      : (const void *)column_join<FLASHBEV_BF16>;
            if ((rc = launch_kernel(fn, (uint64_t)(p->N + 15) / 16, 256, c, 0, st))) return rc;
        }
    }
    void *partial = ws + b.d_bytes + b.sum_bytes;
    if (want_w) {
        Epilogue e{grad_weight, nullptr, nullptr, nullptr, ldgw, 0, 0, alpha, FLASHBLOCK_ACT_NONE,
                   dt == FLASHBEV_F32};
        if ((rc = product<true, true>(plan_grad_weight(p), dt, d, ldd, x, p->ldx, p->N, p->K, p->M,
                                      b.slope, e, partial, st)))
            return rc;
    }
    if (want_x) {
        Epilogue e{grad_x, nullptr, nullptr, nullptr, ldgx, 0, 0, alpha, FLASHBLOCK_ACT_NONE,
                   dt == FLASHBEV_F32};
        if ((rc = product<false, true>(plan_grad_x(p), dt, d, ldd, weight, p->ldw, p->M, p->K, p->N,
                                       b.slope, e, partial, st)))
            return rc;
    }
    return FLASHBEV_OK;
}

}  // extern "C"

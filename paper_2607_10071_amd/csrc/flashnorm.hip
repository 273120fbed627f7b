// The norms before and after a block with its gate and residual scale, and
// their gradients, for AMD MI355X (gfx950).  C ABI: include/block/flashblock.h.
//
//   u = N_post(x) post_weight + post_bias,  s = residual + (scale gate) u,
//   y = N(s) weight + bias
//
// Memory bounds both directions (about 30 operations an element forward, where
// HBM at 5 TB/s leaves time for 64 with four 16-bit tensors), so a row is read
// once, stays in registers through its statistics (mean, then the sum of squared
// differences from it), and each output is written once.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block_common.h"

namespace {

// ---------------------------------------------------------------------------
// a row over T lanes, NV vectors of V consecutive channels each
// ---------------------------------------------------------------------------
// T = 8 to 64 lanes share a wavefront with other rows; T = 128 takes half a
// workgroup, T = 256 to 1024 one of their own.  Lane t holds channels
// V (v T + t) .. + V - 1 of vector v.
template <int T, int NV, int V>
struct Row {
    static constexpr int E = V * NV;                     // channels a lane holds
    static constexpr int ROWS = T >= 256 ? 1 : 256 / T;  // rows of a workgroup

    static __device__ __forceinline__ int col(int t, int v) { return V * (v * T + t); }

    static __device__ __forceinline__ bool inside(int t, int e, int C)
    {
        return col(t, e / V) + e % V < C;
    }

    // a lane's channels as they are stored, 0 past C, in 16-byte pieces (8-byte ones
    // for four 16-bit channels)
    template <int DT>
    struct Raw {
        static constexpr int PIECES = V * elem_size(DT) >= 16 ? V * elem_size(DT) / 16 : 0;
        u32x4 w[NV][PIECES ? PIECES : 1];
        u32x2 h[NV];
    };

    template <int DT>
    static __device__ __forceinline__ void fetch(const void *p, int64_t off, int t, int C, Raw<DT> &r)
    {
        constexpr int ES = elem_size(DT), G = 16 / ES;
        const char *row = static_cast<const char *>(p) + off * ES;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (Raw<DT>::PIECES == 0) {
                const int c = col(t, v);
                if (c + 4 <= C) r.h[v] = load8(row + (int64_t)c * ES);
                else r.h[v] = c < C ? load_half_granule_edge(row, c, C) : u32x2{0, 0};
            } else {
#pragma unroll
                for (int k = 0; k < Raw<DT>::PIECES; ++k) {
                    const int c = col(t, v) + k * G;
                    if (c + G <= C) r.w[v][k] = load16(row + (int64_t)c * ES);
                    else r.w[v][k] = c < C ? load_granule_edge<DT>(row, c, C) : u32x4{0, 0, 0, 0};
                }
            }
        }
    }

    template <int DT>
    static __device__ __forceinline__ void unpack(const Raw<DT> &raw, float (&r)[E])
    {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (Raw<DT>::PIECES == 0) {
                const u32x4 wide[1] = {{raw.h[v][0], raw.h[v][1], 0, 0}};
                float w[8];
                elems_of<DT>(wide, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) r[4 * v + e] = w[e];
            } else {
                float w[V];
                elems_of<DT>(raw.w[v], w);
#pragma unroll
                for (int e = 0; e < V; ++e) r[V * v + e] = w[e];
            }
        }
    }

    template <int DT>
    static __device__ __forceinline__ void load(const void *p, int64_t off, int t, int C, float (&r)[E])
    {
        Raw<DT> raw;
        fetch<DT>(p, off, t, C, raw);
        unpack<DT>(raw, r);
    }

    template <int DT>
    static __device__ __forceinline__ void store(void *p, int64_t off, int t, int C, const float (&r)[E])
    {
        char *row = static_cast<char *>(p) + off * elem_size(DT);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = col(t, v);
            if (c + V <= C) {
                char *q = row + (int64_t)c * elem_size(DT);
                if constexpr (V * elem_size(DT) == 8) {
                    store8(q, u32x2{pack2<DT>(r[4 * v], r[4 * v + 1]), pack2<DT>(r[4 * v + 2], r[4 * v + 3])});
                } else {
                    float w[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) w[e] = r[V * v + e];
                    store_elems<DT>(q, w);
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (c + e < C) store_elem<DT>(row, c + e, r[V * v + e]);
            }
        }
    }

    // a vector of the parameters' type (float32 or the rows'), `fill` where absent
    template <int DT>
    static __device__ __forceinline__ void params(const void *p, int64_t off, bool f32, int t, int C,
                                                  float fill, float (&r)[E])
    {
        if (!p) {
#pragma unroll
            for (int e = 0; e < E; ++e) r[e] = fill;
        } else if (f32) {
            load<FLASHBEV_F32>(p, off, t, C, r);
        } else {
            load<DT>(p, off, t, C, r);
        }
    }

    // differences from the mean, 0 past C so that they add nothing
    static __device__ __forceinline__ void centre(const float (&r)[E], float mean, int t, int C,
                                                  float (&d)[E])
    {
#pragma unroll
        for (int e = 0; e < E; ++e) d[e] = inside(t, e, C) ? r[e] - mean : 0.0f;
    }

    static __device__ __forceinline__ float sum(const float (&r)[E])
    {
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) s += r[e];
        return s;
    }

    static __device__ __forceinline__ float dot(const float (&a)[E], const float (&b)[E])
    {
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) s = __builtin_fmaf(a[e], b[e], s);
        return s;
    }
};

template <int CTRL>
__device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf,
                                                              true));
}

// Sums of K values over the T lanes of a row, in every lane and in a fixed order.
// Lane exchanges: quad_perm 1 and 2 apart, half-row and row mirrors (whose other
// lanes hold equal sums by then), then the row and half-wavefront swaps.  Across
// wavefronts through `lds` (a slot of its own for each of a row's rounds).
template <int T, int K>
__device__ __forceinline__ void row_sum(float (&v)[K], float *lds)
{
#pragma unroll
    for (int k = 0; k < K; ++k) {
        v[k] += dpp<0xb1>(v[k]);
        v[k] += dpp<0x4e>(v[k]);
        v[k] += dpp<0x141>(v[k]);
        if constexpr (T >= 16) v[k] += dpp<0x140>(v[k]);
        if constexpr (T >= 32) {
            const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v[k]),
                                                            __builtin_bit_cast(unsigned, v[k]), false,
                                                            false);
            const unsigned a = r[0], b = r[1];
            v[k] = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
        }
        if constexpr (T >= 64) {
            const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v[k]),
                                                            __builtin_bit_cast(unsigned, v[k]), false,
                                                            false);
            const unsigned a = r[0], b = r[1];
            v[k] = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
        }
    }
    if constexpr (T > 64) {
        constexpr int W = T / 64;
        const int wave = threadIdx.x >> 6, first = wave / W * W;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) lds[wave * K + k] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) v[k] += lds[(first + w) * K + k];
        }
    }
}

constexpr int kSlot = 64;   // floats of an LDS slot: 16 wavefronts, up to 4 sums

struct Norm {
    const void *x, *residual, *gate, *weight, *bias, *post_weight, *post_bias;
    void *s, *y;
    int64_t ldx, ldr, lds, ldy;
    int64_t M, per_group;      // rows; rows of a sample
    int C, norm, params_f32;
    int post;                  // kind of the post norm
    float eps, scale;
};

// Eight wavefronts a SIMD (64 registers) where 16-bit rows allow it: with 66, a row of
// 4096 left room for three workgroups of four (124 us for 4 x 4096 x 4096, 112 with it).
template <int DT, int SDT, int T, int NV, bool POST>
__global__ void __launch_bounds__(T > 256 ? T : 256, DT != FLASHBEV_F32 && NV == 1 ? 8 : 1)
    norm_forward(Norm p)
{
    using R = Row<T, NV, 8>;
    constexpr int E = R::E;
    __shared__ float slots[T > 64 ? 4 * kSlot : 1];
    const int t = threadIdx.x % T;
    const int64_t row0 = (int64_t)block_index() * R::ROWS;
    if (row0 >= p.M) return;
    const int64_t row = R::ROWS > 1 ? row0 + threadIdx.x / T : row0;
    // lanes past the last row take it again (the sums' barriers need every
    // wavefront) and store nothing
    const bool in = R::ROWS == 1 || row < p.M;
    const int64_t m = in ? row : p.M - 1;
    const float inv = 1.0f / (float)p.C;
    float u[E], a[E], b[E];
    R::template load<DT>(p.x, m * p.ldx, t, p.C, u);
    float res[E];
    if (p.residual) R::template load<SDT>(p.residual, m * p.ldr, t, p.C, res);
    if constexpr (POST) {
        float mean = 0.0f;
        if (p.post == FLASHBLOCK_NORM_LAYER) {
            float v[1] = {R::sum(u)};
            row_sum<T>(v, slots);
            mean = v[0] * inv;
        }
        R::centre(u, mean, t, p.C, u);
        float v[1] = {R::dot(u, u)};
        row_sum<T>(v, slots + kSlot);
        const float r = 1.0f / sqrtf(v[0] * inv + p.eps);
        R::template params<DT>(p.post_weight, 0, p.params_f32, t, p.C, 1.0f, a);
        R::template params<DT>(p.post_bias, 0, p.params_f32, t, p.C, 0.0f, b);
#pragma unroll
        for (int e = 0; e < E; ++e) u[e] = u[e] * r * a[e] + b[e];
    }
    if (p.gate) {
        const uint32_t group = (uint32_t)m / (uint32_t)p.per_group;
        R::template params<DT>(p.gate, (int64_t)group * p.C, p.params_f32, t, p.C, 1.0f, a);
#pragma unroll
        for (int e = 0; e < E; ++e) u[e] *= p.scale * a[e];
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) u[e] *= p.scale;
    }
    if (p.residual) {
#pragma unroll
        for (int e = 0; e < E; ++e) u[e] += res[e];
    }
    // the norm reads the stream as it is stored
    if constexpr (SDT == FLASHBEV_BF16) {
#pragma unroll
        for (int e = 0; e < E; ++e) u[e] = (float)(__bf16)u[e];
    } else if constexpr (SDT == FLASHBEV_F16) {
#pragma unroll
        for (int e = 0; e < E; ++e) u[e] = (float)(_Float16)u[e];
    }
    if (in && p.s) R::template store<SDT>(p.s, m * p.lds, t, p.C, u);
    if (p.norm == FLASHBLOCK_NORM_NONE) return;
    R::template params<DT>(p.weight, 0, p.params_f32, t, p.C, 1.0f, a);
    R::template params<DT>(p.bias, 0, p.params_f32, t, p.C, 0.0f, b);
    float mean = 0.0f;
    if (p.norm == FLASHBLOCK_NORM_LAYER) {
        float v[1] = {R::sum(u)};
        row_sum<T>(v, slots + 2 * kSlot);
        mean = v[0] * inv;
    }
    R::centre(u, mean, t, p.C, u);
    float v[1] = {R::dot(u, u)};
    row_sum<T>(v, slots + 3 * kSlot);
    const float r = 1.0f / sqrtf(v[0] * inv + p.eps);
#pragma unroll
    for (int e = 0; e < E; ++e) u[e] = u[e] * r * a[e] + b[e];
    if (in) R::template store<DT>(p.y, m * p.ldy, t, p.C, u);
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
// A workgroup takes a range of one sample's rows; its lanes keep the vectors'
// gradients of their channels in registers over the range and write them to the
// range's row of `partial` (the sums of its rows' lanes through LDS first), which
// norm_join adds in order.
enum { kGate, kWeight, kBias, kPostWeight, kPostBias, kVectors };

struct NormBackward {
    const void *x, *s, *grad_y, *grad_s, *gate, *weight, *post_weight, *post_bias;
    void *grad_x, *grad_residual;
    float *partial[kVectors];   // [ranges][pld], null where not wanted
    int64_t pld;
    int64_t ldx, lds, ldgy, ldgs, ldgx, ldgr;
    int64_t M, per_group, range;   // rows; of a sample; of a range
    int64_t ranges_per_group;
    int C, norm, post, params_f32;
    float eps, scale;
};

template <int DT, int SDT, int T, int NV, bool POST>
__global__ void __launch_bounds__(T > 256 ? T : 256) norm_backward(NormBackward p)
{
    constexpr int V = 4;
    using R = Row<T, NV, V>;
    constexpr int E = R::E;
    __shared__ float slots[T > 64 ? 3 * kSlot : 1];
    __shared__ float lanes[R::ROWS > 1 ? R::ROWS * T * V : 1];   // one vector's sums at a time
    const int t = threadIdx.x % T, lane_row = threadIdx.x / T;
    const int64_t group = block_index() / p.ranges_per_group, range = block_index() % p.ranges_per_group;
    const int64_t m0 = group * p.per_group + range * p.range;
    if (m0 >= p.M) return;
    int64_t m1 = m0 + p.range;
    if (m1 > (group + 1) * p.per_group) m1 = (group + 1) * p.per_group;
    const float inv = 1.0f / (float)p.C;
    const bool norm = p.norm != FLASHBLOCK_NORM_NONE && p.grad_y;
    const bool reads_x = POST || p.partial[kGate];
    // The vectors of this sample, in registers over the range (read again for each
    // row where a lane holds more than four channels), and their gradients.
    constexpr bool HOLD = NV == 1;
    float weight[E], gate[E], post_weight[E], post_bias[E];
    auto read_weight = [&] { R::template params<DT>(p.weight, 0, p.params_f32, t, p.C, 1.0f, weight); };
    auto read_gate = [&] {
        R::template params<DT>(p.gate, group * p.C, p.params_f32, t, p.C, 1.0f, gate);
#pragma unroll
        for (int e = 0; e < E; ++e) gate[e] *= p.scale;
    };
    auto read_post_weight = [&] {
        if constexpr (POST) R::template params<DT>(p.post_weight, 0, p.params_f32, t, p.C, 1.0f, post_weight);
    };
    auto read_post_bias = [&] {
        if constexpr (POST) R::template params<DT>(p.post_bias, 0, p.params_f32, t, p.C, 0.0f, post_bias);
    };
    if constexpr (HOLD) {
        read_weight();
        read_gate();
        read_post_weight();
        read_post_bias();
    }
    float acc[kVectors][E];
#pragma unroll
    for (int k = 0; k < kVectors; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[k][e] = 0.0f;

    // The next row's loads are in flight while a row's three sums are formed (a row
    // at a time, 8331 x 771 half took 82 us).  Rows of more than 4096 channels have no
    // registers for that.
    constexpr bool AHEAD = NV == 1;
    typename R::template Raw<SDT> raw_ds, raw_s;
    typename R::template Raw<DT> raw_x, raw_g;
    auto fetch = [&](int64_t first) {
        const int64_t m = first + lane_row < m1 ? first + lane_row : m1 - 1;
        if (p.grad_s) R::template fetch<SDT>(p.grad_s, m * p.ldgs, t, p.C, raw_ds);
        if (reads_x) R::template fetch<DT>(p.x, m * p.ldx, t, p.C, raw_x);
        if (norm) {
            R::template fetch<SDT>(p.s, m * p.lds, t, p.C, raw_s);
            R::template fetch<DT>(p.grad_y, m * p.ldgy, t, p.C, raw_g);
        }
    };
    if (m0 < m1) fetch(m0);
    for (int64_t first = m0; first < m1; first += R::ROWS) {
        // lanes past the range take its last row again and add and store nothing
        const bool in = first + lane_row < m1;
        const int64_t m = in ? first + lane_row : m1 - 1;
        float ds[E], x[E], s[E], g[E];
        if (p.grad_s) {
            R::template unpack<SDT>(raw_ds, ds);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) ds[e] = 0.0f;
        }
        if (reads_x) R::template unpack<DT>(raw_x, x);
        if (norm) {
            R::template unpack<SDT>(raw_s, s);
            R::template unpack<DT>(raw_g, g);
        }
        if (AHEAD && first + R::ROWS < m1) fetch(first + R::ROWS);
        float one[3] = {0.0f, 0.0f, 0.0f};
        if (norm) {
            if constexpr (!HOLD) read_weight();
            one[0] = R::sum(s);
            one[1] = R::dot(g, weight);
        }
        if constexpr (POST) one[2] = R::sum(x);
        row_sum<T>(one, slots);
        float two[3] = {0.0f, 0.0f, 0.0f};
        if (norm) {
            R::centre(s, p.norm == FLASHBLOCK_NORM_LAYER ? one[0] * inv : 0.0f, t, p.C, s);
            two[0] = R::dot(s, s);
#pragma unroll
            for (int e = 0; e < E; ++e) two[1] = __builtin_fmaf(g[e] * weight[e], s[e], two[1]);
        }
        if constexpr (POST) {
            R::centre(x, p.post == FLASHBLOCK_NORM_LAYER ? one[2] * inv : 0.0f, t, p.C, x);
            two[2] = R::dot(x, x);
        }
        row_sum<T>(two, slots + kSlot);
        if (norm) {
            const float r = 1.0f / sqrtf(two[0] * inv + p.eps);
            const float mg = p.norm == FLASHBLOCK_NORM_LAYER ? one[1] * inv : 0.0f;
            const float mgs = two[1] * r * inv;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float sh = s[e] * r;
                if (in) {
                    acc[kWeight][e] = __builtin_fmaf(g[e], sh, acc[kWeight][e]);
                    acc[kBias][e] += g[e];
                }
                ds[e] = __builtin_fmaf(r, g[e] * weight[e] - mg - sh * mgs, ds[e]);
            }
        }
        if (in && p.grad_residual)
            R::template store<SDT>(p.grad_residual, m * p.ldgr, t, p.C, ds);
        if (!reads_x && !p.grad_x) {
            if (!AHEAD && first + R::ROWS < m1) fetch(first + R::ROWS);
            continue;
        }
        float rx = 0.0f;
        if constexpr (POST) {
            rx = 1.0f / sqrtf(two[2] * inv + p.eps);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] *= rx;
        }
        if constexpr (!HOLD) read_post_weight();
        if (p.partial[kGate]) {
            if constexpr (!HOLD) read_post_bias();
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float u = x[e];
                if constexpr (POST) u = __builtin_fmaf(u, post_weight[e], post_bias[e]);
                if (in) acc[kGate][e] = __builtin_fmaf(ds[e], u, acc[kGate][e]);
            }
        }
        if constexpr (!HOLD) read_gate();
#pragma unroll
        for (int e = 0; e < E; ++e) ds[e] *= gate[e];
        if constexpr (POST) {
            float three[2] = {0.0f, 0.0f};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (in) {
                    acc[kPostWeight][e] = __builtin_fmaf(ds[e], x[e], acc[kPostWeight][e]);
                    acc[kPostBias][e] += ds[e];
                }
                // ds past C is -r mean(g), not 0
                ds[e] = R::inside(t, e, p.C) ? ds[e] * post_weight[e] : 0.0f;
                three[0] += ds[e];
                three[1] = __builtin_fmaf(ds[e], x[e], three[1]);
            }
            row_sum<T>(three, slots + 2 * kSlot);
            const float mh = p.post == FLASHBLOCK_NORM_LAYER ? three[0] * inv : 0.0f;
            const float mhx = three[1] * inv;
#pragma unroll
            for (int e = 0; e < E; ++e) ds[e] = rx * (ds[e] - mh - x[e] * mhx);
        }
        if (in && p.grad_x) R::template store<DT>(p.grad_x, m * p.ldgx, t, p.C, ds);
        if (!AHEAD && first + R::ROWS < m1) fetch(first + R::ROWS);
    }

#pragma unroll
    for (int k = 0; k < kVectors; ++k) {
        if (!p.partial[k]) continue;
        const float f = k == kGate ? p.scale : 1.0f;
        float *dst = p.partial[k] + (int64_t)block_index() * p.pld;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float w[V];
#pragma unroll
            for (int e = 0; e < V; ++e) w[e] = acc[k][V * v + e];
            if constexpr (R::ROWS > 1) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < V; ++e) lanes[(lane_row * T + t) * V + e] = w[e];
                __syncthreads();
                if (lane_row == 0) {
                    for (int q = 1; q < R::ROWS; ++q)
#pragma unroll
                        for (int e = 0; e < V; ++e) w[e] += lanes[(q * T + t) * V + e];
                }
            }
            const int c = R::col(t, v);
            if (lane_row == 0 && c < p.C) {   // pld is a multiple of 8
#pragma unroll
                for (int e = 0; e < V; ++e) w[e] *= f;
                store_elems<FLASHBEV_F32>(dst + c, w);
            }
        }
    }
}

// sums of the ranges' rows: 16 columns per workgroup, 16 lanes over the ranges of
// each; the gate's ranges of one sample, the others' of all
struct NormJoin {
    const float *partial[kVectors];
    void *out[kVectors];
    int64_t pld;
    int64_t ranges[kVectors];   // summed for one output row
    int64_t rows[kVectors];     // output rows
    int which[kVectors];        // vectors in use, in order
    int col_blocks, C;
    int out_f32;
    uint32_t blocks;
};

template <int DT>
__global__ void __launch_bounds__(256) norm_join(NormJoin p)
{
    if (block_index() >= p.blocks) return;
    int64_t b = block_index() / p.col_blocks;
    int k = 0;
    while (b >= p.rows[p.which[k]]) b -= p.rows[p.which[k++]];
    k = p.which[k];
    const int n = (int)(block_index() % p.col_blocks) * 16 + (threadIdx.x & 15), r0 = threadIdx.x >> 4;
    float s = 0.0f;
    if (n < p.C) {
        const float *src = p.partial[k] + b * p.ranges[k] * p.pld + n;
#pragma unroll 8
        for (int64_t r = r0; r < p.ranges[k]; r += 16) s += src[r * p.pld];
    }
    __shared__ float part[16][17];
    part[r0][threadIdx.x & 15] = s;
    __syncthreads();
    if (r0 != 0 || n >= p.C) return;
    s = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) s += part[r][threadIdx.x];
    if (p.out_f32) store_elem<FLASHBEV_F32>(p.out[k], b * p.C + n, s);
    else store_elem<DT>(p.out[k], b * p.C + n, s);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
// The lanes of a row: a vector of `v` channels each, up to 1024 lanes.  Forward, 8
// channels; backward, 4, for its five sums and four vectors in registers (with 8, at
// 145 to 200 of them, two or three wavefronts fit a SIMD: 40000 x 256 bfloat16 took 52
// us and takes 34, 16384 x 4096 303 and 197).  Wider rows of the backward spill: up to
// 8192 channels 512 lanes with 256 registers do it less than 1024 with 128 (8192 x 8192
// with both norms 483 us and 749, without a post norm 261 and 244).
struct Shape {
    int lanes, rows, threads;   // of a row; rows and threads of a workgroup
};

Shape shape_of(int C, int v)
{
    int t = 8;
    while (t < 1024 && v * t < C) t *= 2;
    if (v == 4 && C > 4096 && C <= 8192) t = 512;
    return {t, t >= 256 ? 1 : 256 / t, t > 256 ? t : 256};
}

template <int DT, int SDT, bool POST>
const void *forward_kernel(int C)
{
    if (C > 8192) return (const void *)norm_forward<DT, SDT, 1024, 2, POST>;
    switch (shape_of(C, 8).lanes) {
    case 8: return (const void *)norm_forward<DT, SDT, 8, 1, POST>;
    case 16: return (const void *)norm_forward<DT, SDT, 16, 1, POST>;
    case 32: return (const void *)norm_forward<DT, SDT, 32, 1, POST>;
    case 64: return (const void *)norm_forward<DT, SDT, 64, 1, POST>;
    case 128: return (const void *)norm_forward<DT, SDT, 128, 1, POST>;
    case 256: return (const void *)norm_forward<DT, SDT, 256, 1, POST>;
    case 512: return (const void *)norm_forward<DT, SDT, 512, 1, POST>;
    default: return (const void *)norm_forward<DT, SDT, 1024, 1, POST>;
    }
}

template <int DT, int SDT, bool POST>
const void *backward_kernel(int C)
{
    if (C > 8192) return (const void *)norm_backward<DT, SDT, 1024, 4, POST>;
    if (C > 4096) return (const void *)norm_backward<DT, SDT, 512, 4, POST>;
    switch (shape_of(C, 4).lanes) {
    case 8: return (const void *)norm_backward<DT, SDT, 8, 1, POST>;
    case 16: return (const void *)norm_backward<DT, SDT, 16, 1, POST>;
    case 32: return (const void *)norm_backward<DT, SDT, 32, 1, POST>;
    case 64: return (const void *)norm_backward<DT, SDT, 64, 1, POST>;
    case 128: return (const void *)norm_backward<DT, SDT, 128, 1, POST>;
    case 256: return (const void *)norm_backward<DT, SDT, 256, 1, POST>;
    case 512: return (const void *)norm_backward<DT, SDT, 512, 1, POST>;
    default: return (const void *)norm_backward<DT, SDT, 1024, 1, POST>;
    }
}

template <bool BACKWARD, bool POST>
const void *kernel_of(int dt, int sdt, int C)
{
#define FLASHBLOCK_PICK(D, S) \
    (BACKWARD ? backward_kernel<D, S, POST>(C) : forward_kernel<D, S, POST>(C))
    if (dt == FLASHBEV_F32) return FLASHBLOCK_PICK(FLASHBEV_F32, FLASHBEV_F32);
    if (dt == FLASHBEV_F16)
        return sdt == FLASHBEV_F32 ? FLASHBLOCK_PICK(FLASHBEV_F16, FLASHBEV_F32)
                                   : FLASHBLOCK_PICK(FLASHBEV_F16, FLASHBEV_F16);
    return sdt == FLASHBEV_F32 ? FLASHBLOCK_PICK(FLASHBEV_BF16, FLASHBEV_F32)
                               : FLASHBLOCK_PICK(FLASHBEV_BF16, FLASHBEV_BF16);
#undef FLASHBLOCK_PICK
}

bool known_kind(int k) { return k >= FLASHBLOCK_NORM_NONE && k <= FLASHBLOCK_NORM_RMS; }

int check_norm(const flashblock_norm *p)
{
    if (!p) return FLASHBEV_ERR_NULLPTR;
    if (p->M < 0 || p->C < 0 || p->groups < 1 || p->M % p->groups) return FLASHBEV_ERR_SHAPE;
    if (!known_dtype(p->dtype) ||
        (p->stream_dtype != p->dtype && p->stream_dtype != FLASHBEV_F32) ||
        (p->param_dtype != p->dtype && p->param_dtype != FLASHBEV_F32))
        return FLASHBEV_ERR_DTYPE;
    if (!known_kind(p->norm) || !known_kind(p->post_norm) ||
        (p->norm == FLASHBLOCK_NORM_NONE && p->post_norm == FLASHBLOCK_NORM_NONE) ||
        !finite_value(p->scale) || !finite_value(p->eps) || !(p->eps > 0.0f))
        return FLASHBEV_ERR_VALUE;
    if (p->M > FLASHBLOCK_ROWS_MAX || p->C > FLASHBLOCK_NORM_MAX) return FLASHBEV_ERR_UNSUPPORTED;
    return FLASHBEV_OK;
}

int check_params(const flashblock_norm *p, const flashblock_norm_params *v)
{
    if (!v) return FLASHBEV_ERR_NULLPTR;
    if ((p->norm == FLASHBLOCK_NORM_NONE && (v->weight || v->bias)) ||
        (p->post_norm == FLASHBLOCK_NORM_NONE && (v->post_weight || v->post_bias)))
        return FLASHBEV_ERR_VALUE;
    for (const void *q : {v->gate, v->weight, v->bias, v->post_weight, v->post_bias})
        if (misaligned(q, elem_size(p->param_dtype))) return FLASHBEV_ERR_ALIGN;
    return FLASHBEV_OK;
}

struct NormRange {
    const void *p;
    uint64_t n;
};

int check_overlaps(const NormRange *outs, int n_outs, const NormRange *ins, int n_ins, int out_skip,
                   int in_skip)
{
    for (int o = 0; o < n_outs; ++o) {
        for (int i = 0; i < n_ins; ++i)
            if (!(o == out_skip && i == in_skip) &&
                ranges_overlap(outs[o].p, outs[o].n, ins[i].p, ins[i].n))
                return FLASHBEV_ERR_ALIAS;
        for (int q = 0; q < o; ++q)
            if (ranges_overlap(outs[o].p, outs[o].n, outs[q].p, outs[q].n)) return FLASHBEV_ERR_ALIAS;
    }
    return FLASHBEV_OK;
}

// The ranges of a backward: about four workgroups of 256 threads per CU, of four
// rows for each of a workgroup's lanes or more, none across two samples.
struct NormRanges {
    int64_t per_group, range, per;   // rows of a sample, rows of a range, ranges of a sample
    uint64_t bytes;                  // of one vector's partial sums
    int64_t pld;
};

NormRanges plan_ranges(const flashblock_norm *p)
{
    NormRanges r;
    const Shape s = shape_of(p->C, 4);
    r.per_group = p->M / p->groups;
    const int64_t want = (int64_t)256 * 4 * 256 / s.threads;
    int64_t per = (want + p->groups - 1) / p->groups;
    const int64_t most = r.per_group / (4 * s.rows);
    if (per > most) per = most;
    if (per < 1) per = 1;
    r.range = (r.per_group + per - 1) / per;
    if (r.range < 1) r.range = 1;
    r.per = (r.per_group + r.range - 1) / r.range;
    r.pld = (p->C + 7) / 8 * 8;
    r.bytes = ((uint64_t)p->groups * r.per * r.pld * 4 + 255) / 256 * 256;
    return r;
}

void *const *grad_list(const flashblock_norm_grads *g, void *(&v)[kVectors])
{
    v[kGate] = g ? g->gate : nullptr;
    v[kWeight] = g ? g->weight : nullptr;
    v[kBias] = g ? g->bias : nullptr;
    v[kPostWeight] = g ? g->post_weight : nullptr;
    v[kPostBias] = g ? g->post_bias : nullptr;
    return v;
}

uint64_t norm_workspace(const flashblock_norm *p, void *const *grads)
{
    int n = 0;
    for (int k = 0; k < kVectors; ++k) n += grads[k] != nullptr;
    return n ? n * plan_ranges(p).bytes : 0;
}

int check_norm_rows(const void *p, int64_t rows, int64_t ld, int64_t width, int es)
{
    if (!p) return FLASHBEV_ERR_NULLPTR;
    if (rows && ld < width) return FLASHBEV_ERR_SHAPE;
    if (ld > FLASHBLOCK_LD_MAX) return FLASHBEV_ERR_UNSUPPORTED;
    return misaligned(p, es) ? FLASHBEV_ERR_ALIGN : FLASHBEV_OK;
}

}  // namespace

extern "C" {

int flashblock_norm_forward(const flashblock_norm *p, const flashblock_norm_params *v, const void *x,
                            const void *residual, void *s, void *y, void *stream)
{
    int rc = check_norm(p);
    if (rc || (rc = check_params(p, v))) return rc;
    if (p->M == 0 || p->C == 0) return FLASHBEV_OK;
    const int es = elem_size(p->dtype), ss = elem_size(p->stream_dtype);
    const int ps = elem_size(p->param_dtype);
    const bool has_y = p->norm != FLASHBLOCK_NORM_NONE;
    if (!has_y && y) return FLASHBEV_ERR_VALUE;
    if (!has_y && !s) return FLASHBEV_ERR_NULLPTR;
    if ((rc = check_norm_rows(x, p->M, p->ldx, p->C, es)) ||
        (residual && (rc = check_norm_rows(residual, p->M, p->ldr, p->C, ss))) ||
        (s && (rc = check_norm_rows(s, p->M, p->lds, p->C, ss))) ||
        (has_y && (rc = check_norm_rows(y, p->M, p->ldy, p->C, es))))
        return rc;
    const uint64_t vec = (uint64_t)p->C * ps;
    const NormRange ins[] = {{x, span_bytes(p->M, p->ldx, p->C, es)},
                             {residual, span_bytes(p->M, p->ldr, p->C, ss)},
                             {v->gate, vec * p->groups},
                             {v->weight, vec},
                             {v->bias, vec},
                             {v->post_weight, vec},
                             {v->post_bias, vec}};
    const NormRange outs[] = {{s, span_bytes(p->M, p->lds, p->C, ss)},
                              {y, span_bytes(p->M, p->ldy, p->C, es)}};
    const bool in_place = residual && residual == s && p->ldr == p->lds;
    if ((rc = check_overlaps(outs, 2, ins, 7, in_place ? 0 : -1, in_place ? 1 : -1))) return rc;
    Norm n{x, residual, v->gate, v->weight, v->bias, v->post_weight, v->post_bias, s, y,
           p->ldx, p->ldr, p->lds, p->ldy, p->M, p->M / p->groups, p->C, p->norm,
           p->param_dtype == FLASHBEV_F32, p->post_norm, p->eps, p->scale};
    const Shape h = shape_of(p->C, 8);
    const void *fn = p->post_norm != FLASHBLOCK_NORM_NONE
                         ? kernel_of<false, true>(p->dtype, p->stream_dtype, p->C)
                         : kernel_of<false, false>(p->dtype, p->stream_dtype, p->C);
    return launch_rows(fn, (uint64_t)(p->M + h.rows - 1) / h.rows, h.threads, n,
                       static_cast<hipStream_t>(stream));
}

int flashblock_norm_backward_workspace_size(const flashblock_norm *p,
                                            const flashblock_norm_grads *grads, uint64_t *bytes)
{
    if (!bytes) return FLASHBEV_ERR_NULLPTR;
    if (const int rc = check_norm(p)) return rc;
    void *g[kVectors];
    *bytes = p->C ? norm_workspace(p, grad_list(grads, g)) : 0;
    return FLASHBEV_OK;
}

int flashblock_norm_backward(const flashblock_norm *p, const flashblock_norm_params *v,
                             const void *grad_y, const void *grad_s, const void *x, const void *s,
                             void *grad_x, int64_t ldgx, void *grad_residual, int64_t ldgr,
                             const flashblock_norm_grads *grads, void *workspace,
                             uint64_t workspace_bytes, void *stream)
{
    int rc = check_norm(p);
    if (rc || (rc = check_params(p, v))) return rc;
    if (p->C == 0) return FLASHBEV_OK;
    void *g[kVectors];
    grad_list(grads, g);
    const int es = elem_size(p->dtype), ss = elem_size(p->stream_dtype);
    const int ps = elem_size(p->param_dtype);
    bool vectors = false;
    for (int k = 0; k < kVectors; ++k) {
        vectors |= g[k] != nullptr;
        if (misaligned(g[k], ps)) return FLASHBEV_ERR_ALIGN;
    }
    if (p->norm == FLASHBLOCK_NORM_NONE && (grad_y || g[kWeight] || g[kBias])) return FLASHBEV_ERR_VALUE;
    if (p->post_norm == FLASHBLOCK_NORM_NONE && (g[kPostWeight] || g[kPostBias]))
        return FLASHBEV_ERR_VALUE;
    if (p->M > 0 && ((!grad_x && !grad_residual && !vectors) || (!grad_y && !grad_s)))
        return FLASHBEV_ERR_NULLPTR;
    if (!vectors && p->M == 0) return FLASHBEV_OK;
    const bool norm = p->norm != FLASHBLOCK_NORM_NONE && grad_y;
    const bool reads_x = p->post_norm != FLASHBLOCK_NORM_NONE || g[kGate];
    if (p->M > 0) {
        if ((grad_y && (rc = check_norm_rows(grad_y, p->M, p->ldy, p->C, es))) ||
            (grad_s && (rc = check_norm_rows(grad_s, p->M, p->ldr, p->C, ss))) ||
            (reads_x && (rc = check_norm_rows(x, p->M, p->ldx, p->C, es))) ||
            (norm && (rc = check_norm_rows(s, p->M, p->lds, p->C, ss))) ||
            (grad_x && (rc = check_norm_rows(grad_x, p->M, ldgx, p->C, es))) ||
            (grad_residual && (rc = check_norm_rows(grad_residual, p->M, ldgr, p->C, ss))))
            return rc;
    }
    const uint64_t need = norm_workspace(p, g);
    if (need) {
        if (!workspace) return FLASHBEV_ERR_NULLPTR;
        if (misaligned(workspace, 256)) return FLASHBEV_ERR_ALIGN;
        if (workspace_bytes < need) return FLASHBEV_ERR_SCRATCH;
    }
    const uint64_t vec = (uint64_t)p->C * ps;
    const NormRange ins[] = {{grad_y, span_bytes(p->M, p->ldy, p->C, es)},
                             {grad_s, span_bytes(p->M, p->ldr, p->C, ss)},
                             {reads_x ? x : nullptr, span_bytes(p->M, p->ldx, p->C, es)},
                             {norm ? s : nullptr, span_bytes(p->M, p->lds, p->C, ss)},
                             {v->gate, vec * p->groups},
                             {v->weight, vec},
                             {v->post_weight, vec},
                             {v->post_bias, vec}};
    const NormRange outs[] = {{grad_x, span_bytes(p->M, ldgx, p->C, es)},
                              {grad_residual, span_bytes(p->M, ldgr, p->C, ss)},
                              {g[kGate], vec * p->groups},
                              {g[kWeight], vec},
                              {g[kBias], vec},
                              {g[kPostWeight], vec},
                              {g[kPostBias], vec},
                              {need ? workspace : nullptr, need}};
    if ((rc = check_overlaps(outs, 8, ins, 8, -1, -1))) return rc;

    hipStream_t st = static_cast<hipStream_t>(stream);
    const NormRanges q = plan_ranges(p);
    NormBackward n{};
    n.x = x;
    n.s = s;
    n.grad_y = grad_y;
    n.grad_s = grad_s;
    n.gate = v->gate;
    n.weight = v->weight;
    n.post_weight = v->post_weight;
    n.post_bias = v->post_bias;
    n.grad_x = grad_x;
    n.grad_residual = grad_residual;
    n.pld = q.pld;
    n.ldx = p->ldx;
    n.lds = p->lds;
    n.ldgy = p->ldy;
    n.ldgs = p->ldr;
    n.ldgx = ldgx;
    n.ldgr = ldgr;
    n.M = p->M;
    n.per_group = q.per_group;
    n.range = q.range;
    n.ranges_per_group = q.per;
    n.C = p->C;
    n.norm = p->norm;
    n.post = p->post_norm;
    n.params_f32 = p->param_dtype == FLASHBEV_F32;
    n.eps = p->eps;
    n.scale = p->scale;
    NormJoin j{};
    j.pld = q.pld;
    j.col_blocks = (p->C + 15) / 16;
    j.C = p->C;
    j.out_f32 = n.params_f32;
    int used = 0;
    int64_t out_rows = 0;
    char *ws = static_cast<char *>(workspace);
    for (int k = 0; k < kVectors; ++k) {
        if (!g[k]) continue;
        n.partial[k] = reinterpret_cast<float *>(ws);
        ws += q.bytes;
        j.partial[k] = n.partial[k];
        j.out[k] = g[k];
        j.rows[k] = k == kGate ? p->groups : 1;
        j.ranges[k] = k == kGate ? q.per : p->groups * q.per;
        j.which[used++] = k;
        out_rows += j.rows[k];
    }
    if (p->M > 0) {
        const Shape h = shape_of(p->C, 4);
        const void *fn = p->post_norm != FLASHBLOCK_NORM_NONE
                             ? kernel_of<true, true>(p->dtype, p->stream_dtype, p->C)
                             : kernel_of<true, false>(p->dtype, p->stream_dtype, p->C);
        if ((rc = launch_rows(fn, (uint64_t)p->groups * q.per, h.threads, n, st))) return rc;
    } else {
        for (int k = 0; k < kVectors; ++k) j.ranges[k] = 0;   // sums of nothing
    }
    if (!used) return FLASHBEV_OK;
    const void *fn = p->dtype == FLASHBEV_F32   ? (const void *)norm_join<FLASHBEV_F32>
                     : p->dtype == FLASHBEV_F16 ? (const void *)norm_join<FLASHBEV_F16>
                                                : (const void *)norm_join<FLASHBEV_BF16>;
    const uint64_t blocks = (uint64_t)out_rows * j.col_blocks;
    j.blocks = (uint32_t)blocks;   // (more than 32 bits are refused below)
    return launch_rows(fn, blocks, 256, j, st);
}

}  // extern "C"

// Helpers of the encoder block's operators (flashlinear.hip, flashnorm.hip): 8- and
// 16-byte vectors at any element alignment, conversion of stored elements to
// float32 and back, and on the host the byte ranges of strided tensors.
#pragma once

#include "block/flashblock.h"
#include "hip_common.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));   // 16 bytes at any 16-bit alignment

// Rows of odd widths start at any element; gfx950 loads and stores 16 bytes at
// any 2-byte address in one instruction.
__device__ __forceinline__ u32x4 load16(const void *p)
{
    return *reinterpret_cast<const u32x4_any *>(p);
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));

__device__ __forceinline__ u32x2 load8(const void *p)
{
    return *reinterpret_cast<const u32x2_any *>(p);
}

__device__ __forceinline__ void store8(void *p, u32x2 v)
{
    *reinterpret_cast<u32x2_any *>(p) = v;
}

__device__ __forceinline__ void store16(void *p, u32x4 v)
{
    *reinterpret_cast<u32x4_any *>(p) = v;
}

constexpr int elem_size(int dt) { return dt == FLASHBEV_F32 ? 4 : 2; }

// The workgroups of a row of the grid (2^31 threads at most), and a workgroup's number
// over all rows.
constexpr uint32_t kGridRow = 1u << 21;

__device__ __forceinline__ uint32_t block_index() { return blockIdx.y * kGridRow + blockIdx.x; }

// One stored element as float32 (exact) and a float32 rounded to it.
template <int DT>
__device__ __forceinline__ float load_elem(const void *p, int64_t i)
{
    if constexpr (DT == FLASHBEV_F32) {
        return static_cast<const float *>(p)[i];
    } else if constexpr (DT == FLASHBEV_F16) {
        return (float)static_cast<const _Float16 *>(p)[i];
    } else {
        return (float)static_cast<const __bf16 *>(p)[i];
    }
}

template <int DT>
__device__ __forceinline__ void store_elem(void *p, int64_t i, float v)
{
    if constexpr (DT == FLASHBEV_F32) {
        static_cast<float *>(p)[i] = v;
    } else if constexpr (DT == FLASHBEV_F16) {
        static_cast<_Float16 *>(p)[i] = (_Float16)v;
    } else {
        static_cast<__bf16 *>(p)[i] = (__bf16)v;
    }
}

// V consecutive elements (V times the element size is a multiple of 16 bytes)
// as float32, in 16-byte vectors.
template <int DT, int W, int V>
__device__ __forceinline__ void elems_of(const u32x4 (&raw)[W], float (&v)[V])
{
    static_assert(V * elem_size(DT) == W * 16, "whole vectors");
#pragma unroll
    for (int q = 0; q < W; ++q) {
        const u32x4 r = raw[q];
        if constexpr (DT == FLASHBEV_F32) {
            const f32x4 f = __builtin_bit_cast(f32x4, r);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] = f[e];
        } else if constexpr (DT == FLASHBEV_BF16) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[8 * q + 2 * e] = __builtin_bit_cast(float, r[e] << 16);
                v[8 * q + 2 * e + 1] = __builtin_bit_cast(float, r[e] & 0xffff0000u);
            }
        } else {
            typedef _Float16 h2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t w = r[e];
                const h2 h = __builtin_bit_cast(h2, w);
                v[8 * q + 2 * e] = (float)h[0];
                v[8 * q + 2 * e + 1] = (float)h[1];
            }
        }
    }
}

template <int DT, int V>
__device__ __forceinline__ void load_elems(const void *p, float (&v)[V])
{
    constexpr int W = V * elem_size(DT) / 16;
    u32x4 raw[W];
#pragma unroll
    for (int q = 0; q < W; ++q) raw[q] = load16(static_cast<const char *>(p) + 16 * q);
    elems_of<DT>(raw, v);
}

template <int DT>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    if constexpr (DT == FLASHBEV_BF16) {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, b2{(__bf16)a, (__bf16)b});
    } else {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, h2{(_Float16)a, (_Float16)b});
    }
}

template <int DT, int V>
__device__ __forceinline__ void store_elems(void *p, const float (&v)[V])
{
    constexpr int E = 16 / elem_size(DT);
    static_assert(V % E == 0, "whole vectors");
#pragma unroll
    for (int q = 0; q < V / E; ++q) {
        u32x4 r;
        if constexpr (DT == FLASHBEV_F32) {
            r = __builtin_bit_cast(u32x4, f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]});
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = pack2<DT>(v[8 * q + 2 * e], v[8 * q + 2 * e + 1]);
        }
        store16(static_cast<char *>(p) + 16 * q, r);
    }
}

// 16 bytes at element `i` of a row that ends at element `end`, zeros past it: the
// row's last 16 bytes where they begin before `i`, shifted down.
template <int DT>
__device__ __forceinline__ u32x4 load_granule_edge(const char *row, int i, int end)
{
    constexpr int ES = elem_size(DT), E = 16 / ES;
    u32x4 v = {0, 0, 0, 0};
    if (end >= E) {
        const int at = min(i, end - E);
        v = load16(row + (int64_t)at * ES);
        const int shift = (i - at) * ES * 8;   // bits
        uint64_t lo = v[0] | (uint64_t)v[1] << 32, hi = v[2] | (uint64_t)v[3] << 32;
        if (shift >= 64) {
            lo = shift < 128 ? hi >> (shift - 64) : 0;
            hi = 0;
        } else if (shift > 0) {
            lo = lo >> shift | hi << (64 - shift);
            hi >>= shift;
        }
        v = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
    } else {
#pragma unroll
        for (int q = 0; q < E; ++q) {
            if (i + q >= end) continue;
            if constexpr (DT == FLASHBEV_F32) {
                v[q] = reinterpret_cast<const uint32_t *>(row)[i + q];
            } else {
                v[q >> 1] |= (uint32_t)reinterpret_cast<const uint16_t *>(row)[i + q] << (16 * (q & 1));
            }
        }
    }
    return v;
}

// The same for 8 bytes of 16-bit elements.
__device__ __forceinline__ u32x2 load_half_granule_edge(const char *row, int i, int end)
{
    uint64_t v = 0;
    if (end >= 4) {
        const int at = min(i, end - 4);
        const u32x2 w = load8(row + (int64_t)at * 2);
        const int shift = (i - at) * 16;
        v = shift < 64 ? (w[0] | (uint64_t)w[1] << 32) >> shift : 0;
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (i + q < end) v |= (uint64_t)reinterpret_cast<const uint16_t *>(row)[i + q] << (16 * q);
    }
    return u32x2{(uint32_t)v, (uint32_t)(v >> 32)};
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
inline bool ranges_overlap(const void *a, uint64_t na, const void *b, uint64_t nb)
{
    if (!na || !nb || !a || !b) return false;
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    return a0 < b0 + nb && b0 < a0 + na;
}

// bytes from the first to the last element of `rows` rows at a stride
inline uint64_t span_bytes(int64_t rows, int64_t ld, int64_t width, int es)
{
    return rows <= 0 || width <= 0 ? 0 : ((uint64_t)(rows - 1) * ld + width) * es;
}

inline bool finite_value(float v) { return v == v && v - v == 0.0f; }

inline bool known_dtype(int dt) { return dt >= FLASHBEV_F32 && dt <= FLASHBEV_BF16; }

inline bool misaligned(const void *p, int a) { return ((uintptr_t)p & (uintptr_t)(a - 1)) != 0; }

template <class P>
int launch_kernel(const void *fn, uint64_t blocks, int threads, P &p, size_t lds, hipStream_t st,
                  unsigned grid_rows = 1)
{
    if (blocks == 0) return FLASHBEV_OK;
    if (blocks > 0x7fffffffull || !grid_fits((int64_t)blocks, threads)) return FLASHBEV_ERR_UNSUPPORTED;
    void *args[] = {&p};
    return hipLaunchKernel(fn, dim3((unsigned)blocks, grid_rows), dim3(threads), args, lds, st) == hipSuccess
               ? FLASHBEV_OK : FLASHBEV_ERR_HIP;
}

// For kernels that go by block_index() and leave at once past their last workgroup: more
// workgroups than one row of the grid takes go over several.
template <class P>
int launch_rows(const void *fn, uint64_t blocks, int threads, P &p, hipStream_t st)
{
    if (blocks > 0x7fffffffull) return FLASHBEV_ERR_UNSUPPORTED;
    if (blocks <= kGridRow) return launch_kernel(fn, blocks, threads, p, 0, st);
    return launch_kernel(fn, kGridRow, threads, p, 0, st, (unsigned)((blocks + kGridRow - 1) / kGridRow));
}

}  // namespace

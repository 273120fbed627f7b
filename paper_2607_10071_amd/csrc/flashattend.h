// What the forward and the backward of attention share (flashattend.hip,
// flashattend_grad.hip): a call's arguments in device form, panels of rows in LDS and the
// fragments that the matrix units take from them, masks, and on the host the checks.
//
// Rows.  The query heads that share a head of the states are rows of one problem: for batch b
// and head g of the states, row r is query r / share and query head g share + r % share.  Keys
// and values are then read once for all of them, their gradients are sums over rows, and the
// single new token of a serving step has `share` rows.
//
// Products.  A wavefront forms the scores of 32 keys and 32 rows with keys down and rows
// across: a lane then holds 16 of its row's scores (row lane % 32, keys 8 k + 4 h + 0..3 for
// k = 0..3 and its half h), a row's maximum and sum stay within a lane and its other half, and the
// same registers, packed, are the operand of the product with v, whose reduction runs over
// the keys in the order that the registers have.
#pragma once

#include <algorithm>

#include "block/flashlayer.h"
#include "block_mma.h"
#include "block_stream.h"

namespace {

constexpr float kLog2 = 1.4426950408889634f;   // of e
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float log2_fast(float v) { return __builtin_amdgcn_logf(v); }

struct Attend {
    const char *q, *k, *v, *g;       // g: the output's gradient
    char *o;
    const char *mask;                // null: none
    const int32_t *lengths;          // null: all Lk
    int64_t qb, qr, qh, kb, kr, kh, vb, vr, vh, ob, orow, oh, mb, mh, mr;   // bytes
    int B, Lq, Lk, H, Hk, D;
    int share, rows;                 // rows = Lq share
    uint32_t share_inv;              // ceil(2^32 / share), share > 1
    int kind;                        // flashlayer_mask
    int drops;                       // a boolean mask that is the same for all rows of a problem
    const uint32_t *words;           // with drops, without other masks: bits of the keys that take part,
    int64_t words_b, words_g;        // `words_b` words from batch to batch, `words_g` from head to head
    int Dk;                          // channels of k's and v's rows: D, or that up to whole granules
    float scale;
    int tiles;                       // of rows (forward, grad_q) or of keys (grad_k, grad_v)
    int splits;
    uint32_t blocks, per_xcd;

    __device__ __forceinline__ void row(int r, int &i, int &j) const   // query, head within the share
    {
        i = share > 1 ? (int)__umulhi((uint32_t)r, share_inv) : r;
        j = r - i * share;
    }

    __device__ __forceinline__ int keys(int b) const
    {
        return lengths ? max(0, min(lengths[b], Lk)) : Lk;
    }
};

// An XCD's workgroups (one in eight of the grid) take a contiguous share of the items: the
// tiles that read the same keys meet in one L2.
__device__ __forceinline__ uint32_t item_of(const Attend &p)
{
    return blockIdx.x / 8 < p.per_xcd ? blockIdx.x % 8 * p.per_xcd + blockIdx.x / 8 : p.blocks;
}

// R rows of up to DP elements in LDS, 16-byte granules.  Rows stand an odd multiple of 64 bytes
// apart and granule g of row r at place g ^ (r / 4 & 3): 16 lanes that read one granule of 16
// rows use all 64 banks, and so do half a wavefront's transposed reads of 4 rows x 64 bytes.
template <int DT, int DP, int R>
struct Panel {
    static constexpr int ES = elem_size(DT), E = 16 / ES;
    static constexpr int GR = DP * ES / 16;                    // granules of a row
    static constexpr int STRIDE = DP * ES + (DP * ES / 64 % 2 ? 0 : 64);
    static constexpr int BYTES = R * STRIDE;
    static constexpr int RP = 256 / GR < R ? 256 / GR : R;     // rows that the workgroup takes at once
    static constexpr int G = (R + RP - 1) / RP;                // granules of a thread
    static constexpr int CHUNKS = GR / 2;                      // of an MFMA's reduction, in DP
    static constexpr int STEPS = E == 8 ? 2 : 4;               // ..., in 32 rows

    static __device__ __forceinline__ int place(int row, int g) { return row * STRIDE + ((g ^ (row >> 2 & 3)) << 4); }

    // A row's granule, zeros past its D elements.
    static __device__ __forceinline__ u32x4 granule(const char *row, int g, int D)
    {
        if ((g + 1) * E <= D) return load16(row + g * 16);
        if (g * E < D) return load_granule_edge<DT>(row, g * E, D);
        return u32x4{0, 0, 0, 0};
    }

    // Rows on their way from memory to LDS: thread tid takes granule tid % GR of rows tid / GR, + RP,
    // ..., and a tile's loads are under way while the last one is worked on.
    struct Mover {
        int row, g;
        uint32_t off;      // of the granule from the tile's first row
        bool mine;         // D a multiple of E: the granule is there

        __device__ __forceinline__ void start(int tid, int D, int64_t stride)
        {
            row = tid / GR;
            g = tid - row * GR;
            off = (uint32_t)row * (uint32_t)stride + g * 16;
            mine = row < RP && g * E < D;
        }

        // whether the thread's i-th row lies within the tile
        __device__ __forceinline__ bool inside(int i) const { return R % RP == 0 || i < G - 1 || row + i * RP < R; }

        __device__ __forceinline__ void clear(u32x4 (&v)[G]) const
        {
#pragma unroll
            for (int i = 0; i < G; ++i) v[i] = u32x4{0, 0, 0, 0};
        }

        // `base`: the tile's first row, of which `left` >= 1 are there; past them the last one
        // again, whose scores the caller cuts
        __device__ __forceinline__ void load(u32x4 (&v)[G], const char *base, int64_t stride, int left) const
        {
            if (!mine) return;
            if (left >= R) {
#pragma unroll
                for (int i = 0; i < G; ++i)
                    if (inside(i)) v[i] = load16(base + i * RP * stride + off);
            } else {
                asm volatile("");
#pragma unroll
                for (int i = 0; i < G; ++i)
                    v[i] = load16(base + (uint32_t)min(row + i * RP, left - 1) * (uint32_t)stride + g * 16);
            }
        }

        __device__ __forceinline__ void store(const u32x4 (&v)[G], char *lds) const
        {
            if (row >= RP) return;
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (inside(i)) *reinterpret_cast<u32x4 *>(lds + place(row + i * RP, g)) = v[i];
        }

        // Any width, rows that there(i) says are wanted, zeros for the others: when it is their
        // turn.
        template <class There>
        __device__ __forceinline__ void copy(char *lds, const char *base, int64_t stride, int left, int D,
                                             There there) const
        {
            if (row >= RP) return;
#pragma unroll 1
            for (int i = row; i < R; i += RP) {
                u32x4 v = {0, 0, 0, 0};
                if (i < left && there(i)) v = granule(base + i * stride, g, D);
                *reinterpret_cast<u32x4 *>(lds + place(i, g)) = v;
            }
        }
    };

    // A lane's places in a panel: all it reads is at these and distances that are known ahead.
    struct Reader {
        int along_[2], across_[2];

        __device__ __forceinline__ void start(int lane)
        {
            const int i = lane & 31, h = lane >> 5;
#pragma unroll
            for (int e = 0; e < 2; ++e) along_[e] = place(i, 2 * e + h);
            if constexpr (ES == 2) {
                const int j = lane & 15, a = lane >> 4 & 1, b = j >> 1 & 1;
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    across_[q] = (4 * h + (j >> 2)) * STRIDE + ((2 * (a ^ q) + (b ^ h)) << 4) + (j & 1) * 8;
            } else {
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    across_[e] = 4 * h * STRIDE + ((i >> 2 ^ (2 * e + h)) << 4) + (i & 3) * 4;
            }
        }

        // Reduction along the rows' elements: the lane's granule of chunk c of row r0 + lane % 32.
        __device__ __forceinline__ u32x4 along(const char *lds, int r0, int c) const
        {
            return *reinterpret_cast<const u32x4 *>(lds + along_[c & 1] + r0 * STRIDE + (c >> 1) * 64);
        }

        // Reduction over the rows, in the order of a block's registers (above): the lane's granule
        // of step u of rows r0 .. r0 + 31 for element d0 + lane % 32.
        __device__ __forceinline__ u32x4 across(const char *lds, int r0, int u, int d0) const
        {
            u32x4 v;
            if constexpr (ES == 2) {
                // ds_read_b64_tr_b16: 16 lanes take 4 rows x 16 elements, each ends with one
                // element's 4 rows
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const s16x4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s16x4 *)(lds + across_[q] + (r0 + 16 * u + 8 * q) * STRIDE +
                                                                    d0 * 2));
                    const uint64_t w = __builtin_bit_cast(uint64_t, t);
                    v[2 * q] = (uint32_t)w;
                    v[2 * q + 1] = (uint32_t)(w >> 32);
                }
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    v[q] = *reinterpret_cast<const uint32_t *>(lds + across_[u & 1] + (r0 + 8 * u + q) * STRIDE + d0 * 4);
            }
            return v;
        }
    };
};

// Rows of DP elements in LDS as global_load_lds leaves them, four wavefronts loading: 64 granules to
// a wavefront's instruction, one after the other, so the rows are not padded.  Granule g of row r
// stands at place g ^ turn(r) of its row: lanes that read one granule of 16 rows, and half a
// wavefront that reads 4 rows x 64 bytes transposed, use all 64 banks.
template <int DT, int DP, int R>
struct Strip {
    static constexpr int W = 4;
    static constexpr int ES = elem_size(DT), E = 16 / ES;
    static constexpr int ROW = DP * ES, GR = ROW / 16, BYTES = R * ROW;
    static constexpr int PIECES = BYTES / 1024;                // instructions
    static constexpr int LOADS = (PIECES + W - 1) / W;         // of a wavefront
    static constexpr int CHUNKS = GR / 2, STEPS = E == 8 ? 2 : 4;
    static_assert(BYTES % 1024 == 0, "whole instructions");

    static __device__ __forceinline__ int turn(int r)
    {
        if constexpr (GR % 16 == 0) return (r & 3) << 2 | (r >> 2 & 3);
        if constexpr (GR % 16 == 8) return (r >> 1 & 1) << 2 | (r >> 2 & 3);
        return r >> 2 & 3;
    }

    // A lane's granules of a strip: its rows and their offsets from the strip's first one.
    struct Loader {
        int row[LOADS];
        uint32_t off[LOADS];
        bool mine[LOADS];
        uint32_t place;    // the wavefront's first instruction's, within the strip

        __device__ __forceinline__ void start(int wave, int lane, int D, int64_t stride)
        {
            place = wave * 1024;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int n = (wave + i * W) * 64 + lane;
                row[i] = n / GR;
                const int g = (n - row[i] * GR) ^ turn(row[i]);
                off[i] = (uint32_t)row[i] * (uint32_t)stride + g * 16;
                mine[i] = g * E < D;
            }
        }

        // `left` of the strip's rows are there; zeros for the others and past D
        __device__ __forceinline__ void load(const char *base, int left, uint32_t lds, int wave) const
        {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                if (PIECES % W != 0 && wave + i * W >= PIECES) break;
                const char *p = base + off[i];
                to_lds(mine[i] && row[i] < left ? p : reinterpret_cast<const char *>(kZeros), lds + place + i * W * 1024);
            }
        }
    };

    // The same of a problem's rows: row r is query r / share, head r % share, at `base` + its offset
    // from the tile's first query.  Past the last one it comes again.
    struct RowLoader {
        int row[LOADS], g[LOADS];
        uint32_t off[LOADS];

        __device__ __forceinline__ void start(int wave, int lane)
        {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int n = (wave + i * W) * 64 + lane;
                row[i] = n / GR;
                g[i] = (n - row[i] * GR) ^ turn(row[i]);
            }
        }

        template <class A>
        __device__ __forceinline__ void places(const A &p, int r0, int i0, int64_t stride, int64_t head)
        {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                int qi, qj;
                p.part_of(min(r0 + row[i], p.rows - 1), qi, qj);
                off[i] = (uint32_t)(qi - i0) * (uint32_t)stride + (uint32_t)qj * (uint32_t)head + g[i] * 16;
            }
        }

        __device__ __forceinline__ void load(const char *base, int D, uint32_t lds, int wave) const
        {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                if (PIECES % W != 0 && wave + i * W >= PIECES) break;
                const char *p = base + off[i];
                to_lds(g[i] * E < D ? p : reinterpret_cast<const char *>(kZeros), lds + (wave + i * W) * 1024);
            }
        }
    };

    // A lane's places: sums of a part of its own, an exclusive or with what is known ahead, and
    // distances that are known ahead.
    struct Reader {
        int along_row, along_turn, across_row, across_turn;

        __device__ __forceinline__ void start(int lane)
        {
            const int i = lane & 31, h = lane >> 5;
            along_row = i * ROW;
            along_turn = (h ^ turn(i)) << 4;
            if constexpr (ES == 2) {
                const int j = lane & 15, a = lane >> 4 & 1, b = j >> 1 & 1;
                across_row = (4 * h + (j >> 2)) * ROW + (j & 1) * 8;
                across_turn = ((2 * a + b) ^ turn(4 * h + (j >> 2))) << 4;
            } else {
                across_row = 4 * h * ROW + (i & 3) * 4;
                across_turn = ((i >> 2) ^ h) << 4;
            }
        }

        // As Panel's.
        __device__ __forceinline__ u32x4 along(const char *lds, int r0, int c) const
        {
            return *reinterpret_cast<const u32x4 *>(lds + along_row + (along_turn ^ (c << 5)) + r0 * ROW);
        }

        __device__ __forceinline__ u32x4 across(const char *lds, int r0, int u, int d0) const
        {
            u32x4 v;
            if constexpr (ES == 2) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {   // (rows 8 q further on turn by 2 q more)
                    const s16x4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s16x4 *)(lds + across_row +
                                                                    (across_turn ^ (d0 * 2 ^ q << 5)) +
                                                                    (r0 + 16 * u + 8 * q) * ROW));
                    const uint64_t w = __builtin_bit_cast(uint64_t, t);
                    v[2 * q] = (uint32_t)w;
                    v[2 * q + 1] = (uint32_t)(w >> 32);
                }
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    v[q] = *reinterpret_cast<const uint32_t *>(
                        lds + across_row + (across_turn ^ (d0 * 4 ^ (turn(8 * u + q) << 4))) + (r0 + 8 * u + q) * ROW);
            }
            return v;
        }
    };
};

// Until this wavefront's loads to LDS are done, and then all wavefronts'.
__device__ __forceinline__ void meet()
{
    wait_loads<0>();
    __builtin_amdgcn_s_waitcnt(0xc07f);   // its reads of LDS too: lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Step u's operand of a block's registers, rounded to the inputs' type.
template <int DT>
__device__ __forceinline__ u32x4 operand(const f32x16 &v, int u)
{
    if constexpr (DT == FLASHBEV_F32) {
        return __builtin_bit_cast(u32x4, f32x4{v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]});
    } else {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack2<DT>(v[8 * u + 2 * i], v[8 * u + 2 * i + 1]);
        return w;
    }
}

__device__ __forceinline__ f32x16 zeros16()
{
    f32x16 v;
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = 0.0f;
    return v;
}

// A lane's row of a block with the rows across: its fragments, straight from memory.
template <int DT, int DP, int N>
__device__ __forceinline__ void row_fragments(u32x4 (&f)[N], const char *row, bool there, int D, int lane)
{
    using P = Panel<DT, DP, 32>;
    static_assert(N == P::CHUNKS, "a row's granules");
#pragma unroll
    for (int c = 0; c < N; ++c) {
        f[c] = u32x4{0, 0, 0, 0};
        if (there) f[c] = P::granule(row, 2 * c + (lane >> 5), D);
    }
}

// ---------------------------------------------------------------------------
// masks
// ---------------------------------------------------------------------------
typedef uint32_t u32_any __attribute__((aligned(1)));
typedef u32x4 u32x4_f __attribute__((aligned(4)));

constexpr int kAddF16 = 16 + FLASHLAYER_MASK_ADD, kAddBf16 = 32 + FLASHLAYER_MASK_ADD;   // kinds

// A block's mask as it is stored.  Its loads are issued before the block's products and used
// behind them.
struct MaskBlock {
    u32x4 w[4];

    // Keys key0 + 8 k + 4 h + 0 .. 3 for k = 0 .. 3 of a lane's row; Lk keys to a row.
    __device__ __forceinline__ void load_row(const Attend &p, const char *row, int key0, int h)
    {
        if (p.kind == FLASHLAYER_MASK_NONE) return;
        const bool whole = key0 + 32 <= p.Lk;
        const int size = p.kind == FLASHLAYER_MASK_BOOL ? 1 : p.kind == FLASHLAYER_MASK_ADD_F32 ? 4 : 2;
        const char *at = row + (int64_t)(key0 + 4 * h) * size;
        if (!whole) {
            asm volatile("");
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                u32x4 v = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (key0 + 8 * k + 4 * h + i >= p.Lk) continue;
                    const char *e = at + (8 * k + i) * size;
                    if (size == 1) {
                        v[0] |= (uint32_t)(uint8_t)*e << (8 * i);
                    } else if (size == 2) {
                        v[i / 2] |= (uint32_t)*reinterpret_cast<const uint16_t *>(e) << (16 * (i & 1));
                    } else {
                        v[i] = *reinterpret_cast<const uint32_t *>(e);
                    }
                }
                w[k] = v;
            }
        } else if (size == 1) {
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k][0] = *reinterpret_cast<const u32_any *>(at + 8 * k);
        } else if (size == 2) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const u32x2 v = load8(at + 16 * k);
                w[k][0] = v[0];
                w[k][1] = v[1];
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = *reinterpret_cast<const u32x4_f *>(at + 32 * k);
        }
    }

    // x = scale x + mask.  (Without a mask too: these kernels serve odd widths.)
    __device__ __forceinline__ void apply_row(const Attend &p, f32x16 &x) const
    {
        if (p.kind == FLASHLAYER_MASK_NONE) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] *= p.scale;
        } else if (p.kind == FLASHLAYER_MASK_BOOL) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                x[i] = w[i / 4][0] >> (8 * (i & 3)) & 0xff ? x[i] * p.scale : -__builtin_inff();
        } else if (p.kind == FLASHLAYER_MASK_ADD_F32) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t v = w[i / 4][i & 3];
                x[i] = __builtin_fmaf(x[i], p.scale, __builtin_bit_cast(float, v));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = __builtin_fmaf(x[i], p.scale, half_at(p, w[i / 4][i / 2 & 1] >> (16 * (i & 1))));
        }
    }

    // One key of a lane, rows at `offsets` (in bytes, from `base`).
    __device__ __forceinline__ void load_key(const Attend &p, const char *base, const int64_t *offsets, int key)
    {
        if (p.kind == FLASHLAYER_MASK_NONE) return;
        if (p.kind == FLASHLAYER_MASK_BOOL) {
            base += key;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                w[i / 4][i & 3] = *reinterpret_cast<const uint8_t *>(base + offsets[8 * (i >> 2) + (i & 3)]);
        } else if (p.kind == FLASHLAYER_MASK_ADD_F32) {
            base += (int64_t)key * 4;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                w[i / 4][i & 3] = *reinterpret_cast<const uint32_t *>(base + offsets[8 * (i >> 2) + (i & 3)]);
        } else {
            base += (int64_t)key * 2;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                w[i / 4][i & 3] = *reinterpret_cast<const uint16_t *>(base + offsets[8 * (i >> 2) + (i & 3)]);
        }
    }

    __device__ __forceinline__ void apply_key(const Attend &p, f32x16 &x) const
    {
        if (p.kind == FLASHLAYER_MASK_NONE) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] *= p.scale;
        } else if (p.kind == FLASHLAYER_MASK_BOOL) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = w[i / 4][i & 3] ? x[i] * p.scale : -__builtin_inff();
        } else if (p.kind == FLASHLAYER_MASK_ADD_F32) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t v = w[i / 4][i & 3];
                x[i] = __builtin_fmaf(x[i], p.scale, __builtin_bit_cast(float, v));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = __builtin_fmaf(x[i], p.scale, half_at(p, w[i / 4][i & 3]));
        }
    }

    static __device__ __forceinline__ float half_at(const Attend &p, uint32_t w)
    {
        const uint16_t v = (uint16_t)w;
        return p.kind == kAddF16 ? (float)__builtin_bit_cast(_Float16, v) : __builtin_bit_cast(float, w << 16);
    }
};

// Scores of keys from `end` on leave a row.  (The empty statement keeps the last tile's branch a
// branch: as selections every tile paid for it, 100 of 280 vector instructions.)
__device__ __forceinline__ void cut_keys(f32x16 &x, int key0, int h, int end)
{
    asm volatile("");
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (key0 + 8 * (i >> 2) + 4 * h + (i & 3) >= end) x[i] = -__builtin_inff();
}

// The same by a word of the keys' bits.
__device__ __forceinline__ void cut_word(f32x16 &x, uint32_t word, int h)
{
    asm volatile("");
    word >>= 4 * h;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (!(word >> (8 * (i >> 2) + (i & 3)) & 1)) x[i] = -__builtin_inff();
}

// The other half's value of the lane's column joined with its own.
__device__ __forceinline__ float both_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v),
                                                    false, false);
    const unsigned a = r[0], b = r[1];
    return __builtin_fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

__device__ __forceinline__ float both_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v),
                                                    false, false);
    const unsigned a = r[0], b = r[1];
    return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}

// ---------------------------------------------------------------------------
// results: a block has row lane % 32 across and 32 channels down
// ---------------------------------------------------------------------------
// Channels d .. d + 7 of a row of D, and what their rounding took.
template <int DT>
__device__ __forceinline__ void put8(char *row, int d, int D, const float (&v)[8])
{
    if (d + 8 <= D) {
        store_elems<DT>(row + d * elem_size(DT), v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (d + i < D) store_elem<DT>(row, d + i, v[i]);
    }
}

template <int DT>
__device__ __forceinline__ float rounded(float v)
{
    if constexpr (DT == FLASHBEV_F16) {
        return (float)(_Float16)v;
    } else if constexpr (DT == FLASHBEV_BF16) {
        return (float)(__bf16)v;
    } else {
        return v;
    }
}

// ---------------------------------------------------------------------------
// copies
// ---------------------------------------------------------------------------
// Rows of a problem (the keys of a head of the states, or the rows of a problem) to whole granules.
struct Copy {
    const char *from[2];
    char *to[2];
    int64_t batch[2], row[2], head[2], group[2];   // bytes: row r at row (r / share) + head (r % share)
    const uint32_t *words;                         // null: all rows are there
    int64_t words_b, words_g;
    const int32_t *lengths;                        // null: all
    uint64_t items;                                // granules of one tensor
    int heads, rows, share, D, granules;
};

template <int DT>
__global__ void __launch_bounds__(256) attend_copy(Copy p)
{
    const uint64_t t = (uint64_t)block_index() * 256 + threadIdx.x;
    if (t >= 2 * p.items) return;
    const int which = t >= p.items;
    const uint64_t at = t - (which ? p.items : 0);
    uint64_t n = at / p.granules;
    const int granule = (int)(at - n * p.granules);
    const uint64_t m = n / p.rows;
    const int r = (int)(n - m * p.rows);
    const int b = (int)(m / p.heads), g = (int)(m - (uint64_t)b * p.heads);
    u32x4 v = {0, 0, 0, 0};
    const bool there = (!p.words || p.words[b * p.words_b + g * p.words_g + (r >> 5)] >> (r & 31) & 1) &&
                       (!p.lengths || r < p.lengths[b]);
    if (there) {
        const int i = r / p.share, j = r - i * p.share;
        const char *row = (which ? p.from[1] : p.from[0]) + b * (which ? p.batch[1] : p.batch[0]) +
                          g * (which ? p.group[1] : p.group[0]) + i * (which ? p.row[1] : p.row[0]) +
                          j * (which ? p.head[1] : p.head[0]);
        v = Panel<DT, 32, 32>::granule(row, granule, p.D);
    }
    *reinterpret_cast<u32x4 *>((which ? p.to[1] : p.to[0]) + at * 16) = v;
}

// The keys' bits, from a boolean mask.
struct Bits {
    const char *mask;
    int64_t batch, head;   // bytes
    uint32_t *words;
    const int32_t *lengths;
    int64_t per;           // words of a row
    uint64_t items;        // words
    int heads, Lk;
};

template <int UNUSED>
__global__ void __launch_bounds__(256) attend_bits(Bits p)
{
    const uint64_t t = (uint64_t)block_index() * 256 + threadIdx.x;
    if (t >= p.items) return;
    const uint64_t m = t / p.per;
    const int key0 = (int)(t - m * p.per) * 32, b = (int)(m / p.heads), g = (int)(m - (uint64_t)b * p.heads);
    const int end = p.lengths ? max(0, min(p.lengths[b], p.Lk)) : p.Lk;
    const char *row = p.mask + b * p.batch + g * p.head;
    uint32_t w = 0;
    for (int i = 0; i < 32; ++i)
        if (key0 + i < end && row[key0 + i]) w |= 1u << i;
    p.words[t] = w;
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
constexpr int kCusOfCard = 256;

inline uint64_t align256(uint64_t v) { return (v + 255) & ~255ull; }

inline int check_attention(const flashlayer_attention *a)
{
    if (!a) return FLASHBEV_ERR_NULLPTR;
    if (a->B < 0 || a->Lq < 0 || a->Lk < 0 || a->H < 0 || a->Hk < 0 || a->D < 0) return FLASHBEV_ERR_SHAPE;
    if (a->Hk ? a->H % a->Hk : a->H) return FLASHBEV_ERR_SHAPE;
    for (const int64_t s : {a->q_batch, a->q_row, a->q_head, a->k_batch, a->k_row, a->k_head, a->v_batch, a->v_row,
                            a->v_head, a->o_batch, a->o_row, a->o_head, a->mask_batch, a->mask_head, a->mask_row})
        if (s < 0) return FLASHBEV_ERR_SHAPE;
    if (!known_dtype(a->dtype)) return FLASHBEV_ERR_DTYPE;
    if (a->mask < FLASHLAYER_MASK_NONE || a->mask > FLASHLAYER_MASK_ADD_F32) return FLASHBEV_ERR_VALUE;
    if (!(a->scale > 0.0f) || !finite_value(a->scale)) return FLASHBEV_ERR_VALUE;
    if (a->D > FLASHLAYER_HEAD_MAX) return FLASHBEV_ERR_UNSUPPORTED;
    // (a tile's rows lie within 32 bits)
    for (const int64_t s : {a->q_row, a->q_head, a->k_row, a->v_row, a->o_row, a->o_head})
        if (s > FLASHBLOCK_LD_MAX) return FLASHBEV_ERR_UNSUPPORTED;
    const uint64_t share = a->Hk ? a->H / a->Hk : 0;
    for (const int64_t s : {a->q_head, a->o_head})
        if (size_prod({share, (uint64_t)s}) > 1ull << 28) return FLASHBEV_ERR_UNSUPPORTED;
    // (rows by their share's reciprocal; places of the last tile within 31 bits)
    if (size_prod({(uint64_t)a->Lq, share, share}) > 0xffffffffull ||
        size_prod({(uint64_t)a->Lq, share}) > 0x7ffffe00ull || a->Lk > 0x7ffffe00)
        return FLASHBEV_ERR_UNSUPPORTED;
    return FLASHBEV_OK;
}

// Bytes from the first to the last element of a tensor [n0, n1, n2, D] by its strides;
// kSizeOver past 2^62.
inline uint64_t span4(int n0, int64_t s0, int n1, int64_t s1, int n2, int64_t s2, int D, int es)
{
    if (!n0 || !n1 || !n2 || !D) return 0;
    uint64_t last = (uint64_t)D;
    for (const auto &d : {std::pair<int, int64_t>{n0, s0}, {n1, s1}, {n2, s2}}) {
        const uint64_t part = size_prod({(uint64_t)(d.first - 1), (uint64_t)d.second});
        if (part > kSizeCap / 16) return kSizeOver;
        last += part;
    }
    return last * es;
}

// Whether no two elements of such a tensor share a place (by each dimension clearing those of
// smaller strides).
inline bool apart(int n0, int64_t s0, int n1, int64_t s1, int n2, int64_t s2, int D)
{
    std::pair<int64_t, int> dims[3] = {{s0, n0}, {s1, n1}, {s2, n2}};
    std::sort(dims, dims + 3);
    uint64_t span = (uint64_t)D;
    for (const auto &d : dims) {
        if (d.second <= 1) continue;
        if ((uint64_t)d.first < span) return false;
        span += size_prod({(uint64_t)(d.second - 1), (uint64_t)d.first});
    }
    return true;
}

inline int padded_head(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : D <= 96 ? 96 : 128; }

inline int share_of(const flashlayer_attention *a) { return a->Hk ? a->H / a->Hk : 1; }

// A boolean mask that is the same for all rows of a problem leaves its keys out altogether.
inline bool drops_of(const flashlayer_attention *a)
{
    return a->mask == FLASHLAYER_MASK_BOOL && (a->mask_row == 0 || a->Lq == 1) &&
           (a->mask_head == 0 || share_of(a) == 1);
}

// A mask that differs from row to row.
inline bool pairs_of(const flashlayer_attention *a) { return a->mask != FLASHLAYER_MASK_NONE && !drops_of(a); }

// Rows that end inside a granule.
inline bool odd_of(const flashlayer_attention *a) { return a->D % (16 / elem_size(a->dtype)) != 0; }

// Whether a call of one workgroup's few rows takes the kernels that do all.
inline bool any_of(const flashlayer_attention *a) { return a->mask != FLASHLAYER_MASK_NONE || odd_of(a); }

inline int whole_head(const flashlayer_attention *a)
{
    const int E = 16 / elem_size(a->dtype);
    return (a->D + E - 1) / E * E;
}

// Copies that keep loads to LDS simple: rows of whole granules, zeros past D and in place of keys
// that are left out, [B][heads][rows][whole_head]; and the bits of the keys that take part.
inline uint64_t rows_copy_bytes(const flashlayer_attention *a, int64_t rows, int heads)
{
    return align256(size_prod({(uint64_t)a->B, (uint64_t)heads, (uint64_t)rows, (uint64_t)whole_head(a),
                               (uint64_t)elem_size(a->dtype)}));
}

inline int64_t words_of(const flashlayer_attention *a) { return ((int64_t)a->Lk + 127) / 128 * 4; }

inline uint64_t words_bytes(const flashlayer_attention *a)
{
    return align256((uint64_t)a->B * (a->mask_head ? a->Hk : 1) * words_of(a) * 4);
}

inline bool copies_keys(const flashlayer_attention *a) { return !pairs_of(a) && (odd_of(a) || drops_of(a)); }

inline uint64_t keys_copy_bytes(const flashlayer_attention *a)
{
    if (!copies_keys(a)) return 0;
    return 2 * rows_copy_bytes(a, a->Lk, a->Hk) + (drops_of(a) ? words_bytes(a) : 0);
}

inline Attend attend_of(const flashlayer_attention *a)
{
    Attend p{};
    const int es = elem_size(a->dtype);
    const int ms = a->mask == FLASHLAYER_MASK_BOOL ? 1 : a->mask == FLASHLAYER_MASK_ADD_F32 ? 4 : es;
    p.qb = a->q_batch * es;
    p.qr = a->q_row * es;
    p.qh = a->q_head * es;
    p.kb = a->k_batch * es;
    p.kr = a->k_row * es;
    p.kh = a->k_head * es;
    p.vb = a->v_batch * es;
    p.vr = a->v_row * es;
    p.vh = a->v_head * es;
    p.ob = a->o_batch * es;
    p.orow = a->o_row * es;
    p.oh = a->o_head * es;
    p.mb = a->mask_batch * ms;
    p.mh = a->mask_head * ms;
    p.mr = a->mask_row * ms;
    p.B = a->B;
    p.Lq = a->Lq;
    p.Lk = a->Lk;
    p.H = a->H;
    p.Hk = a->Hk;
    p.D = a->D;
    p.share = a->Hk ? a->H / a->Hk : 1;
    p.rows = a->Lq * p.share;
    p.share_inv = p.share > 1 ? (uint32_t)((0x100000000ull + p.share - 1) / p.share) : 0;
    // additive masks of the inputs' type: float32 ones are one kind, float16 and bfloat16 two
    p.kind = a->mask != FLASHLAYER_MASK_ADD      ? a->mask
             : a->dtype == FLASHBEV_F32          ? FLASHLAYER_MASK_ADD_F32
             : a->dtype == FLASHBEV_F16          ? kAddF16
                                                 : kAddBf16;
    p.drops = drops_of(a);
    p.Dk = a->D;
    p.scale = a->scale;
    return p;
}

// The grid's items, dealt to the XCDs.
inline int deal(Attend &p, uint64_t items)
{
    if (items > 0x7fffffffull / 2) return FLASHBEV_ERR_UNSUPPORTED;
    p.blocks = (uint32_t)items;
    p.per_xcd = (uint32_t)((items + 7) / 8);
    return FLASHBEV_OK;
}

// Whether loads to LDS may read a tensor's rows: they take 16 bytes at addresses that are multiples of
// them.  Elsewhere the kernels with masks, whose loads to registers go to any element, take the call: 2 x
// 2048 x 4096 of 16 heads x 128 on 4, bf16, forward 151 -> 240 us and grad_q 214 -> 365 with k one element
// further on, grad_k and grad_v 276 -> 627 with q.
struct Step {
    int n;
    int64_t bytes;
};

inline bool to_lds_reads(const void *base, std::initializer_list<Step> steps)
{
    if (misaligned(base, 16)) return false;
    for (const Step &s : steps)
        if (s.n > 1 && s.bytes % 16 != 0) return false;
    return true;
}

inline bool keys_to_lds(const Attend &p)
{
    return to_lds_reads(p.k, {{p.B, p.kb}, {p.Lk, p.kr}, {p.Hk, p.kh}}) &&
           to_lds_reads(p.v, {{p.B, p.vb}, {p.Lk, p.vr}, {p.Hk, p.vh}});
}

template <class P>
int launch_lds(const void *fn, uint64_t blocks, P &p, size_t lds, hipStream_t st)
{
    if (lds > 65536 && hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
        return FLASHBEV_ERR_HIP;
    return launch_kernel(fn, blocks, 256, p, lds, st);
}

template <int DT>
int copy_rows(Copy &c, int64_t batches, hipStream_t st)
{
    c.items = (uint64_t)batches * c.heads * c.rows * c.granules;
    return launch_rows((const void *)attend_copy<DT>, (2 * c.items + 255) / 256, 256, c, st);
}

// k's and v's copies and bits, in `ws` of keys_copy_bytes; p reads them from here on.
template <int DT>
int copy_keys(const flashlayer_attention *a, Attend &p, char *ws, hipStream_t st)
{
    constexpr int ES = elem_size(DT);
    const uint64_t each = rows_copy_bytes(a, a->Lk, a->Hk);
    if (p.drops) {
        Bits bits{p.mask, p.mb, p.mh, reinterpret_cast<uint32_t *>(ws + 2 * each), p.lengths, words_of(a), 0,
                  a->mask_head ? a->Hk : 1, a->Lk};
        bits.items = (uint64_t)a->B * bits.heads * bits.per;
        if (const int rc = launch_rows((const void *)attend_bits<0>, (bits.items + 255) / 256, 256, bits, st)) return rc;
        p.words = bits.words;
        p.words_g = a->mask_head ? bits.per : 0;
        p.words_b = bits.per * bits.heads;
    }
    Copy c{};
    c.from[0] = p.k;
    c.from[1] = p.v;
    c.to[0] = ws;
    c.to[1] = ws + each;
    c.batch[0] = p.kb;
    c.batch[1] = p.vb;
    c.row[0] = p.kr;
    c.row[1] = p.vr;
    c.group[0] = p.kh;
    c.group[1] = p.vh;
    c.words = p.words;
    c.words_b = p.words_b;
    c.words_g = p.words_g;
    c.lengths = p.lengths;
    c.heads = a->Hk;
    c.rows = a->Lk;
    c.share = 1;
    c.D = a->D;
    p.Dk = whole_head(a);
    c.granules = p.Dk * ES / 16;
    p.k = c.to[0];
    p.v = c.to[1];
    p.kr = p.vr = (int64_t)p.Dk * ES;
    p.kh = p.vh = p.kr * a->Lk;
    p.kb = p.vb = p.kh * a->Hk;
    return copy_rows<DT>(c, a->B, st);
}

struct Bytes {
    const void *p;
    uint64_t n;
};

inline int check_overlaps(std::initializer_list<Bytes> outs, std::initializer_list<Bytes> ins)
{
    for (const Bytes *o = outs.begin(); o != outs.end(); ++o) {
        if (o->n == kSizeOver) return FLASHBEV_ERR_UNSUPPORTED;
        for (const Bytes &i : ins) {
            if (i.n == kSizeOver) return FLASHBEV_ERR_UNSUPPORTED;
            if (ranges_overlap(o->p, o->n, i.p, i.n)) return FLASHBEV_ERR_ALIAS;
        }
        for (const Bytes *q = outs.begin(); q != o; ++q)
            if (ranges_overlap(o->p, o->n, q->p, q->n)) return FLASHBEV_ERR_ALIAS;
    }
    return FLASHBEV_OK;
}

// Into how many parts a long axis of `steps` tiles is split, for `base` workgroups without
// that and per_cu that run on a CU at once: the number that takes the fewest steps one after
// another.  A workgroup's start and end count as 1 1/2 steps, the joining launch as one and an eighth
// more for each part.  (Gradients of 3 x 777 queries of 2 heads' shares of 3 by 1333 keys x 72 half with
// a bias, 66 workgroups of grad_k and grad_v, one to a CU: 195, 106, 78 us in 1, 2, 3 parts, 116
// in 4, whose last workgroups take a round of their own, 89 in 6 and 107 in 12.)
inline int splits_of(int64_t base, int64_t steps, int per_cu)
{
    const int64_t slots = (int64_t)kCusOfCard / 8 * per_cu;   // of an XCD
    if (base <= 0 || base >= 8 * slots || steps <= 1) return 1;
    uint32_t best = 1, least = ~0u;
    const uint32_t most = (uint32_t)std::min<int64_t>(steps, 3 * kCusOfCard), n = (uint32_t)steps;
    for (uint32_t s = 1; s <= most; s += 1 + s / 16) {
        const uint32_t rounds = ((uint32_t)((base * s + 7) / 8) + (uint32_t)slots - 1) / (uint32_t)slots;
        const uint32_t cost = rounds * (2 * ((n + s - 1) / s) + 3) + (s > 1 ? 2 + s / 4 : 0);
        if (cost < least) {
            least = cost;
            best = s;
        }
        if (rounds > 4) break;
    }
    return (int)best;
}

inline int check_scratch(const void *ws, uint64_t bytes, uint64_t need)
{
    if (!need) return FLASHBEV_OK;
    if (!ws) return FLASHBEV_ERR_NULLPTR;
    if (misaligned(ws, 256)) return FLASHBEV_ERR_ALIGN;
    return bytes < need ? FLASHBEV_ERR_SCRATCH : FLASHBEV_OK;
}

}  // namespace

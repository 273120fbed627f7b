// Dropout from a counter-based generator, onto a residual, and its gradient, for AMD MI355X
// (gfx950).  C ABI: include/block/flashlayer.h.
//
//   out = residual + (word >= threshold ? factor x : 0),   grad_x = word >= threshold ? factor g : 0
//
// Both are one map of a tensor to another, so one kernel serves both.  The words come from
// Philox 4x32-10 at the element's place, so nothing of the mask is stored: a block of the
// generator serves four elements and takes 20 wide products (v_mad_u64_u32, a quarter of the
// full rate) and 40 exclusive ors.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "block/flashlayer.h"
#include "block_common.h"

namespace {

struct Drop {
    const char *in, *residual;   // residual null: none
    char *out;
    const uint64_t *state;       // null: seed and offset from here
    uint64_t seed, offset;
    int64_t n;                   // elements
    int64_t ldi, ldr, ldo;       // elements
    int64_t width;               // elements of a row: n where all rows follow each other
    uint32_t threshold;
    int all;                     // everything is dropped
    float factor;
};

// Block `i` of the generator.
__device__ __forceinline__ void philox(uint64_t i, uint64_t offset, uint64_t seed, uint32_t (&w)[4])
{
    uint32_t a = (uint32_t)i, b = (uint32_t)(i >> 32);
    uint32_t c = (uint32_t)offset, d = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t u = (uint64_t)a * 0xD2511F53u, v = (uint64_t)c * 0xCD9E8D57u;
        a = (uint32_t)(v >> 32) ^ b ^ k0;
        b = (uint32_t)v;
        c = (uint32_t)(u >> 32) ^ d ^ k1;
        d = (uint32_t)u;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    w[0] = a;
    w[1] = b;
    w[2] = c;
    w[3] = d;
}

constexpr int kVec = 8;   // elements a lane takes: two blocks, 16 bytes of 16-bit elements

// The words' verdicts on elements e .. e + 7 (e a multiple of 8), bit i for element e + i.
__device__ __forceinline__ uint32_t kept(const Drop &p, uint64_t seed, uint64_t offset, int64_t e)
{
    if (p.all) return 0;
    if (p.threshold == 0) return 0xff;
    uint32_t bits = 0;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        uint32_t w[4];
        philox((uint64_t)(e >> 2) + q, offset, seed, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) bits |= (w[i] >= p.threshold ? 1u : 0u) << (4 * q + i);
    }
    return bits;
}

template <int IN, int OUT>
__device__ __forceinline__ float one(const Drop &p, uint32_t bits, int i, const char *x, const char *r)
{
    const float v = bits >> i & 1 ? load_elem<IN>(x, 0) * p.factor : 0.0f;
    return r ? load_elem<OUT>(r, 0) + v : v;
}

// EVEN: rows of whole vectors, or all rows one; else a vector may run over rows' ends.  Memory and the
// generator's products take alike long: 16384 x 8192 bf16 98 us, 5.5 TB/s (the last-level cache
// holds some of it), the vector units busy all the time.
template <int IN, int OUT, bool RES, bool EVEN>
__global__ void __launch_bounds__(256) drop_map(Drop p)
{
    const uint64_t vec = (uint64_t)block_index() * 256 + threadIdx.x;
    const int64_t e = (int64_t)vec * kVec;
    if (e >= p.n) return;
    const uint64_t seed = p.state ? p.state[0] : p.seed, offset = p.state ? p.state[1] : p.offset;
    constexpr int IS = elem_size(IN), OS = elem_size(OUT);
    int64_t row = 0, col = e;
    if (p.width != p.n) {   // a 64-bit division takes some 100 instructions
        if (p.n <= 0xffffffffll) {
            row = (uint32_t)e / (uint32_t)p.width;
        } else {
            row = e / p.width;
        }
        col = e - row * p.width;
    }
    const char *x = p.in + (row * p.ldi + col) * IS;
    const char *r = RES ? p.residual + (row * p.ldr + col) * OS : nullptr;
    char *o = p.out + (row * p.ldo + col) * OS;
    if (EVEN && e + kVec <= p.n) {
        float v[kVec], b[kVec];
        load_elems<IN>(x, v);
        if (RES) load_elems<OUT>(r, b);
        const uint32_t bits = kept(p, seed, offset, e);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            v[i] = bits >> i & 1 ? v[i] * p.factor : 0.0f;   // (what is dropped may be NaN)
            if (RES) v[i] += b[i];
        }
        store_elems<OUT>(o, v);
        return;
    }
    const uint32_t bits = kept(p, seed, offset, e);
    for (int i = 0; i < kVec && e + i < p.n; ++i) {
        store_elem<OUT>(o, 0, one<IN, OUT>(p, bits, i, x, r));
        if (++col == p.width) {
            col = 0;
            x += (p.ldi - p.width + 1) * IS;
            if (RES) r += (p.ldr - p.width + 1) * OS;
            o += (p.ldo - p.width + 1) * OS;
        } else {
            x += IS;
            if (RES) r += OS;
            o += OS;
        }
    }
}

template <int IN, int OUT>
const void *kernel_of(bool res, bool even)
{
    if (res) return even ? (const void *)drop_map<IN, OUT, true, true> : (const void *)drop_map<IN, OUT, true, false>;
    return even ? (const void *)drop_map<IN, OUT, false, true> : (const void *)drop_map<IN, OUT, false, false>;
}

int check(const flashlayer_dropout *a)
{
    if (!a) return FLASHBEV_ERR_NULLPTR;
    if (a->M < 0 || a->C < 0) return FLASHBEV_ERR_SHAPE;
    if (!known_dtype(a->dtype)) return FLASHBEV_ERR_DTYPE;
    if (a->stream_dtype != a->dtype && a->stream_dtype != FLASHBEV_F32) return FLASHBEV_ERR_DTYPE;
    if (!(a->p >= 0.0 && a->p <= 1.0) || !finite_value(a->scale)) return FLASHBEV_ERR_VALUE;
    if (a->M > FLASHBLOCK_ROWS_MAX || a->C > FLASHBLOCK_WIDTH_MAX) return FLASHBEV_ERR_UNSUPPORTED;
    return FLASHBEV_OK;
}

int check_ld(int64_t ld, int64_t C)
{
    return ld < C ? FLASHBEV_ERR_SHAPE : ld > FLASHBLOCK_LD_MAX ? FLASHBEV_ERR_UNSUPPORTED : FLASHBEV_OK;
}

// The call on checked arguments: `in` of type it to `out` of type ot.
int launch(const flashlayer_dropout *a, const void *in, int it, int64_t ldi, const void *residual, int64_t ldr,
           const uint64_t *state, void *out, int ot, int64_t ldo, void *stream)
{
    Drop p{};
    p.in = static_cast<const char *>(in);
    p.residual = static_cast<const char *>(residual);
    p.out = static_cast<char *>(out);
    p.state = state;
    p.seed = a->seed;
    p.offset = a->offset;
    p.n = a->M * a->C;
    p.ldi = ldi;
    p.ldr = residual ? ldr : a->C;
    p.ldo = ldo;
    const bool one_row = a->M == 1 || (ldi == a->C && p.ldr == a->C && ldo == a->C);
    p.width = one_row ? p.n : a->C;
    const double t = nearbyint(a->p * 4294967296.0);
    p.all = t >= 4294967296.0;
    p.threshold = p.all ? 0 : (uint32_t)t;
    p.factor = a->p < 1.0 ? (float)(a->scale / (1.0 - a->p)) : 0.0f;
    const bool res = residual != nullptr, even = one_row || a->C % kVec == 0;
    const void *fn = nullptr;
    if (it == FLASHBEV_F32 && ot == FLASHBEV_F32) fn = kernel_of<FLASHBEV_F32, FLASHBEV_F32>(res, even);
    if (it == FLASHBEV_F16 && ot == FLASHBEV_F16) fn = kernel_of<FLASHBEV_F16, FLASHBEV_F16>(res, even);
    if (it == FLASHBEV_BF16 && ot == FLASHBEV_BF16) fn = kernel_of<FLASHBEV_BF16, FLASHBEV_BF16>(res, even);
    if (it == FLASHBEV_F16 && ot == FLASHBEV_F32) fn = kernel_of<FLASHBEV_F16, FLASHBEV_F32>(res, even);
    if (it == FLASHBEV_BF16 && ot == FLASHBEV_F32) fn = kernel_of<FLASHBEV_BF16, FLASHBEV_F32>(res, even);
    if (it == FLASHBEV_F32 && ot == FLASHBEV_F16) fn = kernel_of<FLASHBEV_F32, FLASHBEV_F16>(res, even);
    if (it == FLASHBEV_F32 && ot == FLASHBEV_BF16) fn = kernel_of<FLASHBEV_F32, FLASHBEV_BF16>(res, even);
    return launch_rows(fn, ((uint64_t)p.n + 256 * kVec - 1) / (256 * kVec), 256, p, static_cast<hipStream_t>(stream));
}

int check_pointers(const void *in, int it, const void *out, int ot, const uint64_t *state)
{
    if (!in || !out) return FLASHBEV_ERR_NULLPTR;
    if (misaligned(in, elem_size(it)) || misaligned(out, elem_size(ot)) || misaligned(state, 8))
        return FLASHBEV_ERR_ALIGN;
    return FLASHBEV_OK;
}

}  // namespace

extern "C" int flashlayer_dropout_forward(const flashlayer_dropout *args, const void *x,
                                          const void *residual, const uint64_t *state, void *out,
                                          void *stream)
{
    if (const int rc = check(args)) return rc;
    const int xt = args->dtype, st = args->stream_dtype;
    const int64_t M = args->M, C = args->C;
    for (const int64_t ld : {args->ldx, args->ldo, residual ? args->ldr : C})
        if (const int rc = check_ld(ld, C)) return rc;
    if (M == 0 || C == 0) return FLASHBEV_OK;
    if (const int rc = check_pointers(x, xt, out, st, state)) return rc;
    if (misaligned(residual, elem_size(st))) return FLASHBEV_ERR_ALIGN;
    const uint64_t out_bytes = span_bytes(M, args->ldo, C, elem_size(st));
    if (ranges_overlap(out, out_bytes, x, span_bytes(M, args->ldx, C, elem_size(xt))) ||
        ranges_overlap(out, out_bytes, state, 16))
        return FLASHBEV_ERR_ALIAS;
    if (residual && !(residual == out && args->ldr == args->ldo) &&
        ranges_overlap(out, out_bytes, residual, span_bytes(M, args->ldr, C, elem_size(st))))
        return FLASHBEV_ERR_ALIAS;
    return launch(args, x, xt, args->ldx, residual, args->ldr, state, out, st, args->ldo, stream);
}

extern "C" int flashlayer_dropout_backward(const flashlayer_dropout *args, const void *grad_out,
                                           const uint64_t *state, void *grad_x, void *stream)
{
    if (const int rc = check(args)) return rc;
    const int xt = args->dtype, st = args->stream_dtype;
    const int64_t M = args->M, C = args->C;
    for (const int64_t ld : {args->ldx, args->ldo})
        if (const int rc = check_ld(ld, C)) return rc;
    if (M == 0 || C == 0) return FLASHBEV_OK;
    if (const int rc = check_pointers(grad_out, st, grad_x, xt, state)) return rc;
    const uint64_t bytes = span_bytes(M, args->ldx, C, elem_size(xt));
    if (ranges_overlap(grad_x, bytes, grad_out, span_bytes(M, args->ldo, C, elem_size(st))) ||
        ranges_overlap(grad_x, bytes, state, 16))
        return FLASHBEV_ERR_ALIAS;
    return launch(args, grad_out, st, args->ldo, nullptr, C, state, grad_x, xt, args->ldx, stream);
}

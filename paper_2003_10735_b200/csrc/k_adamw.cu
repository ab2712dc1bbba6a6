// st_adamw — OptimStep of Algorithm 1 (Adam, Section 5.2; here with decoupled weight decay) over any number of the caller's
// tensors in one launch, moments in fp32 or in 8 bits.  The formulas stand in include/shadowtutor.h.
//
// All tensors are cut into chunks of kChunk values; a table on the device says which tensor a chunk belongs to, and each block of a
// launch takes an equal part of them (how many blocks: at st_adamw_create).  A warp takes 256 consecutive values of a chunk, which are also a block of 8-bit
// moments: the two maxima that a block's scales need are warp reductions, and a lane keeps its eight values in registers from the
// load to the store, so that every buffer is read once and written once.
//
// The gradients' norm needs every gradient before the first step is taken: a kernel of its own (double accumulators, partial
// sums per block added in block order, a lane's values in theirs wherever the gradients lie: the result depends on the values, the tensors' sizes and
// the number of blocks that the device holds).
#include "../../include/shadowtutor.h"
#include "st_internal.h"

#include <cuda_fp16.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>
#include <string>
#include <vector>

namespace st {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kBlockVals = ST_ADAMW_BLOCK;                  // one warp's values: a block of 8-bit moments
constexpr int kChunk = kWarps * kBlockVals;
constexpr int kPer = kBlockVals / 32;                       // values of a lane
static_assert(kPer == 8, "the vector path below moves eight values per lane");

struct TensorRec {              // does not change as long as the optimiser lives (the gradients' addresses may: Plan::grads)
    void* param; float* master;
    void *m, *v; float *m_scale, *v_scale;
    int64_t n;
    float wd, lr_scale;
    uint8_t param_type, grad_type, vec, pad;                // vec: all buffers but the gradient lie as the vector path needs them
};
struct ChunkRec { int32_t tensor, index; };
struct __align__(32) Scalars {
    long long t;                // steps taken
    float bias[2][2];           // of step t at [t % 2]: 1 / (1 - beta1^t) and 1 / sqrt(1 - beta2^t)
    float lr;
    float factor;               // of the gradients, from the norm
    int skip;                   // the norm is not finite and the step is to be left out
    unsigned int norm_ticket, step_ticket;
    double power[2];            // beta1^t and beta2^t of the next step
};
struct Plan {
    const TensorRec* tensors; const ChunkRec* chunks; int64_t n_chunks;
    const void** grads;
    Scalars* sc; double* partials;
    double beta1, beta2, max_norm;
    float b1, b2, omb1, omb2, eps, one;
    int skip_nonfinite;
};

// ---- moving a warp's 256 values -------------------------------------------------------------------------
// Vector path: lane l has values 8 l .. 8 l + 7, one access per buffer (32 bytes of fp32, 16 of 16-bit values, 8 of codes).  Otherwise (a
// block that a tensor's end cuts, or buffers that lie unaligned): values l, 32 + l, ..., which moves whole sectors too, with
// eight times the accesses.
__device__ __forceinline__ void load_256(uint32_t* r, const void* src)
{
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(src) : "memory");
}
struct Raw { uint32_t w[kPer]; };
template <bool VEC>
__device__ __forceinline__ void fetch(Raw& r, const void* base, int type, int64_t at, int count, int lane)
{
    if (VEC) {
        if (type == ST_F32) load_256(r.w, (const float*)base + at + kPer * lane);
        else {
            const uint4 q = *(const uint4*)((const uint16_t*)base + at + kPer * lane);
            r.w[0] = q.x; r.w[1] = q.y; r.w[2] = q.z; r.w[3] = q.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int i = 32 * j + lane;
            r.w[j] = i >= count ? 0u : type == ST_F32 ? ((const uint32_t*)base)[at + i] : (uint32_t)((const uint16_t*)base)[at + i];
        }
    }
}
__device__ __forceinline__ float from16(uint32_t h, int type)
{
    return type == ST_BF16 ? __uint_as_float(h << 16) : __half2float(__ushort_as_half((unsigned short)h));
}
template <bool VEC>
__device__ __forceinline__ void convert(float (&x)[kPer], const Raw& r, int type)
{
    if (type == ST_F32) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) x[j] = __uint_as_float(r.w[j]);
    } else {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const uint32_t h = VEC ? (r.w[j >> 1] >> ((j & 1) * 16)) & 0xffffu : r.w[j];
            x[j] = from16(h, type);
        }
    }
}
__device__ __forceinline__ uint32_t to16(float x, int type)
{
    return type == ST_BF16 ? (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(x)) : (uint32_t)__half_as_ushort(__float2half_rn(x));
}
__device__ __forceinline__ uint32_t pair16(float lo, float hi, int type)
{
    if (type == ST_BF16) { const __nv_bfloat162 q = __floats2bfloat162_rn(lo, hi); return *(const uint32_t*)&q; }
    const __half2 q = __floats2half2_rn(lo, hi);
    return *(const uint32_t*)&q;
}
template <bool VEC>
__device__ __forceinline__ void put(const float (&x)[kPer], void* base, int type, int64_t at, int count, int lane)
{
    if (VEC) {
        if (type == ST_F32) {
            const uint32_t r[kPer] = {__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]),
                                      __float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])};
            store_256((float*)base + at + kPer * lane, r);
        } else {
            *(uint4*)((uint16_t*)base + at + kPer * lane) = make_uint4(pair16(x[0], x[1], type), pair16(x[2], x[3], type), pair16(x[4], x[5], type), pair16(x[6], x[7], type));
        }
    } else {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int i = 32 * j + lane;
            if (i >= count) continue;
            if (type == ST_F32) ((float*)base)[at + i] = x[j];
            else ((uint16_t*)base)[at + i] = (uint16_t)to16(x[j], type);
        }
    }
}
template <bool VEC>
__device__ __forceinline__ void fetch_codes(Raw& r, const void* base, int64_t at, int count, int lane)
{
    const uint8_t* b = (const uint8_t*)base + at;
    if (VEC) {
        const uint2 q = *(const uint2*)(b + kPer * lane);
        r.w[0] = q.x; r.w[4] = q.y;
    } else {
#pragma unroll
        for (int j = 0; j < kPer; ++j) { const int i = 32 * j + lane; r.w[j] = i < count ? b[i] : 0u; }
    }
}
// Code j of a lane as fp32: its byte becomes the low byte of 2^23's mantissa (one permutation and one sum, where a conversion of an
// integer goes through a slower unit).  `flip` and `base`: 0x80 in each byte and 2^23 + 128 for signed codes, 0 and 2^23 for others.
template <bool VEC> __device__ __forceinline__ float code(const Raw& r, int j, uint32_t flip, float base)
{
    return VEC ? __uint_as_float(__byte_perm(r.w[j & 4] ^ flip, 0x4b000000u, 0x7440u | (j & 3))) - base
               : __uint_as_float(__byte_perm(r.w[j] ^ flip, 0x4b000000u, 0x7440u)) - base;
}
__device__ __forceinline__ uint32_t low_bytes(const uint32_t* c) { return __byte_perm(__byte_perm(c[0], c[1], 0x0040u), __byte_perm(c[2], c[3], 0x0040u), 0x5410u); }
// Codes come as the low bytes of 32-bit words
template <bool VEC>
__device__ __forceinline__ void put_codes(const uint32_t (&c)[kPer], void* base, int64_t at, int count, int lane)
{
    uint8_t* b = (uint8_t*)base + at;
    if (VEC) {
        *(uint2*)(b + kPer * lane) = make_uint2(low_bytes(c), low_bytes(c + 4));
    } else {
#pragma unroll
        for (int j = 0; j < kPer; ++j) { const int i = 32 * j + lane; if (i < count) b[i] = (uint8_t)c[j]; }
    }
}

// ---- moments in 8 bits ------------------------------------------------------------------------------------
// Every product and sum that decides on a level is rounded by itself (no fused multiply-add), so that the levels follow from the
// formulas in the header alone, on any device.
template <bool VEC>
__device__ __forceinline__ void decode(float (&m)[kPer], float (&root)[kPer], const Raw& rm, const Raw& rv, float m_scale, float v_scale)
{
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const float c = code<VEC>(rm, j, 0x80808080u, 8388608.f + 128.f), d = code<VEC>(rv, j, 0u, 8388608.f);
        m[j] = __fmul_rn(__fmul_rn(c, fabsf(c)), m_scale);
        root[j] = __fmul_rn(__fmul_rn(d, d), v_scale);
    }
}

// The level floor(sqrt(r) + 1/2).  The approximate root lies within 2^-23 of the root.  The ratio of sqrt(v) is formed from an approximate root (2^-23 of
// itself) and rounded, the one that defines the level from the rounded root (2^-24) and rounded too: 2.5 * 2^-23 between the two, half of it between
// their roots.  So rounding the approximate root to the nearest whole number gives the level unless it lies next to a border: within 127 * 2^-23 = 1.6e-5
// of one for m, 255 * 2.25 * 2^-23 = 6.9e-5 for sqrt(v).  There the border, which fp32 holds exactly, decides.
constexpr float kNearM = 2e-5f, kNearV = 7e-5f, kRound = 12582912.f;      // adding 1.5 * 2^23 rounds to a whole number and leaves it in the low bits
static_assert(kNearM > 127 * 0x1p-23 && kNearV > 255 * 2.25 * 0x1p-23, "values next to a border would not be looked at exactly");
__device__ __forceinline__ float approximate_root(float r)
{
    float s;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(r));
    return s;
}
__device__ __forceinline__ float exact_level(float r)
{
    float c = floorf(approximate_root(r) + 0.5f);
    const float below = c - 0.5f, above = c + 0.5f;
    if (r < below * below && c > 0.f) c -= 1.f;
    if (r >= above * above) c += 1.f;
    return c;
}
// Levels (low bytes) of a warp's block from m and sqrt(v), and its two scales.  No level leaves its range: the largest ratio is 127^2 or 255^2
// to within 2^-22.
__device__ __forceinline__ void encode(const float (&m)[kPer], const float (&root)[kPer], uint32_t (&cm)[kPer], uint32_t (&cv)[kPer], float& m_scale, float& v_scale)
{
    uint32_t top = 0, top_root = 0;             // of values that are not negative the bits are in the values' order, and NaN is above infinity
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        top = max(top, __float_as_uint(m[j]) & 0x7fffffffu);
        top_root = max(top_root, __float_as_uint(root[j]) & 0x7fffffffu);
    }
    const float a = __uint_as_float(__reduce_max_sync(0xffffffffu, top)), b = __uint_as_float(__reduce_max_sync(0xffffffffu, top_root));
    m_scale = a < 0x1p-100f ? 0.f : __fdiv_rn(a, 127.f * 127.f);
    v_scale = __fdiv_rn(b, 255.f * 255.f);
    const float im = m_scale > 0.f ? __frcp_rn(m_scale) : 0.f, iv = v_scale > 0.f ? __frcp_rn(v_scale) : 0.f;
    float far_m = 0.f, far_v = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const float s = copysignf(approximate_root(__fmul_rn(fabsf(m[j]), im)), m[j]), y = s + kRound;
        // a second moment that is not 0 has level 1 at least (the least root is 3.7e-23)
        const float r = fmaxf(approximate_root(__fmul_rn(root[j], iv)), __saturatef(root[j] * FLT_MAX)), z = r + kRound;
        far_m = fmaxf(far_m, fabsf(s - (y - kRound)));
        far_v = fmaxf(far_v, fabsf(r - (z - kRound)));
        cm[j] = __float_as_uint(y);
        cv[j] = __float_as_uint(z);
    }
    if (far_m > 0.5f - kNearM || far_v > 0.5f - kNearV) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const float c = exact_level(__fmul_rn(fabsf(m[j]), im)), d = exact_level(__fmul_rn(root[j], iv));
            cm[j] = __float_as_uint(copysignf(c, m[j]) + kRound);
            cv[j] = __float_as_uint(fmaxf(d, __saturatef(root[j] * FLT_MAX)) + kRound);
        }
    }
}

// ---- which values are a block's ---------------------------------------------------------------------------------
// Part b of a launch's parts takes the b-th share of the chunks, consecutive ones, so that the record of a tensor is read once per share and
// what follows are addresses that need no further look-up.  (A table entry per chunk, read in turn, put two dependent loads in front of
// each chunk's own.)  The first record is read ahead of pdl_wait().
struct Share { int64_t c, end; ChunkRec chunk; TensorRec tensor; };
__device__ __forceinline__ Share share_of(const Plan& p, int64_t from, int64_t to, int part, int parts)
{
    Share s;
    s.c = from + (to - from) * part / parts;
    s.end = from + (to - from) * (part + 1) / parts;
    if (s.c < s.end) { s.chunk = p.chunks[s.c]; s.tensor = p.tensors[s.chunk.tensor]; }
    return s;
}
// f(index of the tensor, its record, first value of the share's part of it, end of that part)
template <typename F>
__device__ __forceinline__ void walk(const Plan& p, Share& s, F&& f)
{
    while (s.c < s.end) {
        const int64_t here = min((s.tensor.n + kChunk - 1) / kChunk - s.chunk.index, s.end - s.c);
        f(s.chunk.tensor, s.tensor, (int64_t)s.chunk.index * kChunk, min((s.chunk.index + here) * kChunk, s.tensor.n));
        s.c += here;
        if (s.c < s.end) { s.chunk = p.chunks[s.c]; s.tensor = p.tensors[s.chunk.tensor]; }
    }
}

// ---- one step ----------------------------------------------------------------------------------------------
struct StepNow { float lr1_over_lr, r2, lr, factor, b1, b2, omb1, omb2, eps, one; };

// m and sqrt(v) of a step from those before it and the gradient
__device__ __forceinline__ void moments_8(const StepNow& k, float g, float& m, float& root)
{
    g = __fmul_rn(g, k.factor);
    m = __fadd_rn(__fmul_rn(m, k.b1), __fmul_rn(g, k.omb1));
    root = __fsqrt_rn(__fadd_rn(__fmul_rn(__fmul_rn(root, root), k.b2), __fmul_rn(__fmul_rn(g, g), k.omb2)));
}

// Square root and quotient to within a rounding for any value, without the library's branches for operands at the ends of the range: a unit without
// a gradient has v = 0, and its m shrinks until it is the last subnormals for good, so that a step of 44 M such values took 278 us instead of 222.
// The root of small values is that of 2^96 times the value; the quotient is the approximate one after a Newton step with the residual.
__device__ __forceinline__ float root_of(float v)
{
    const bool small = v < 0x1p-96f;
    const float r = __fsqrt_rn(v == 0.f ? 1.f : small ? v * 0x1p96f : v);
    return v == 0.f ? 0.f : small ? r * 0x1p-48f : r;
}
__device__ __forceinline__ float approximate_reciprocal(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
// Below kMostEps a denominator above 2^125, whose reciprocal leaves fp32's normal range, has a root that has left fp32: finite roots end at 1.9e19, times
// r2 of 9.5e7 at most (the largest beta2 below 1).
constexpr double kMostEps = 0x1p100;
__device__ __forceinline__ float quotient(float m, float den)       // den >= FLT_MIN, or NaN
{
    const float y = approximate_reciprocal(den), q = m * y;
    if (den > 0x1p125f) return m * 0.f;                                 // sqrt(v) that left fp32: no step, NaN if m has left it too
    return fabsf(q) <= FLT_MAX ? fmaf(fmaf(-q, den, m), y, q) : q;
}

// A warp's 256 values
template <int BITS, bool VEC>
__device__ __forceinline__ void step_block(const TensorRec& t, int param_type, int grad_type, bool has_master, const void* grad, const StepNow& k, int64_t at, int count, int lane)
{
    const void* from = has_master ? (const void*)t.master : t.param;
    const int from_type = has_master ? ST_F32 : param_type;
    Raw rg, rp, rm, rv;
    fetch<VEC>(rg, grad, grad_type, at, count, lane);
    fetch<VEC>(rp, from, from_type, at, count, lane);
    float m_scale = 0.f, v_scale = 0.f;
    const int64_t block = at / kBlockVals;
    if (BITS == 32) {
        fetch<VEC>(rm, t.m, ST_F32, at, count, lane);
        fetch<VEC>(rv, t.v, ST_F32, at, count, lane);
    } else {
        fetch_codes<VEC>(rm, t.m, at, count, lane);
        fetch_codes<VEC>(rv, t.v, at, count, lane);
        m_scale = t.m_scale[block]; v_scale = t.v_scale[block];
    }
    const float lr = k.lr * t.lr_scale, lr1 = lr * k.lr1_over_lr, decay = lr * t.wd;
    float g[kPer], x[kPer], m[kPer], root[kPer], v[kPer];
    convert<VEC>(g, rg, grad_type);
    convert<VEC>(x, rp, from_type);
    if (BITS == 32) {
        convert<VEC>(m, rm, ST_F32);
        convert<VEC>(v, rv, ST_F32);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const float gj = g[j] * k.factor;
            m[j] = fmaf(k.b1, m[j], k.omb1 * gj);
            v[j] = fmaf(k.b2, v[j], k.omb2 * gj * gj);
            root[j] = root_of(v[j]);
        }
        put<VEC>(m, t.m, ST_F32, at, count, lane);
        put<VEC>(v, t.v, ST_F32, at, count, lane);
    } else {
        decode<VEC>(m, root, rm, rv, m_scale, v_scale);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            moments_8(k, g[j], m[j], root[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const float kept = fmaf(-decay, x[j], x[j]);
        // 8 bits: the quotient to 2^-22 of itself (its moments are levels 1 per cent and more apart)
        const float den = fmaf(root[j], k.r2, k.eps);
        x[j] = fmaf(-lr1, BITS == 32 ? quotient(m[j], den) : __fdividef(m[j], den), kept);
    }
    put<VEC>(x, t.param, param_type, at, count, lane);
    if (has_master) put<VEC>(x, t.master, ST_F32, at, count, lane);
    if (BITS == 8) {
        uint32_t cm[kPer], cv[kPer];
        encode(m, root, cm, cv, m_scale, v_scale);
        put_codes<VEC>(cm, t.m, at, count, lane);
        put_codes<VEC>(cv, t.v, at, count, lane);
        if (lane == 0) { t.m_scale[block] = m_scale; t.v_scale[block] = v_scale; }
    }
}

__device__ __forceinline__ bool grad_aligned(const void* grad, int type) { return ((uintptr_t)grad & (type == ST_F32 ? 31u : 15u)) == 0; }

// Two fp32 operations in one instruction, each rounded by itself
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void unpack2(f32x2 x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) { f32x2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
// a + b where both are products that are rounded by themselves: the assembler makes one fused operation of mul.rn.f32x2 and add.rn.f32x2, but
// not of a product and a multiplication by a factor that it does not know (`one` is 1)
__device__ __forceinline__ f32x2 sum2(f32x2 a, f32x2 b, f32x2 one) { return fma2(a, one, b); }
__device__ __forceinline__ f32x2 both(float a) { return pack2(a, a); }

// The 8-bit step of whole blocks: the same results for the moments as step_block<8>, with fewer instructions, whose issue bounds it.
// Pairs of values go through one instruction; square roots are approximate (2^-23 of themselves: parameters need no more, and a level only
// next to a border, where exact_codes decides).
struct Loads8 { Raw g, p, m, v; float m_scale, v_scale; };
template <int PARAM, int GRAD, bool MASTER>
__device__ __forceinline__ void fetch_8(Loads8& l, const TensorRec& t, const void* grad, int64_t at, int lane)
{
    fetch<true>(l.g, grad, GRAD, at, kBlockVals, lane);
    fetch_codes<true>(l.m, t.m, at, kBlockVals, lane);
    fetch_codes<true>(l.v, t.v, at, kBlockVals, lane);
    l.m_scale = t.m_scale[at / kBlockVals];
    l.v_scale = t.v_scale[at / kBlockVals];
    if (MASTER) fetch<true>(l.p, t.master, ST_F32, at, kBlockVals, lane);
    else fetch<true>(l.p, t.param, PARAM, at, kBlockVals, lane);
}
// A lane's codes of a block, exactly, from what the block's step reads (old codes and scales, which must not have been overwritten) and the
// reciprocals of its new scales.  Out of line: a lane in 690 comes here, and its registers are not the step's.
template <int GRAD>
__device__ __noinline__ uint4 exact_codes(const TensorRec* t, const void* grad, StepNow k, int64_t at, float im, float iv)
{
    const int lane = threadIdx.x % 32;
    Raw rg, rm, rv;
    float g[kPer], m[kPer], root[kPer];
    fetch<true>(rg, grad, GRAD, at, kBlockVals, lane);
    fetch_codes<true>(rm, t->m, at, kBlockVals, lane);
    fetch_codes<true>(rv, t->v, at, kBlockVals, lane);
    convert<true>(g, rg, GRAD);
    decode<true>(m, root, rm, rv, t->m_scale[at / kBlockVals], t->v_scale[at / kBlockVals]);
    uint32_t cm[kPer], cv[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        moments_8(k, g[j], m[j], root[j]);
        cm[j] = __float_as_uint(copysignf(exact_level(__fmul_rn(fabsf(m[j]), im)), m[j]) + kRound);
        cv[j] = __float_as_uint(fmaxf(exact_level(__fmul_rn(root[j], iv)), __saturatef(root[j] * FLT_MAX)) + kRound);
    }
    return make_uint4(low_bytes(cm), low_bytes(cm + 4), low_bytes(cv), low_bytes(cv + 4));
}

template <int PARAM, int GRAD, bool MASTER>
__device__ __forceinline__ void step_block_8(const TensorRec* record, const TensorRec& t, const void* grad, const Loads8& l, const StepNow& k, int64_t at, int lane)
{
    constexpr int kPairs = kPer / 2;
    float root[kPer], m[kPer];
    // the largest |m| and v of the block (bits of values that are not negative are in the values' order, NaN above infinity)
    uint32_t top = 0, top_v = 0;
    {
        float g[kPer];
        convert<true>(g, l.g, GRAD);
        const f32x2 ms = both(l.m_scale), vs = both(l.v_scale), factor = both(k.factor), b1 = both(k.b1), b2 = both(k.b2), omb1 = both(k.omb1), omb2 = both(k.omb2), one = both(k.one);
#pragma unroll
        for (int q = 0; q < kPairs; ++q) {
            const float c0 = code<true>(l.m, 2 * q, 0x80808080u, 8388608.f + 128.f), c1 = code<true>(l.m, 2 * q + 1, 0x80808080u, 8388608.f + 128.f);
            const f32x2 d = pack2(code<true>(l.v, 2 * q, 0u, 8388608.f), code<true>(l.v, 2 * q + 1, 0u, 8388608.f));
            const f32x2 gj = mul2(pack2(g[2 * q], g[2 * q + 1]), factor);
            const f32x2 mj = sum2(mul2(mul2(pack2(__fmul_rn(c0, fabsf(c0)), __fmul_rn(c1, fabsf(c1))), ms), b1), mul2(gj, omb1), one);
            const f32x2 r = mul2(mul2(d, d), vs);
            float v0, v1;
            unpack2(sum2(mul2(mul2(r, r), b2), mul2(mul2(gj, gj), omb2), one), v0, v1);
            unpack2(mj, m[2 * q], m[2 * q + 1]);
            top = max(top, max(__float_as_uint(m[2 * q]) & 0x7fffffffu, __float_as_uint(m[2 * q + 1]) & 0x7fffffffu));
            top_v = max(top_v, max(__float_as_uint(v0), __float_as_uint(v1)));
            asm("sqrt.approx.f32 %0, %1;" : "=f"(root[2 * q]) : "f"(v0));
            asm("sqrt.approx.f32 %0, %1;" : "=f"(root[2 * q + 1]) : "f"(v1));
        }
    }
    // the two scales and their reciprocals, m's in the lower lanes and v's in the upper ones: one division and one reciprocal for both
    const float a = __uint_as_float(__reduce_max_sync(0xffffffffu, top)), b = __fsqrt_rn(__uint_as_float(__reduce_max_sync(0xffffffffu, top_v)));
    const bool low = lane < 16;
    const float scale = low && a < 0x1p-100f ? 0.f : __fdiv_rn(low ? a : b, low ? 127.f * 127.f : 255.f * 255.f);    // roots are rounded in the values' order: b is the largest root
    const float inverse = scale > 0.f ? __frcp_rn(scale) : 0.f, im = __shfl_sync(0xffffffffu, inverse, 0), iv = __shfl_sync(0xffffffffu, inverse, 16);
    {
        float x[kPer];
        convert<true>(x, l.p, MASTER ? ST_F32 : PARAM);
        const float lr = k.lr * t.lr_scale;
        const f32x2 lr1 = both(-lr * k.lr1_over_lr), decay = both(-lr * t.wd), r2 = both(k.r2), eps = both(k.eps);
#pragma unroll
        for (int q = 0; q < kPairs; ++q) {
            const f32x2 xj = pack2(x[2 * q], x[2 * q + 1]);
            const f32x2 kept = fma2(decay, xj, xj);
            float d0, d1;
            unpack2(fma2(pack2(root[2 * q], root[2 * q + 1]), r2, eps), d0, d1);
            // the quotient to 2^-22 of itself: the moments are levels 1 per cent and more apart
            const f32x2 u = mul2(pack2(m[2 * q], m[2 * q + 1]), pack2(approximate_reciprocal(d0), approximate_reciprocal(d1)));
            unpack2(fma2(lr1, u, kept), x[2 * q], x[2 * q + 1]);
        }
        put<true>(x, t.param, PARAM, at, kBlockVals, lane);
        if (MASTER) put<true>(x, t.master, ST_F32, at, kBlockVals, lane);
    }
    uint32_t cm[kPer], cv[kPer];
    float far_m = 0.f, far_v = 0.f;
    const f32x2 im2 = both(im), iv2 = both(iv), up = both(kRound), down = both(-kRound), minus = both(-1.f);
#pragma unroll
    for (int q = 0; q < kPairs; ++q) {
        float t0, t1, r0, r1, e0, e1;
        unpack2(mul2(pack2(m[2 * q], m[2 * q + 1]), im2), t0, t1);
        unpack2(mul2(pack2(root[2 * q], root[2 * q + 1]), iv2), r0, r1);
        const f32x2 s = pack2(copysignf(approximate_root(fabsf(t0)), t0), copysignf(approximate_root(fabsf(t1)), t1));
        const f32x2 r = pack2(fmaxf(approximate_root(r0), __saturatef(root[2 * q] * FLT_MAX)), fmaxf(approximate_root(r1), __saturatef(root[2 * q + 1] * FLT_MAX)));
        const f32x2 y = add2(s, up), z = add2(r, up);
        unpack2(fma2(add2(y, down), minus, s), e0, e1);
        far_m = fmaxf(far_m, fmaxf(fabsf(e0), fabsf(e1)));
        unpack2(fma2(add2(z, down), minus, r), e0, e1);
        far_v = fmaxf(far_v, fmaxf(fabsf(e0), fabsf(e1)));
        cm[2 * q] = (uint32_t)y; cm[2 * q + 1] = (uint32_t)(y >> 32);
        cv[2 * q] = (uint32_t)z; cv[2 * q + 1] = (uint32_t)(z >> 32);
    }
    uint4 codes = make_uint4(low_bytes(cm), low_bytes(cm + 4), low_bytes(cv), low_bytes(cv + 4));
    if (far_m > 0.5f - kNearM || far_v > 0.5f - kNearV) codes = exact_codes<GRAD>(record, grad, k, at, im, iv);
    __syncwarp();                                               // nobody reads the old scales any more
    *(uint2*)((uint8_t*)t.m + at + kPer * lane) = make_uint2(codes.x, codes.y);
    *(uint2*)((uint8_t*)t.v + at + kPer * lane) = make_uint2(codes.z, codes.w);
    if ((lane & 15) == 0) (low ? t.m_scale : t.v_scale)[at / kBlockVals] = scale;
}

// All whole blocks of a tensor's part; returns where it stopped.  A function of its own for each combination of types: the conversions
// are decided outside the loop, and the registers are this loop's alone (inlined into the walk, the 8-bit step of 200 M bf16
// values took 738 us with all combinations side by side and 545 with one compiled alone).  A warp loads a block, works it out and stores it; what covers
// its loads are the other warps of the SM.
template <int BITS, int PARAM, int GRAD, bool MASTER>
__device__ __noinline__ int64_t step_blocks(const TensorRec* record, const void* grad, StepNow k, int64_t at, int64_t end)
{
    const int lane = threadIdx.x % 32;
    const TensorRec t = *record;
    if (BITS == 8) {
        Loads8 now;
        for (; at + kBlockVals <= end; at += kChunk) {
            fetch_8<PARAM, GRAD, MASTER>(now, t, grad, at, lane);
            step_block_8<PARAM, GRAD, MASTER>(record, t, grad, now, k, at, lane);
        }
    } else {
        for (; at + kBlockVals <= end; at += kChunk) step_block<32, true>(t, PARAM, GRAD, MASTER, grad, k, at, kBlockVals, lane);
    }
    return at;
}
template <int BITS, int PARAM, bool MASTER, typename... A>
__device__ __forceinline__ int64_t step_blocks_of(int grad_type, const A&... a)
{
    return grad_type == ST_F32 ? step_blocks<BITS, PARAM, ST_F32, MASTER>(a...) : grad_type == ST_BF16 ? step_blocks<BITS, PARAM, ST_BF16, MASTER>(a...)
                                                                                                      : step_blocks<BITS, PARAM, ST_F16, MASTER>(a...);
}
template <int BITS, bool MASTER, typename... A>
__device__ __forceinline__ int64_t step_blocks_of(int param_type, int grad_type, const A&... a)
{
    return param_type == ST_F32 ? step_blocks_of<BITS, ST_F32, MASTER>(grad_type, a...) : param_type == ST_BF16 ? step_blocks_of<BITS, ST_BF16, MASTER>(grad_type, a...)
                                                                                                             : step_blocks_of<BITS, ST_F16, MASTER>(grad_type, a...);
}

// The path of single values, out of line: its registers are not the vector path's
template <int BITS>
__device__ __noinline__ void step_block_slow(const TensorRec* t, const void* grad, StepNow k, int64_t at, int lane)
{
    step_block<BITS, false>(*t, t->param_type, t->grad_type, t->master != nullptr, grad, k, at, (int)min(t->n - at, (int64_t)kBlockVals), lane);
}

__host__ __device__ inline void bias_corrections(const double (&power)[2], float (&out)[2])
{
    out[0] = (float)(1.0 / (1.0 - power[0]));
    out[1] = (float)(1.0 / sqrt(1.0 - power[1]));
}

// Block 0 works the next step's bias corrections out; the others step the tensors.  (As exponentials they took over a microsecond; a product
// per step is off by 1e-16 of itself a step, when the power has long ceased to matter.)
template <int BITS>
__global__ void __launch_bounds__(kThreads, BITS == 32 ? 4 : 5) adamw_step_kernel(const __grid_constant__ Plan p, float grad_scale, int with_norm)
{
    Share share;
    if (blockIdx.x) share = share_of(p, 0, p.n_chunks, blockIdx.x - 1, gridDim.x - 1);
    pdl_wait();
    pdl_launch_dependents();
    Scalars* const sc = p.sc;
    const long long t = sc->t + 1;                      // every thread reads it: the step that is taken
    const float bias[2][2] = {{sc->bias[0][0], sc->bias[0][1]}, {sc->bias[1][0], sc->bias[1][1]}}, lr = sc->lr, factor = sc->factor;   // all on their way together
    const bool skip = with_norm && sc->skip;
    if (blockIdx.x == 0) {
        if (threadIdx.x == 0 && !skip) {
            const double power[2] = {sc->power[0] * p.beta1, sc->power[1] * p.beta2};
            float next[2];
            bias_corrections(power, next);
            sc->power[0] = power[0]; sc->power[1] = power[1];
            sc->bias[(t + 1) & 1][0] = next[0]; sc->bias[(t + 1) & 1][1] = next[1];
        }
    } else if (!skip) {
        const StepNow k = {t & 1 ? bias[1][0] : bias[0][0], t & 1 ? bias[1][1] : bias[0][1], lr, with_norm ? factor : grad_scale,
                           p.b1, p.b2, p.omb1, p.omb2, p.eps, p.one};
        const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
        walk(p, share, [&](int i, const TensorRec& t, int64_t begin, int64_t end) {
            const void* grad = p.grads[i];
            if (!grad) return;
            int64_t at = begin + warp * kBlockVals;
            if (t.vec && grad_aligned(grad, t.grad_type))
                at = t.master ? step_blocks_of<BITS, true>(t.param_type, t.grad_type, p.tensors + i, grad, k, at, end)
                              : step_blocks_of<BITS, false>(t.param_type, t.grad_type, p.tensors + i, grad, k, at, end);
            for (; at < end; at += kChunk) step_block_slow<BITS>(p.tensors + i, grad, k, at, lane);
        });
    }
    // The block that finishes last counts the step: every thread of every block has read the count by then.  (No fence: nothing that the
    // blocks have written is read before the kernel is complete.)
    __syncthreads();
    if (threadIdx.x == 0 && atomicAdd(&sc->step_ticket, 1u) == gridDim.x - 1) {
        sc->step_ticket = 0;
        if (!skip) sc->t = t;
    }
}

// ---- norm of all gradients -----------------------------------------------------------------------------------
__device__ __forceinline__ double block_sum(double x, double (&shared)[kWarps])
{
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = x;
    __syncthreads();
    x = 0;
    for (int i = 0; i < kWarps; ++i) x += shared[i];
    __syncthreads();
    return x;
}

__global__ void __launch_bounds__(kThreads) adamw_norm_kernel(const __grid_constant__ Plan p, float grad_scale, float* norm_out)
{
    __shared__ double shared[kWarps];
    __shared__ bool last;
    Share share = share_of(p, 0, p.n_chunks, blockIdx.x, gridDim.x);
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    double sum = 0;
    const auto add = [&](const float (&g)[kPer]) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) { const double d = g[j]; sum = fma(d, d, sum); }
    };
    walk(p, share, [&](int i, const TensorRec& t, int64_t begin, int64_t end) {
        const void* grad = p.grads[i];
        if (!grad) return;
        const int type = t.grad_type;
        int64_t at = begin + warp * kBlockVals;
        if (grad_aligned(grad, type)) {
            constexpr int kFlight = 4;          // a warp's blocks whose loads are on their way together
            for (; at + (kFlight - 1) * kChunk + kBlockVals <= end; at += kFlight * kChunk) {
                Raw r[kFlight];
#pragma unroll
                for (int u = 0; u < kFlight; ++u) fetch<true>(r[u], grad, type, at + u * kChunk, kBlockVals, lane);
#pragma unroll
                for (int u = 0; u < kFlight; ++u) { float g[kPer]; convert<true>(g, r[u], type); add(g); }
            }
            for (; at + kBlockVals <= end; at += kChunk) { Raw r; float g[kPer]; fetch<true>(r, grad, type, at, kBlockVals, lane); convert<true>(g, r, type); add(g); }
        }
        // one by one, each lane the eight values that it has on the vector path
        for (; at < end; at += kChunk) {
            const int64_t first = at + kPer * lane;
            const int count = (int)min(max(end - first, (int64_t)0), (int64_t)kPer);
            float g[kPer];
            if (type == ST_F32) {
                const float* q = (const float*)grad + first;
                if (count == kPer) {                    // in pairs where they lie at multiples of 8 bytes: half of the accesses
                    const bool odd = (uintptr_t)q & 4;
                    if (odd) { g[0] = q[0]; g[7] = q[7]; ++q; }
                    const float2 a = *(const float2*)q, b = *(const float2*)(q + 2), c = *(const float2*)(q + 4);
                    if (odd) { g[1] = a.x; g[2] = a.y; g[3] = b.x; g[4] = b.y; g[5] = c.x; g[6] = c.y; }
                    else { const float2 d = *(const float2*)(q + 6); g[0] = a.x; g[1] = a.y; g[2] = b.x; g[3] = b.y; g[4] = c.x; g[5] = c.y; g[6] = d.x; g[7] = d.y; }
                } else {
#pragma unroll
                    for (int j = 0; j < kPer; ++j) g[j] = j < count ? q[j] : 0.f;
                }
            } else {
#pragma unroll
                for (int j = 0; j < kPer; ++j) g[j] = from16(j < count ? ((const uint16_t*)grad)[first + j] : 0u, type);
            }
            add(g);
        }
    });
    sum = block_sum(sum, shared);
    if (threadIdx.x == 0) {
        p.partials[blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(&p.sc->norm_ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum = 0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += kThreads) sum += __ldcg(p.partials + i);
    sum = block_sum(sum, shared);
    if (threadIdx.x == 0) {
        const double norm = sqrt(sum) * fabs((double)grad_scale);
        const double ratio = p.max_norm > 0 ? p.max_norm / (norm + 1e-6) : 1.0;
        p.sc->factor = (float)((double)grad_scale * (ratio >= 1.0 ? 1.0 : ratio));      // a norm that is NaN makes the gradients NaN
        p.sc->skip = p.skip_nonfinite && !isfinite(norm);
        p.sc->norm_ticket = 0;
        if (norm_out) *norm_out = (float)norm;
    }
}

// ---- where things are; the learning rate -----------------------------------------------------------------------
constexpr int kPointers = 448;      // of one launch: with the rest of the arguments inside the 4 KB that any launch may carry
struct PointerArgs { const void* q[kPointers]; };

__global__ void adamw_set_grads_kernel(const void** grads, int first, int count, const PointerArgs a)
{
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < count) grads[first + i] = a.q[i];
}
__global__ void adamw_set_lr_kernel(Scalars* sc, float lr) { sc->lr = lr; }

// ---- moments as fp32 values and back -----------------------------------------------------------------------
// Tensors [first, ...) of chunks [chunk_begin, chunk_end) with their pointers in the arguments: m's at 2 i, v's at 2 i + 1
struct Moments { Raw m, v; float m_scale, v_scale; };
template <int BITS, bool VEC>
__device__ __forceinline__ void fetch_moments(Moments& l, const TensorRec& t, int64_t at, int count, int lane)
{
    if (BITS == 32) {
        fetch<VEC>(l.m, t.m, ST_F32, at, count, lane);
        fetch<VEC>(l.v, t.v, ST_F32, at, count, lane);
    } else {
        fetch_codes<VEC>(l.m, t.m, at, count, lane);
        fetch_codes<VEC>(l.v, t.v, at, count, lane);
        l.m_scale = t.m_scale[at / kBlockVals];
        l.v_scale = t.v_scale[at / kBlockVals];
    }
}
template <int BITS, bool VEC>
__device__ __forceinline__ void put_moments(const Moments& l, float* m_out, float* v_out, int64_t at, int count, int lane)
{
    float m[kPer], v[kPer];
    if (BITS == 32) {
        convert<VEC>(m, l.m, ST_F32);
        convert<VEC>(v, l.v, ST_F32);
    } else {
        decode<VEC>(m, v, l.m, l.v, l.m_scale, l.v_scale);
#pragma unroll
        for (int j = 0; j < kPer; ++j) v[j] = __fmul_rn(v[j], v[j]);
    }
    if (m_out) put<VEC>(m, m_out, ST_F32, at, count, lane);
    if (v_out) put<VEC>(v, v_out, ST_F32, at, count, lane);
}
template <int BITS>
__global__ void __launch_bounds__(kThreads) adamw_read_kernel(const __grid_constant__ Plan p, int first, int64_t chunk_begin, int64_t chunk_end, const __grid_constant__ PointerArgs a)
{
    Share share = share_of(p, chunk_begin, chunk_end, blockIdx.x, gridDim.x);
    pdl_wait();
    pdl_launch_dependents();
    constexpr int kFlight = BITS == 8 ? 2 : 1;          // a warp's blocks whose loads are on their way together
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    walk(p, share, [&](int i, const TensorRec& t, int64_t begin, int64_t end) {
        float *m_out = (float*)a.q[2 * (i - first)], *v_out = (float*)a.q[2 * (i - first) + 1];
        const bool vec = t.vec && (((uintptr_t)m_out | (uintptr_t)v_out) & 31) == 0;
        int64_t at = begin + warp * kBlockVals;
        Moments l[kFlight];
        if (vec) {
            for (; at + (kFlight - 1) * kChunk + kBlockVals <= end; at += kFlight * kChunk) {
#pragma unroll
                for (int u = 0; u < kFlight; ++u) fetch_moments<BITS, true>(l[u], t, at + u * kChunk, kBlockVals, lane);
#pragma unroll
                for (int u = 0; u < kFlight; ++u) put_moments<BITS, true>(l[u], m_out, v_out, at + u * kChunk, kBlockVals, lane);
            }
            for (; at + kBlockVals <= end; at += kChunk) { fetch_moments<BITS, true>(l[0], t, at, kBlockVals, lane); put_moments<BITS, true>(l[0], m_out, v_out, at, kBlockVals, lane); }
        }
        for (; at < end; at += kChunk) {
            const int count = (int)min(end - at, (int64_t)kBlockVals);
            fetch_moments<BITS, false>(l[0], t, at, count, lane);
            put_moments<BITS, false>(l[0], m_out, v_out, at, count, lane);
        }
    });
}

template <int BITS>
__global__ void __launch_bounds__(kThreads) adamw_write_kernel(const __grid_constant__ Plan p, int first, int64_t chunk_begin, int64_t chunk_end, const __grid_constant__ PointerArgs a)
{
    Share share = share_of(p, chunk_begin, chunk_end, blockIdx.x, gridDim.x);
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    walk(p, share, [&](int i, const TensorRec& t, int64_t begin, int64_t end) {
        const float *m_in = (const float*)a.q[2 * (i - first)], *v_in = (const float*)a.q[2 * (i - first) + 1];
        for (int64_t at = begin + warp * kBlockVals; at < end; at += kChunk) {
            const int count = (int)min(t.n - at, (int64_t)kBlockVals);
            float m[kPer] = {}, v[kPer] = {};
            Raw r;
            if (m_in) { fetch<false>(r, m_in, ST_F32, at, count, lane); convert<false>(m, r, ST_F32); }
            if (v_in) { fetch<false>(r, v_in, ST_F32, at, count, lane); convert<false>(v, r, ST_F32); }
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[j] = v[j] < 0.f ? 0.f : v[j];
            if (BITS == 32) {
                if (m_in) put<false>(m, t.m, ST_F32, at, count, lane);
                if (v_in) put<false>(v, t.v, ST_F32, at, count, lane);
            } else {
#pragma unroll
                for (int j = 0; j < kPer; ++j) v[j] = __fsqrt_rn(v[j]);
                uint32_t cm[kPer], cv[kPer];
                float ms, vs;
                encode(m, v, cm, cv, ms, vs);
                if (m_in) { put_codes<false>(cm, t.m, at, count, lane); if (lane == 0) t.m_scale[at / kBlockVals] = ms; }
                if (v_in) { put_codes<false>(cv, t.v, at, count, lane); if (lane == 0) t.v_scale[at / kBlockVals] = vs; }
            }
        }
    });
}

}  // namespace
}  // namespace st

using namespace st;

// ---- C interface ---------------------------------------------------------------------------------------------
struct st_adamw {
    Plan plan = {};
    int device = 0, n = 0, bits = 32;
    cudaStream_t stream = nullptr;
    int step_grid = 0, norm_grid = 0, moments_span = 0, moments_resident = 0;
    bool always_norm = false;
    void* block = nullptr;                  // the one allocation: scalars, partial sums, tables
    std::vector<int64_t> first_chunk;       // [n + 1]
    std::vector<uint8_t> grad_type;
    std::vector<int64_t> values;
    struct Range { uintptr_t begin, end; };
    std::vector<Range> written;             // what a step writes, sorted and disjoint
    std::string err;
};

namespace {

st_status fail(st_adamw* o, st_status code, const char* fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    if (!o) return (st_status)fail_on_thread(code, "%s", buf);
    try { o->err = buf; } catch (...) {}
    return code;
}

// Calls work on the optimiser's device, whichever is current
struct OnDevice {
    int before = -1;
    bool ok = true;
    explicit OnDevice(int device)
    {
        ok = cudaGetDevice(&before) == cudaSuccess;
        if (ok && before != device) ok = cudaSetDevice(device) == cudaSuccess; else before = -1;
    }
    ~OnDevice() { if (before >= 0) cudaSetDevice(before); }
};

bool on_device(const void* q, int device)
{
    cudaPointerAttributes at;
    if (cudaPointerGetAttributes(&at, q) != cudaSuccess) { cudaGetLastError(); return false; }
    return at.type == cudaMemoryTypeManaged || (at.type == cudaMemoryTypeDevice && at.device == device);
}
size_t type_size(int type) { return type == ST_F32 ? 4 : 2; }
bool known_type(int type) { return type == ST_F32 || type == ST_BF16 || type == ST_F16; }
bool aligned(const void* q, size_t a) { return ((uintptr_t)q & (a - 1)) == 0; }

// nullptr where a buffer is fine, else what is wrong with it
const char* buffer_fault(const void* q, size_t element, int device)
{
    if (!q) return "is NULL";
    if (!aligned(q, element)) return "is not aligned to its elements";
    if (!on_device(q, device)) return "is not memory of the optimiser's device";
    return nullptr;
}

bool touches(const std::vector<st_adamw::Range>& sorted, uintptr_t begin, uintptr_t end)
{
    auto it = std::upper_bound(sorted.begin(), sorted.end(), begin, [](uintptr_t b, const st_adamw::Range& r) { return b < r.end; });
    return it != sorted.end() && it->begin < end;
}

// Sorts them
bool overlap(std::vector<st_adamw::Range>& ranges)
{
    std::sort(ranges.begin(), ranges.end(), [](const st_adamw::Range& a, const st_adamw::Range& b) { return a.begin < b.begin; });
    for (size_t i = 1; i < ranges.size(); ++i)
        if (ranges[i].begin < ranges[i - 1].end) return true;
    return false;
}

const char* grad_fault(const st_adamw* o, int i, const void* grad)
{
    if (!grad || o->values[i] == 0) return nullptr;
    const size_t size = type_size(o->grad_type[i]);
    if (const char* f = buffer_fault(grad, size, o->device)) return f;
    if (touches(o->written, (uintptr_t)grad, (uintptr_t)grad + size * o->values[i])) return "overlaps a buffer that the step writes";
    return nullptr;
}

// From what the launches returned: the thread's last error may be an earlier call's, and a step that is reported as failed must not have been enqueued
st_status check_launch(st_adamw* o, cudaError_t e, const char* what)
{
    if (e == cudaSuccess) return ST_OK;
    cudaGetLastError();
    return fail(o, ST_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

st_status create(const st_adamw_desc& d, const st_adamw_tensor* tensors, st_adamw* o)
{
    o->n = d.n_tensors; o->bits = d.state_bits; o->stream = (cudaStream_t)d.cuda_stream;
    if (cudaGetDevice(&o->device) != cudaSuccess) { cudaGetLastError(); return fail(nullptr, ST_ERR_CUDA, "st_adamw_create: no current device"); }
    std::vector<TensorRec> recs(d.n_tensors);
    o->first_chunk.assign(d.n_tensors + 1, 0);
    o->values.resize(d.n_tensors); o->grad_type.resize(d.n_tensors);
    int64_t total = 0;
    for (int i = 0; i < d.n_tensors; ++i) {
        const st_adamw_tensor& t = tensors[i];
        TensorRec& r = recs[i];
        if (t.n < 0 || !known_type(t.param_type) || !known_type(t.grad_type) || !std::isfinite(t.weight_decay) || !std::isfinite(t.lr_scale))
            return fail(nullptr, ST_ERR_INVALID_ARG, "st_adamw_create: tensor %d: negative size, unknown type, or weight_decay or lr_scale not finite", i);
        if (t.n > ((int64_t)1 << 42) - total) return fail(nullptr, ST_ERR_UNSUPPORTED, "st_adamw_create: more than 2^42 values");
        total += t.n;
        o->values[i] = t.n; o->grad_type[i] = (uint8_t)t.grad_type;
        o->first_chunk[i + 1] = o->first_chunk[i] + (t.n + kChunk - 1) / kChunk;
        r = TensorRec{t.param, t.master, t.exp_avg, t.exp_avg_sq, t.exp_avg_scale, t.exp_avg_sq_scale, t.n, t.weight_decay, t.lr_scale,
                      (uint8_t)t.param_type, (uint8_t)t.grad_type, 0, 0};
        if (t.n == 0) continue;
        const size_t moment = d.state_bits == 32 ? 4 : 1, scales = 4 * (size_t)((t.n + kBlockVals - 1) / kBlockVals);
        const struct { const char* name; const void* q; size_t element, bytes; bool needed; } buffers[] = {
            {"param", t.param, type_size(t.param_type), type_size(t.param_type) * t.n, true},
            {"master", t.master, 4, 4 * (size_t)t.n, t.master != nullptr},
            {"exp_avg", t.exp_avg, moment, moment * t.n, true},
            {"exp_avg_sq", t.exp_avg_sq, moment, moment * t.n, true},
            {"exp_avg_scale", t.exp_avg_scale, 4, scales, d.state_bits == 8},
            {"exp_avg_sq_scale", t.exp_avg_sq_scale, 4, scales, d.state_bits == 8}};
        for (const auto& b : buffers) {
            if (!b.needed) continue;
            if (const char* f = buffer_fault(b.q, b.element, o->device)) return fail(nullptr, ST_ERR_INVALID_ARG, "st_adamw_create: tensor %d: %s %s", i, b.name, f);
            o->written.push_back({(uintptr_t)b.q, (uintptr_t)b.q + b.bytes});
        }
        r.vec = aligned(t.param, kPer * type_size(t.param_type)) && aligned(t.master, kPer * 4) && aligned(t.exp_avg, kPer * moment) && aligned(t.exp_avg_sq, kPer * moment);
    }
    if (overlap(o->written)) return fail(nullptr, ST_ERR_INVALID_ARG, "st_adamw_create: two buffers that a step writes overlap");
    for (int i = 0; i < d.n_tensors; ++i)
        if (const char* f = grad_fault(o, i, tensors[i].grad)) return fail(nullptr, ST_ERR_INVALID_ARG, "st_adamw_create: tensor %d: grad %s", i, f);

    const int64_t n_chunks = o->first_chunk[d.n_tensors];
    int sms = 0, step = 0, norm = 0;
    cudaError_t e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, o->device);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&step, d.state_bits == 32 ? adamw_step_kernel<32> : adamw_step_kernel<8>, kThreads, 0);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&norm, adamw_norm_kernel, kThreads, 0);
    if (e != cudaSuccess) { cudaGetLastError(); return fail(nullptr, ST_ERR_CUDA, "st_adamw_create: %s", cudaGetErrorString(e)); }
    // Blocks of a launch: as many as the GPU holds at once, or one per `span` chunks where that is more.  A step with fp32 moments and the reading
    // of moments wait for memory, and short shares that the GPU hands out as blocks end keep all of it busy (150 M fp32 values with
    // spans of 4 / 8 chunks / one share per resident block: 633 / 648 / 690 us; reading 200 M values: 327 with 8, 353).  A step with 8-bit
    // moments and the norm have more to work out per byte, and a block's beginning and end cost more than an uneven end (200 M: 744 us with
    // spans of 8, 520 with one share each; norm 77 and 63).
    const auto blocks = [&](int per_sm, int span) {
        const int64_t resident = (int64_t)sms * std::max(per_sm, 1), most = span ? std::max(resident, n_chunks / span) : resident;
        return (int)std::max<int64_t>(1, std::min(n_chunks, most));
    };
    o->step_grid = 1 + blocks(step, d.state_bits == 32 ? 4 : 0);
    o->norm_grid = blocks(norm, 0);
    o->moments_span = 8; o->moments_resident = sms * 8;

    std::vector<ChunkRec> chunks((size_t)n_chunks);
    for (int i = 0; i < d.n_tensors; ++i)
        for (int64_t c = o->first_chunk[i]; c < o->first_chunk[i + 1]; ++c) chunks[c] = {i, (int32_t)(c - o->first_chunk[i])};
    const auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t at_partials = up(sizeof(Scalars)), at_tensors = at_partials + up(sizeof(double) * o->norm_grid),
                 at_grads = at_tensors + up(sizeof(TensorRec) * recs.size()),
                 at_chunks = at_grads + up(sizeof(void*) * recs.size()), bytes = at_chunks + up(sizeof(ChunkRec) * chunks.size());
    e = cudaMalloc(&o->block, bytes);
    if (e != cudaSuccess) { cudaGetLastError(); return fail(nullptr, e == cudaErrorMemoryAllocation ? ST_ERR_OOM : ST_ERR_CUDA, "st_adamw_create: %s", cudaGetErrorString(e)); }
    char* b = (char*)o->block;
    Plan& p = o->plan;
    p.sc = (Scalars*)b; p.partials = (double*)(b + at_partials); p.tensors = (const TensorRec*)(b + at_tensors); p.grads = (const void**)(b + at_grads);
    p.chunks = (const ChunkRec*)(b + at_chunks);
    p.n_chunks = n_chunks;
    p.beta1 = d.beta1; p.beta2 = d.beta2; p.max_norm = d.max_norm;
    p.b1 = (float)d.beta1; p.b2 = (float)d.beta2; p.omb1 = (float)(1.0 - d.beta1); p.omb2 = (float)(1.0 - d.beta2); p.eps = (float)d.eps; p.one = 1.f;
    p.skip_nonfinite = d.skip_nonfinite;
    o->always_norm = d.max_norm > 0 || d.skip_nonfinite;
    Scalars sc = {};
    sc.t = d.first_step; sc.lr = (float)d.lr; sc.factor = 1.f;
    sc.power[0] = pow(d.beta1, (double)d.first_step + 1); sc.power[1] = pow(d.beta2, (double)d.first_step + 1);
    bias_corrections(sc.power, sc.bias[(d.first_step + 1) & 1]);
    std::vector<const void*> grads(d.n_tensors);
    for (int i = 0; i < d.n_tensors; ++i) grads[i] = tensors[i].n ? tensors[i].grad : nullptr;
    const struct { void* to; const void* from; size_t bytes; } copies[] = {
        {p.sc, &sc, sizeof sc}, {(void*)p.tensors, recs.data(), sizeof(TensorRec) * recs.size()}, {p.grads, grads.data(), sizeof(void*) * grads.size()},
         {(void*)p.chunks, chunks.data(), sizeof(ChunkRec) * chunks.size()}};
    for (const auto& c : copies)
        if (e == cudaSuccess && c.bytes) e = cudaMemcpyAsync(c.to, c.from, c.bytes, cudaMemcpyHostToDevice, o->stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(o->stream);
    if (e != cudaSuccess) { cudaGetLastError(); return fail(nullptr, ST_ERR_CUDA, "st_adamw_create: %s", cudaGetErrorString(e)); }
    return ST_OK;
}

// Reading (write = false) or writing the moments of tensors in groups whose pointers fit a launch
st_status move_moments(st_adamw* o, const void* const* m, const void* const* v, bool write, const char* what)
{
    OnDevice guard(o->device);
    if (!guard.ok) return fail(o, ST_ERR_CUDA, "%s: cannot use the optimiser's device", what);
    std::vector<st_adamw::Range> to;
    for (int i = 0; i < o->n; ++i)
        for (const void* q : {m ? m[i] : nullptr, v ? v[i] : nullptr}) {
            if (!q || o->values[i] == 0) continue;
            if (!write) to.push_back({(uintptr_t)q, (uintptr_t)q + 4 * o->values[i]});
            const char* f = buffer_fault(q, 4, o->device);
            if (!f && touches(o->written, (uintptr_t)q, (uintptr_t)q + 4 * o->values[i])) f = "overlaps a buffer of the optimiser";
            if (f) return fail(o, ST_ERR_INVALID_ARG, "%s: tensor %d: a buffer %s", what, i, f);
        }
    if (overlap(to)) return fail(o, ST_ERR_INVALID_ARG, "%s: two buffers that are written overlap", what);
    constexpr int group = kPointers / 2;
    cudaError_t e = cudaSuccess;
    for (int first = 0; first < o->n && e == cudaSuccess; first += group) {
        const int last = std::min(o->n, first + group);
        PointerArgs a;
        for (int i = first; i < last; ++i) { a.q[2 * (i - first)] = m ? m[i] : nullptr; a.q[2 * (i - first) + 1] = v ? v[i] : nullptr; }
        const int64_t begin = o->first_chunk[first], end = o->first_chunk[last];
        if (begin == end) continue;
        const int grid = (int)std::min<int64_t>(end - begin, std::max<int64_t>(o->moments_resident, (end - begin) / o->moments_span));
        auto kernel = write ? (o->bits == 32 ? adamw_write_kernel<32> : adamw_write_kernel<8>) : (o->bits == 32 ? adamw_read_kernel<32> : adamw_read_kernel<8>);
        e = launch_early(pdl_enabled(), kernel, dim3(grid), dim3(kThreads), 0, o->stream, o->plan, first, begin, end, a);
    }
    return check_launch(o, e, what);
}

}  // namespace

extern "C" {

st_status st_adamw_create(const st_adamw_desc* desc, const st_adamw_tensor* tensors, st_adamw** out)
{
    if (!desc || !tensors || !out) return (st_status)fail_on_thread(ST_ERR_INVALID_ARG, "st_adamw_create: NULL argument");
    *out = nullptr;
    const st_adamw_desc& d = *desc;
    if (d.n_tensors < 1 || d.n_tensors > 65535) return (st_status)fail_on_thread(ST_ERR_INVALID_ARG, "st_adamw_create: n_tensors %d outside 1..65535", d.n_tensors);
    if (d.state_bits != 32 && d.state_bits != 8) return (st_status)fail_on_thread(ST_ERR_INVALID_ARG, "st_adamw_create: state_bits must be 32 or 8");
    if (!(d.lr >= 0 && d.lr <= FLT_MAX) || !(d.beta1 >= 0 && d.beta1 < 1) || !(d.beta2 >= 0 && d.beta2 < 1) || !(d.eps >= FLT_MIN && d.eps <= kMostEps))
        return (st_status)fail_on_thread(ST_ERR_INVALID_ARG, "st_adamw_create: needs lr >= 0, beta1 and beta2 in [0, 1) and eps in %g..%g", (double)FLT_MIN, kMostEps);
    if (!(d.max_norm >= 0) || !std::isfinite(d.max_norm) || d.first_step < 0 || (d.skip_nonfinite & ~1))
        return (st_status)fail_on_thread(ST_ERR_INVALID_ARG, "st_adamw_create: needs max_norm >= 0, first_step >= 0 and skip_nonfinite 0 or 1");
    st_adamw* o = new (std::nothrow) st_adamw;
    if (!o) return (st_status)fail_on_thread(ST_ERR_OOM, "st_adamw_create: host allocation failed");
    st_status st;
    try { st = create(d, tensors, o); } catch (const std::exception&) { st = (st_status)fail_on_thread(ST_ERR_OOM, "st_adamw_create: host allocation failed"); }
    if (st != ST_OK) { st_adamw_destroy(o); return st; }
    *out = o;
    return ST_OK;
}

st_status st_adamw_set_grads(st_adamw* o, const void* const* grads)
{
    if (!o) return ST_ERR_INVALID_ARG;
    if (!grads) return fail(o, ST_ERR_INVALID_ARG, "st_adamw_set_grads: NULL argument");
    OnDevice guard(o->device);
    if (!guard.ok) return fail(o, ST_ERR_CUDA, "st_adamw_set_grads: cannot use the optimiser's device");
    for (int i = 0; i < o->n; ++i)
        if (const char* f = grad_fault(o, i, grads[i])) return fail(o, ST_ERR_INVALID_ARG, "st_adamw_set_grads: gradient %d %s", i, f);
    cudaError_t e = cudaSuccess;
    for (int first = 0; first < o->n && e == cudaSuccess; first += kPointers) {
        const int count = std::min(kPointers, o->n - first);
        PointerArgs a;
        std::copy(grads + first, grads + first + count, a.q);
        e = launch_early(false, adamw_set_grads_kernel, dim3((count + 127) / 128), dim3(128), 0, o->stream, o->plan.grads, first, count, a);
    }
    return check_launch(o, e, "st_adamw_set_grads");
}

st_status st_adamw_set_lr(st_adamw* o, double lr)
{
    if (!o) return ST_ERR_INVALID_ARG;
    if (!(lr >= 0 && lr <= FLT_MAX)) return fail(o, ST_ERR_INVALID_ARG, "st_adamw_set_lr: lr must be >= 0 and finite in fp32");
    OnDevice guard(o->device);
    if (!guard.ok) return fail(o, ST_ERR_CUDA, "st_adamw_set_lr: cannot use the optimiser's device");
    return check_launch(o, launch_early(false, adamw_set_lr_kernel, dim3(1), dim3(1), 0, o->stream, o->plan.sc, (float)lr), "st_adamw_set_lr");
}

st_status st_adamw_step(st_adamw* o, float grad_scale, float* norm_out)
{
    if (!o) return ST_ERR_INVALID_ARG;
    if (!std::isfinite(grad_scale)) return fail(o, ST_ERR_INVALID_ARG, "st_adamw_step: grad_scale must be finite");
    OnDevice guard(o->device);
    if (!guard.ok) return fail(o, ST_ERR_CUDA, "st_adamw_step: cannot use the optimiser's device");
    if (norm_out) {
        const char* f = buffer_fault(norm_out, 4, o->device);
        if (!f && touches(o->written, (uintptr_t)norm_out, (uintptr_t)norm_out + 4)) f = "overlaps a buffer that the step writes";
        if (f) return fail(o, ST_ERR_INVALID_ARG, "st_adamw_step: norm_out %s", f);
    }
    const int with_norm = o->always_norm || norm_out;
    cudaError_t e = cudaSuccess;
    if (with_norm) e = launch_early(pdl_enabled(), adamw_norm_kernel, dim3(o->norm_grid), dim3(kThreads), 0, o->stream, o->plan, grad_scale, norm_out);
    // no step without the norm that it was to be clipped by
    if (e == cudaSuccess) e = launch_early(pdl_enabled(), o->bits == 32 ? adamw_step_kernel<32> : adamw_step_kernel<8>, dim3(o->step_grid), dim3(kThreads), 0, o->stream,
                                           o->plan, grad_scale, with_norm);
    return check_launch(o, e, "st_adamw_step");
}

st_status st_adamw_read_moments(st_adamw* o, float* const* m, float* const* v)
{
    if (!o) return ST_ERR_INVALID_ARG;
    try { return move_moments(o, (const void* const*)m, (const void* const*)v, false, "st_adamw_read_moments"); }
    catch (const std::exception&) { return fail(o, ST_ERR_OOM, "st_adamw_read_moments: host allocation failed"); }
}

st_status st_adamw_write_moments(st_adamw* o, const float* const* m, const float* const* v)
{
    if (!o) return ST_ERR_INVALID_ARG;
    return move_moments(o, (const void* const*)m, (const void* const*)v, true, "st_adamw_write_moments");
}

st_status st_adamw_step_count(st_adamw* o, int64_t* steps)
{
    if (!o) return ST_ERR_INVALID_ARG;
    if (!steps) return fail(o, ST_ERR_INVALID_ARG, "st_adamw_step_count: NULL argument");
    OnDevice guard(o->device);
    long long t = 0;
    cudaError_t e = guard.ok ? cudaMemcpyAsync(&t, &o->plan.sc->t, sizeof t, cudaMemcpyDeviceToHost, o->stream) : cudaErrorInvalidDevice;
    if (e == cudaSuccess) e = cudaStreamSynchronize(o->stream);
    if (e != cudaSuccess) { cudaGetLastError(); return fail(o, ST_ERR_CUDA, "st_adamw_step_count: %s", cudaGetErrorString(e)); }
    *steps = t;
    return ST_OK;
}

void st_adamw_destroy(st_adamw* o)
{
    if (!o) return;
    if (o->block) {
        OnDevice guard(o->device);
        cudaStreamSynchronize(o->stream);
        cudaFree(o->block);
    }
    delete o;
}

const char* st_adamw_last_error(const st_adamw* o) { return o ? o->err.c_str() : st_last_error(nullptr); }

}  // extern "C"

// st_adamw — OptimStep of Algorithm 1 (Adam, Section 5.2; here with decoupled weight decay) over any number of the caller's
// tensors in one launch, moments in fp32 or in 8 bits.  The formulas stand in include/shadowtutor.h.
//
// All tensors are cut into chunks of kChunk values; a table on the device says which tensor a chunk belongs to, and the blocks of a
// launch that fills the GPU once walk over it.  A warp takes 256 consecutive values of a chunk, which are also a block of 8-bit
// moments: the two maxima that a block's scales need are warp reductions, and a lane keeps its eight values in registers from the
// load to the store, so that every buffer is read once and written once.
//
// The gradients' norm needs every gradient before the first step is taken: a kernel of its own (double accumulators, partial
// sums per block added in block order: the result depends on nothing but the values and the launch).  The step then walks the
// chunks from the last to the first, so that it begins with the gradients that the norm has just left in L2.
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
static_assert(kPer == 8, "the vector path below moves two groups of four values per lane");

struct TensorRec {
    void* param; float* master; const void* grad;
    void *m, *v; float *m_scale, *v_scale;
    int64_t n;
    float wd, lr_scale;
    uint8_t param_type, grad_type, vec, pad;                // vec: all buffers but the gradient lie as the vector path needs them
};
struct ChunkRec { int32_t tensor, index; };
struct Scalars {
    long long t;                // steps taken
    double lr;
    float factor;               // of the gradients, from the norm
    int skip;                   // the norm is not finite and the step is to be left out
    unsigned int norm_ticket, step_ticket;
};
struct Plan {
    TensorRec* tensors; const ChunkRec* chunks; int64_t n_chunks;
    Scalars* sc; double* partials;
    double ln_b1, ln_b2, max_norm;
    float b1, b2, omb1, omb2, eps;
    int skip_nonfinite;
};

// ---- moving a warp's 256 values -------------------------------------------------------------------------
// Vector path: lane l has values 4 l .. 4 l + 3 of each half of 128.  Otherwise (a block that a tensor's end cuts, or buffers
// that lie unaligned): values l, 32 + l, ..., which moves whole sectors too, with four times the instructions.
struct Raw { uint32_t w[kPer]; };
template <bool VEC>
__device__ __forceinline__ void fetch(Raw& r, const void* base, int type, int64_t at, int count, int lane)
{
    if (VEC) {
        if (type == ST_F32) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint4 q = *(const uint4*)((const float*)base + at + u * 128 + 4 * lane);
                r.w[4 * u] = q.x; r.w[4 * u + 1] = q.y; r.w[4 * u + 2] = q.z; r.w[4 * u + 3] = q.w;
            }
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint2 q = *(const uint2*)((const uint16_t*)base + at + u * 128 + 4 * lane);
                r.w[4 * u] = q.x; r.w[4 * u + 1] = q.y;
            }
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
            const uint32_t h = VEC ? (r.w[(j & 4) + ((j & 3) >> 1)] >> ((j & 1) * 16)) & 0xffffu : r.w[j];
            x[j] = from16(h, type);
        }
    }
}
__device__ __forceinline__ uint32_t to16(float x, int type)
{
    return type == ST_BF16 ? (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(x)) : (uint32_t)__half_as_ushort(__float2half_rn(x));
}
template <bool VEC>
__device__ __forceinline__ void put(const float (&x)[kPer], void* base, int type, int64_t at, int count, int lane)
{
    if (VEC) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float* y = x + 4 * u;
            if (type == ST_F32) *(float4*)((float*)base + at + u * 128 + 4 * lane) = make_float4(y[0], y[1], y[2], y[3]);
            else *(uint2*)((uint16_t*)base + at + u * 128 + 4 * lane) = make_uint2(to16(y[0], type) | to16(y[1], type) << 16, to16(y[2], type) | to16(y[3], type) << 16);
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
        r.w[0] = *(const uint32_t*)(b + 4 * lane);
        r.w[4] = *(const uint32_t*)(b + 128 + 4 * lane);
    } else {
#pragma unroll
        for (int j = 0; j < kPer; ++j) { const int i = 32 * j + lane; r.w[j] = i < count ? b[i] : 0u; }
    }
}
template <bool VEC> __device__ __forceinline__ uint32_t code(const Raw& r, int j) { return VEC ? (r.w[j & 4] >> (8 * (j & 3))) & 0xffu : r.w[j]; }
template <bool VEC>
__device__ __forceinline__ void put_codes(const int (&c)[kPer], void* base, int64_t at, int count, int lane)
{
    uint8_t* b = (uint8_t*)base + at;
    if (VEC) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int* q = c + 4 * u;
            *(uint32_t*)(b + u * 128 + 4 * lane) = (q[0] & 0xff) | (q[1] & 0xff) << 8 | (q[2] & 0xff) << 16 | (uint32_t)q[3] << 24;
        }
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
        const int c = (int)(int8_t)code<VEC>(rm, j), d = (int)code<VEC>(rv, j);
        m[j] = __fmul_rn((float)(c * abs(c)), m_scale);
        root[j] = __fmul_rn((float)(d * d), v_scale);
    }
}

// floor(sqrt(r) + 1/2), at most `most`.  The approximate root is within 2^-22 of the root; where that can matter the two borders next
// to the level, which fp32 holds exactly, decide.
__device__ __forceinline__ int nearest_level(float r, int most)
{
    float s;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(s) : "f"(r));
    float c = floorf(s + 0.5f);
    const float below = c - 0.5f, above = c + 0.5f;
    if (r < below * below && c > 0.f) c -= 1.f;
    if (r >= above * above) c += 1.f;
    return min(__float2int_rz(c), most);        // NaN (a block that is not finite): 0
}
// Levels of a warp's block from m and sqrt(v), and its two scales
__device__ __forceinline__ void encode(const float (&m)[kPer], const float (&root)[kPer], int (&cm)[kPer], int (&cv)[kPer], float& m_scale, float& v_scale)
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
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int c = nearest_level(__fmul_rn(fabsf(m[j]), im), 127);
        cm[j] = m[j] < 0.f ? -c : c;
        const int d = nearest_level(__fmul_rn(root[j], iv), 255);
        cv[j] = root[j] > 0.f ? max(d, 1) : d;
    }
}

// ---- one step ----------------------------------------------------------------------------------------------
struct StepShared { float lr1_over_lr, r2, lr, factor; int skip; };

// A warp's 256 values
template <int BITS, bool VEC>
__device__ __forceinline__ void step_block(const Plan& p, const TensorRec& t, const void* grad, const StepShared& k, int64_t at, int count, int lane)
{
    const bool has_master = t.master != nullptr;
    const void* from = has_master ? (const void*)t.master : t.param;
    const int from_type = has_master ? ST_F32 : t.param_type;
    Raw rg, rp, rm, rv;
    fetch<VEC>(rg, grad, t.grad_type, at, count, lane);
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
    convert<VEC>(g, rg, t.grad_type);
    convert<VEC>(x, rp, from_type);
    if (BITS == 32) {
        convert<VEC>(m, rm, ST_F32);
        convert<VEC>(v, rv, ST_F32);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const float gj = g[j] * k.factor;
            m[j] = fmaf(p.b1, m[j], p.omb1 * gj);
            v[j] = fmaf(p.b2, v[j], p.omb2 * gj * gj);
            root[j] = __fsqrt_rn(v[j]);
        }
        put<VEC>(m, t.m, ST_F32, at, count, lane);
        put<VEC>(v, t.v, ST_F32, at, count, lane);
    } else {
        decode<VEC>(m, root, rm, rv, m_scale, v_scale);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const float gj = __fmul_rn(g[j], k.factor);
            m[j] = __fadd_rn(__fmul_rn(m[j], p.b1), __fmul_rn(gj, p.omb1));
            root[j] = __fsqrt_rn(__fadd_rn(__fmul_rn(__fmul_rn(root[j], root[j]), p.b2), __fmul_rn(__fmul_rn(gj, gj), p.omb2)));
        }
        int cm[kPer], cv[kPer];
        encode(m, root, cm, cv, m_scale, v_scale);
        put_codes<VEC>(cm, t.m, at, count, lane);
        put_codes<VEC>(cv, t.v, at, count, lane);
        if (lane == 0) { t.m_scale[block] = m_scale; t.v_scale[block] = v_scale; }
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const float kept = fmaf(-decay, x[j], x[j]);
        x[j] = fmaf(-lr1, __fdiv_rn(m[j], fmaf(root[j], k.r2, p.eps)), kept);
    }
    put<VEC>(x, t.param, t.param_type, at, count, lane);
    if (has_master) put<VEC>(x, t.master, ST_F32, at, count, lane);
}

__device__ __forceinline__ bool grad_aligned(const void* grad, int type) { return ((uintptr_t)grad & (type == ST_F32 ? 15u : 7u)) == 0; }

template <int BITS>
__global__ void __launch_bounds__(kThreads) adamw_step_kernel(const Plan p, float grad_scale, int with_norm)
{
    __shared__ StepShared k;
    pdl_wait();
    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        const double t = (double)(p.sc->t + 1), lr = p.sc->lr;
        k.lr = (float)lr;
        k.lr1_over_lr = (float)(-1.0 / expm1(t * p.ln_b1));
        k.r2 = (float)(1.0 / sqrt(-expm1(t * p.ln_b2)));
        k.factor = with_norm ? p.sc->factor : grad_scale;
        k.skip = with_norm && p.sc->skip;
    }
    __syncthreads();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    if (!k.skip) {
        for (int64_t c = blockIdx.x; c < p.n_chunks; c += gridDim.x) {
            const ChunkRec ck = p.chunks[p.n_chunks - 1 - c];
            const TensorRec& t = p.tensors[ck.tensor];
            const void* grad = t.grad;
            const int64_t at = (int64_t)ck.index * kChunk + warp * kBlockVals, left = t.n - at;
            if (!grad || left <= 0) continue;
            if (left >= kBlockVals && t.vec && grad_aligned(grad, t.grad_type)) step_block<BITS, true>(p, t, grad, k, at, kBlockVals, lane);
            else step_block<BITS, false>(p, t, grad, k, at, (int)min(left, (int64_t)kBlockVals), lane);
        }
    }
    // the block that finishes last counts the step: every block has read the count by then
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        if (atomicAdd(&p.sc->step_ticket, 1u) == gridDim.x - 1) {
            p.sc->step_ticket = 0;
            if (!k.skip) p.sc->t += 1;
        }
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

__global__ void __launch_bounds__(kThreads) adamw_norm_kernel(const Plan p, float grad_scale, float* norm_out)
{
    __shared__ double shared[kWarps];
    __shared__ bool last;
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    double sum = 0;
    for (int64_t c = blockIdx.x; c < p.n_chunks; c += gridDim.x) {
        const ChunkRec ck = p.chunks[c];
        const TensorRec& t = p.tensors[ck.tensor];
        const void* grad = t.grad;
        const int64_t at = (int64_t)ck.index * kChunk + warp * kBlockVals, left = t.n - at;
        if (!grad || left <= 0) continue;
        Raw r;
        float g[kPer];
        if (left >= kBlockVals && grad_aligned(grad, t.grad_type)) { fetch<true>(r, grad, t.grad_type, at, kBlockVals, lane); convert<true>(g, r, t.grad_type); }
        else { fetch<false>(r, grad, t.grad_type, at, (int)min(left, (int64_t)kBlockVals), lane); convert<false>(g, r, t.grad_type); }
#pragma unroll
        for (int j = 0; j < kPer; ++j) { const double d = g[j]; sum = fma(d, d, sum); }
    }
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

__global__ void adamw_set_grads_kernel(TensorRec* tensors, int first, int count, const PointerArgs a)
{
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < count) tensors[first + i].grad = a.q[i];
}
__global__ void adamw_set_lr_kernel(Scalars* sc, double lr) { sc->lr = lr; }

// ---- moments as fp32 values and back -----------------------------------------------------------------------
// Tensors [first, first + count) with their pointers in the arguments: m's at 2 i, v's at 2 i + 1
__device__ __forceinline__ bool moment_block(const Plan& p, int64_t c, int first, int warp, TensorRec& t, int& i, int64_t& at, int& count)
{
    const ChunkRec ck = p.chunks[c];
    t = p.tensors[ck.tensor];
    i = ck.tensor - first;
    at = (int64_t)ck.index * kChunk + warp * kBlockVals;
    const int64_t left = t.n - at;
    count = (int)min(left, (int64_t)kBlockVals);
    return left > 0;
}

template <int BITS>
__global__ void __launch_bounds__(kThreads) adamw_read_kernel(const Plan p, int first, int64_t chunk_begin, int64_t chunk_end, const PointerArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int64_t c = chunk_begin + blockIdx.x; c < chunk_end; c += gridDim.x) {
        TensorRec t; int i, count; int64_t at;
        if (!moment_block(p, c, first, warp, t, i, at, count)) continue;
        float* out[2] = {(float*)a.q[2 * i], (float*)a.q[2 * i + 1]};
        float m[kPer], v[kPer];
        Raw rm, rv;
        const bool vec = count == kBlockVals && t.vec && (((uintptr_t)out[0] | (uintptr_t)out[1]) & 15) == 0;
        if (BITS == 32) {
            if (vec) { fetch<true>(rm, t.m, ST_F32, at, count, lane); fetch<true>(rv, t.v, ST_F32, at, count, lane); convert<true>(m, rm, ST_F32); convert<true>(v, rv, ST_F32); }
            else { fetch<false>(rm, t.m, ST_F32, at, count, lane); fetch<false>(rv, t.v, ST_F32, at, count, lane); convert<false>(m, rm, ST_F32); convert<false>(v, rv, ST_F32); }
        } else {
            const float ms = t.m_scale[at / kBlockVals], vs = t.v_scale[at / kBlockVals];
            if (vec) { fetch_codes<true>(rm, t.m, at, count, lane); fetch_codes<true>(rv, t.v, at, count, lane); decode<true>(m, v, rm, rv, ms, vs); }
            else { fetch_codes<false>(rm, t.m, at, count, lane); fetch_codes<false>(rv, t.v, at, count, lane); decode<false>(m, v, rm, rv, ms, vs); }
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[j] = __fmul_rn(v[j], v[j]);
        }
        if (vec) {
            if (out[0]) put<true>(m, out[0], ST_F32, at, count, lane);
            if (out[1]) put<true>(v, out[1], ST_F32, at, count, lane);
        } else {
            if (out[0]) put<false>(m, out[0], ST_F32, at, count, lane);
            if (out[1]) put<false>(v, out[1], ST_F32, at, count, lane);
        }
    }
}

template <int BITS>
__global__ void __launch_bounds__(kThreads) adamw_write_kernel(const Plan p, int first, int64_t chunk_begin, int64_t chunk_end, const PointerArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int64_t c = chunk_begin + blockIdx.x; c < chunk_end; c += gridDim.x) {
        TensorRec t; int i, count; int64_t at;
        if (!moment_block(p, c, first, warp, t, i, at, count)) continue;
        const float* in[2] = {(const float*)a.q[2 * i], (const float*)a.q[2 * i + 1]};
        float m[kPer] = {}, v[kPer] = {};
        Raw r;
        if (in[0]) { fetch<false>(r, in[0], ST_F32, at, count, lane); convert<false>(m, r, ST_F32); }
        if (in[1]) { fetch<false>(r, in[1], ST_F32, at, count, lane); convert<false>(v, r, ST_F32); }
#pragma unroll
        for (int j = 0; j < kPer; ++j) v[j] = v[j] < 0.f ? 0.f : v[j];
        if (BITS == 32) {
            if (in[0]) put<false>(m, t.m, ST_F32, at, count, lane);
            if (in[1]) put<false>(v, t.v, ST_F32, at, count, lane);
        } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[j] = __fsqrt_rn(v[j]);
            int cm[kPer], cv[kPer];
            float ms, vs;
            encode(m, v, cm, cv, ms, vs);
            if (in[0]) { put_codes<false>(cm, t.m, at, count, lane); if (lane == 0) t.m_scale[at / kBlockVals] = ms; }
            if (in[1]) { put_codes<false>(cv, t.v, at, count, lane); if (lane == 0) t.v_scale[at / kBlockVals] = vs; }
        }
    }
}

}  // namespace
}  // namespace st

using namespace st;

// ---- C interface ---------------------------------------------------------------------------------------------
struct st_adamw {
    Plan plan = {};
    int device = 0, n = 0, bits = 32;
    cudaStream_t stream = nullptr;
    int step_grid = 0, norm_grid = 0, any_grid = 0;
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

const char* grad_fault(const st_adamw* o, int i, const void* grad)
{
    if (!grad || o->values[i] == 0) return nullptr;
    const size_t size = type_size(o->grad_type[i]);
    if (const char* f = buffer_fault(grad, size, o->device)) return f;
    if (touches(o->written, (uintptr_t)grad, (uintptr_t)grad + size * o->values[i])) return "overlaps a buffer that the step writes";
    return nullptr;
}

st_status check_launch(st_adamw* o, const char* what)
{
    cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? ST_OK : fail(o, ST_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
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
        r = TensorRec{t.param, t.master, t.grad, t.exp_avg, t.exp_avg_sq, t.exp_avg_scale, t.exp_avg_sq_scale, t.n, t.weight_decay, t.lr_scale,
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
        const size_t four = d.state_bits == 32 ? 16 : 4;
        r.vec = aligned(t.param, 4 * type_size(t.param_type)) && aligned(t.master, 16) && aligned(t.exp_avg, four) && aligned(t.exp_avg_sq, four);
    }
    std::sort(o->written.begin(), o->written.end(), [](const st_adamw::Range& a, const st_adamw::Range& b) { return a.begin < b.begin; });
    for (size_t i = 1; i < o->written.size(); ++i)
        if (o->written[i].begin < o->written[i - 1].end) return fail(nullptr, ST_ERR_INVALID_ARG, "st_adamw_create: two buffers that a step writes overlap");
    for (int i = 0; i < d.n_tensors; ++i)
        if (const char* f = grad_fault(o, i, tensors[i].grad)) return fail(nullptr, ST_ERR_INVALID_ARG, "st_adamw_create: tensor %d: grad %s", i, f);

    const int64_t n_chunks = o->first_chunk[d.n_tensors];
    int sms = 0, step = 0, norm = 0;
    cudaError_t e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, o->device);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&step, d.state_bits == 32 ? adamw_step_kernel<32> : adamw_step_kernel<8>, kThreads, 0);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&norm, adamw_norm_kernel, kThreads, 0);
    if (e != cudaSuccess) { cudaGetLastError(); return fail(nullptr, ST_ERR_CUDA, "st_adamw_create: %s", cudaGetErrorString(e)); }
    const auto grid = [&](int per_sm) { return (int)std::max<int64_t>(1, std::min<int64_t>(n_chunks, (int64_t)sms * std::max(per_sm, 1))); };
    o->step_grid = grid(step); o->norm_grid = grid(norm); o->any_grid = grid(8);

    std::vector<ChunkRec> chunks((size_t)n_chunks);
    for (int i = 0; i < d.n_tensors; ++i)
        for (int64_t c = o->first_chunk[i]; c < o->first_chunk[i + 1]; ++c) chunks[c] = {i, (int32_t)(c - o->first_chunk[i])};
    const auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t at_partials = up(sizeof(Scalars)), at_tensors = at_partials + up(sizeof(double) * o->norm_grid),
                 at_chunks = at_tensors + up(sizeof(TensorRec) * recs.size()), bytes = at_chunks + up(sizeof(ChunkRec) * chunks.size());
    e = cudaMalloc(&o->block, bytes);
    if (e != cudaSuccess) { cudaGetLastError(); return fail(nullptr, e == cudaErrorMemoryAllocation ? ST_ERR_OOM : ST_ERR_CUDA, "st_adamw_create: %s", cudaGetErrorString(e)); }
    char* b = (char*)o->block;
    Plan& p = o->plan;
    p.sc = (Scalars*)b; p.partials = (double*)(b + at_partials); p.tensors = (TensorRec*)(b + at_tensors); p.chunks = (const ChunkRec*)(b + at_chunks);
    p.n_chunks = n_chunks;
    p.ln_b1 = log(d.beta1); p.ln_b2 = log(d.beta2); p.max_norm = d.max_norm;
    p.b1 = (float)d.beta1; p.b2 = (float)d.beta2; p.omb1 = (float)(1.0 - d.beta1); p.omb2 = (float)(1.0 - d.beta2); p.eps = (float)d.eps;
    p.skip_nonfinite = d.skip_nonfinite;
    o->always_norm = d.max_norm > 0 || d.skip_nonfinite;
    Scalars sc = {};
    sc.t = d.first_step; sc.lr = d.lr; sc.factor = 1.f;
    const struct { void* to; const void* from; size_t bytes; } copies[] = {
        {p.sc, &sc, sizeof sc}, {p.tensors, recs.data(), sizeof(TensorRec) * recs.size()}, {(void*)p.chunks, chunks.data(), sizeof(ChunkRec) * chunks.size()}};
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
    for (int i = 0; i < o->n; ++i)
        for (const void* q : {m ? m[i] : nullptr, v ? v[i] : nullptr}) {
            if (!q || o->values[i] == 0) continue;
            const char* f = buffer_fault(q, 4, o->device);
            if (!f && touches(o->written, (uintptr_t)q, (uintptr_t)q + 4 * o->values[i])) f = "overlaps a buffer of the optimiser";
            if (f) return fail(o, ST_ERR_INVALID_ARG, "%s: tensor %d: a buffer %s", what, i, f);
        }
    constexpr int group = kPointers / 2;
    for (int first = 0; first < o->n; first += group) {
        const int last = std::min(o->n, first + group);
        PointerArgs a;
        for (int i = first; i < last; ++i) { a.q[2 * (i - first)] = m ? m[i] : nullptr; a.q[2 * (i - first) + 1] = v ? v[i] : nullptr; }
        const int64_t begin = o->first_chunk[first], end = o->first_chunk[last];
        if (begin == end) continue;
        const int grid = (int)std::min<int64_t>(end - begin, o->any_grid);
        auto kernel = write ? (o->bits == 32 ? adamw_write_kernel<32> : adamw_write_kernel<8>) : (o->bits == 32 ? adamw_read_kernel<32> : adamw_read_kernel<8>);
        launch_early(pdl_enabled(), kernel, dim3(grid), dim3(kThreads), 0, o->stream, o->plan, first, begin, end, a);
    }
    return check_launch(o, what);
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
    if (!(d.lr >= 0) || !std::isfinite(d.lr) || !(d.beta1 >= 0 && d.beta1 < 1) || !(d.beta2 >= 0 && d.beta2 < 1) || !(d.eps >= FLT_MIN && d.eps <= FLT_MAX))
        return (st_status)fail_on_thread(ST_ERR_INVALID_ARG, "st_adamw_create: needs lr >= 0, beta1 and beta2 in [0, 1) and eps >= %g", (double)FLT_MIN);
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
    for (int first = 0; first < o->n; first += kPointers) {
        const int count = std::min(kPointers, o->n - first);
        PointerArgs a;
        std::copy(grads + first, grads + first + count, a.q);
        adamw_set_grads_kernel<<<(count + 127) / 128, 128, 0, o->stream>>>(o->plan.tensors, first, count, a);
    }
    return check_launch(o, "st_adamw_set_grads");
}

st_status st_adamw_set_lr(st_adamw* o, double lr)
{
    if (!o) return ST_ERR_INVALID_ARG;
    if (!(lr >= 0) || !std::isfinite(lr)) return fail(o, ST_ERR_INVALID_ARG, "st_adamw_set_lr: lr must be >= 0");
    OnDevice guard(o->device);
    if (!guard.ok) return fail(o, ST_ERR_CUDA, "st_adamw_set_lr: cannot use the optimiser's device");
    adamw_set_lr_kernel<<<1, 1, 0, o->stream>>>(o->plan.sc, lr);
    return check_launch(o, "st_adamw_set_lr");
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
    if (with_norm) launch_early(pdl_enabled(), adamw_norm_kernel, dim3(o->norm_grid), dim3(kThreads), 0, o->stream, o->plan, grad_scale, norm_out);
    launch_early(pdl_enabled(), o->bits == 32 ? adamw_step_kernel<32> : adamw_step_kernel<8>, dim3(o->step_grid), dim3(kThreads), 0, o->stream,
                 o->plan, grad_scale, with_norm);
    return check_launch(o, "st_adamw_step");
}

st_status st_adamw_read_moments(st_adamw* o, float* const* m, float* const* v)
{
    if (!o) return ST_ERR_INVALID_ARG;
    return move_moments(o, (const void* const*)m, (const void* const*)v, false, "st_adamw_read_moments");
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

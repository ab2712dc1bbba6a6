// st_quantize_rows — rows of activations or weights to 8-bit integers with one scale per row: scale = max |x| / 127, q = x / scale rounded to
// the nearest whole number (half to even), exactly.
//
// Bound by memory: 4 or 2 bytes read and 1 written per value.  Two forms, both reading x once where a row fits registers:
//   rows whose values lie side by side (tokens, weights): 1 to 8 warps to a row
//   other strides (planar feature maps, whose rows are pixels): a block takes 32 rows and reads them channel by channel, a row to a
//     lane, so that planes are read in whole sectors; the integers are turned round in shared memory
//
// The quotient is x * (1 / scale), off by at most 127 * 2^-23 of a step (1.5e-5), so it gives the whole number unless it lies within kNear
// of a half.  There (one value in 25000; a lane then takes all values of its piece that way) the quotient in double decides: of two fp32
// numbers it is either a half exactly or at least 2^-32 away from one.
#include "../../include/shadowtutor.h"
#include "st_internal.h"
#include "int8_common.h"

#include <cuda_fp16.h>

#include <algorithm>

namespace st {
namespace {

constexpr int kThreads = 256;
constexpr float kRound = 12582912.f;            // adding 1.5 * 2^23 rounds to a whole number and leaves it in the low bits
constexpr float kNear = 2e-5f;
constexpr float kLeastScale = 0x1p-100f;        // below it every quotient is formed in double

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

// `doubt`: added to a value's distance from the whole numbers; 1 sends every value through the quotient in double.  `mask`: 0 makes all integers 0.
struct RowScale { float scale, inverse, doubt; uint32_t mask; };
// From the bits of the row's largest |x| (NaN lies above infinity).  A row that is not finite has scale NaN and integers 0.
__device__ __forceinline__ RowScale row_scale(uint32_t top)
{
    RowScale r;
    const bool finite = top < 0x7f800000u;
    r.scale = finite ? __fdiv_rn(__uint_as_float(top), 127.f) : __uint_as_float(0x7fffffffu);
    r.doubt = r.scale < kLeastScale && r.scale > 0.f ? 1.f : 0.f;
    r.inverse = r.scale >= kLeastScale ? __frcp_rn(r.scale) : 0.f;
    r.mask = finite ? 0xffffffffu : 0u;
    return r;
}
__device__ __noinline__ uint32_t exact_quotient(float x, float scale)
{
    const double q = rint((double)x / (double)scale);
    return (uint32_t)(int)fmin(fmax(q, -127.0), 127.0);
}
__device__ __forceinline__ uint32_t low_bytes(const uint32_t* c) { return __byte_perm(__byte_perm(c[0], c[1], 0x0040u), __byte_perm(c[2], c[3], 0x0040u), 0x5410u); }
// the integers of V values in the low bytes of words
template <int V>
__device__ __forceinline__ void quantized(uint32_t (&b)[V], const float (&x)[V], const RowScale& r)
{
    float far = r.doubt;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float t = x[j] * r.inverse, y = t + kRound;
        far = fmaxf(far, fabsf(t - (y - kRound)));
        b[j] = __float_as_uint(y);
    }
    if (far > 0.5f - kNear)
#pragma unroll
        for (int j = 0; j < V; ++j) b[j] = exact_quotient(x[j], r.scale);
}
__device__ __forceinline__ uint32_t bits_of_size(float x) { return __float_as_uint(x) & 0x7fffffffu; }

template <typename T, int V> struct Piece { T v[V]; };
template <typename T, int V>
__device__ __forceinline__ void load_piece(Piece<T, V>& p, const T* src)
{
    if constexpr (V == 1) p.v[0] = *src;
    else *(uint4*)p.v = *(const uint4*)src;
}

// W warps to a row, V values to an access (16 bytes, or one value).  KEEP: the row fits ITEMS pieces per lane; otherwise it is read twice.
template <typename T, int V, int W, bool KEEP>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(const T* __restrict__ x, int64_t rows, int cols, int64_t row_stride,
                                                                 int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale)
{
    constexpr int ITEMS = V == 1 ? 16 : 4, STEP = 32 * W * V, kRows = kThreads / 32 / W;
    __shared__ uint32_t tops[kThreads / 32];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, at = (threadIdx.x % (32 * W)) * V;
    const int64_t row = (int64_t)blockIdx.x * kRows + warp / W;
    if (W == 1 && row >= rows) return;
    const bool mine = row < rows;
    const T* src = x + row * row_stride;
    Piece<T, V> kept[KEEP ? ITEMS : 1];
    uint32_t top = 0;
    if (mine) {
        if (KEEP) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (at + i * STEP < cols) load_piece(kept[i], src + at + i * STEP);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (at + i * STEP < cols) {
#pragma unroll
                    for (int j = 0; j < V; ++j) top = max(top, bits_of_size(to_float(kept[i].v[j])));
                }
        } else {
#pragma unroll 4
            for (int c = at; c < cols; c += STEP) {
                load_piece(kept[0], src + c);
#pragma unroll
                for (int j = 0; j < V; ++j) top = max(top, bits_of_size(to_float(kept[0].v[j])));
            }
        }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (W > 1) {
        if (lane == 0) tops[warp] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < W; ++i) top = max(top, tops[warp / W * W + i]);
        if (!mine) return;
    }
    const RowScale r = row_scale(top);
    int8_t* dst = q + row * ldq;
    const auto put = [&](const Piece<T, V>& p, int c) {
        float v[V];
        uint32_t b[V];
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = to_float(p.v[j]);
        quantized(b, v, r);
        if constexpr (V == 1) dst[c] = (int8_t)(b[0] & r.mask);
        else if constexpr (V == 8) *(uint2*)(dst + c) = make_uint2(low_bytes(b) & r.mask, low_bytes(b + 4) & r.mask);
        else *(uint32_t*)(dst + c) = low_bytes(b) & r.mask;
    };
    if (KEEP) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (at + i * STEP < cols) put(kept[i], at + i * STEP);
    } else {
#pragma unroll 4
        for (int c = at; c < cols; c += STEP) { load_piece(kept[0], src + c); put(kept[0], c); }
    }
    if (threadIdx.x % (32 * W) == 0) scale[row] = r.scale;
}

// 32 P rows to a block, rows lane, 32 + lane, ... to a lane (256 bytes of a plane are read together); warp w reads columns 4 w .. 4 w + 3 of every 32.
// KEEP: at most kSlab columns, held in registers.
constexpr int kSlab = 256, kSlabPitch = kSlab + 4;          // an odd number of words: the lanes of a store lie in different banks
template <typename T, bool KEEP>
__global__ void __launch_bounds__(kThreads) quantize_planes_kernel(const T* __restrict__ x, int64_t rows, int cols, int64_t row_stride, int64_t col_stride,
                                                                   int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale, int words)
{
    constexpr int P = 8 / sizeof(T), kRows = 32 * P, kMine = kSlab / 8;
    __shared__ uint32_t tops[8][kRows];
    __shared__ __align__(16) uint8_t turned[kRows * kSlabPitch];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t row0 = (int64_t)blockIdx.x * kRows;
    const T* src[P];
    bool mine[P];
#pragma unroll
    for (int u = 0; u < P; ++u) {
        mine[u] = row0 + 32 * u + lane < rows;
        src[u] = x + (mine[u] ? row0 + 32 * u + lane : 0) * row_stride;
    }
    T kept[P][KEEP ? kMine : 1];
    uint32_t top[P] = {};
    if (KEEP) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int c = i / 4 * 32 + 4 * warp + i % 4;
#pragma unroll
            for (int u = 0; u < P; ++u)
                if (c < cols && mine[u]) kept[u][i] = src[u][c * col_stride];
        }
#pragma unroll
        for (int i = 0; i < kMine; ++i)
#pragma unroll
            for (int u = 0; u < P; ++u)
                if (i / 4 * 32 + 4 * warp + i % 4 < cols && mine[u]) top[u] = max(top[u], bits_of_size(to_float(kept[u][i])));
    } else {
#pragma unroll 8
        for (int c = warp; c < cols; c += 8)
#pragma unroll
            for (int u = 0; u < P; ++u)
                if (mine[u]) top[u] = max(top[u], bits_of_size(to_float(src[u][c * col_stride])));
    }
#pragma unroll
    for (int u = 0; u < P; ++u) tops[warp][32 * u + lane] = top[u];
    __syncthreads();
    RowScale r[P];
#pragma unroll
    for (int u = 0; u < P; ++u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) top[u] = max(top[u], tops[i][32 * u + lane]);
        r[u] = row_scale(top[u]);
        if (warp == 0 && mine[u]) scale[row0 + 32 * u + lane] = r[u].scale;
    }
    for (int slab = 0; slab < cols; slab += kSlab) {
        const int n = min(cols - slab, kSlab);
#pragma unroll
        for (int u = 0; u < P; ++u)
#pragma unroll
            for (int i = 0; i < kSlab / 32; ++i) {
                const int c = i * 32 + 4 * warp;
                if (c >= n || !mine[u]) continue;
                float v[4] = {};
                uint32_t b[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (c + k < n) v[k] = to_float(KEEP ? kept[u][KEEP ? 4 * i + k : 0] : src[u][(slab + c + k) * col_stride]);
                quantized(b, v, r[u]);
                *(uint32_t*)(turned + (32 * u + lane) * kSlabPitch + c) = low_bytes(b) & r[u].mask;
            }
        __syncthreads();
        for (int i = warp; i < kRows && row0 + i < rows; i += 8) {
            int8_t* dst = q + (row0 + i) * ldq + slab;
            const uint8_t* from = turned + i * kSlabPitch;
            const int whole = words ? n / 4 : 0;
            for (int c = lane; c < whole; c += 32) ((uint32_t*)dst)[c] = *(const uint32_t*)(from + 4 * c);
            for (int c = 4 * whole + lane; c < n; c += 32) dst[c] = (int8_t)from[c];
        }
        __syncthreads();
    }
}

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

template <typename T>
cudaError_t launch(const T* x, int64_t rows, int64_t cols, int64_t rs, int64_t cs, int8_t* q, int64_t ldq, float* scale, cudaStream_t s)
{
    const bool early = pdl_enabled();
    const int n = (int)cols;
    if (cs != 1 && cols > 1) {
        const int words = aligned(q, 4) && (ldq % 4 == 0 || rows == 1);
        constexpr int per = 32 * 8 / sizeof(T);
        const dim3 grid((unsigned)((rows + per - 1) / per));
        return n <= kSlab ? launch_early(early, quantize_planes_kernel<T, true>, grid, dim3(kThreads), 0, s, x, rows, n, rs, cs, q, ldq, scale, words)
                          : launch_early(early, quantize_planes_kernel<T, false>, grid, dim3(kThreads), 0, s, x, rows, n, rs, cs, q, ldq, scale, words);
    }
    constexpr int V = 16 / sizeof(T);
    const bool vec = aligned(x, 16) && (rows == 1 || rs * sizeof(T) % 16 == 0) && cols % V == 0 && aligned(q, V) && (rows == 1 || ldq % V == 0);
    const auto go = [&](auto kernel, int warps) {
        const int per = kThreads / 32 / warps;
        return launch_early(early, kernel, dim3((unsigned)((rows + per - 1) / per)), dim3(kThreads), 0, s, x, rows, n, rs, q, ldq, scale);
    };
    // as few warps to a row as hold it in registers: 32 values per lane in pieces of 16 bytes, 16 single ones
    const int64_t room = vec ? 32 * 4 * V : 32 * 16;
    if (vec) {
        if (cols <= room) return go(quantize_rows_kernel<T, V, 1, true>, 1);
        if (cols <= 2 * room) return go(quantize_rows_kernel<T, V, 2, true>, 2);
        if (cols <= 4 * room) return go(quantize_rows_kernel<T, V, 4, true>, 4);
        if (cols <= 8 * room) return go(quantize_rows_kernel<T, V, 8, true>, 8);
        return go(quantize_rows_kernel<T, V, 8, false>, 8);
    }
    if (cols <= room) return go(quantize_rows_kernel<T, 1, 1, true>, 1);
    if (cols <= 2 * room) return go(quantize_rows_kernel<T, 1, 2, true>, 2);
    if (cols <= 4 * room) return go(quantize_rows_kernel<T, 1, 4, true>, 4);
    if (cols <= 8 * room) return go(quantize_rows_kernel<T, 1, 8, true>, 8);
    return go(quantize_rows_kernel<T, 1, 8, false>, 8);
}

}  // namespace
}  // namespace st

using namespace st;

extern "C" st_status st_quantize_rows(const void* x, int32_t x_type, int64_t rows, int64_t cols, int64_t row_stride, int64_t col_stride,
                                      int8_t* q, int64_t ldq, float* scale, void* cuda_stream)
{
    const auto bad = [](const char* what) { return (st_status)fail_on_thread(ST_ERR_INVALID_ARG, "st_quantize_rows: %s", what); };
    if (x_type != ST_F32 && x_type != ST_BF16 && x_type != ST_F16) return bad("x_type is not an st_dtype");
    if (rows < 0 || cols < 1 || row_stride < 0 || col_stride < 0) return bad("needs rows >= 0, cols >= 1 and strides >= 0");
    if (rows > kMaxInt8Extent || cols > kMaxInt8Extent) return (st_status)fail_on_thread(ST_ERR_UNSUPPORTED, "st_quantize_rows: more than 2^31 - 1 rows or columns");
    if (ldq < cols) return bad("ldq is below cols");
    if (!extent_fits(rows, row_stride, cols, col_stride) || !extent_fits(rows, ldq, cols, 1)) return (st_status)fail_on_thread(ST_ERR_UNSUPPORTED, "st_quantize_rows: strides reach beyond 2^48 elements");
    if (rows == 0) return ST_OK;
    const int64_t size = x_type == ST_F32 ? 4 : 2;
    Int8Buffers b("st_quantize_rows");
    b.add("x", x, size, (rows - 1) * row_stride + (cols - 1) * col_stride + 1, false);
    b.add("q", q, 1, (rows - 1) * ldq + cols, true);
    b.add("scale", scale, 4, rows, true);
    if (!b.ok()) return b.status();
    cudaStream_t s = (cudaStream_t)cuda_stream;
    cudaError_t e = x_type == ST_F32 ? launch((const float*)x, rows, cols, row_stride, col_stride, q, ldq, scale, s)
                  : x_type == ST_BF16 ? launch((const bf16*)x, rows, cols, row_stride, col_stride, q, ldq, scale, s)
                                      : launch((const __half*)x, rows, cols, row_stride, col_stride, q, ldq, scale, s);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) { cudaGetLastError(); return (st_status)fail_on_thread(ST_ERR_CUDA, "st_quantize_rows: %s", cudaGetErrorString(e)); }
    return ST_OK;
}

// st_quantize_rows — rows of activations or weights to 8-bit integers with one scale per row: scale = max |x| / 127, q = x / scale rounded to
// the nearest whole number (half to even), exactly.
//
// Bound by memory: 4 or 2 bytes read and 1 written per value.  Two forms, which read x once where a row fits registers:
//   rows whose values lie side by side (tokens, weights): 1 to 8 warps to a row, 16 bytes to an access wherever a row begins; rows that are not
//     aligned are read a second time, from L1
//   other strides (planar feature maps, whose rows are pixels): a block takes 64 or 128 rows and reads them channel by channel, so that
//     planes are read 256 bytes at a time; the integers are turned round in shared memory
//
// The quotient is x * (1 / scale), off by at most 127 * 2^-23 of a step (1.5e-5), so it gives the whole number unless it lies within kNear
// of a half h.  There the sign of x - h scale decides, which a fused multiply-add has exactly.  Rows whose scale is so small that this could
// underflow take the quotient in double: of two fp32 numbers it is either a half exactly or at least 2^-32 away from one.
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

// 16 bytes of a row, and the largest |x| met so far (NaN if one was NaN); 16-bit types in pairs
template <typename T> struct Piece;
template <> struct Piece<float> {
    static constexpr int V = 4;
    float v[4];
    __device__ __forceinline__ void get(float (&x)[4]) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = v[j];
    }
};
template <> struct Piece<bf16> {
    static constexpr int V = 8;
    __nv_bfloat162 v[4];
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) { x[2 * j] = __low2float(v[j]); x[2 * j + 1] = __high2float(v[j]); }
    }
};
template <> struct Piece<__half> {
    static constexpr int V = 8;
    __half2 v[4];
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) { x[2 * j] = __low2float(v[j]); x[2 * j + 1] = __high2float(v[j]); }
    }
};
__device__ __forceinline__ float larger(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
template <typename T> struct Top;
template <> struct Top<float> {
    float t = 0.f;
    __device__ __forceinline__ void add(const Piece<float>& p)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) t = larger(t, fabsf(p.v[j]));
    }
    __device__ __forceinline__ void add(float x) { t = larger(t, fabsf(x)); }
    __device__ __forceinline__ uint32_t bits() const { return __float_as_uint(t) & 0x7fffffffu; }
};
template <> struct Top<bf16> {
    __nv_bfloat162 t = {0, 0};
    __device__ __forceinline__ void add(const Piece<bf16>& p)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) t = __hmax2_nan(t, __habs2(p.v[j]));
    }
    __device__ __forceinline__ void add(bf16 x) { t.x = __hmax_nan(t.x, __habs(x)); }
    __device__ __forceinline__ uint32_t bits() const { return __float_as_uint(larger(__low2float(t), __high2float(t))) & 0x7fffffffu; }
};
template <> struct Top<__half> {
    __half2 t = {0, 0};
    __device__ __forceinline__ void add(const Piece<__half>& p)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) t = __hmax2_nan(t, __habs2(p.v[j]));
    }
    __device__ __forceinline__ void add(__half x) { t.x = __hmax_nan(t.x, __habs(x)); }
    __device__ __forceinline__ uint32_t bits() const { return __float_as_uint(larger(__low2float(t), __high2float(t))) & 0x7fffffffu; }
};

// `doubt`: 0, or 1 for a row whose values take the quotient in double.  `mask`: 0 makes all integers 0.
struct __align__(16) RowScale { float scale, inverse, doubt; uint32_t mask; };
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
__device__ __forceinline__ uint32_t low_bytes(const uint32_t* c) { return __byte_perm(__byte_perm(c[0], c[1], 0x0040u), __byte_perm(c[2], c[3], 0x0040u), 0x5410u); }
// The integers of n <= 4 values, read again, from quotients in double; packed
template <typename T>
__device__ __noinline__ uint32_t exact_integers(const T* x, int64_t stride, int n, float scale)
{
    uint32_t w = 0;
    for (int j = 0; j < n; ++j) {
        const double q = rint((double)to_float(x[j * stride]) / (double)scale);
        w |= ((uint32_t)(int)fmin(fmax(q, -127.0), 127.0) & 0xffu) << (8 * j);
    }
    return w;
}
// x / scale to the nearest whole number, for a quotient t next to a half
__device__ __forceinline__ float beside_half(float x, float t, float scale)
{
    const float k = (t + kRound) - kRound, d = t - k;
    if (fabsf(d) <= 0.5f - kNear) return k;
    const float h = k + copysignf(0.5f, d), over = fmaf(-h, scale, x);
    return over > 0.f ? h + 0.5f : over < 0.f ? h - 0.5f : rintf(h);
}
// The integers of V values (4 or 8), packed in words
template <int V>
__device__ __forceinline__ void quantize(uint32_t (&w)[V / 4], const float (&x)[V], const RowScale& r)
{
    float far = 0.f;
    uint32_t b[V];
#pragma unroll
    for (int j = 0; j < V; j += 2) {
        unsigned long long t, y, d;             // two values to an instruction
        asm("{\n\t.reg .b64 v, s, up, down, minus;\n\t"
            "mov.b64 v, {%3, %4};\n\tmov.b64 s, {%5, %5};\n\tmov.b64 up, {%6, %6};\n\tmov.b64 down, {%7, %7};\n\tmov.b64 minus, {%8, %8};\n\t"
            "mul.rn.f32x2 %0, v, s;\n\tadd.rn.f32x2 %1, %0, up;\n\tadd.rn.f32x2 %2, %1, down;\n\tfma.rn.f32x2 %2, %2, minus, %0;\n\t}"
            : "=&l"(t), "=&l"(y), "=&l"(d) : "f"(x[j]), "f"(x[j + 1]), "f"(r.inverse), "f"(kRound), "f"(-kRound), "f"(-1.f));
        far = fmaxf(far, fmaxf(fabsf(__uint_as_float((uint32_t)d)), fabsf(__uint_as_float((uint32_t)(d >> 32)))));
        b[j] = (uint32_t)y;
        b[j + 1] = (uint32_t)(y >> 32);
    }
    if (far > 0.5f - kNear)
#pragma unroll
        for (int j = 0; j < V; ++j) b[j] = __float_as_uint(beside_half(x[j], x[j] * r.inverse, r.scale) + kRound);
#pragma unroll
    for (int i = 0; i < V / 4; ++i) w[i] = low_bytes(b + 4 * i) & r.mask;
}
template <typename T>
__device__ __forceinline__ uint8_t quantize_one(const T* at, const RowScale& r)
{
    const float x = to_float(*at);
    if (r.doubt != 0.f) return (uint8_t)exact_integers(at, 0, 1, r.scale);
    return (uint8_t)(__float_as_uint(beside_half(x, x * r.inverse, r.scale) + kRound) & r.mask);
}

// A row's memory: `head` single values up to a 16-byte boundary, `pieces` of 16 bytes, single values from `tail` on.
struct RowParts { int head, pieces, tail; };
template <typename T>
__device__ __forceinline__ RowParts parts_of(const T* row, int cols)
{
    constexpr int V = Piece<T>::V;
    RowParts p;
    p.head = min((int)((16u - ((uint32_t)(uintptr_t)row & 15u)) & 15u) / (int)sizeof(T), cols);
    p.pieces = (cols - p.head) / V;
    p.tail = p.head + p.pieces * V;
    return p;
}

// W warps to a row.  ALIGNED: rows of x and q begin where whole pieces can be read and written, and cols is a multiple of V.  Otherwise the integers
// of a row are gathered in shared memory and written from there in aligned words, whatever the alignment of x's and q's rows.
// KEEP (aligned rows only): a row's pieces stay in registers, kItems of them per lane; otherwise it is read twice, the second time in stretches of
// that many.
// Pieces of a lane's stretch, and blocks an SM should hold.  Where pieces go straight to q they stay in registers, and many small blocks are best (8192 x
// 4096 bf16: 21.0 us with four pieces and six blocks, 24.8 with eight and three).  Rows that go through shared memory are read again from
// L1 instead (23890 x 3259 fp32: 135 us; 238 with eight pieces in registers and half of the warps).
constexpr int kItemsStraight = 4, kItemsGathered = 8;
template <typename T, int W, bool ALIGNED, bool KEEP>
__global__ void __launch_bounds__(kThreads, ALIGNED ? 6 : 4) quantize_rows_kernel(const T* __restrict__ x, int64_t rows, int cols, int64_t row_stride,
                                                                 int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale)
{
    static_assert(ALIGNED || !KEEP, "rows that go through shared memory are read again");
    constexpr int V = Piece<T>::V, kLanes = 32 * W, kItems = ALIGNED ? kItemsStraight : kItemsGathered, kRows = kThreads / kLanes, kStretch = kItems * kLanes;     // pieces
    constexpr int kPitch = kStretch * V + 32;               // bytes of a row's stretch with its head and tail, and what aligning it takes
    __shared__ uint32_t tops[kThreads / 32];
    __shared__ __align__(16) uint8_t gathered[ALIGNED ? 16 : kRows * kPitch];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, me = threadIdx.x % kLanes;
    const int64_t row = (int64_t)blockIdx.x * kRows + warp / W;
    const bool mine = row < rows;
    if (W == 1 && !mine) return;
    const T* src = x + (mine ? row : 0) * row_stride;
    int8_t* dst = q + (mine ? row : 0) * ldq;
    const RowParts p = ALIGNED ? RowParts{0, cols / V, cols} : parts_of(src, cols);
    const uint4* body = (const uint4*)(src + p.head);
    Piece<T> kept[kItems];
    Top<T> top;
    const auto get = [&](Piece<T>& k, int i) { *(uint4*)k.v = body[i]; };
    if (mine) {
        if (KEEP) {
#pragma unroll
            for (int i = 0; i < kItems; ++i)
                if (me + i * kLanes < p.pieces) get(kept[i], me + i * kLanes);
        }
        if (!ALIGNED) {
            if (me < p.head) top.add(src[me]);
            if (me < cols - p.tail) top.add(src[p.tail + me]);
        }
        if (KEEP) {
#pragma unroll
            for (int i = 0; i < kItems; ++i)
                if (me + i * kLanes < p.pieces) top.add(kept[i]);
        } else {
#pragma unroll 4
            for (int i = me; i < p.pieces; i += kLanes) { get(kept[0], i); top.add(kept[0]); }
        }
    }
    uint32_t bits = __reduce_max_sync(0xffffffffu, top.bits());
    if (W > 1) {
        if (lane == 0) tops[warp] = bits;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < W; ++i) bits = max(bits, tops[warp / W * W + i]);
    }
    const RowScale r = row_scale(bits);
    if (mine && me == 0) scale[row] = r.scale;
    const auto pack = [&](uint32_t (&w)[V / 4], const Piece<T>& k) {
        float v[V];
        k.get(v);
        quantize<V>(w, v, r);
    };
    if (ALIGNED) {
        if (!mine) return;
        const auto put = [&](const Piece<T>& k, int i) {
            uint32_t w[V / 4];
            pack(w, k);
            if constexpr (V == 8) *(uint2*)(dst + i * V) = make_uint2(w[0], w[1]);
            else *(uint32_t*)(dst + i * V) = w[0];
        };
        if (KEEP) {
#pragma unroll
            for (int i = 0; i < kItems; ++i)
                if (me + i * kLanes < p.pieces) put(kept[i], me + i * kLanes);
        } else {
#pragma unroll 4
            for (int i = me; i < p.pieces; i += kLanes) { get(kept[0], i); put(kept[0], i); }
        }
        if (r.doubt != 0.f)                     // the row once more, the same lanes at the same places
            for (int i = me; i < p.pieces; i += kLanes)
                for (int j = 0; j < V; j += 4) *(uint32_t*)(dst + i * V + j) = exact_integers(src + i * V + j, 1, 4, r.scale);
        return;
    }
    // integer c of the row lies at buf[c - first]; buf is placed so that pieces lie at multiples of 8
    uint8_t* const area = gathered + (threadIdx.x / kLanes) * kPitch;
    for (int begin = 0; begin == 0 || begin < p.pieces; begin += kStretch) {
        const bool is_first = begin == 0, is_last = begin + kStretch >= p.pieces;
        const int first = is_first ? 0 : p.head + begin * V, last = is_last ? cols : p.head + (begin + kStretch) * V;
        uint8_t* const buf = area + ((8 - p.head) & 7) * is_first;
        if (mine) {
            if (is_first && me < p.head) buf[me] = quantize_one(src + me, r);
            if (is_last && me < cols - p.tail) buf[p.tail + me - first] = quantize_one(src + p.tail + me, r);
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                const int at = begin + me + i * kLanes;
                if (at >= p.pieces) continue;
                get(kept[i], at);
                uint32_t w[V / 4];
                pack(w, kept[i]);
                uint8_t* to = buf + p.head + at * V - first;
                if constexpr (V == 8) *(uint2*)to = make_uint2(w[0], w[1]);
                else *(uint32_t*)to = w[0];
            }
            if (r.doubt != 0.f)                 // once more, the same lanes at the same places
                for (int at = begin + me; at < min(begin + kStretch, p.pieces); at += kLanes)
                    for (int j = 0; j < V; j += 4) *(uint32_t*)(buf + p.head + at * V + j - first) = exact_integers(src + p.head + at * V + j, 1, 4, r.scale);
        }
        if (W == 1) __syncwarp(); else __syncthreads();
        if (mine) {
            // single bytes up to the first word of q, words put together from two of the buffer's, single bytes behind
            const int n = last - first, lead = min((int)(-(uint32_t)(uintptr_t)(dst + first) & 3u), n), words = (n - lead) / 4;
            if (me < lead) dst[first + me] = (int8_t)buf[me];
            const uint32_t off = (uint32_t)(uintptr_t)(buf + lead) & 3u;
            const uint32_t* from = (const uint32_t*)(buf + lead - off);
            uint32_t* to = (uint32_t*)(dst + first + lead);
            for (int i = me; i < words; i += kLanes) to[i] = off ? __funnelshift_r(from[i], from[i + 1], 8 * off) : from[i];
            if (lead + 4 * words + me < n) dst[first + lead + 4 * words + me] = (int8_t)buf[lead + 4 * words + me];
        }
        if (W == 1) __syncwarp(); else __syncthreads();
    }
}

// Rows whose values do not lie side by side.  A block takes 32 P rows, rows lane, 32 + lane, ... to a lane (256 bytes of a plane are read together);
// warp w reads columns 4 w .. 4 w + 3 of every 4 kPlaneWarps.  KEEP: at most kSlab columns, held in registers.  Lanes and columns beyond the
// matrix read its last row and column again, which changes nothing, and write nothing.
constexpr int kPlaneWarps = 16, kSlab = 256, kSlabPitch = kSlab + 4;        // an odd number of words: the lanes of a store lie in different banks
template <typename T, bool KEEP, bool UNIT>
__global__ void __launch_bounds__(32 * kPlaneWarps, 2) quantize_planes_kernel(const T* __restrict__ x, int64_t rows, int cols, int64_t row_stride, int64_t col_stride,
                                                                              int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale, int words)
{
    constexpr int P = 8 / sizeof(T), kRows = 32 * P, kGroups = kSlab / 4 / kPlaneWarps;
    __shared__ uint32_t tops[kPlaneWarps][kRows];
    __shared__ RowScale scales[kRows];
    __shared__ __align__(16) uint8_t turned[kRows * kSlabPitch];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t row0 = (int64_t)blockIdx.x * kRows;
    // UNIT: rows lie side by side and all of the block's exist
    const T* src[UNIT ? 1 : P];
#pragma unroll
    for (int u = 0; u < (UNIT ? 1 : P); ++u) src[u] = UNIT ? x + row0 + lane : x + min(row0 + 32 * u + lane, rows - 1) * row_stride;
    T kept[kGroups][4][P];
    Top<T> top[P];
    const auto fetch = [&](T (&k)[4][P], int c) {
        const int last = cols - 1 - c;
        int64_t at = c * col_stride;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int u = 0; u < P; ++u) k[j][u] = UNIT ? src[0][at + 32 * u] : src[UNIT ? 0 : u][at];
            at += j < last ? col_stride : 0;
        }
    };
    for (int slab = 0;; slab += kSlab) {            // cols may be 2^31 - 1: no sum goes beyond it
#pragma unroll
        for (int i = 0; i < kGroups; ++i)
            if (4 * (warp + kPlaneWarps * i) < cols - slab) fetch(kept[i], slab + 4 * (warp + kPlaneWarps * i));
#pragma unroll
        for (int i = 0; i < kGroups; ++i)
            if (4 * (warp + kPlaneWarps * i) < cols - slab)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int u = 0; u < P; ++u) top[u].add(kept[i][j][u]);
        if (KEEP || cols - slab <= kSlab) break;
    }
#pragma unroll
    for (int u = 0; u < P; ++u) tops[warp][32 * u + lane] = top[u].bits();
    __syncthreads();
    if (threadIdx.x < kRows) {
        uint32_t bits = 0;
#pragma unroll
        for (int i = 0; i < kPlaneWarps; ++i) bits = max(bits, tops[i][threadIdx.x]);
        const RowScale r = row_scale(bits);
        scales[threadIdx.x] = r;
        if (row0 + threadIdx.x < rows) scale[row0 + threadIdx.x] = r.scale;
    }
    __syncthreads();
    for (int slab = 0;; slab += kSlab) {
        const int n = min(cols - slab, kSlab);
        if (!KEEP) {
#pragma unroll
            for (int i = 0; i < kGroups; ++i)
                if (4 * (warp + kPlaneWarps * i) < n) fetch(kept[i], slab + 4 * (warp + kPlaneWarps * i));
        }
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const RowScale r = scales[32 * u + lane];
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
                const int c = 4 * (warp + kPlaneWarps * i);
                if (c >= n) continue;
                const float v[4] = {to_float(kept[i][0][u]), to_float(kept[i][1][u]), to_float(kept[i][2][u]), to_float(kept[i][3][u])};
                uint32_t w[1];
                quantize<4>(w, v, r);
                *(uint32_t*)(turned + (32 * u + lane) * kSlabPitch + c) = w[0];
                if (r.doubt != 0.f)
                    *(uint32_t*)(turned + (32 * u + lane) * kSlabPitch + c) =
                        exact_integers((UNIT ? src[0] + 32 * u : src[UNIT ? 0 : u]) + (slab + c) * col_stride, col_stride, min(n - c, 4), r.scale);
            }
        }
        __syncthreads();
        const int rows_in = (int)min((int64_t)kRows, rows - row0);
        for (int i = warp; i < rows_in; i += kPlaneWarps) {
            int8_t* dst = q + (row0 + i) * ldq + slab;
            const uint8_t* from = turned + i * kSlabPitch;
            if (words && n == kSlab) {
                const uint32_t a = *(const uint32_t*)(from + 4 * lane), b = *(const uint32_t*)(from + 128 + 4 * lane);
                ((uint32_t*)dst)[lane] = a;
                ((uint32_t*)dst)[32 + lane] = b;
            } else {
                const int whole = words ? n / 4 : 0;
                for (int c = lane; c < whole; c += 32) ((uint32_t*)dst)[c] = *(const uint32_t*)(from + 4 * c);
                for (int c = 4 * whole + lane; c < n; c += 32) dst[c] = (int8_t)from[c];
            }
        }
        if (KEEP || cols - slab <= kSlab) break;
        __syncthreads();
    }
}

// The same where blocks of whole rows would leave most SMs idle (74 rows x 4332 columns of bf16: 170 us, 13 in this way): a block takes kSlab columns of its rows.  First the largest
// |x| of every row, as bits in `scale`, joined with atomicMax (whose order does not matter); then the integers; then the scales.  Block i: rows from
// 32 (i % groups) and columns from kSlab (i / groups), in one extent of the grid, since only its first holds the slabs of 2^31 - 1 columns.
template <typename T>
__global__ void __launch_bounds__(32 * kPlaneWarps) plane_tops_kernel(const T* __restrict__ x, int64_t rows, int cols, int64_t row_stride, int64_t col_stride, uint32_t* __restrict__ tops, int groups)
{
    __shared__ uint32_t top[32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, begin = (int)(blockIdx.x / groups) * kSlab, n = min(cols - begin, kSlab);
    const int64_t row = (int64_t)(blockIdx.x % groups) * 32 + lane;
    if (warp == 0) top[lane] = 0;
    __syncthreads();
    Top<T> mine;
    if (row < rows)
#pragma unroll 8
        for (int c = warp; c < n; c += kPlaneWarps) mine.add(x[row * row_stride + (begin + c) * col_stride]);
    atomicMax(&top[lane], mine.bits());
    __syncthreads();
    if (warp == 0 && row < rows) atomicMax(tops + row, top[lane]);
}
template <typename T>
__global__ void __launch_bounds__(32 * kPlaneWarps) plane_integers_kernel(const T* __restrict__ x, int64_t rows, int cols, int64_t row_stride, int64_t col_stride,
                                                                          int8_t* __restrict__ q, int64_t ldq, const uint32_t* __restrict__ tops, int groups)
{
    __shared__ uint8_t turned[32 * kSlabPitch];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, begin = (int)(blockIdx.x / groups) * kSlab, n = min(cols - begin, kSlab);
    const int64_t row0 = (int64_t)(blockIdx.x % groups) * 32, row = row0 + lane;
    if (row < rows) {
        const RowScale r = row_scale(tops[row]);
#pragma unroll 4
        for (int c = warp; c < n; c += kPlaneWarps) turned[lane * kSlabPitch + c] = quantize_one(x + row * row_stride + (begin + c) * col_stride, r);
    }
    __syncthreads();
    for (int i = warp; i < 32 && row0 + i < rows; i += kPlaneWarps)
        for (int c = lane; c < n; c += 32) q[(row0 + i) * ldq + begin + c] = (int8_t)turned[i * kSlabPitch + c];
}
__global__ void plane_scales_kernel(float* scale, int64_t rows)
{
    const int64_t row = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (row < rows) scale[row] = row_scale(__float_as_uint(scale[row])).scale;
}

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

template <typename T>
cudaError_t launch(const T* x, int64_t rows, int64_t cols, int64_t rs, int64_t cs, int8_t* q, int64_t ldq, float* scale, int device, cudaStream_t s)
{
    const bool early = pdl_enabled();
    const int n = (int)cols;
    if (cs != 1 && cols > 1) {
        const int words = aligned(q, 4) && (ldq % 4 == 0 || rows == 1);
        constexpr int per = 32 * 8 / sizeof(T);
        int sms = 0;
        cudaError_t e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
        if (e != cudaSuccess) return e;
        if (n > kSlab && (rows + per - 1) / per < sms / 2) {    // blocks of whole rows would leave more than half of the SMs idle
            const int groups = (int)((rows + 31) / 32);
            const unsigned grid = (unsigned)(groups * ((cols + kSlab - 1) / kSlab));
            e = cudaMemsetAsync(scale, 0, sizeof(float) * rows, s);
            if (e != cudaSuccess) return e;
            e = launch_early(false, plane_tops_kernel<T>, dim3(grid), dim3(32 * kPlaneWarps), 0, s, x, rows, n, rs, cs, (uint32_t*)scale, groups);
            if (e == cudaSuccess) e = launch_early(false, plane_integers_kernel<T>, dim3(grid), dim3(32 * kPlaneWarps), 0, s, x, rows, n, rs, cs, q, ldq, (const uint32_t*)scale, groups);
            if (e == cudaSuccess) e = launch_early(false, plane_scales_kernel, dim3((unsigned)((rows + 255) / 256)), dim3(256), 0, s, scale, rows);
            return e;
        }
        const auto go = [&](auto kernel, const T* from, int64_t first, int64_t count) {
            return launch_early(early, kernel, dim3((unsigned)((count + per - 1) / per)), dim3(32 * kPlaneWarps), 0, s, from, count, n, rs, cs, q + first * ldq, ldq, scale + first, words);
        };
        // whole blocks of pixels that lie side by side, then what is left
        const int64_t unit = rs == 1 ? rows / per * per : 0;
        if (unit) e = n <= kSlab ? go(quantize_planes_kernel<T, true, true>, x, 0, unit) : go(quantize_planes_kernel<T, false, true>, x, 0, unit);
        if (e == cudaSuccess && unit < rows)
            e = n <= kSlab ? go(quantize_planes_kernel<T, true, false>, x + unit * rs, unit, rows - unit) : go(quantize_planes_kernel<T, false, false>, x + unit * rs, unit, rows - unit);
        return e;
    }
    constexpr int V = Piece<T>::V;
    const bool whole = aligned(x, 16) && (rows == 1 || rs * sizeof(T) % 16 == 0) && cols % V == 0 && aligned(q, V) && (rows == 1 || ldq % V == 0);
    const auto go = [&](auto kernel, int warps) {
        const int per = kThreads / 32 / warps;
        return launch_early(early, kernel, dim3((unsigned)((rows + per - 1) / per)), dim3(kThreads), 0, s, x, rows, n, rs, q, ldq, scale);
    };
    // as few warps to a row as have it in one stretch
    const int64_t room = 32 * (whole ? kItemsStraight : kItemsGathered) * V;
    if (whole) {
        if (cols <= room) return go(quantize_rows_kernel<T, 1, true, true>, 1);
        if (cols <= 2 * room) return go(quantize_rows_kernel<T, 2, true, true>, 2);
        if (cols <= 4 * room) return go(quantize_rows_kernel<T, 4, true, true>, 4);
        if (cols <= 8 * room) return go(quantize_rows_kernel<T, 8, true, true>, 8);
        return go(quantize_rows_kernel<T, 8, true, false>, 8);
    }
    if (cols <= room) return go(quantize_rows_kernel<T, 1, false, false>, 1);
    if (cols <= 2 * room) return go(quantize_rows_kernel<T, 2, false, false>, 2);
    if (cols <= 4 * room) return go(quantize_rows_kernel<T, 4, false, false>, 4);
    return go(quantize_rows_kernel<T, 8, false, false>, 8);
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
    if (col_stride == 1 || cols == 1) b.add("x", x, size, rows, cols, row_stride, false);
    else if (row_stride == 1 || rows == 1) b.add("x", x, size, cols, rows, col_stride, false);
    else b.add("x", x, size, (rows - 1) * row_stride + (cols - 1) * col_stride + 1, false);
    b.add("q", q, 1, rows, cols, ldq, true);
    b.add("scale", scale, 4, rows, true);
    if (!b.ok()) return b.status();
    cudaStream_t s = (cudaStream_t)cuda_stream;
    cudaError_t e = x_type == ST_F32 ? launch((const float*)x, rows, cols, row_stride, col_stride, q, ldq, scale, b.device(), s)
                  : x_type == ST_BF16 ? launch((const bf16*)x, rows, cols, row_stride, col_stride, q, ldq, scale, b.device(), s)
                                      : launch((const __half*)x, rows, cols, row_stride, col_stride, q, ldq, scale, b.device(), s);
    if (e != cudaSuccess) { cudaGetLastError(); return (st_status)fail_on_thread(ST_ERR_CUDA, "st_quantize_rows: %s", cudaGetErrorString(e)); }
    return ST_OK;
}

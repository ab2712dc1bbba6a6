// st_int8_matmul — product of 8-bit integers with a scale per token (row of x) and per output channel (row of w):
//   y[m][n] = act((sum_k x[m][k] w[n][k]) sx[m] sw[n] + b[n])
// Sums are exact in 32-bit integers; the four fp32 operations behind them are rounded one by one, in the order above.
//
// Both operands are K-major, so TMA's 128-byte-swizzled tiles go into tcgen05.mma kind::i8 (K = 32 bytes an instruction) as they
// are; extents that are no multiples of a tile are TMA's zero fill.  Four forms:
//   int8_tiles_kernel   more tokens: tokens are the accumulator's lanes, 64, 128 or 256 channels its columns; a persistent block per SM, ring of
//                       128-byte slices of K, two or four accumulators so that some are scaled and stored while the next is summed.
//   int8_pair_kernel    deep K: two SMs to a tile of 256 x 256.
//   int8_split_kernel   up to 128 tokens: channels are the lanes, tokens the columns; the blocks of a cluster share a tile's K range and add
//                       their sums through distributed shared memory.
//   int8_plain_kernel   operands that TMA cannot read (bases or pitches that are no multiples of 16 bytes): dp4a.
#include "../../include/shadowtutor.h"
#include "st_internal.h"
#include "int8_common.h"
#include "tc_common.cuh"

#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <mutex>

namespace st {

using namespace tc;

namespace {

constexpr int kTile = 128;                      // lanes of an accumulator
constexpr int kSlice = 128;                     // bytes of K in a stage: one swizzled row
constexpr int kSmemAlign = 1024;

// Instruction descriptor of tcgen05.mma kind::i8: D format 2 (s32), A and B format 1 (s8), both K-major
__host__ __device__ constexpr uint32_t instr_desc_i8(int M, int N)
{
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
__device__ __forceinline__ void umma_i8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"((uint64_t)map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int c0, int c1)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"((uint64_t)map), "r"(src), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ int std_min(int a, int b) { return a < b ? a : b; }
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ uint32_t cluster_address(uint32_t addr, uint32_t rank)
{
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
    return at;
}
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }

struct Out {
    void* y; int64_t ldy; int type, wide;       // wide: rows of y take whole 16-byte stores
    const float *sx, *sw, *bias; float least, one;
    int M, N;
};
// `least`: 0 with ReLU, else minus infinity; NaN (a token or channel that is not finite) stays NaN.  Without a bias 0 is added, which changes nothing.
__device__ __forceinline__ float at_least(float y, float least) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(y), "f"(least)); return r; }
__device__ __forceinline__ float finish(int acc, float sx, float sw, float bias, float least)
{
    return at_least(__fadd_rn(__fmul_rn(__fmul_rn((float)acc, sx), sw), bias), least);
}
// Two of them, two fp32 operations to an instruction.  The sum is a multiplication by a factor that the assembler does not know (`one` is 1):
// it fuses mul.rn.f32x2 and add.rn.f32x2, which are to be rounded one by one
__device__ __forceinline__ void finish2(float& a, float& b, float sx, float sw_a, float sw_b, float bias_a, float bias_b, float least, float one)
{
    const float x = (float)__float_as_int(a), y = (float)__float_as_int(b);
    asm("{\n\t.reg .b64 v, s, w, c, o;\n\t"
        "mov.b64 v, {%2, %3};\n\tmov.b64 s, {%4, %4};\n\tmov.b64 w, {%5, %6};\n\tmov.b64 c, {%7, %8};\n\tmov.b64 o, {%9, %9};\n\t"
        "mul.rn.f32x2 v, v, s;\n\tmul.rn.f32x2 v, v, w;\n\tfma.rn.f32x2 v, v, o, c;\n\tmov.b64 {%0, %1}, v;\n\t}"
        : "=f"(a), "=f"(b) : "f"(x), "f"(y), "f"(sx), "f"(sw_a), "f"(sw_b), "f"(bias_a), "f"(bias_b), "f"(one));
    a = at_least(a, least);
    b = at_least(b, least);
}
__device__ __forceinline__ uint16_t round16(float y, int type)
{
    return type == ST_BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(y)) : __half_as_ushort(__float2half_rn(y));
}
__device__ __forceinline__ uint32_t round16x2(float lo, float hi, int type)
{
    if (type == ST_BF16) { const __nv_bfloat162 q = __floats2bfloat162_rn(lo, hi); return *(const uint32_t*)&q; }
    const __half2 q = __floats2half2_rn(lo, hi);
    return *(const uint32_t*)&q;
}
__device__ __forceinline__ void put_one(const Out& o, int64_t at, float y)
{
    if (o.type == ST_F32) ((float*)o.y)[at] = y;
    else ((uint16_t*)o.y)[at] = round16(y, o.type);
}

// ---- many tokens ------------------------------------------------------------------------------------------------
constexpr int kPieceRow = 64, kPieceBytes = 32 * kPieceRow;        // what a warp stages at a time: 32 rows of 64 bytes
constexpr int kMaxStages = 8, kMaxResident = 16;                    // stages of the ring; slices of weights that stay in shared memory
constexpr int kMaxGroups = 4, kTilesThreads = 128 + 128 * kMaxGroups;     // producer, issuer, two that idle; groups that store
constexpr int kTilesSmem = 218 * 1024;                              // of a block, beside scales, bias and barriers
// `groups` of four warps scale and store, `slots` tiles at a time, each tile by groups / slots of them, which share its columns.  `resident`: all
// weights of the block's columns stay in shared memory and only tokens go through the ring; the launch's blocks are a multiple of
// n_tiles, so that a block's tiles have the same columns.  `stall`: 0; a test of the give-up path makes the first stage expect bytes that
// no copy delivers, so that the waits behind it run out.
struct TilesArgs { Out out; int tile_m, m_tiles, n_tiles, slices, stages, resident, groups, slots; unsigned int* err; uint32_t stall; };

// (Blocks of 256 columns read 12 KB of operands per 128 cycles of multiplication, of 128 columns 8 KB per 64: shared memory's rate.)
template <int BN>
struct TilesShape {
    static constexpr int accs = BN == 256 ? 2 : 4, cols = accs * BN, x_bytes = kTile * kSlice, w_bytes = BN * kSlice;
    static constexpr int bytes(int slices, int stages, bool resident, int groups)
    {
        return kSmemAlign + 4 * groups * kPieceBytes + stages * (resident ? x_bytes : x_bytes + w_bytes) + (resident ? slices * w_bytes : 0);
    }
    static constexpr int stages(int slices, bool resident, int groups)
    {
        return std::min((kTilesSmem - bytes(slices, 0, resident, groups)) / (resident ? x_bytes : x_bytes + w_bytes), kMaxStages);
    }
};

// A warp's 32 rows x 32 columns (a row to a lane) to y by TMA: staged in rows of 64 bytes, their 16-byte pieces where TMA's 64-byte swizzle has them
template <int TYPE>
__device__ __forceinline__ void stage_and_store(const float (&v)[32], uint32_t piece, int lane, const CUtensorMap* map, int col, int row, int N)
{
#pragma unroll
    for (int h = 0; h < (TYPE == ST_F32 ? 2 : 1); ++h) {
        if (lane == 0) tma_store_wait_read<0>();
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t to = piece + lane * kPieceRow + ((k ^ ((lane >> 1) & 3)) * 16);
            const float* x = v + (TYPE == ST_F32 ? 16 * h + 4 * k : 8 * k);
            if (TYPE == ST_F32) st_shared_128(to, __float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
            else st_shared_128(to, round16x2(x[0], x[1], TYPE), round16x2(x[2], x[3], TYPE), round16x2(x[4], x[5], TYPE), round16x2(x[6], x[7], TYPE));
        }
        fence_async_shared();
        __syncwarp();
        if (lane == 0) {
            if (col + 16 * h < N) tma_store_2d(map, piece, col + 16 * h, row);
            tma_store_commit();
        }
    }
}

// A warp's 32 rows x 32 columns to rows of y at any address: turned round in shared memory (2 KB), so that a warp's store is a piece of a row.
// (30000 x 300 x 300: 157 us with each lane storing its own row value by value.)  fp32: 16 rows at a time, 128 bytes to a store
__device__ __forceinline__ void store_rows_32(const float (&v)[32], float* buf, int lane, float* y, int64_t ldy, int rows)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        __syncwarp();
        if (lane / 16 == h) {
#pragma unroll
            for (int j = 0; j < 32; ++j) buf[(lane & 15) * 32 + ((j + lane) & 31)] = v[j];
        }
        __syncwarp();
        float* to = y + 16 * h * ldy + lane;
        const int turn = (lane + 16 * h) & 31;
#pragma unroll
        for (int r = 0; r < 16; ++r, to += ldy)
            if (16 * h + r < rows) *to = buf[r * 32 + ((turn + r) & 31)];
    }
    __syncwarp();
}
// 16 bits: two rows to a store, in words of two values; a row that begins between two words is moved by one value and its ends are stored alone
__device__ __forceinline__ void store_rows_16(const float (&v)[32], uint32_t* buf, int lane, uint16_t* y, int64_t ldy, int rows, int type)
{
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const uint32_t w = type == ST_BF16 ? round16x2(v[2 * k], v[2 * k + 1], ST_BF16) : round16x2(v[2 * k], v[2 * k + 1], ST_F16);
        buf[lane * 16 + ((k + lane) & 15)] = w;
    }
    __syncwarp();
    // a lane's rows are two apart: where one of them begins, to a word, the others do too
    const int k = lane & 15, r0 = lane >> 4;
    uint16_t* row = y + r0 * ldy;
    const bool whole = ((uintptr_t)row & 3) == 0;
    uint16_t* to = row + (whole ? 2 * k : 2 * k + 1);
#pragma unroll
    for (int i = 0; i < 16; ++i, to += 2 * ldy) {
        const int r = r0 + 2 * i;
        uint32_t w = buf[r * 16 + ((k + r) & 15)];
        const uint32_t after = whole ? 0u : buf[r * 16 + ((k + 1 + r) & 15)];
        if (r >= rows) continue;
        if (whole || k < 15) *(uint32_t*)to = whole ? w : __byte_perm(w, after, 0x5432);
        else { to[0] = (uint16_t)(w >> 16); to[-31] = (uint16_t)after; }              // word 15's end, and round to word 0
    }
    __syncwarp();
}
// The last columns of y, fewer than 32: 16 at a time
__device__ __forceinline__ void store_end(const float (&v)[32], float* buf, int lane, const Out& o, int64_t first, int rows, int columns)
{
    const int r0 = lane / 16, c = lane % 16;
#pragma unroll
    for (int h = 0; h < 32; h += 16) {
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 16; ++j) buf[lane * 16 + ((j + lane) & 15)] = v[h + j];
        __syncwarp();
        if (h + c < columns)
#pragma unroll 1
            for (int r = r0; r < rows; r += 2) put_one(o, first + r * o.ldy + h + c, buf[r * 16 + ((c + r) & 15)]);
    }
    __syncwarp();
}

// What the groups of warps that store do.  `rank` of BLOCKS that share a tile: the tile's rows are split between them.  acc_full: this block's barriers;
// acc_empty: those of the block that issues (cluster addresses where it may be another).  False: a wait gave up.
template <int BN, int ACCS, int BLOCKS>
__device__ __forceinline__ bool scale_and_store(const TilesArgs& a, const CUtensorMap& tm_y, const CUtensorMap& tm_y_rest, uint8_t* smem_raw, uint32_t staging, float* column,
                                                uint32_t tmem, uint32_t acc_full, uint32_t acc_empty, int warp, int lane, int first, int step, int tiles, int rank)
{
    constexpr int kWidth = BN == 256 ? 128 : BN;            // columns of a group's share, of four groups; two have the room of four
    bool ok = true;
    const int group = (warp - 4) / 4, quarter = warp % 4, tid = threadIdx.x - 128 - 128 * group;
    const int shares = std_min(a.groups / a.slots, BN / 32), width = BN / shares, slot = group / shares, c_begin = group % shares * width, c_most = c_begin + width;
    const Out& o = a.out;
    const bool whole_end = o.N * (o.type == ST_F32 ? 4 : 2) % 16 == 0;       // TMA leaves out the 16-byte pieces beyond y, but not the rest of one that y ends in
    const uint32_t piece = staging + (warp - 4) * kPieceBytes;
    float* const columns = column + group * 4 * (a.groups == 2 && BN == 256 ? 256 : kWidth);
    int index = 0, turn = 0;
    for (int t = first; t < tiles; t += step, ++index) {
        if (index % a.slots != slot) continue;
        const int acc = index % ACCS, acc_phase = index / ACCS & 1;
        float *const scales = columns + turn * 2 * width - c_begin, *const biases = scales + width;       // of column c at [c]
        turn ^= 1;
        const int m0 = (t / a.n_tiles * BLOCKS + rank) * a.tile_m, n0 = t % a.n_tiles * BN;
        const int64_t row = (int64_t)m0 + quarter * 32 + lane;
        const bool mine = quarter * 32 + lane < a.tile_m && row < o.M;
        const float sx = mine ? o.sx[row] : 0.f;
        for (int c = c_begin + tid; c < c_most; c += 128) {
            const bool in = n0 + c < o.N;
            scales[c] = in ? o.sw[n0 + c] : 0.f;
            biases[c] = in && o.bias ? o.bias[n0 + c] : 0.f;
        }
        asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory");
        // a warp whose wait has given up goes on through the tiles without storing: the others wait for it above
        if (ok) ok = mbar_wait(acc_full + 8 * acc, acc_phase, a.err, kWaitDone);
        tc_fence_after_sync();
        const int rows_in = min(min(a.tile_m, o.M - m0) - quarter * 32, 32);       // of this warp's 32
        const CUtensorMap* tm_out = a.tile_m - quarter * 32 >= 32 ? &tm_y : &tm_y_rest;
        const uint32_t lanes = tmem + acc * BN + ((uint32_t)(quarter * 32) << 16);
        const int c_end = ok && rows_in > 0 ? min(c_most, o.N - n0) : 0;
#pragma unroll 1
        for (int c0 = c_begin; c0 < c_end; c0 += 32) {
            float v[32];
            __syncwarp();
            tmem_ld_32x32(lanes + c0, v);
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const float4 sw = *(const float4*)(scales + c0 + j), b = *(const float4*)(biases + c0 + j);
                finish2(v[j], v[j + 1], sx, sw.x, sw.y, b.x, b.y, o.least, o.one);
                finish2(v[j + 2], v[j + 3], sx, sw.z, sw.w, b.z, b.w, o.least, o.one);
            }
            if (o.wide && (whole_end || n0 + c0 + 32 <= o.N)) {
                // (57600 x 512 x 256 with the three compared: 27 us with lanes storing their own rows, 18.5 with the warp storing from shared memory,
                // 17.3 in this way)
                const int at_row = m0 + quarter * 32, at_col = n0 + c0;
                if (o.type == ST_BF16) stage_and_store<ST_BF16>(v, piece, lane, tm_out, at_col, at_row, o.N);
                else if (o.type == ST_F16) stage_and_store<ST_F16>(v, piece, lane, tm_out, at_col, at_row, o.N);
                else stage_and_store<ST_F32>(v, piece, lane, tm_out, at_col, at_row, o.N);
            } else {
                if (lane == 0) tma_store_wait_read<0>();            // the copy of columns before these
                uint32_t* buf = (uint32_t*)(smem_raw + (piece - smem_u32(smem_raw)));
                const int64_t first = ((int64_t)m0 + quarter * 32) * o.ldy + n0 + c0;
                if (n0 + c0 + 32 > o.N) store_end(v, (float*)buf, lane, o, first, rows_in, o.N - n0 - c0);
                else if (o.type == ST_F32) store_rows_32(v, (float*)buf, lane, (float*)o.y + first, o.ldy, rows_in);
                else store_rows_16(v, buf, lane, (uint16_t*)o.y + first, o.ldy, rows_in, o.type);
            }
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) { if (BLOCKS == 1) mbar_arrive(acc_empty + 8 * acc); else mbar_arrive_cluster(acc_empty + 8 * acc); }
    }
    if (lane == 0) tma_store_wait();
    __syncwarp();
    return ok;
}

template <int BN>
__global__ void __launch_bounds__(kTilesThreads, 1) int8_tiles_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_y, const __grid_constant__ CUtensorMap tm_y_rest, const TilesArgs a)
{
    using Shape = TilesShape<BN>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t staging = (smem_u32(smem_raw) + kSmemAlign - 1) & ~(uint32_t)(kSmemAlign - 1), ring = staging + 4 * a.groups * kPieceBytes;
    const uint32_t stage_bytes = a.resident ? Shape::x_bytes : Shape::x_bytes + Shape::w_bytes, weights = ring + a.stages * stage_bytes;
    __shared__ __align__(8) uint64_t full[kMaxStages], empty[kMaxStages], acc_full[Shape::accs], acc_empty[Shape::accs], w_full[kMaxResident];
    __shared__ uint32_t tmem_slot;
    // scales and bias of a tile's columns, for each group twice: a warp may be a tile ahead of the others of its group
    constexpr int kWidth = BN == 256 ? 128 : BN;
    __shared__ __align__(16) float column[kMaxGroups * 4 * kWidth];
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (warp == 2) tmem_alloc(smem_u32(&tmem_slot), Shape::cols);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kMaxStages; ++i) { mbar_init(smem_u32(&full[i]), 1); mbar_init(smem_u32(&empty[i]), 1); }
        for (int i = 0; i < Shape::accs; ++i) { mbar_init(smem_u32(&acc_full[i]), 1); mbar_init(smem_u32(&acc_empty[i]), 4 * std_min(a.groups / a.slots, BN / 32)); }
        for (int i = 0; i < kMaxResident; ++i) mbar_init(smem_u32(&w_full[i]), 1);
        fence_barrier_init();
        prefetch_map(&tm_x); prefetch_map(&tm_w);
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    pdl_wait();
    pdl_launch_dependents();
    const int tiles = a.m_tiles * a.n_tiles;
    bool ok = true;
    // Producer and issuer are one thread each that looks at the next barrier before it waits for this one's (as whole warps that vote and
    // elect they took 500 cycles a slice, whatever its width)
    if (warp == 0) {                            // producer
        if (elect_one()) {
            uint32_t stage = 0, phase = 1;      // a fresh barrier's phase before the first counts as completed
            for (int t = (int)blockIdx.x; t < tiles && ok; t += gridDim.x) {
                const int m0 = t / a.n_tiles * a.tile_m, n0 = t % a.n_tiles * BN;
                const bool first = t == (int)blockIdx.x;
                for (int s = 0; s < a.slices; ++s) {
                    ok = mbar_wait_from(false, smem_u32(&empty[stage]), phase, a.err, kWaitEmpty);
                    if (!ok) break;
                    const uint32_t bar = smem_u32(&full[stage]), dst = ring + stage * stage_bytes;
                    mbar_expect_tx(bar, a.tile_m * kSlice + (a.resident ? 0 : Shape::w_bytes) + (first && s == 0 ? a.stall : 0u));
                    tma_load_2d(dst, &tm_x, bar, s * kSlice, m0);
                    if (!a.resident) tma_load_2d(dst + Shape::x_bytes, &tm_w, bar, s * kSlice, n0);
                    else if (first) {
                        mbar_expect_tx(smem_u32(&w_full[s]), Shape::w_bytes);
                        tma_load_2d(weights + s * Shape::w_bytes, &tm_w, smem_u32(&w_full[s]), s * kSlice, n0);
                    }
                    if (++stage == (uint32_t)a.stages) { stage = 0; phase ^= 1; }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {                     // issuer
        if (elect_one()) {
            constexpr uint32_t idesc = instr_desc_i8(kTile, BN);
            const uint64_t desc0 = smem_desc(ring, 16, 1024), w_desc0 = smem_desc(a.resident ? weights : ring + Shape::x_bytes, 16, 1024);
            const uint32_t step = stage_bytes >> 4, w_step = a.resident ? Shape::w_bytes >> 4 : step;
            uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 1;
            bool ready = false;                 // the next stage's data has been seen to be there
            for (int t = (int)blockIdx.x; t < tiles && ok; t += gridDim.x) {
                const bool first = t == (int)blockIdx.x;
                ok = mbar_wait_from(false, smem_u32(&acc_empty[acc]), acc_phase, a.err, kWaitDone);
                if (!ok) break;
                for (int s = 0; s < a.slices; ++s) {
                    ok = mbar_wait_from(ready, smem_u32(&full[stage]), phase, a.err, kWaitFull) && (!a.resident || !first || mbar_wait_from(false, smem_u32(&w_full[s]), 0, a.err, kWaitFull));
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint32_t now = stage;
                    if (++stage == (uint32_t)a.stages) { stage = 0; phase ^= 1; }
                    ready = mbar_try_wait(smem_u32(&full[stage]), phase);
                    const uint64_t da = desc0 + now * step, db = w_desc0 + (a.resident ? (uint32_t)s : now) * w_step;
#pragma unroll
                    for (int k = 0; k < kSlice / 32; ++k) umma_i8(tmem + acc * BN, da + 2 * k, db + 2 * k, idesc, (s | k) != 0);
                    umma_commit(smem_u32(&empty[now]));
                }
                if (!ok) break;
                umma_commit(smem_u32(&acc_full[acc]));
                if (++acc == Shape::accs) { acc = 0; acc_phase ^= 1; }
            }
        }
        __syncwarp();
    } else if (warp >= 4) {
        ok = scale_and_store<BN, Shape::accs, 1>(a, tm_y, tm_y_rest, smem_raw, staging, column, tmem, smem_u32(acc_full), smem_u32(acc_empty), warp, lane, blockIdx.x, gridDim.x, tiles, 0);
    }
    if (!ok) drain_after_error();
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 2) tmem_dealloc(tmem, Shape::cols);
}

// ---- many tokens, deep K: two SMs to a tile -----------------------------------------------------------------------
// A cluster of two blocks works on tiles of 256 rows x 256 columns: each holds half of the rows and half of the weights of a slice, one multiplication
// (cta_group::2, issued by the first block) uses both halves of both, and each block's tensor memory receives its rows.  A block's
// copies per slice are 32 KB instead of 48 KB, which leaves room for six stages instead of four.
constexpr int kPairStages = 6, kPairGroups = 2, kPairThreads = 128 + 128 * kPairGroups, kPairStageBytes = 2 * kTile * kSlice;
constexpr size_t kPairSmem = kSmemAlign + 4 * kPairGroups * kPieceBytes + kPairStages * kPairStageBytes;

__device__ __forceinline__ void tmem_alloc_pair(uint32_t smem_slot, uint32_t n_cols)
{
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_slot), "r"(n_cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t n_cols)
{
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(n_cols) : "memory");
}
// Into this block's shared memory, completion on a barrier of either block (a cluster address)
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"((uint64_t)map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void umma_i8_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
// Arrive on the barrier at this place of both blocks once all multiplications issued so far have completed
__device__ __forceinline__ void umma_commit_pair(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}

__global__ void __launch_bounds__(kPairThreads, 1) __cluster_dims__(2, 1, 1) int8_pair_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_y, const __grid_constant__ CUtensorMap tm_y_rest, const TilesArgs a)
{
    constexpr int BN = 256, kAccs = 2;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t staging = (smem_u32(smem_raw) + kSmemAlign - 1) & ~(uint32_t)(kSmemAlign - 1), ring = staging + 4 * kPairGroups * kPieceBytes;
    // full, acc_empty: the first block's are used; empty, acc_full: each block's own
    __shared__ __align__(8) uint64_t full[kPairStages], empty[kPairStages], acc_full[kAccs], acc_empty[kAccs];
    __shared__ uint32_t tmem_slot;
    __shared__ __align__(16) float column[kPairGroups * 4 * BN];
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, rank = blockIdx.x & 1;
    if (warp == 2) tmem_alloc_pair(smem_u32(&tmem_slot), kAccs * BN);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kPairStages; ++i) { mbar_init(smem_u32(&full[i]), 1); mbar_init(smem_u32(&empty[i]), 1); }
        for (int i = 0; i < kAccs; ++i) { mbar_init(smem_u32(&acc_full[i]), 1); mbar_init(smem_u32(&acc_empty[i]), 2 * 4 * (kPairGroups / a.slots)); }
        fence_barrier_init();
        prefetch_map(&tm_x); prefetch_map(&tm_w);
    }
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync();                             // both blocks' barriers are there
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    pdl_wait();
    pdl_launch_dependents();
    const int tiles = a.m_tiles * a.n_tiles, first = blockIdx.x >> 1, step = gridDim.x >> 1;
    bool ok = true;
    if (warp == 0) {                            // producer of this block's halves
        if (elect_one()) {
            uint32_t stage = 0, phase = 1;
            for (int t = first; t < tiles && ok; t += step) {
                const int m0 = (t / a.n_tiles * 2 + rank) * a.tile_m, n0 = t % a.n_tiles * BN + rank * (BN / 2);
                for (int s = 0; s < a.slices; ++s) {
                    ok = mbar_wait_from(false, smem_u32(&empty[stage]), phase, a.err, kWaitEmpty);
                    if (!ok) break;
                    const uint32_t bar = cluster_address(smem_u32(&full[stage]), 0), dst = ring + stage * kPairStageBytes;
                    if (rank == 0) mbar_expect_tx(smem_u32(&full[stage]), 2 * (a.tile_m + BN / 2) * kSlice + (t == first && s == 0 ? a.stall : 0u));
                    tma_load_2d_pair(dst, &tm_x, bar, s * kSlice, m0);
                    tma_load_2d_pair(dst + kTile * kSlice, &tm_w, bar, s * kSlice, n0);
                    if (++stage == kPairStages) { stage = 0; phase ^= 1; }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1 && rank == 0) {        // issuer for both
        if (elect_one()) {
            constexpr uint32_t idesc = instr_desc_i8(2 * kTile, BN);
            const uint64_t desc0 = smem_desc(ring, 16, 1024);
            uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 1;
            bool ready = false;
            for (int t = first; t < tiles && ok; t += step) {
                ok = mbar_wait_from(false, smem_u32(&acc_empty[acc]), acc_phase, a.err, kWaitDone);
                if (!ok) break;
                for (int s = 0; s < a.slices; ++s) {
                    ok = mbar_wait_from(ready, smem_u32(&full[stage]), phase, a.err, kWaitFull);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint32_t now = stage;
                    if (++stage == kPairStages) { stage = 0; phase ^= 1; }
                    ready = mbar_try_wait(smem_u32(&full[stage]), phase);
                    const uint64_t da = desc0 + now * (kPairStageBytes >> 4), db = da + (kTile * kSlice >> 4);
#pragma unroll
                    for (int k = 0; k < kSlice / 32; ++k) umma_i8_pair(tmem + acc * BN, da + 2 * k, db + 2 * k, idesc, (s | k) != 0);
                    umma_commit_pair(smem_u32(&empty[now]));
                }
                if (!ok) break;
                umma_commit_pair(smem_u32(&acc_full[acc]));
                if (++acc == kAccs) { acc = 0; acc_phase ^= 1; }
            }
        }
        __syncwarp();
    } else if (warp >= 4) {
        ok = scale_and_store<BN, kAccs, 2>(a, tm_y, tm_y_rest, smem_raw, staging, column, tmem, smem_u32(acc_full), cluster_address(smem_u32(acc_empty), 0), warp, lane, first, step, tiles, rank);
    }
    if (!ok) drain_after_error();
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync();                             // nobody leaves while the other block's copies, multiplications or arrivals may still reach it
    tc_fence_after_sync();
    if (warp == 2) tmem_dealloc_pair(tmem, kAccs * BN);
}

// ---- few tokens --------------------------------------------------------------------------------------
constexpr int kSplitThreads = 192;              // four warps that store, producer, issuer
constexpr int kMaxSplitStages = 8, kMaxSplits = 8;
struct SplitArgs { Out out; int slices, splits, stages; unsigned int* err; uint32_t stall; };

__device__ __forceinline__ int4 load_cluster(uint32_t addr, uint32_t rank)
{
    int4 v;
    asm volatile("ld.shared::cluster.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(cluster_address(addr, rank)) : "memory");
    return v;
}
// Four channels of a token; where rows of y are aligned and hold all four, one store
__device__ __forceinline__ void put_four(const Out& o, int64_t token, int channel, const int4& acc, float sx, const float4& sw, const float4& bias)
{
    const float y[4] = {finish(acc.x, sx, sw.x, bias.x, o.least), finish(acc.y, sx, sw.y, bias.y, o.least), finish(acc.z, sx, sw.z, bias.z, o.least),
                        finish(acc.w, sx, sw.w, bias.w, o.least)};
    const int64_t at = token * o.ldy + channel;
    if (o.wide && channel + 4 <= o.N) {
        if (o.type == ST_F32) *(float4*)((float*)o.y + at) = make_float4(y[0], y[1], y[2], y[3]);
        else *(uint2*)((uint16_t*)o.y + at) = make_uint2(round16x2(y[0], y[1], o.type), round16x2(y[2], y[3], o.type));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (channel + j < o.N) put_one(o, at + j, y[j]);
    }
}

// Block r of a cluster of `splits` sums slices [r, r + 1) / splits of K for 128 channels x BT tokens; sums are whole numbers, so their order does not
// matter.  Token t of the tile is then added up over the blocks, scaled and stored by block t % splits.
template <int BT>
__global__ void __launch_bounds__(kSplitThreads) int8_split_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const SplitArgs a)
{
    constexpr int kStage = (kTile + BT) * kSlice, kCols = BT < 32 ? 32 : BT;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t ring = (smem_u32(smem_raw) + kSmemAlign - 1) & ~(uint32_t)(kSmemAlign - 1);
    __shared__ __align__(8) uint64_t full[kMaxSplitStages], empty[kMaxSplitStages], acc_full;
    __shared__ uint32_t tmem_slot;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (warp == 0) tmem_alloc(smem_u32(&tmem_slot), kCols);
    if (threadIdx.x == 0) {
        for (int i = 0; i < a.stages; ++i) { mbar_init(smem_u32(&full[i]), 1); mbar_init(smem_u32(&empty[i]), 1); }
        mbar_init(smem_u32(&acc_full), 1);
        fence_barrier_init();
        prefetch_map(&tm_x); prefetch_map(&tm_w);
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    const int split = blockIdx.x % a.splits, n0 = blockIdx.x / a.splits * kTile;
    const int begin = (int)((int64_t)a.slices * split / a.splits), end = (int)((int64_t)a.slices * (split + 1) / a.splits);
    const Out& o = a.out;
    pdl_wait();
    pdl_launch_dependents();
    bool ok = true;
    const int count = o.M;                      // tokens, at most BT
    if (warp == 4) {
        if (elect_one()) {
            uint32_t stage = 0, phase = 1;
            for (int s = begin; s < end; ++s) {
                ok = mbar_wait_from(false, smem_u32(&empty[stage]), phase, a.err, kWaitEmpty);
                if (!ok) break;
                const uint32_t bar = smem_u32(&full[stage]), dst = ring + stage * kStage;
                mbar_expect_tx(bar, kStage + (s == begin ? a.stall : 0u));
                tma_load_2d(dst, &tm_w, bar, s * kSlice, n0);
                tma_load_2d(dst + kTile * kSlice, &tm_x, bar, s * kSlice, 0);
                if (++stage == (uint32_t)a.stages) { stage = 0; phase ^= 1; }
            }
        }
        __syncwarp();
    } else if (warp == 5) {
        if (elect_one()) {
            constexpr uint32_t idesc = instr_desc_i8(kTile, BT);
            const uint64_t desc0 = smem_desc(ring, 16, 1024);
            uint32_t stage = 0, phase = 0;
            bool ready = false;
            for (int s = begin; s < end; ++s) {
                ok = mbar_wait_from(ready, smem_u32(&full[stage]), phase, a.err, kWaitFull);
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t now = stage;
                if (++stage == (uint32_t)a.stages) { stage = 0; phase ^= 1; }
                ready = mbar_try_wait(smem_u32(&full[stage]), phase);
                const uint64_t da = desc0 + now * (kStage >> 4), db = da + (kTile * kSlice >> 4);
#pragma unroll
                for (int k = 0; k < kSlice / 32; ++k) umma_i8(tmem, da + 2 * k, db + 2 * k, idesc, (s != begin) | (k != 0));
                umma_commit(smem_u32(&empty[now]));
            }
            if (ok) umma_commit(smem_u32(&acc_full));
        }
        __syncwarp();
    } else if (warp < 4) {
        const int channel = n0 + threadIdx.x;
        const bool mine = channel < o.N;
        const float sw = mine ? o.sw[channel] : 0.f, bias = mine && o.bias ? o.bias[channel] : 0.f;
        ok = mbar_wait(smem_u32(&acc_full), 0, a.err, kWaitDone);
        tc_fence_after_sync();
        if (ok) {
#pragma unroll
            for (int c0 = 0; c0 < BT; c0 += 16) {
                if (c0 >= count) break;
                float v[16];
                __syncwarp();
                tmem_ld_32x16(tmem + ((uint32_t)(warp * 32) << 16) + c0, v);
                if (a.splits == 1) {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (mine && c0 + j < count) put_one(o, (int64_t)(c0 + j) * o.ldy + channel, finish(__float_as_int(v[j]), o.sx[c0 + j], sw, bias, o.least));
                } else {                        // every MMA has read its operands: the ring is free
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (c0 + j < count) asm volatile("st.shared.b32 [%0], %1;" ::"r"(ring + ((c0 + j) * kTile + threadIdx.x) * 4), "r"(__float_as_int(v[j])) : "memory");
                }
            }
        }
    }
    if (!ok) drain_after_error();
    __syncwarp();
    if (a.splits > 1) {
        const int all_ok = __syncthreads_and(ok);
        cluster_sync();
        if (warp < 4 && all_ok) {
            // a warp to a token, four channels to a lane; the sums of all blocks are on their way together
            const int channel = n0 + 4 * lane;
            float scales[4], biases[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                scales[j] = channel + j < o.N ? o.sw[channel + j] : 0.f;
                biases[j] = channel + j < o.N && o.bias ? o.bias[channel + j] : 0.f;
            }
            const float4 sw = make_float4(scales[0], scales[1], scales[2], scales[3]), bias = make_float4(biases[0], biases[1], biases[2], biases[3]);
            for (int c = split + a.splits * warp; c < count; c += 4 * a.splits) {
                const uint32_t at = ring + (c * kTile + 4 * lane) * 4;
                int4 part[kMaxSplits];
#pragma unroll
                for (int r = 0; r < kMaxSplits; ++r) part[r] = r < a.splits ? load_cluster(at, r) : make_int4(0, 0, 0, 0);
                int4 sum = part[0];
#pragma unroll
                for (int r = 1; r < kMaxSplits; ++r) { sum.x += part[r].x; sum.y += part[r].y; sum.z += part[r].z; sum.w += part[r].w; }
                put_four(o, c, channel, sum, o.sx[c], sw, bias);
            }
        }
        __syncwarp();
        cluster_sync();                         // nobody leaves while others read its sums
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, kCols);
}

// ---- operands at any address ----------------------------------------------------------------------------------------
constexpr int kPlainTile = 64, kPlainK = 64, kPlainPitch = kPlainK / 4 + 1;
__global__ void __launch_bounds__(256) int8_plain_kernel(const int8_t* __restrict__ x, int64_t ldx, const int8_t* __restrict__ w, int64_t ldw, int K, const Out o)
{
    __shared__ uint32_t xs[kPlainTile * kPlainPitch], ws[kPlainTile * kPlainPitch];
    pdl_wait();
    pdl_launch_dependents();
    const int64_t m0 = (int64_t)blockIdx.x * kPlainTile;
    const int n0 = blockIdx.y * kPlainTile, tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    int acc[4][4] = {};
    for (int k0 = 0; k0 < K; k0 += kPlainK) {
        for (int i = threadIdx.x; i < kPlainTile * kPlainK; i += 256) {
            const int r = i / kPlainK, c = i % kPlainK;
            const bool k_in = k0 + c < K;
            ((int8_t*)xs)[r * kPlainPitch * 4 + c] = k_in && m0 + r < o.M ? x[(m0 + r) * ldx + k0 + c] : (int8_t)0;
            ((int8_t*)ws)[r * kPlainPitch * 4 + c] = k_in && n0 + r < o.N ? w[(int64_t)(n0 + r) * ldw + k0 + c] : (int8_t)0;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPlainK / 4; ++k) {
            uint32_t a[4], b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { a[i] = xs[(ty + 16 * i) * kPlainPitch + k]; b[i] = ws[(tx + 16 * i) * kPlainPitch + k]; }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a((int)a[i], (int)b[j], acc[i][j]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + ty + 16 * i;
        if (m >= o.M) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int n = n0 + tx + 16 * j;
            if (n < o.N) put_one(o, m * o.ldy + n, finish(acc[i][j], o.sx[m], o.sw[n], o.bias ? o.bias[n] : 0.f, o.least));
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------
// What a device needs before its first launch: the kernels' limits of shared memory, and words in pinned host memory in which a wait that gave up
// leaves its code, so that the next call on the same stream can tell without waiting for the device.  Streams, by their handles, have words of their
// own, up to kErrWords of them; any more share.  (Their numbers, cudaStreamGetId, cannot be asked for while they are captured.)  One more word is for
// launches that become part of a graph: it may be replayed on any stream, and the one that was captured may see no call again, so that whichever
// call comes next tells of them.
constexpr int kMaxDevices = 64, kErrWords = 1024;
struct Device { bool ready = false; int sms = 0; unsigned int *err = nullptr, *err_dev = nullptr; uintptr_t owner[kErrWords] = {}; };
Device g_devices[kMaxDevices];
std::mutex g_mutex;

// `word`: which of the device's words is the stream's
cudaError_t device_for(int index, cudaStream_t s, Device** out, int* word)
{
    if (index < 0 || index >= kMaxDevices) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(g_mutex);
    Device& d = g_devices[index];
    *out = &d;
    const uintptr_t key = (uintptr_t)s + 1;             // the default stream's handle is 0, and so is a word without an owner
    uint32_t at = (uint32_t)((uint64_t)key * 0x9e3779b97f4a7c15u >> 54);
    for (int i = 0; i < kErrWords && d.owner[at] != key && d.owner[at]; ++i) at = (at + 1) % kErrWords;
    if (!d.owner[at]) d.owner[at] = key;
    *word = (int)at;
    if (d.ready) return cudaSuccess;
    cudaError_t e = cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, index);
    for (const void* k : {(const void*)int8_tiles_kernel<64>, (const void*)int8_tiles_kernel<128>, (const void*)int8_tiles_kernel<256>, (const void*)int8_pair_kernel,
                          (const void*)int8_split_kernel<16>, (const void*)int8_split_kernel<32>, (const void*)int8_split_kernel<64>, (const void*)int8_split_kernel<128>})
        if (e == cudaSuccess) e = allow_shared_memory(k);
    if (e == cudaSuccess && !d.err) e = cudaHostAlloc((void**)&d.err, (kErrWords + 1) * sizeof(unsigned int), cudaHostAllocMapped | cudaHostAllocPortable);
    if (e == cudaSuccess) { std::fill_n(d.err, kErrWords + 1, 0u); e = cudaHostGetDevicePointer((void**)&d.err_dev, d.err, 0); }
    d.ready = e == cudaSuccess;
    return e;
}

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

uint32_t stall_bytes()
{
    const char* e = getenv("ST_TEST_STALL_INT8");
    return e && e[0] == '1' ? 16u : 0u;
}

bool operand_map(CUtensorMap* m, const int8_t* q, int64_t rows, int64_t ld, int64_t K, int box_rows, char* msg, size_t msg_len, const char* what)
{
    const uint64_t dims[2] = {(uint64_t)K, (uint64_t)rows}, strides[1] = {(uint64_t)(rows == 1 ? (K + 15) / 16 * 16 : ld)};
    const uint32_t box[2] = {kSlice, (uint32_t)box_rows};
    return encode_tensor_map(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, CU_TENSOR_MAP_SWIZZLE_128B, q, 2, dims, strides, box, msg, msg_len, what);
}

int launch(const Int8Product& p, unsigned int* err, const Device* d, cudaStream_t s)
{
    const auto cuda_fail = [](cudaError_t e) { cudaGetLastError(); return fail_on_thread(ST_ERR_CUDA, "st_int8_matmul: %s", cudaGetErrorString(e)); };
    cudaError_t e;
    Out o = {p.y, p.ldy, p.y_type, 0, p.x_scale, p.w_scale, p.bias, p.relu ? 0.f : -INFINITY, 1.f, (int)p.M, (int)p.N};
    const int64_t size = p.y_type == ST_F32 ? 4 : 2;
    o.wide = aligned(p.y, 16) && (p.M == 1 || p.ldy * size % 16 == 0);
    const bool tma = aligned(p.x, 16) && aligned(p.w, 16) && (p.M == 1 || p.ldx % 16 == 0) && (p.N == 1 || p.ldw % 16 == 0);
    if (!tma) {
        const dim3 grid((unsigned)((p.M + kPlainTile - 1) / kPlainTile), (unsigned)((p.N + kPlainTile - 1) / kPlainTile));
        e = launch_early(pdl_enabled(), int8_plain_kernel, grid, dim3(256), 0, s, p.x, p.ldx, p.w, p.ldw, (int)p.K, o);
        return e == cudaSuccess ? (int)ST_OK : cuda_fail(e);
    }
    char msg[160] = "";
    CUtensorMap tx, tw;
    const int slices = (int)((p.K + kSlice - 1) / kSlice);
    // What the forms would take, in microseconds: launch and ends, then for each round of tiles the slices and what storing adds, fitted to 40 shapes
    // from 1 x 256 x 256 to 57600 x 512 x 256 that several were run on (off by 20 per cent at most; 16 x 4096 x 4096: 6.3 measured for clusters, 9.7
    // for tiles of 64 columns; 128 x 4096 x 4096: 12 and 10; 4096 x 1024 x 1024: 11.4, 8.7 and 7.5 for tiles of 64, 128 and 256 columns;
    // 8192 x 4096 x 4096: 99.6 for tiles of 256 columns, 87 for pairs of SMs; 57600 x 512 x 256: 18.8 and 25).
    const auto time_of = [&](int rows, int columns, int at_once, double slice, double store) {
        const int64_t tiles = (p.M + rows - 1) / rows * ((p.N + columns - 1) / columns), rounds = (tiles + at_once - 1) / at_once;
        return 3.3 + (double)rounds * (slices * slice + store);
    };
    const auto tiles_time = [&](int columns) { return time_of(kTile, columns, d->sms, columns == 64 ? 0.20 : columns == 128 ? 0.22 : 0.34, columns / 160.0); };
    int bn = 64;
    for (int columns : {128, 256})
        if (tiles_time(columns) < tiles_time(bn)) bn = columns;
    const bool pair = d->sms >= 2 && time_of(2 * kTile, 256, d->sms / 2, 0.30, 2.3) < tiles_time(bn);
    const int bt = p.M <= 16 ? 16 : p.M <= 32 ? 32 : p.M <= 64 ? 64 : 128;
    const int64_t n_split_tiles = (p.N + kTile - 1) / kTile;
    // As many blocks to a tile as the SMs allow, with a slice of K each at least.  A few more blocks than SMs are let in: where a block's stages take
    // less than half of an SM's shared memory two fit one, otherwise (128 tokens x 4096 x 2560: 160 blocks of 128 KB) the last clusters wait for the first
    int splits = 1;
    while (splits < kMaxSplits && n_split_tiles * splits * 2 <= d->sms + 20 && slices >= splits * 2) splits *= 2;
    const double weight_time = (double)p.N * (double)p.K / 5.5e6, slice_time = 0.16 * ((slices + splits - 1) / splits) * (double)((n_split_tiles * splits + d->sms - 1) / d->sms);
    if (p.M <= 128 && 2.6 + std::max(weight_time, slice_time) + 0.04 * bt < tiles_time(bn)) {
        SplitArgs a;
        a.out = o; a.slices = slices; a.splits = splits; a.err = err; a.stall = stall_bytes();
        const int stage = (kTile + bt) * kSlice, per = (slices + splits - 1) / splits;
        a.stages = std::min({kMaxSplitStages, per, 200 * 1024 / stage});
        // At least as large a share of an SM's shared memory as its columns are of tensor memory: blocks of a cluster wait for one another, and would
        // do so for good if clusters of several streams each held columns that another one's blocks wait for
        const size_t bytes = std::max<size_t>((size_t)std::max(a.stages * stage, splits > 1 ? bt * kTile * 4 : 0) + kSmemAlign, (size_t)std::max(bt, 32) * (227 * 1024 / 512));
        if (!operand_map(&tx, p.x, p.M, p.ldx, p.K, bt, msg, sizeof msg, "x") || !operand_map(&tw, p.w, p.N, p.ldw, p.K, kTile, msg, sizeof msg, "w"))
            return fail_on_thread(ST_ERR_CUDA, "st_int8_matmul: %s", msg);
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(n_split_tiles * splits)); cfg.blockDim = dim3(kSplitThreads); cfg.dynamicSmemBytes = bytes; cfg.stream = s;
        cudaLaunchAttribute at[2];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = (unsigned)splits; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
        at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = at; cfg.numAttrs = pdl_enabled() ? 2 : 1;
        e = bt == 16 ? cudaLaunchKernelEx(&cfg, int8_split_kernel<16>, tx, tw, a) : bt == 32 ? cudaLaunchKernelEx(&cfg, int8_split_kernel<32>, tx, tw, a)
          : bt == 64 ? cudaLaunchKernelEx(&cfg, int8_split_kernel<64>, tx, tw, a) : cudaLaunchKernelEx(&cfg, int8_split_kernel<128>, tx, tw, a);
        return e == cudaSuccess ? (int)ST_OK : cuda_fail(e);
    }
    TilesArgs a;
    const int tile_n = pair ? 256 : bn, box_n = pair ? 128 : bn;        // columns of a tile, and of what one block fetches of it
    a.out = o; a.n_tiles = (int)((p.N + tile_n - 1) / tile_n); a.slices = slices; a.err = err; a.stall = stall_bytes();
    // Rows of a tile: 128, or fewer where as many rounds of tiles then fill all SMs evenly.  (57600 x 512 x 256: 450 tiles of 128 rows are 3.04
    // rounds of 148, the fourth nearly empty; tiles of 98 rows fill four.)
    const auto even_rows = [&](int64_t per_round) {
        const int64_t rounds = ((p.M + kTile - 1) / kTile + per_round - 1) / per_round;
        return (int)std::min<int64_t>(kTile, (p.M + rounds * per_round - 1) / (rounds * per_round));
    };
    int64_t blocks;
    size_t bytes;
    if (pair) {
        const int64_t pairs = d->sms / 2, rounds = ((p.M + 2 * kTile - 1) / (2 * kTile) * a.n_tiles + pairs - 1) / pairs, most = std::max<int64_t>(1, rounds * pairs / a.n_tiles);
        a.tile_m = (int)std::min<int64_t>(kTile, (p.M + 2 * most - 1) / (2 * most));
        a.m_tiles = (int)((p.M + 2 * a.tile_m - 1) / (2 * a.tile_m));
        const int64_t tiles = (int64_t)a.m_tiles * a.n_tiles;
        blocks = 2 * std::min(tiles, pairs);
        a.stages = kPairStages; a.resident = 0; a.groups = kPairGroups; a.slots = 2 * tiles <= blocks ? 1 : 2;
        bytes = kPairSmem;
    } else {
        const auto shape = [&](auto f) { return bn == 64 ? f(TilesShape<64>()) : bn == 128 ? f(TilesShape<128>()) : f(TilesShape<256>()); };
        // The weights of a block's columns stay in shared memory where they leave room for three stages of tokens and a block has two tiles at least
        const int64_t columns = d->sms / a.n_tiles;          // blocks that share the same weights
        const int kept_stages = shape([&](auto q) { return q.stages(slices, true, kMaxGroups); });
        a.resident = slices <= kMaxResident && kept_stages >= 3 && columns * a.n_tiles * 10 >= d->sms * 9 && (p.M + kTile - 1) / kTile >= 2 * columns;
        if (a.resident) a.tile_m = even_rows(columns);
        else {
            const int64_t rounds = ((p.M + kTile - 1) / kTile * a.n_tiles + d->sms - 1) / d->sms, most = rounds * d->sms / a.n_tiles;
            a.tile_m = (int)std::min<int64_t>(kTile, (p.M + most - 1) / most);
        }
        a.m_tiles = (int)((p.M + a.tile_m - 1) / a.tile_m);
        // Four groups that store where their staging leaves the ring four stages (three beside resident weights, or where rows of y at any address
        // make storing the slower part: 3751 x 653 x 6518), else two
        a.groups = kMaxGroups;
        a.stages = a.resident ? kept_stages : shape([&](auto q) { return q.stages(slices, false, kMaxGroups); });
        if (!a.resident && a.stages < (o.wide ? 4 : 3)) { a.groups = 2; a.stages = shape([&](auto q) { return q.stages(slices, false, 2); }); }
        const int64_t tiles = (int64_t)a.m_tiles * a.n_tiles;
        blocks = std::min<int64_t>(tiles, a.resident ? columns * a.n_tiles : d->sms);
        a.slots = tiles <= blocks ? 1 : shape([&](auto q) { return std::min(a.groups, q.accs); });
        bytes = shape([&](auto q) { return (size_t)q.bytes(slices, a.stages, a.resident, a.groups); });
    }
    CUtensorMap ty = {}, ty_rest = {};               // of 32 rows, and of the rows that a tile has beyond multiples of 32
    if (o.wide) {
        const uint64_t dims[2] = {(uint64_t)p.N, (uint64_t)p.M}, strides[1] = {(uint64_t)(p.M == 1 ? (p.N * size + 15) / 16 * 16 : p.ldy * size)};
        const uint32_t box[2] = {(uint32_t)(kPieceRow / size), 32}, rest[2] = {box[0], (uint32_t)(a.tile_m % 32 ? a.tile_m % 32 : 32)};
        const CUtensorMapDataType type = p.y_type == ST_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : p.y_type == ST_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
        if (!encode_tensor_map(&ty, type, CU_TENSOR_MAP_SWIZZLE_64B, p.y, 2, dims, strides, box, msg, sizeof msg, "y") ||
            !encode_tensor_map(&ty_rest, type, CU_TENSOR_MAP_SWIZZLE_64B, p.y, 2, dims, strides, rest, msg, sizeof msg, "y"))
            return fail_on_thread(ST_ERR_CUDA, "st_int8_matmul: %s", msg);
    }
    if (!operand_map(&tx, p.x, p.M, p.ldx, p.K, a.tile_m, msg, sizeof msg, "x") || !operand_map(&tw, p.w, p.N, p.ldw, p.K, box_n, msg, sizeof msg, "w"))
        return fail_on_thread(ST_ERR_CUDA, "st_int8_matmul: %s", msg);
    const auto go = [&](auto kernel) { return launch_early(pdl_enabled(), kernel, dim3((unsigned)blocks), dim3(128 + 128 * a.groups), bytes, s, tx, tw, ty, ty_rest, a); };
    e = pair ? go(int8_pair_kernel) : bn == 64 ? go(int8_tiles_kernel<64>) : bn == 128 ? go(int8_tiles_kernel<128>) : go(int8_tiles_kernel<256>);
    return e == cudaSuccess ? (int)ST_OK : cuda_fail(e);
}

}  // namespace

int int8_matmul(const Int8Product& p, cudaStream_t s)
{
    const int64_t M = p.M, N = p.N, K = p.K;
    const auto bad = [](const char* what) { return fail_on_thread(ST_ERR_INVALID_ARG, "st_int8_matmul: %s", what); };
    if (M < 0 || N < 0 || K < 1) return bad("needs M >= 0, N >= 0 and K >= 1");
    if (p.y_type != ST_F32 && p.y_type != ST_BF16 && p.y_type != ST_F16) return bad("y_type is not an st_dtype");
    if (p.relu & ~1) return bad("relu must be 0 or 1");
    if (p.ldx < K || p.ldw < K || p.ldy < N) return bad("ldx, ldw below K or ldy below N");
    if (K > kMaxInt8K) return fail_on_thread(ST_ERR_UNSUPPORTED, "st_int8_matmul: K above %d could overflow the 32-bit sums", kMaxInt8K);
    if (M > kMaxInt8Extent - 255 || N > kMaxInt8N || !extent_fits(M, p.ldx, K, 1) || !extent_fits(N, p.ldw, K, 1) || !extent_fits(M, p.ldy, N, 1) ||
        ((M + 127) / 128) * ((N + 63) / 64) > kMaxInt8Extent / 2)
        return fail_on_thread(ST_ERR_UNSUPPORTED, "st_int8_matmul: extents beyond the kernels' 32-bit counts of tiles");
    if (M == 0 || N == 0) return ST_OK;
    Int8Buffers b("st_int8_matmul");
    b.add("x", p.x, 1, M, K, p.ldx, false);
    b.add("x_scale", p.x_scale, 4, M, false);
    b.add("w", p.w, 1, N, K, p.ldw, false);
    b.add("w_scale", p.w_scale, 4, N, false);
    if (p.bias) b.add("bias", p.bias, 4, N, false);
    b.add("y", p.y, p.y_type == ST_F32 ? 4 : 2, M, N, p.ldy, true);
    if (!b.ok()) return b.status();
    const auto cuda_fail = [](cudaError_t e) { cudaGetLastError(); return fail_on_thread(ST_ERR_CUDA, "st_int8_matmul: %s", cudaGetErrorString(e)); };
    Device* d = nullptr;
    int word = 0;
    const cudaError_t e = device_for(b.device(), s, &d, &word);
    if (e != cudaSuccess) return cuda_fail(e);
    if (p.err) return launch(p, p.err, d, s);
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(s, &capture) != cudaSuccess) { cudaGetLastError(); capture = cudaStreamCaptureStatusNone; }
    const int status = launch(p, d->err_dev + (capture == cudaStreamCaptureStatusNone ? word : kErrWords), d, s);
    if (status != ST_OK) return status;
    // what an earlier product has left is told once, and this product is enqueued all the same: what gave up need not be the caller's
    if (const unsigned int code = __atomic_exchange_n(d->err + word, 0u, __ATOMIC_RELAXED))
        return fail_on_thread(ST_ERR_CUDA, "st_int8_matmul: a device wait of a product on this stream gave up (code %u); its result is not complete", code);
    if (const unsigned int code = __atomic_exchange_n(d->err + kErrWords, 0u, __ATOMIC_RELAXED))
        return fail_on_thread(ST_ERR_CUDA, "st_int8_matmul: a device wait of a product in a replayed graph gave up (code %u); its result is not complete", code);
    return ST_OK;
}

}  // namespace st

using namespace st;

extern "C" st_status st_int8_matmul(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w, int64_t ldw, const float* w_scale,
                                    const float* bias, int32_t relu, int64_t M, int64_t N, int64_t K, void* y, int32_t y_type, int64_t ldy, void* cuda_stream)
{
    return (st_status)int8_matmul({x, ldx, x_scale, w, ldw, w_scale, bias, relu, M, N, K, y, y_type, ldy, nullptr}, (cudaStream_t)cuda_stream);
}

// Linear layers with 4-bit weights and group scales on few rows of real activations (decoding).
//
// Mathematics.  y[r][o] = sum_g s[o][g] sum_{k in g} (q[o][k] - z[o][g]) x[r][k] + b[o].
//   up to 8 rows   The codes meet the integer matrix instructions (m16n8k32) as they are: eight are cut from a word by three logic
//                  operations.  Each row's 256 columns at hand are written as 2^(e - 21) (d_2 2^16 + d_1 2^8 + d_0), e the exponent
//                  of their largest value, d in [-128, 127]: 22 bits below it, more than the 11 or 8 that a value has; one operand
//                  column for each digit.  Integer sums are exact; scale, digit weight and zero point (through the sum of x over the
//                  group) multiply them in fp32.
//   more rows      fp16 / bf16 matrix instructions (m16n8k16) with q - z as an exact operand: two codes are cut from a word by one
//                  logic operation that also writes the exponent (1024 + q in fp16, 128 + q in bf16), one packed operation takes the
//                  offset off; the scale multiplies the fp32 sum of its group, or of the 64 columns of it that are at hand.
// Nothing is rounded to 16 bits before y.
//
// What bounds it: half a byte of weight is read for 2 flops an activation row.  At the measured copy rate that is 46 weights a clock
// and SM, for which the SM issues 2.8 operations a weight: the second form needs about 2.3, the first 0.8 for one row and 1.9 for
// eight, where its matrix instructions (2048 products a clock) still take 85 weights a clock.  With 32 rows the second form's
// matrix instructions (1024 products a clock) take 32 weights a clock: they bound it.
// The weights are read once, in the order of use, as contiguous blocks of 32 rows x 256 columns with their scales and zero points
// behind the codes; every warp streams its blocks through a ring of its own (bulk copies, several blocks ahead).  Activations are
// few: the eight warps of a CTA work on the same columns of 256 rows and share them in shared memory.
// The (256 rows, 256 columns) units form one sequence that is dealt out in equal contiguous shares to a grid that fills the GPU
// once; rows whose columns lie in several CTAs are joined by the last of those to arrive, in the order of the columns.
#include <new>
#include <type_traits>

#include "qtz_half_util.cuh"
#include "qtz_internal.cuh"
#include "qtz_ptx.cuh"

struct qtz_linear {
    qtz_ctx* h = nullptr;
    qtz_linear_desc d{};
    int row_tiles = 0, k_blocks = 0;   // of 32 rows, of 256 columns
    int scales = 0;                    // scales of a row in a block of 256 columns: 2, 4 or 8
    int block_bytes = 0;
    uint8_t* blocks = nullptr;         // [row_tiles][k_blocks][block_bytes]: codes, scales, zero points
    void* bias = nullptr;              // [n], behind the blocks in the same allocation; null: none
};

namespace {

using namespace qtz_ptx;

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kRowTile = 32, kKBlock = 256;
constexpr int kCodeBytes = kRowTile * kKBlock / 2;
constexpr int kMaxStages = 8;
constexpr int kMaxTokens = 32;             // activation rows of one pass over the weights
constexpr int kSmemLimit = 227 * 1024;

// ------------------------------------------------------------------------------------
// preparation
// ------------------------------------------------------------------------------------
struct PackArgs {
    const uint8_t* codes;
    const uint16_t* scales;
    const uint8_t* zeros;
    int n, k, group, groups, k_blocks, per_block, block_bytes;
    bool is_signed;
    uint8_t* out;
};

// One thread per 32-bit word of codes: word (chunk of 64 columns, half of the 32 rows, lane, w) holds eight columns of one row, in
// the order in which the lanes of a matrix instruction hold their operand: columns 0 .. 3 in the low nibbles of the four bytes,
// 4 .. 7 in the high ones.
__global__ void __launch_bounds__(256)
pack_kernel(PackArgs a)
{
    uint8_t* block = a.out + (static_cast<int64_t>(blockIdx.y) * a.k_blocks + blockIdx.x) * a.block_bytes;
    const int row0 = blockIdx.y * kRowTile, k0 = blockIdx.x * kKBlock;
    for (int i = threadIdx.x; i < kCodeBytes / 4; i += 256) {
        const int w = i & 3, lane = (i >> 2) & 31, half = (i >> 7) & 1, chunk = i >> 8;
        const int row = row0 + half * 16 + (lane >> 2) + 8 * (w & 1), k = k0 + chunk * 64 + (w >> 1) * 32 + 8 * (lane & 3);
        uint32_t v = 0;
        for (int j = 0; j < 8; ++j) {
            uint32_t q = a.is_signed ? 8 : 0;          // beyond the matrix: the code of zero
            if (row < a.n && k + j < a.k) {
                const uint8_t byte = a.codes[static_cast<int64_t>(row) * ((a.k + 1) / 2) + ((k + j) >> 1)];
                q = ((k + j) & 1 ? byte >> 4 : byte & 15) ^ (a.is_signed ? 8 : 0);
            } else if (row < a.n && a.zeros) {
                const int g = min((k + j) / a.group, a.groups - 1);
                q = min(static_cast<int>(a.zeros[static_cast<int64_t>(row) * a.groups + g]), 15);
            }
            v |= q << (8 * (j & 3) + 4 * (j >> 2));
        }
        reinterpret_cast<uint32_t*>(block)[i] = v;
    }
    // scales [s][half][g][row g, row g + 8], zero points likewise
    for (int i = threadIdx.x; i < a.per_block * kRowTile; i += 256) {
        const int s = i / kRowTile, half = (i >> 4) & 1, g = (i >> 1) & 7, row = row0 + half * 16 + g + 8 * (i & 1);
        const int group = min((k0 + s * (kKBlock / a.per_block)) / a.group, a.groups - 1);
        const int64_t at = static_cast<int64_t>(row) * a.groups + group;
        reinterpret_cast<uint16_t*>(block + kCodeBytes)[i] = row < a.n ? a.scales[at] : 0;
        if (a.zeros) block[kCodeBytes + a.per_block * kRowTile * 2 + i] = row < a.n ? min(static_cast<int>(a.zeros[at]), 15) : 0;
    }
}

// ------------------------------------------------------------------------------------
// product
// ------------------------------------------------------------------------------------
struct LinearArgs {
    const uint8_t* blocks;
    const void* x;
    int64_t x_stride, rows;
    const void* bias;
    void* y;
    int64_t y_stride;
    int32_t n, k, row_tiles, k_blocks, row_blocks, units, share;
    int32_t per_block, block_bytes, stages;
    float* parts;                          // [CTAs][2][256 * kMaxTokens]
    int32_t* counters;                     // [CTAs]
    int64_t wait_budget;
    int32_t* status;
};

template <typename T>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same<T, __half>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <typename T>
__device__ __forceinline__ void mma_from_zero(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same<T, __half>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// (a & mask) | exponent in one operation
__device__ __forceinline__ uint32_t cut(uint32_t a, uint32_t mask, uint32_t exponent)
{
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(a), "r"(mask), "r"(exponent));
    return r;
}

template <typename H2> __device__ __forceinline__ H2 as(uint32_t v) { return *reinterpret_cast<const H2*>(&v); }
template <typename H2> __device__ __forceinline__ uint32_t bits(H2 v) { return *reinterpret_cast<const uint32_t*>(&v); }

// The pairs of columns (0 2), (4 6), (1 3), (5 7) of a word as q - z; `zero`: z (0..15) in both halves.  fp16: 1024 + q - (1024 + z),
// and (1024 + 16 q) / 16 - (64 + z) for the pairs in odd nibbles.  bf16 has no room for the latter: 128 + q - (128 + z) after a shift.
template <typename T>
__device__ __forceinline__ void unpack_codes(uint32_t w, uint32_t zero, uint32_t (&out)[4])
{
    if constexpr (std::is_same<T, __half>::value) {
        const __half2 even = as<__half2>(0x64006400u | zero), odd = as<__half2>(0xd400d400u | (zero << 4));
        const uint32_t v = w >> 8;
        out[0] = bits(__hsub2(as<__half2>(cut(w, 0x000f000fu, 0x64006400u)), even));
        out[1] = bits(__hfma2(as<__half2>(cut(w, 0x00f000f0u, 0x64006400u)), as<__half2>(0x2c002c00u), odd));
        out[2] = bits(__hsub2(as<__half2>(cut(v, 0x000f000fu, 0x64006400u)), even));
        out[3] = bits(__hfma2(as<__half2>(cut(v, 0x00f000f0u, 0x64006400u)), as<__half2>(0x2c002c00u), odd));
    } else {
        const __nv_bfloat162 offset = as<__nv_bfloat162>(0x43004300u | zero);
#pragma unroll
        for (int p = 0; p < 4; ++p) out[p] = bits(__hsub2(as<__nv_bfloat162>(cut(w >> (4 * p), 0x000f000fu, 0x43004300u)), offset));
    }
}

// D = A B + c, the same c everywhere
__device__ __forceinline__ void mma_digits_from(int (&d)[4], const uint32_t (&a)[4], uint2 b, int c)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y), "r"(c));
}

// D (16 x 8, int32) += A (16 x 32, unsigned bytes) B (32 x 8, signed bytes)
__device__ __forceinline__ void mma_digits(int (&d)[4], const uint32_t (&a)[4], uint2 b)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y));
}

__device__ __forceinline__ uint4 lds128(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t addr)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t addr)
{
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr));
    return v;
}

// What both kernels share: a warp's stream of weight blocks, the writing of rows, the joining of parts.  A lane holds eight values
// of each block of eight activation rows: v[j][c] belongs to output row g + 8 (c >> 1) of half j and activation row 2 t4 + (c & 1).
struct Place {                             // a unit: (rows of x, 256 rows of W, 256 columns), the columns fastest
    int kb, rb, pass;
    __device__ __forceinline__ Place(const LinearArgs& a, int unit)
    {
        const int rows = unit / a.k_blocks;
        kb = unit - rows * a.k_blocks;
        pass = rows / a.row_blocks;
        rb = rows - pass * a.row_blocks;
    }
    __device__ __forceinline__ void next(const LinearArgs& a)
    {
        if (++kb < a.k_blocks) return;
        kb = 0;
        if (++rb < a.row_blocks) return;
        rb = 0;
        ++pass;
    }
};

struct Stream {
    const LinearArgs& a;
    uint32_t ring;
    uint64_t* full;                        // [kMaxStages] of this warp
    int u0, u1, warp, lane;
    Place here, ahead;                     // the unit at work; the next to be issued
    int unit, issued, stage;
    uint32_t phase;

    __device__ __forceinline__ Stream(const LinearArgs& args, uint32_t ring_, uint64_t* full_)
        : a(args), ring(ring_), full(full_), u0(min(static_cast<int>(blockIdx.x) * args.share, args.units)), u1(min(u0 + args.share, args.units)),
          warp(threadIdx.x >> 5), lane(threadIdx.x & 31), here(args, u0), ahead(here), unit(u0), issued(0), stage(0), phase(0)
    {
    }
    __device__ __forceinline__ void start()
    {
        for (int i = 0; i < min(a.stages, u1 - u0); ++i) issue(i);
    }
    __device__ __forceinline__ int tile(const Place& p) const { return p.rb * kWarps + warp; }
    __device__ __forceinline__ bool has_rows() const { return tile(here) < a.row_tiles; }
    __device__ __forceinline__ bool ends() const { return here.kb == a.k_blocks - 1; }
    __device__ __forceinline__ bool finishes() const { return ends() || unit == u1 - 1; }
    __device__ __forceinline__ void issue(int to)
    {
        if (lane == 0) {
            const uint32_t bar = smem_u32(&full[to]);
            if (tile(ahead) >= a.row_tiles) {          // no rows for this warp
                mbar_arrive(bar);
            } else {
                mbar_arrive_expect_tx(bar, a.block_bytes);
                bulk_load(ring + to * a.block_bytes, a.blocks + (static_cast<int64_t>(tile(ahead)) * a.k_blocks + ahead.kb) * a.block_bytes, a.block_bytes, bar);
            }
        }
        ahead.next(a);
        ++issued;
    }
    // After a wait that gave up nothing more is issued, but what is in flight is still waited for (with the same limit).
    __device__ __forceinline__ bool wait() const
    {
        return unit - u0 >= issued || __all_sync(0xffffffffu, mbar_wait(smem_u32(&full[stage]), phase, a.wait_budget));
    }
    __device__ __forceinline__ uint32_t block() const { return ring + stage * a.block_bytes; }
    __device__ __forceinline__ void release(bool ok)
    {
        __syncwarp();                                  // every lane has read the stage
        if (ok && issued < u1 - u0) issue(stage);
        if (++stage == a.stages) {
            stage = 0;
            phase ^= 1;
        }
    }
    __device__ __forceinline__ void next()
    {
        here.next(a);
        ++unit;
    }
};

__device__ __forceinline__ void timed_out(const LinearArgs& a)
{
    if ((threadIdx.x & 31) == 0 && atomicCAS(a.status, 0, QTZ_ERR_DEVICE_TIMEOUT) == 0) a.status[1] = QTZ_SITE_LINEAR;
}

// Rows of y of the warp's tile; `rows` of them at most (an activation block may be narrower than eight).
template <typename T, int kNt>
__device__ __forceinline__ void write_rows(const LinearArgs& a, const Stream& s, const Place& at, const float (&v)[2][kNt][4], int rows)
{
    const int t4 = s.lane & 3, o0 = s.tile(at) * kRowTile + (s.lane >> 2);
    const int64_t r0 = static_cast<int64_t>(at.pass) * (8 * kNt) + 2 * t4;
    if (2 * t4 >= rows) return;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
            const int o = o0 + 16 * j + 8 * hi;
            if (o >= a.n) continue;
            const float b = a.bias ? qtz_dev::to_f32(static_cast<const T*>(a.bias)[o]) : 0.f;
#pragma unroll
            for (int nt = 0; nt < kNt; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int64_t r = r0 + 8 * nt + c;
                    if (r < a.rows) static_cast<T*>(a.y)[r * a.y_stride + o] = qtz_dev::from_f32<T>(v[j][nt][2 * hi + c] + b);
                }
        }
}

// Where the parts of a warp lie: slot 0, rows that began in an earlier CTA; slot 1, rows that go on in a later one.
template <int kNt>
__device__ __forceinline__ float* part_of(const LinearArgs& a, const Stream& s, int cta, int slot)
{
    return a.parts + ((static_cast<int64_t>(cta) * 2 + slot) * kWarps + s.warp) * (kRowTile * 8 * kNt) + s.lane;
}

// The end of a row block, or of this CTA's columns of it: y, or a part.
template <typename T, int kNt>
__device__ __forceinline__ void finish_rows(const LinearArgs& a, const Stream& s, const float (&v)[2][kNt][4], int rows, int (&open)[2])
{
    const bool begins = s.unit - s.here.kb >= s.u0;
    if (begins && s.ends()) {
        if (s.has_rows()) write_rows<T, kNt>(a, s, s.here, v, rows);
        return;
    }
    if (begins) open[1] = s.unit;
    else open[0] = s.unit;
    float* part = part_of<kNt>(a, s, blockIdx.x, begins ? 1 : 0);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int nt = 0; nt < kNt; ++nt)
#pragma unroll
            for (int c = 0; c < 4; ++c) part[((j * kNt + nt) * 4 + c) * 32] = v[j][nt][c];
}

// Rows whose columns lie in several CTAs, c0 .. c1: the last to arrive joins their parts in order.
template <typename T, int kNt>
__device__ __forceinline__ void join_rows(const LinearArgs& a, const Stream& s, const int (&open)[2], int rows, const int& failed, int (&last)[2])
{
    if (open[0] < 0 && open[1] < 0) return;            // the same for all warps
    __threadfence();
    __syncthreads();
    if (failed) return;                                // the results are void, and the counters have to be cleared
    const Place at[2] = {Place(a, max(open[0], 0)), Place(a, max(open[1], 0))};
    const int c0[2] = {(open[0] - at[0].kb) / a.share, (open[1] - at[1].kb) / a.share};
    const int c1[2] = {(open[0] - at[0].kb + a.k_blocks - 1) / a.share, (open[1] - at[1].kb + a.k_blocks - 1) / a.share};
#pragma unroll
    for (int which = 0; which < 2; ++which)
        if (threadIdx.x == 32 * which && open[which] >= 0) {
            last[which] = atomicAdd(a.counters + c0[which], 1) == c1[which] - c0[which];
            if (last[which]) a.counters[c0[which]] = 0;    // ready for the next call
        }
    __syncthreads();
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (open[which] < 0 || !last[which] || s.tile(at[which]) >= a.row_tiles) continue;
        __threadfence();
        constexpr int kFlight = kNt == 1 ? 8 : kNt == 2 ? 4 : 2;       // parts in flight: what the registers hold
        float v[2][kNt][4] = {};
        for (int c = c0[which]; c <= c1[which]; c += kFlight) {
            float p[kFlight][2][kNt][4];
#pragma unroll
            for (int x = 0; x < kFlight; ++x) {
                const float* part = part_of<kNt>(a, s, min(c + x, c1[which]), c + x == c0[which] ? 1 : 0);
#pragma unroll
                for (int i = 0; i < 8 * kNt; ++i) (&p[x][0][0][0])[i] = __ldcg(part + i * 32);
            }
#pragma unroll
            for (int x = 0; x < kFlight; ++x)
#pragma unroll
                for (int i = 0; i < 8 * kNt; ++i) (&v[0][0][0])[i] += c + x <= c1[which] ? (&p[x][0][0][0])[i] : 0.f;
        }
        write_rows<T, kNt>(a, s, at[which], v, rows);
    }
}

// ---- up to eight rows: digits of x, integer matrix instructions ----
constexpr int kDigitBuffers = 3;           // units whose digits are held: the one at work, the next, the one before
constexpr int kDigitPitch = kKBlock + 32;  // bytes of an operand column: the lanes of a load meet all banks

template <int kTiles>
struct Digits {                            // of the rows' columns in one unit
    uint8_t operand[8 * kTiles][kDigitPitch];
    float factor[8 * kTiles];              // of a column's digit: a power of two, 0 for a column that holds none
    float sum[8][8 * kTiles];              // per scale of the unit: the sum of x over its columns, at the row's highest digit
};

// Row r's digit d is operand column: 1 tile (2 rows) 2 d + r; 2 tiles (4 rows) digits 2 i + j at tile i, column 4 j + r; 3 tiles
// (8 rows) tile d, column r.  A lane so holds a row's digits itself or shares them with the lanes of its quad.
template <int kTiles>
__device__ __forceinline__ int digit_column(int d, int r)
{
    return kTiles == 1 ? 2 * d + r : kTiles == 2 ? (d >> 1) * 8 + (d & 1) * 4 + r : d * 8 + r;
}

// kSteps: steps of 32 columns to a scale (1, 2 or 4)
template <typename T, int kTiles, int kSteps, bool kZero>
__global__ void __launch_bounds__(kThreads, 2)
linear_digits_kernel(const __grid_constant__ LinearArgs a)
{
    constexpr int kRows = kTiles == 3 ? 8 : 2 * kTiles;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t s_full[kWarps][kMaxStages], s_ready[kDigitBuffers], s_free[kDigitBuffers];
    __shared__ int s_last[2], s_failed;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3, rows = static_cast<int>(a.rows);
    Digits<kTiles>* const digits = reinterpret_cast<Digits<kTiles>*>(smem);
    if (lane < kMaxStages) mbar_init(smem_u32(&s_full[warp][lane]), 1);
    if (tid == 0) {
        s_failed = 0;
        for (int i = 0; i < kDigitBuffers; ++i) {
            mbar_init(smem_u32(&s_ready[i]), rows);
            mbar_init(smem_u32(&s_free[i]), kWarps);
        }
    }
    for (int i = tid; i < kDigitBuffers * 8 * kTiles; i += kThreads) {   // columns that hold no digit count nothing
        Digits<kTiles>& d = digits[i / (8 * kTiles)];
        d.factor[i % (8 * kTiles)] = 0.f;
        for (int k = 0; k < 8; ++k) d.sum[k][i % (8 * kTiles)] = 0.f;
    }
    fence_barrier_init();
    __syncthreads();
    Stream s(a, smem_u32(smem) + kDigitBuffers * static_cast<uint32_t>(sizeof(Digits<kTiles>)) + warp * a.stages * a.block_bytes, s_full[warp]);
    grid_launch_dependents();
    s.start();                                         // the weights were there when the layer was made; all else is waited for
    grid_dependency_wait();
    bool ok = true;

    // Rows of x become digits one unit ahead; row r of the CTA's unit i is the work of warp (i + r) % 8.  `buffer` and `round`: i
    // modulo and divided by the number of buffers.
    auto convert = [&](int i, int kb, int buffer, int round) {
        Digits<kTiles>& to = digits[buffer];
        const int r = (warp - i) & (kWarps - 1);
        if (r < rows) {
            const uint16_t* x = static_cast<const uint16_t*>(a.x) + r * a.x_stride + kb * kKBlock + 8 * lane;
            const int have = a.k - kb * kKBlock - 8 * lane;
            uint4 raw = make_uint4(0, 0, 0, 0);
            if (have > 0) raw = __ldg(reinterpret_cast<const uint4*>(x));
            const uint32_t words[4] = {raw.x, raw.y, raw.z, raw.w};
            float v[8], top = 0.f;
            bool odd = false;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 f = qtz_dev::unpack2(words[k], T());
                v[2 * k] = 2 * k < have ? f.x : 0.f;   // what lies behind the last column is not data
                v[2 * k + 1] = 2 * k + 1 < have ? f.y : 0.f;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                odd = odd || (__float_as_uint(v[k]) & 0x7f800000u) == 0x7f800000u;
                top = fmaxf(top, fabsf(v[k]));
            }
            top = redux_max(top);
            odd = __any_sync(0xffffffffu, odd);
            const int ex = min(max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -100), 127);
            const float mult = __uint_as_float(static_cast<uint32_t>(127 + 21 - ex) << 23);
            uint64_t d[3] = {0, 0, 0};
            int sum = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int q = odd ? 0 : __float2int_rn(v[k] * mult);
                const int d0 = (q << 24) >> 24, q1 = (q - d0) >> 8, d1 = (q1 << 24) >> 24, d2 = (q1 - d1) >> 8;
                sum += q;
                d[0] |= static_cast<uint64_t>(d0 & 0xff) << (8 * k);
                d[1] |= static_cast<uint64_t>(d1 & 0xff) << (8 * k);
                d[2] |= static_cast<uint64_t>(d2 & 0xff) << (8 * k);
            }
            if (round > 0)                             // the buffer's unit before has been used by all warps
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&s_free[buffer]), (round - 1) & 1, a.wait_budget)) && ok;
#pragma unroll
            for (int j = 0; j < 3; ++j) *reinterpret_cast<uint64_t*>(&to.operand[digit_column<kTiles>(j, r)][8 * lane]) = d[j];
            // the sum of a scale's columns: |sum| < 2^22 * 128 fits
            constexpr int kLanes = 4 * kSteps;
#pragma unroll
            for (int off = 1; off < kLanes; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            // a row that holds NaN or infinity gives NaN
            const float unit_of = odd ? __uint_as_float(0x7fc00000u) : __uint_as_float(static_cast<uint32_t>(127 - 21 + ex) << 23);
            const float minus = kZero ? -1.f : -8.f;
            if (lane % kLanes == 0)
                to.sum[lane / kLanes][digit_column<kTiles>(2, r)] = static_cast<float>(sum) * unit_of * minus;
            if (lane < 3) to.factor[digit_column<kTiles>(lane, r)] = unit_of * (lane == 0 ? 1.f : lane == 1 ? 256.f : 65536.f);
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&s_ready[buffer]));
        }
    };

    float acc[2][kTiles][4] = {};
    int open[2] = {-1, -1};                            // units whose rows are shared with an earlier / a later CTA
    if (s.u0 < s.u1) convert(0, s.here.kb, 0, 0);
    int buffer = 0, round = 0, buffer_next = 1 % kDigitBuffers, round_next = 0;
    for (; s.unit < s.u1; s.next()) {
        if (s.unit + 1 < s.u1) convert(s.unit + 1 - s.u0, s.ends() ? 0 : s.here.kb + 1, buffer_next, round_next);
        ok = s.wait() && ok;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&s_ready[buffer]), round & 1, a.wait_budget)) && ok;
        if (ok && s.has_rows()) {
            const uint32_t block = s.block(), scales = block + kCodeBytes, zeros = scales + 8 / kSteps * kRowTile * 2;
            const Digits<kTiles>& dg = digits[buffer];
            const uint32_t operand = smem_u32(&dg.operand[g][8 * t4]);
            int part[2][kTiles][4];
#pragma unroll
            for (int chunk = 0; chunk < 4; ++chunk) {
                uint4 q[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) q[j] = lds128(block + (chunk * 2 + j) * 512 + lane * 16);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    constexpr int kMagic = 0x4b400000; // 1.5 * 2^23: an integer sum in the mantissa
                    const int step = 2 * chunk + h;
                    uint32_t op[2][4];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t lo = h ? q[j].z : q[j].x, hi = h ? q[j].w : q[j].y;     // rows g, g + 8
                        op[j][0] = lo & 0x0f0f0f0fu;
                        op[j][1] = hi & 0x0f0f0f0fu;
                        op[j][2] = (lo >> 4) & 0x0f0f0f0fu;
                        op[j][3] = (hi >> 4) & 0x0f0f0f0fu;
                    }
#pragma unroll
                    for (int nt = 0; nt < kTiles; ++nt) {
                        const uint2 b = lds64(operand + nt * 8 * kDigitPitch + step * 32);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            if (step % kSteps == 0) mma_digits_from(part[j][nt], op[j], b, kMagic);
                            else mma_digits(part[j][nt], op[j], b);
                        }
                    }
                    if ((step + 1) % kSteps == 0) {    // the sums of one scale
                        const int si = step / kSteps;
                        float sc[2][2], z[2][2];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int at = (si * 2 + j) * 8 + g;
                            const float2 f = qtz_dev::unpack2(lds32(scales + 4 * at), T());
                            sc[j][0] = f.x;
                            sc[j][1] = f.y;
                            if (kZero) {               // 2^23 + z - 2^23
                                const uint32_t zz = lds16(zeros + 2 * at);
                                z[j][0] = __uint_as_float(__byte_perm(zz, 0x4b000000u, 0x7550)) - 8388608.f;
                                z[j][1] = __uint_as_float(__byte_perm(zz, 0x4b000000u, 0x7551)) - 8388608.f;
                            }
                        }
#pragma unroll
                        for (int nt = 0; nt < kTiles; ++nt) {
                            const float2 f = *reinterpret_cast<const float2*>(&dg.factor[nt * 8 + 2 * t4]), xs = *reinterpret_cast<const float2*>(&dg.sum[si][nt * 8 + 2 * t4]);
#pragma unroll
                            for (int j = 0; j < 2; ++j)
#pragma unroll
                                for (int c = 0; c < 4; ++c) {
                                    const float p = __int_as_float(part[j][nt][c]) - 12582912.f, xc = c & 1 ? xs.y : xs.x;
                                    const float v = fmaf(p, c & 1 ? f.y : f.x, kZero ? z[j][c >> 1] * xc : xc);
                                    acc[j][nt][c] = fmaf(v, sc[j][c >> 1], acc[j][nt][c]);
                                }
                        }
                    }
                }
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_free[buffer]));
        s.release(ok);
        buffer = buffer_next;
        round = round_next;
        if (++buffer_next == kDigitBuffers) {
            buffer_next = 0;
            ++round_next;
        }
        if (s.finishes()) {
            float v[2][1][4];                          // the digits of a row together
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float t = acc[j][0][c];
                    if (kTiles > 1) t += acc[j][1 % kTiles][c];
                    if (kTiles > 2) t += acc[j][2 % kTiles][c];
                    if (kTiles == 1) t += __shfl_xor_sync(0xffffffffu, t, 1);
                    if (kTiles < 3) t += __shfl_xor_sync(0xffffffffu, t, 2);
                    v[j][0][c] = t;
#pragma unroll
                    for (int nt = 0; nt < kTiles; ++nt) acc[j][nt][c] = 0.f;
                }
            finish_rows<T, 1>(a, s, v, kRows, open);
        }
    }
    if (!ok) {
        timed_out(a);
        s_failed = 1;
    }
    join_rows<T, 1>(a, s, open, kRows, s_failed, s_last);
}

// ---- more rows: 16-bit matrix instructions; kNt: blocks of eight rows; kSteps: steps of 32 columns to a scale (1, 2 or 4) ----
constexpr int kRowPitch = 2 * kKBlock + 64;            // bytes of a row of x in shared memory: the lanes of a load meet all banks

template <typename T, int kNt, int kSteps, bool kZero>
__global__ void __launch_bounds__(kThreads, 2)
linear_wide_kernel(const __grid_constant__ LinearArgs a)
{
    extern __shared__ __align__(128) uint8_t smem[];   // two units of x, the rings
    __shared__ __align__(8) uint64_t s_full[kWarps][kMaxStages];
    __shared__ int s_last[2], s_failed;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
    if (lane < kMaxStages) mbar_init(smem_u32(&s_full[warp][lane]), 1);
    if (tid == 0) s_failed = 0;
    fence_barrier_init();
    __syncthreads();
    Stream s(a, smem_u32(smem) + 2 * 8 * kNt * kRowPitch + warp * a.stages * a.block_bytes, s_full[warp]);

    grid_launch_dependents();
    s.start();                                         // the weights were there when the layer was made; all else is waited for
    grid_dependency_wait();

    // x of a unit: thread i takes eight columns (i % 32) of rows i / 32, + 8, ..; in the order of the operand (0 2, 4 6, 1 3, 5 7)
    uint4 held[kNt];
    auto fetch = [&](const Place& at) {
        const int have = a.k - at.kb * kKBlock - 8 * lane;
        const int64_t r0 = static_cast<int64_t>(at.pass) * (8 * kNt) + warp;
#pragma unroll
        for (int nt = 0; nt < kNt; ++nt) {
            held[nt] = make_uint4(0, 0, 0, 0);
            if (r0 + 8 * nt < a.rows && have > 0)
                held[nt] = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.x) + (r0 + 8 * nt) * a.x_stride + at.kb * kKBlock + 8 * lane));
        }
    };
    auto store = [&](const Place& at, int buffer) {
        const int have = a.k - at.kb * kKBlock - 8 * lane;
#pragma unroll
        for (int nt = 0; nt < kNt; ++nt) {
            uint32_t w[4] = {held[nt].x, held[nt].y, held[nt].z, held[nt].w};
            if (have > 0 && have < 8)                  // the last columns: what lies behind them is not data
#pragma unroll
                for (int c = 0; c < 4; ++c) w[c] = have >= 2 * c + 2 ? w[c] : have == 2 * c + 1 ? w[c] & 0xffffu : 0u;
            *reinterpret_cast<uint4*>(smem + buffer * (8 * kNt * kRowPitch) + (8 * nt + warp) * kRowPitch + lane * 16) =
                make_uint4(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410), __byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632));
        }
    };

    float acc[2][kNt][4] = {};
    int open[2] = {-1, -1};
    bool ok = true;
    if (s.u0 < s.u1) {
        fetch(s.here);
        store(s.here, 0);
        __syncthreads();
    }
    int buffer = 0;
    for (; s.unit < s.u1; s.next(), buffer ^= 1) {
        Place after = s.here;
        after.next(a);
        if (s.unit + 1 < s.u1) fetch(after);
        ok = s.wait() && ok;
        if (ok && s.has_rows()) {
            const uint32_t block = s.block(), scales = block + kCodeBytes, zeros = scales + 8 / kSteps * kRowTile * 2;
            const uint32_t x = smem_u32(smem) + buffer * (8 * kNt * kRowPitch) + g * kRowPitch + t4 * 16;
            float part[2][kNt][4];
#pragma unroll 1
            for (int pair = 0; pair < 2; ++pair) {     // 128 columns
                float sc[2][2];
                uint32_t z[2] = {0x0808u, 0x0808u};
                uint4 q[2];
#pragma unroll
                for (int i = 0; i < 4; ++i) {          // 32 columns
                    const int step = 4 * pair + i;
                    if (i % kSteps == 0)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int at = (step / kSteps * 2 + j) * 8 + g;
                            const float2 f = qtz_dev::unpack2(lds32(scales + 4 * at), T());
                            sc[j][0] = f.x;
                            sc[j][1] = f.y;
                            if (kZero) z[j] = lds16(zeros + 2 * at);
                        }
                    uint32_t w[2][2][4];               // [half of the rows][row g, g + 8][pair]
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (i % 2 == 0) q[j] = lds128(block + (step / 2 * 2 + j) * 512 + lane * 16);
                        unpack_codes<T>(i % 2 ? q[j].z : q[j].x, (z[j] & 0xffu) * 0x00010001u, w[j][0]);
                        unpack_codes<T>(i % 2 ? q[j].w : q[j].y, (z[j] >> 8) * 0x00010001u, w[j][1]);
                    }
                    uint4 b[kNt];
#pragma unroll
                    for (int nt = 0; nt < kNt; ++nt) b[nt] = lds128(x + nt * 8 * kRowPitch + step * 64);
                    // neighbouring instructions write different sums
#pragma unroll
                    for (int nt = 0; nt < kNt; ++nt)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const uint32_t op[4] = {w[j][0][0], w[j][1][0], w[j][0][1], w[j][1][1]};
                            if (i % kSteps == 0) mma_from_zero<T>(part[j][nt], op, b[nt].x, b[nt].y);
                            else mma<T>(part[j][nt], op, b[nt].x, b[nt].y);
                        }
#pragma unroll
                    for (int nt = 0; nt < kNt; ++nt)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const uint32_t op[4] = {w[j][0][2], w[j][1][2], w[j][0][3], w[j][1][3]};
                            mma<T>(part[j][nt], op, b[nt].z, b[nt].w);
                        }
                    if ((i + 1) % kSteps == 0)
#pragma unroll
                        for (int nt = 0; nt < kNt; ++nt)
#pragma unroll
                            for (int j = 0; j < 2; ++j)
#pragma unroll
                                for (int c = 0; c < 4; ++c) acc[j][nt][c] = fmaf(part[j][nt][c], sc[j][c >> 1], acc[j][nt][c]);
                }
            }
        }
        s.release(ok);
        if (s.unit + 1 < s.u1) store(after, buffer ^ 1);
        __syncthreads();                               // the next unit's x is there, this one's is free
        if (s.finishes()) {
            finish_rows<T, kNt>(a, s, acc, 8, open);
#pragma unroll
            for (int i = 0; i < 8 * kNt; ++i) (&acc[0][0][0])[i] = 0.f;
        }
    }
    if (!ok) {
        timed_out(a);
        s_failed = 1;
    }
    join_rows<T, kNt>(a, s, open, 8, s_failed, s_last);
}

// fixed: shared memory beside the rings; kParts: the most parts that a row block is cut into
template <typename K>
qtz_status launch(qtz_linear* p, LinearArgs& a, K kernel, int fixed, int most_parts, cudaStream_t st)
{
    qtz_ctx* h = p->h;
    const int room = (kSmemLimit + 1024) / 2 - 1024 - 1024 - fixed;    // two CTAs an SM; 1 KB: the kernels' static shared memory
    a.stages = room / (kWarps * p->block_bytes);
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    const int smem = fixed + kWarps * a.stages * p->block_bytes, grid = 2 * h->num_sms;
    // A share takes in at least 1 / most_parts of the columns: joining costs more than it brings beyond that.
    a.share = (a.units + grid - 1) / grid;
    if (a.share < (a.k_blocks + most_parts - 1) / most_parts) a.share = (a.k_blocks + most_parts - 1) / most_parts;
    const qtz_status s = qtz_allow_smem(h, kernel);
    if (s != QTZ_OK) return s;
    QTZ_CUDA(h, qtz_launch_dependent(kernel, dim3((a.units + a.share - 1) / a.share), kThreads, smem, st, a));
    return QTZ_OK;
}

template <typename T, int kTiles>
qtz_status launch_digits(qtz_linear* p, LinearArgs& a, bool zero, cudaStream_t st)
{
    constexpr int kFixed = kDigitBuffers * sizeof(Digits<kTiles>);
    if (p->scales == 8)
        return zero ? launch(p, a, linear_digits_kernel<T, kTiles, 1, true>, kFixed, 32, st) : launch(p, a, linear_digits_kernel<T, kTiles, 1, false>, kFixed, 32, st);
    if (p->scales == 4)
        return zero ? launch(p, a, linear_digits_kernel<T, kTiles, 2, true>, kFixed, 32, st) : launch(p, a, linear_digits_kernel<T, kTiles, 2, false>, kFixed, 32, st);
    return zero ? launch(p, a, linear_digits_kernel<T, kTiles, 4, true>, kFixed, 32, st) : launch(p, a, linear_digits_kernel<T, kTiles, 4, false>, kFixed, 32, st);
}

template <typename T, int kNt>
qtz_status launch_wide(qtz_linear* p, LinearArgs& a, bool zero, cudaStream_t st)
{
    constexpr int kFixed = 2 * 8 * kNt * kRowPitch;
    if (p->scales == 8)
        return zero ? launch(p, a, linear_wide_kernel<T, kNt, 1, true>, kFixed, 8, st) : launch(p, a, linear_wide_kernel<T, kNt, 1, false>, kFixed, 8, st);
    if (p->scales == 4)
        return zero ? launch(p, a, linear_wide_kernel<T, kNt, 2, true>, kFixed, 8, st) : launch(p, a, linear_wide_kernel<T, kNt, 2, false>, kFixed, 8, st);
    return zero ? launch(p, a, linear_wide_kernel<T, kNt, 4, true>, kFixed, 8, st) : launch(p, a, linear_wide_kernel<T, kNt, 4, false>, kFixed, 8, st);
}

template <typename T>
qtz_status launch_rows(qtz_linear* p, LinearArgs& a, bool zero, cudaStream_t st)
{
    if (a.rows <= 2) return launch_digits<T, 1>(p, a, zero, st);
    if (a.rows <= 4) return launch_digits<T, 2>(p, a, zero, st);
    if (a.rows <= 8) return launch_digits<T, 3>(p, a, zero, st);
    if (a.rows <= 16) return launch_wide<T, 2>(p, a, zero, st);
    return launch_wide<T, 4>(p, a, zero, st);
}

// Scratch of the joining, shared by the layers of a handle: parts and counters of a full grid.
qtz_status ensure_scratch(qtz_ctx* h, cudaStream_t st)
{
    if (h->linear_dev) return QTZ_OK;
    const int ctas = 2 * h->num_sms;
    const size_t parts = static_cast<size_t>(ctas) * 2 * kWarps * kRowTile * kMaxTokens * sizeof(float);
    QTZ_CUDA(h, cudaMalloc(&h->linear_dev, parts + ctas * sizeof(int32_t)));
    QTZ_CUDA(h, cudaMemsetAsync(static_cast<uint8_t*>(h->linear_dev) + parts, 0, ctas * sizeof(int32_t), st));
    h->linear_counters = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(h->linear_dev) + parts);
    return QTZ_OK;
}

}  // namespace

extern "C" qtz_status qtz_linear_destroy(qtz_linear_plan p)
{
    if (!p) return QTZ_ERR_INVALID_ARG;
    qtz_device_guard guard(p->h->device);
    if (p->blocks) cudaFree(p->blocks);
    (void)cudaGetLastError();
    delete p;
    return QTZ_OK;
}

extern "C" qtz_status qtz_linear_create(qtz_handle h, const qtz_linear_desc* desc, const void* codes_dev, const void* scales_dev,
                                        const uint8_t* zeros_dev, const void* bias_dev, qtz_linear_plan* out, void* stream)
{
    if (!h || !desc || !codes_dev || !scales_dev || !out) return QTZ_ERR_INVALID_ARG;
    *out = nullptr;
    const qtz_linear_desc& d = *desc;
    if (d.n <= 0 || d.k <= 0 || d.group <= 0) return QTZ_ERR_INVALID_ARG;
    if (d.wdtype != QTZ_S4_PACKED && d.wdtype != QTZ_U4_PACKED) return QTZ_ERR_INVALID_ARG;
    if (d.ftype != QTZ_F16 && d.ftype != QTZ_BF16) return QTZ_ERR_INVALID_ARG;
    if (d.wdtype == QTZ_S4_PACKED && zeros_dev) return QTZ_ERR_INVALID_ARG;
    if (d.group != 32 && d.group % 64 != 0) return QTZ_ERR_UNSUPPORTED;
    const int64_t row_tiles = (static_cast<int64_t>(d.n) + kRowTile - 1) / kRowTile, k_blocks = (static_cast<int64_t>(d.k) + kKBlock - 1) / kKBlock;
    if (row_tiles * k_blocks > (1 << 28) || row_tiles > 65535) return QTZ_ERR_TOO_LARGE;
    qtz_device_guard guard(h->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    qtz_status s = ensure_scratch(h, st);
    if (s != QTZ_OK) return s;
    qtz_linear* p = new (std::nothrow) qtz_linear();
    if (!p) return QTZ_ERR_INVALID_ARG;
    p->h = h;
    p->d = d;
    p->row_tiles = static_cast<int>(row_tiles);
    p->k_blocks = static_cast<int>(k_blocks);
    p->scales = d.group == 32 ? 8 : d.group % 128 == 0 ? 2 : 4;
    // unsigned codes without zero points are codes with zero points 0: the kernel's constant stands for 8
    const bool zero = d.wdtype == QTZ_U4_PACKED;
    p->block_bytes = kCodeBytes + p->scales * kRowTile * (zero ? 3 : 2);
    const size_t blocks = static_cast<size_t>(row_tiles) * k_blocks * p->block_bytes, groups = (static_cast<size_t>(d.k) + d.group - 1) / d.group;
    uint8_t* no_zeros = nullptr;
    cudaError_t e = cudaMalloc(reinterpret_cast<void**>(&p->blocks), blocks + 2 * static_cast<size_t>(d.n) + (zero && !zeros_dev ? groups * d.n : 0));
    if (e == cudaSuccess && zero && !zeros_dev) {
        no_zeros = p->blocks + blocks + 2 * static_cast<size_t>(d.n);
        e = cudaMemsetAsync(no_zeros, 0, groups * d.n, st);
    }
    if (e == cudaSuccess && bias_dev) {
        p->bias = p->blocks + blocks;
        e = cudaMemcpyAsync(p->bias, bias_dev, 2 * static_cast<size_t>(d.n), cudaMemcpyDeviceToDevice, st);
    }
    if (e == cudaSuccess) {
        const PackArgs a{static_cast<const uint8_t*>(codes_dev), static_cast<const uint16_t*>(scales_dev), zeros_dev ? zeros_dev : no_zeros, d.n, d.k, d.group,
                         static_cast<int>(groups), p->k_blocks, p->scales, p->block_bytes, d.wdtype == QTZ_S4_PACKED, p->blocks};
        pack_kernel<<<dim3(static_cast<unsigned>(k_blocks), static_cast<unsigned>(row_tiles)), 256, 0, st>>>(a);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);   // later calls may fetch the blocks before they wait for the stream
    if (e != cudaSuccess) {
        qtz_cuda_fail(h, e, "qtz_linear_create");
        qtz_linear_destroy(p);
        return QTZ_ERR_CUDA;
    }
    *out = p;
    return QTZ_OK;
}

extern "C" qtz_status qtz_linear_w4(qtz_linear_plan p, const void* x_dev, int64_t x_stride, int64_t rows, void* y_dev,
                                    int64_t y_stride, void* stream)
{
    if (!p || rows < 0) return QTZ_ERR_INVALID_ARG;
    if (rows == 0) return QTZ_OK;
    if (!x_dev || !y_dev || x_stride < p->d.k || y_stride < p->d.n) return QTZ_ERR_INVALID_ARG;
    if (!qtz_aligned16(x_dev) || x_stride % 8 != 0) return QTZ_ERR_MISALIGNED;
    const int row_blocks = (p->row_tiles + kWarps - 1) / kWarps;
    const int64_t passes = rows <= kMaxTokens ? 1 : (rows + kMaxTokens - 1) / kMaxTokens;
    if (passes * row_blocks * p->k_blocks > 0x3fffffff) return QTZ_ERR_TOO_LARGE;
    qtz_device_guard guard(p->h->device);
    LinearArgs a{p->blocks, x_dev, x_stride, rows, p->bias, y_dev, y_stride, p->d.n, p->d.k, p->row_tiles, p->k_blocks, row_blocks,
                 static_cast<int32_t>(passes * row_blocks * p->k_blocks), 0, p->scales, p->block_bytes, 0, static_cast<float*>(p->h->linear_dev),
                 p->h->linear_counters, p->h->wait_budget, p->h->status_dev};
    const bool zero = p->d.wdtype == QTZ_U4_PACKED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (p->d.ftype == QTZ_F16) return launch_rows<__half>(p, a, zero, st);
    return launch_rows<__nv_bfloat16>(p, a, zero, st);
}

// Linear layers with 4-bit weights and group scales on few rows of real activations (decoding).
//
// Mathematics.  y[r][o] = sum_g s[o][g] sum_{k in g} (q[o][k] - z[o][g]) x[r][k] + b[o].
//   up to 4 rows   The codes meet the integer matrix instructions (m16n8k32) as they are: eight are cut from a word by three logic
//                  operations.  Each row's 256 columns at hand are written as 2^(e - 29) (d_3 2^24 + d_2 2^16 + d_1 2^8 + d_0), e
//                  the exponent of their largest value, d in [-128, 127], one operand column for each digit: 30 bits below that
//                  value, so that fp16 and bf16 values are exact down to 2^-19 and 2^-22 of it, and what smaller ones lose is 2^-29 of it
//                  at most.  (22 bits were not enough: where a strong value meets a weight of zero, the others are all that
//                  counts.)  Integer sums are exact, the zero point's part (through the sums of the digits over the group) among
//                  them; scale and digit weight multiply them in fp32.  Rows with infinities or NaN have no digits and are summed
//                  from the formula in fp32.
//   more rows      fp16 / bf16 tensor cores (tcgen05) with q - z as an exact operand: two codes are cut from a word by one logic
//                  operation that also writes the exponent (1024 + q in fp16, 128 + q in bf16), one packed operation takes the
//                  offset off, and the operand goes to tensor memory without touching shared memory; the scale multiplies the fp32
//                  sum of its group, or of the 128 columns of it that are at hand.
// Nothing is rounded to 16 bits before y.
//
// What bounds it: half a byte of weight is read for 2 flops an activation row.  At the measured copy rate that is 46 weights a clock
// and SM, for which the SM issues 2.8 operations a weight: the first form needs about 1.3 for one row (its matrix instructions, 2048
// products a clock, take 128 weights a clock with four rows), the second less than 2 with 32 rows, by the source.
// The weights are read once, in the order of use, as contiguous blocks of 32 rows x 256 columns with their scales and zero points
// behind the codes; every warp streams its blocks through a ring of its own (bulk copies, several blocks ahead).  Activations are
// few: the eight warps of a CTA work on the same columns of 256 rows and share them in shared memory.
// Measured: one row through 32768 x 8192 27.1 us, 5.2 TB/s of weights, 0.81 of the copy rate; four through 28672 x 8192 31.6 us, where the
// fp32 work for each scale grows with the digit columns; 32 rows through 28672 x 8192 41.8 us, 2.9 TB/s and 0.36 PFLOP/s, the issue slots
// 64 % busy and the tensor pipe 17 %: 3.7 operations a weight are issued, about half of them polls, because a thread waits for each 16
// sums of a product right after it has asked for them and holds too many (32) to have others under way; one row through 1000 x 1024
// 4.7 us, where 2 are the launch.
// The (256 rows, 256 columns) units form one sequence that is dealt out in equal contiguous shares to a grid that fills the GPU
// once; rows whose columns lie in several CTAs are joined by the last of those to arrive, in the order of the columns.
#include <new>
#include <type_traits>

#include "qtz_half_util.cuh"
#include "qtz_internal.cuh"
#include "qtz_plan.cuh"
#include "qtz_ptx.cuh"

struct qtz_linear {
    qtz_ctx* h = nullptr;
    int device = 0;                    // a plan may be destroyed after its handle
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
// the order in which the lanes of a matrix instruction hold their operand: the low nibbles of the four bytes are columns 4 t + 0, 2, 1, 3
// of the 32 at hand (t: the lane's place in its quad), the high ones 16 + 4 t + 0, 2, 1, 3.
__global__ void __launch_bounds__(256)
pack_kernel(PackArgs a)
{
    uint8_t* block = a.out + (static_cast<int64_t>(blockIdx.y) * a.k_blocks + blockIdx.x) * a.block_bytes;
    const int row0 = blockIdx.y * kRowTile, k0 = blockIdx.x * kKBlock;
    for (int i = threadIdx.x; i < kCodeBytes / 4; i += 256) {
        const int w = i & 3, lane = (i >> 2) & 31, half = (i >> 7) & 1, chunk = i >> 8;
        const int row = row0 + half * 16 + (lane >> 2) + 8 * (w & 1), k = k0 + chunk * 64 + (w >> 1) * 32 + 4 * (lane & 3);
        uint32_t v = 0;
        for (int nibble = 0; nibble < 8; ++nibble) {
            const int m = nibble >> 1, c = k + 16 * (nibble & 1) + (m == 1 ? 2 : m == 2 ? 1 : m);
            uint32_t q = a.is_signed ? 8 : 0;          // beyond the matrix: the code of zero
            if (row < a.n && c < a.k) {
                const uint8_t byte = a.codes[static_cast<int64_t>(row) * ((a.k + 1) / 2) + (c >> 1)];
                q = (c & 1 ? byte >> 4 : byte & 15) ^ (a.is_signed ? 8 : 0);
            } else if (row < a.n && a.zeros) {
                const int g = min(c / a.group, a.groups - 1);
                q = min(static_cast<int>(a.zeros[static_cast<int64_t>(row) * a.groups + g]), 15);
            }
            v |= q << (4 * nibble);
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
    int32_t n, k, row_tiles, k_blocks, passes, units, share;
    int32_t per_block, block_bytes, stages;
    float* parts;                          // [CTAs][2][256 * kMaxTokens]
    int32_t* counters;                     // [CTAs]
    int64_t wait_budget;
    int32_t* status;
};

// (a & mask) | exponent in one operation
__device__ __forceinline__ uint32_t cut(uint32_t a, uint32_t mask, uint32_t exponent)
{
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(a), "r"(mask), "r"(exponent));
    return r;
}

template <typename T> __device__ __forceinline__ T bits16_as(uint32_t v)
{
    const uint16_t u = static_cast<uint16_t>(v);
    return *reinterpret_cast<const T*>(&u);
}
template <typename H2> __device__ __forceinline__ H2 as(uint32_t v) { return *reinterpret_cast<const H2*>(&v); }
template <typename H2> __device__ __forceinline__ uint32_t bits(H2 v) { return *reinterpret_cast<const uint32_t*>(&v); }

// The pairs of columns (0 1), (16 17), (2 3), (18 19), from 4 t on, of a word as q - z; `zero`: z (0..15) in both halves.  fp16: 1024 + q - (1024 + z),
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
struct Place {                             // a unit: (256 rows of W, rows of x, 256 columns), the columns fastest: what several passes read of W is in L2
    int kb, rb, pass;
    __device__ __forceinline__ Place(const LinearArgs& a, int unit)
    {
        const int rows = unit / a.k_blocks;
        kb = unit - rows * a.k_blocks;
        rb = rows / a.passes;
        pass = rows - rb * a.passes;
    }
    __device__ __forceinline__ void next(const LinearArgs& a)
    {
        if (++kb < a.k_blocks) return;
        kb = 0;
        if (++pass < a.passes) return;
        pass = 0;
        ++rb;
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
    // After a wait that gave up nothing more is issued.
    __device__ __forceinline__ bool wait(bool ok) const
    {
        return unit - u0 >= issued ? ok : mbar_wait_warp(smem_u32(&full[stage]), phase, a.wait_budget, ok);
    }
    // After one that gave up: nothing may be in flight when the CTA ends.
    __device__ __forceinline__ void drain() const
    {
        for (int j = max(0, issued - a.stages); j < issued; ++j)
            __all_sync(0xffffffffu, mbar_wait(smem_u32(&full[j % a.stages]), (j / a.stages) & 1, kDrainBudget));
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

// A CTA's sums over a part of the columns, [activation row][256 rows of W].  Slot 0: rows that began in an earlier CTA; slot 1, rows
// that go on in a later one.
template <int kRows>
__device__ __forceinline__ float* part_of(const LinearArgs& a, int cta, int slot)
{
    return a.parts + (static_cast<int64_t>(cta) * 2 + slot) * (kWarps * kRowTile * kRows);
}

template <typename T>
__device__ __forceinline__ float bias_of(const LinearArgs& a, int o)
{
    return a.bias && o < a.n ? qtz_dev::to_f32(static_cast<const T*>(a.bias)[o]) : 0.f;
}

template <typename T>
__device__ __forceinline__ void put(const LinearArgs& a, int64_t r, int o, float v)
{
    if (o < a.n && r < a.rows) static_cast<T*>(a.y)[r * a.y_stride + o] = qtz_dev::from_f32<T>(v);
}

// Rows whose columns lie in several CTAs, c0 .. c1: the last to arrive joins their parts in order.  Called by all threads behind a barrier; the first
// kJoin know the units that are open.  All of them read, 16 bytes a load and 16 loads in flight, in short code that comes from memory
// like the parts: a warp for each 32 rows of W with everything unrolled took 7 us of 50 for 32 rows through 28672 x 8192.
template <typename T, int kRows, int kJoin>
__device__ __forceinline__ void join_rows(const LinearArgs& a, const int (&open)[2], const int& failed, int (&last)[2])
{
    constexpr int kQuads = kWarps * kRowTile / 4, kAtOnce = (kRows * kQuads + kJoin - 1) / kJoin, kFlight = 16 / kAtOnce;
    const int tid = threadIdx.x;
    if (failed || tid >= kJoin) return;                // after a wait that gave up the results are void
    auto first = [&](int unit) { return unit / a.k_blocks * a.k_blocks; };
    if ((tid == 0 && open[0] >= 0) || (tid == 32 && open[1] >= 0)) {
        const int begin = first(tid ? open[1] : open[0]), c0 = begin / a.share;
        const bool all = arrive_acq_rel(a.counters + c0) == (begin + a.k_blocks - 1) / a.share - c0;
        last[tid ? 1 : 0] = all;
        if (all) a.counters[c0] = 0;                   // ready for the next call
    }
    named_barrier(1, kJoin);
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        const int unit = which ? open[1] : open[0];
        if (unit < 0 || !last[which]) continue;
        const Place at(a, unit);
        const int c0 = first(unit) / a.share, c1 = (first(unit) + a.k_blocks - 1) / a.share;
        const int64_t r0 = static_cast<int64_t>(at.pass) * kRows;
        const int quads = static_cast<int>(min(static_cast<int64_t>(kRows), a.rows - r0)) * kQuads;
        float4 v[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int c = c0; c <= c1; c += kFlight) {
            float4 p[kFlight][kAtOnce];
#pragma unroll
            for (int x = 0; x < kFlight; ++x) {
                const float4* part = reinterpret_cast<const float4*>(part_of<kRows>(a, c + x, c + x == c0 ? 1 : 0)) + tid;
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
                    p[x][j] = c + x <= c1 && tid + j * kJoin < quads ? __ldcg(part + j * kJoin) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int x = 0; x < kFlight; ++x)
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    v[j].x += p[x][j].x;
                    v[j].y += p[x][j].y;
                    v[j].z += p[x][j].z;
                    v[j].w += p[x][j].w;
                }
        }
        const int o = at.rb * (kWarps * kRowTile) + tid % kQuads * 4;
        const float4 b = make_float4(bias_of<T>(a, o), bias_of<T>(a, o + 1), bias_of<T>(a, o + 2), bias_of<T>(a, o + 3));
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (tid + j * kJoin >= quads) break;
            const int64_t r = r0 + (tid + j * kJoin) / kQuads;
            put<T>(a, r, o, v[j].x + b.x);
            put<T>(a, r, o + 1, v[j].y + b.y);
            put<T>(a, r, o + 2, v[j].z + b.z);
            put<T>(a, r, o + 3, v[j].w + b.w);
        }
    }
}

// ---- up to four rows: digits of x, integer matrix instructions ----
constexpr int kDigitBuffers = 3;           // units whose digits are held: the one at work, the next, the one before
constexpr int kDigitPitch = kKBlock + 32;  // bytes of an operand column: the lanes of a load meet all banks

template <int kTiles>
struct Digits {                            // of the rows' columns in one unit
    uint8_t operand[8 * kTiles][kDigitPitch];
    float factor[8 * kTiles];              // of a column's digit: a power of two, 0 for a column that holds none
    float sum[8][8 * kTiles];              // per scale of the unit: minus the sum of the column's digits times its factor (times 8 without zero points)
};

// Row r's digit d is operand column: 1 tile (2 rows) 2 d + r; 2 tiles (4 rows) digits 2 i + j at tile i, column 4 j + r.  A lane so
// shares a row's digits with the lanes of its quad.
template <int kTiles>
__device__ __forceinline__ int digit_column(int d, int r)
{
    return kTiles == 1 ? 2 * d + r : (d >> 1) * 8 + (d & 1) * 4 + r;
}

// Takes this warp's sums of the activation rows in `odd` again, over all units of the CTA, in fp32 straight from the formula: rows that
// hold infinities or NaN have no digits.  A lane owns a row of W.  Rolled up, since it hardly ever runs, and in place: as a function
// that is called it cost all layers of few rows 2 %.
template <typename T, int kSteps, bool kZero>
__device__ __forceinline__ void redo_rows(const LinearArgs& a, uint32_t odd, int u0, int u1)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int half = lane >> 4, g = lane & 7, upper = (lane >> 3) & 1;     // as pack_kernel lays them out
#pragma unroll 1
    for (int unit = u0; unit < u1;) {
        const Place at(a, unit);
        const int end = min(a.k_blocks, at.kb + u1 - unit), tile = at.rb * kWarps + warp, o = tile * kRowTile + lane;
        for (int r = 0; r < 4 && tile < a.row_tiles; ++r) {
            if (!(odd >> r & 1)) continue;
            const T* const x = static_cast<const T*>(a.x) + r * a.x_stride;
            float sum = 0.f;
#pragma unroll 1
            for (int kb = at.kb; kb < end; ++kb) {
                const uint8_t* block = a.blocks + (static_cast<int64_t>(tile) * a.k_blocks + kb) * a.block_bytes;
#pragma unroll 1
                for (int step = 0; step < 8; step += kSteps) {
                    const int place = step / kSteps * kRowTile + half * 16 + g * 2 + upper;
                    const float scale = qtz_dev::to_f32(reinterpret_cast<const T*>(block + kCodeBytes)[place]);
                    const float zero = kZero ? block[kCodeBytes + 8 / kSteps * kRowTile * 2 + place] : 8;
                    float t = 0.f;
#pragma unroll 1
                    for (int i = 0; i < 4 * kSteps; ++i) {                 // words of eight columns
                        const int s = step + i / 4, l = i % 4;
                        const uint32_t w = reinterpret_cast<const uint32_t*>(block)[(((s >> 1) * 2 + half) * 32 + g * 4 + l) * 4 + (s & 1) * 2 + upper];
                        for (int j = 0; j < 8; ++j) {
                            const int m = j >> 1, c = kb * kKBlock + s * 32 + 4 * l + 16 * (j & 1) + (m == 1 ? 2 : m == 2 ? 1 : m);
                            if (c < a.k) t += qtz_dev::to_f32(x[c]) * (static_cast<float>(w >> (4 * j) & 15) - zero);
                        }
                    }
                    sum += t * scale;
                }
            }
            if (at.kb == 0 && end == a.k_blocks) put<T>(a, r, o, sum + bias_of<T>(a, o));
            else part_of<4>(a, blockIdx.x, at.kb == 0 ? 1 : 0)[r * (kWarps * kRowTile) + warp * kRowTile + lane] = sum;
        }
        unit += end - at.kb;
    }
}

// kSteps: steps of 32 columns to a scale (1, 2 or 4)
template <typename T, int kTiles, int kSteps, bool kZero>
__global__ void __launch_bounds__(kThreads, 2)
linear_digits_kernel(const __grid_constant__ LinearArgs a)
{
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t s_full[kWarps][kMaxStages], s_ready[kDigitBuffers], s_free[kDigitBuffers];
    __shared__ int s_last[2], s_failed;
    __shared__ uint32_t s_odd;                         // activation rows with values that are not finite
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3, rows = static_cast<int>(a.rows);
    Digits<kTiles>* const digits = reinterpret_cast<Digits<kTiles>*>(smem);
    if (lane < kMaxStages) mbar_init(smem_u32(&s_full[warp][lane]), 1);
    if (tid == 0) {
        s_failed = 0;
        s_odd = 0;
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
            // an ordinary load: the call before may have written x while this CTA was up already
            if (have > 0) raw = *reinterpret_cast<const uint4*>(x);
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
            const int ex = min(max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -97), 127);   // below, the unit is no normal number
            const float mult = __uint_as_float(static_cast<uint32_t>(127 + 29 - ex) << 23);
            uint32_t d[4][2];                          // digit, columns 0, 2, 1, 3 of the lane's first and second four
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
                auto bytes_of = [&](float f) {         // of a number, the lower three as signed digits
                    return (static_cast<uint32_t>(odd ? 0 : __float2int_rn(f * mult)) + 0x00808080u) ^ 0x00808080u;
                };
                const uint32_t q0 = bytes_of(v[k]), q1 = bytes_of(v[k + 2]), q2 = bytes_of(v[k + 1]), q3 = bytes_of(v[k + 3]);
                const uint32_t lo01 = __byte_perm(q0, q1, 0x5140), hi01 = __byte_perm(q0, q1, 0x7362), lo23 = __byte_perm(q2, q3, 0x5140), hi23 = __byte_perm(q2, q3, 0x7362);
                d[0][k / 4] = __byte_perm(lo01, lo23, 0x5410);
                d[1][k / 4] = __byte_perm(lo01, lo23, 0x7632);
                d[2][k / 4] = __byte_perm(hi01, hi23, 0x5410);
                d[3][k / 4] = __byte_perm(hi01, hi23, 0x7632);
            }
            if (round > 0)                             // the buffer's unit before has been used by all warps
                ok = mbar_wait_warp(smem_u32(&s_free[buffer]), (round - 1) & 1, a.wait_budget, ok);
#pragma unroll
            for (int j = 0; j < 4; ++j) {              // columns 4 t .. and 16 + 4 t .. of 32 lie side by side
                uint8_t* const row = &to.operand[digit_column<kTiles>(j, r)][(lane >> 2) * 32 + (lane & 1) * 16 + (lane & 2) * 2];
                *reinterpret_cast<uint32_t*>(row) = d[j][0];
                *reinterpret_cast<uint32_t*>(row + 8) = d[j][1];
            }
            // the sums of the digits over a scale's columns, two to a register: 128 times 128 fits 16 bits
            constexpr int kLanes = 4 * kSteps;
            auto digits_of = [&](int j) { return __dp4a(static_cast<int>(d[j][0]), 0x01010101, __dp4a(static_cast<int>(d[j][1]), 0x01010101, 0)); };
            int low = digits_of(0) + (digits_of(1) << 16), high = digits_of(2) + (digits_of(3) << 16);
#pragma unroll
            for (int off = 1; off < kLanes; off <<= 1) {
                low += __shfl_xor_sync(0xffffffffu, low, off);
                high += __shfl_xor_sync(0xffffffffu, high, off);
            }
            // a row that holds NaN or infinity gives NaN, and its sums are taken again at the end
            if (odd && lane == 0) atomicOr(&s_odd, 1u << r);
            const float unit_of = odd ? __uint_as_float(0x7fc00000u) : __uint_as_float(static_cast<uint32_t>(127 - 29 + ex) << 23);
            const float minus = kZero ? -1.f : -8.f;
            if (lane % kLanes == 0) {
                const int s0 = (low << 16) >> 16, s2 = (high << 16) >> 16;
                float* const sums = to.sum[lane / kLanes];
                sums[digit_column<kTiles>(0, r)] = static_cast<float>(s0) * unit_of * minus;
                sums[digit_column<kTiles>(1, r)] = static_cast<float>((low - s0) >> 16) * (unit_of * 256.f) * minus;
                sums[digit_column<kTiles>(2, r)] = static_cast<float>(s2) * (unit_of * 65536.f) * minus;
                sums[digit_column<kTiles>(3, r)] = static_cast<float>((high - s2) >> 16) * (unit_of * 16777216.f) * minus;
            }
            if (lane < 4) to.factor[digit_column<kTiles>(lane, r)] = unit_of * static_cast<float>(1 << (8 * lane));
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
        ok = s.wait(ok);
        ok = mbar_wait_warp(smem_u32(&s_ready[buffer]), round & 1, a.wait_budget, ok);
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
            float v[8];                                // the digits of a row together
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float t = acc[j][0][c];
                    if (kTiles > 1) t += acc[j][1 % kTiles][c];
                    if (kTiles == 1) t += __shfl_xor_sync(0xffffffffu, t, 1);
                    t += __shfl_xor_sync(0xffffffffu, t, 2);
                    v[4 * j + c] = t;
#pragma unroll
                    for (int nt = 0; nt < kTiles; ++nt) acc[j][nt][c] = 0.f;
                }
            // v[2 i + c]: output row g + 8 i, activation row 2 t4 + c
            const bool begins = s.unit - s.here.kb >= s.u0, whole = begins && s.ends();
            if (!whole) {
                if (begins) open[1] = s.unit;
                else open[0] = s.unit;
            }
            float* const part = part_of<4>(a, blockIdx.x, begins ? 1 : 0) + warp * kRowTile + g;
            const int o = s.tile(s.here) * kRowTile + g;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float b = whole ? bias_of<T>(a, o + 8 * i) : 0.f;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int r = 2 * t4 + c;
                    if (r >= rows) continue;
                    if (whole) put<T>(a, r, o + 8 * i, v[2 * i + c] + b);
                    else part[r * (kWarps * kRowTile) + 8 * i] = v[2 * i + c];
                }
            }
        }
    }
    if (!ok) {
        timed_out(a);
        s_failed = 1;
        s.drain();
    }
    __syncthreads();
    if (s_odd && !s_failed) {                          // the same for all threads
        redo_rows<T, kSteps, kZero>(a, s_odd, s.u0, s.u1);
        __syncthreads();
    }
    join_rows<T, 4, kThreads>(a, open, s_failed, s_last);
}

// ---- more rows: 16-bit tensor cores (tcgen05) ----
// Two groups of eight warps turn 32 rows of codes each into 16-bit operands, straight into tensor memory: two tiles of 128 rows.  One
// warp issues the products with kN rows of x, which another brings by TMA, like the weights.  The groups take the scales in turn; each
// hands over at most 64 columns at a time in two operand buffers.  A product lies in one of two buffers, too, and each thread, which
// owns a row of W, adds scale * product to its kN sums while the next one's columns are multiplied.  The groups' sums meet at the end of the rows.  kSteps: steps of 32 columns to a scale (1, 2 or 4).
constexpr int kWideThreads = 2 * kThreads + 96;
constexpr int kExchange = 8;                           // sums of a row that each group hands to the other at a time
constexpr int kXUnits = 4;                             // units of x under way: one takes about as long to come as two take to be used

template <typename T, int kN, int kSteps, bool kZero>
__global__ void __launch_bounds__(kWideThreads, 1)
linear_wide_kernel(const __grid_constant__ LinearArgs a, const __grid_constant__ CUtensorMap x_map)
{
    constexpr int kXBox = kN * 128;                    // 64 columns of x
    constexpr int kXUnit = kKBlock / 64 * kXBox;
    constexpr int kScales = 8 / kSteps;                // of a unit
    constexpr int kHand = kSteps < 2 ? kSteps : 2, kHands = kSteps / kHand;    // steps handed over at a time; times to a scale
    constexpr uint32_t kFormat = std::is_same<T, __half>::value ? 0 : 1;
    constexpr uint32_t kProduct = (1u << 4) | (kFormat << 7) | (kFormat << 10) | (static_cast<uint32_t>(kN >> 3) << 17) | (128u >> 4 << 24);
    extern __shared__ uint8_t smem_raw[];              // units of x, the exchange, the ring
    __shared__ __align__(8) uint64_t s_full[kMaxStages], s_empty[kMaxStages], s_xfull[kXUnits], s_xfree[kXUnits], s_operand[8], s_done[8], s_drain[2];   // [tile][group][buffer]
    __shared__ int s_last[2], s_failed;
    __shared__ uint32_t s_tmem;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    float* const exchange = reinterpret_cast<float*>(smem_raw + (base - smem_u32(smem_raw)) + kXUnits * kXUnit);
    const uint32_t ring = base + kXUnits * kXUnit + 2 * kThreads * kExchange * 4;
    if (tid == 0) {
        s_failed = 0;
        prefetch_tensormap(&x_map);
        mbar_init(smem_u32(&s_drain[0]), 1);
        mbar_init(smem_u32(&s_drain[1]), 1);
        for (int i = 0; i < a.stages; ++i) {
            mbar_init(smem_u32(&s_full[i]), 1);
            mbar_init(smem_u32(&s_empty[i]), 2 * kWarps);
        }
        for (int i = 0; i < kXUnits; ++i) {
            mbar_init(smem_u32(&s_xfull[i]), 1);
            mbar_init(smem_u32(&s_xfree[i]), 2);
        }
        for (int i = 0; i < 8; ++i) {
            mbar_init(smem_u32(&s_operand[i]), 4);
            mbar_init(smem_u32(&s_done[i]), 1);
        }
    }
    if (warp == 2 * kWarps + 1) {
        tmem_alloc(smem_u32(&s_tmem), 512);
        tmem_relinquish();
    }
    fence_barrier_init();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
    // columns: operand [tile][group][buffer], then product [tile][group][buffer]
    auto operand_at = [&](int which) { return tmem + which * 32; };
    auto product_at = [&](int tile, int group, int turn) { return tmem + 256 + (tile * 2 + group) * 64 + (turn & 1) * 32; };
    const int u0 = min(static_cast<int>(blockIdx.x) * a.share, a.units), count = min(u0 + a.share, a.units) - u0;
    Place here(a, u0);
    int open[2] = {-1, -1};                            // units whose rows are shared with an earlier / a later CTA
    bool ok = true;
    auto wait = [&](uint64_t& bar, int parity) { ok = mbar_wait_warp(smem_u32(&bar), parity, a.wait_budget, ok); };
    const int row_tile = warp & (kWarps - 1);
    grid_launch_dependents();

    if (warp == 2 * kWarps) {
        // ======== loads: weights as many units ahead as the ring holds, x two ========
        Place ahead = here;
        int issued = 0;
        auto issue_weights = [&](int stage) {
            const uint32_t bar = smem_u32(&s_full[stage]);
            const int first = ahead.rb * kWarps, tiles = min(kWarps, a.row_tiles - first);
            if (lane == 0) mbar_arrive_expect_tx(bar, tiles * a.block_bytes);
            __syncwarp();
            if (lane < tiles)
                bulk_load(ring + (stage * kWarps + lane) * a.block_bytes, a.blocks + (static_cast<int64_t>(first + lane) * a.k_blocks + ahead.kb) * a.block_bytes,
                          a.block_bytes, bar);
            ahead.next(a);
            ++issued;
        };
        while (issued < min(a.stages, count)) issue_weights(issued);   // the weights were there when the layer was made
        grid_dependency_wait();                        // all else is waited for
        int xi = 0, stage = 0, round = 0;              // units of x; the next place of the ring
        auto issue_x = [&]() {
            const uint32_t bar = smem_u32(&s_xfull[xi % kXUnits]);
            if (elect_one()) {
                mbar_arrive_expect_tx(bar, kXUnit);
#pragma unroll
                for (int c = 0; c < kKBlock / 64; ++c)
                    tma_load_2d(base + xi % kXUnits * kXUnit + c * kXBox, &x_map, bar, (here.kb * kKBlock + c * 64) * 2, here.pass * kN);
            }
            __syncwarp();
            here.next(a);
            ++xi;
        };
        while (xi < min(kXUnits, count)) issue_x();
        for (int i = 0; i < count && ok; ++i) {        // as unit i is used up
            if (issued < count) {
                wait(s_empty[stage], round & 1);
                if (!ok) break;
                issue_weights(stage);
                if (++stage == a.stages) {
                    stage = 0;
                    ++round;
                }
            }
            if (xi < count) {
                wait(s_xfree[i % kXUnits], (i / kXUnits) & 1);
                if (ok) issue_x();
            }
        }
        // nothing may be in flight when the CTA ends
        auto drain = [&](uint64_t& bar, int parity) { ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar), parity, kDrainBudget)) && ok; };
        for (int j = max(0, xi - kXUnits); j < xi; ++j) drain(s_xfull[j % kXUnits], (j / kXUnits) & 1);
        for (int j = max(0, issued - a.stages); j < issued; ++j) drain(s_full[j % a.stages], (j / a.stages) & 1);
    } else if (warp > 2 * kWarps) {
        // ======== products of a group ========
        const int group = __shfl_sync(0xffffffffu, warp - 2 * kWarps - 1, 0);
        int hand = 0, turn = 0, x = 0, x_round = 0;
        for (int i = 0; i < count && ok; ++i) {
            wait(s_xfull[x], x_round & 1);
            const uint64_t x_desc = make_kmajor_desc(base + x * kXUnit, 128);
#pragma unroll
            for (int q = 0; q < kScales; q += 2) {
#pragma unroll
                for (int part = 0; part < kHands; ++part) {
#pragma unroll
                    for (int tile = 0; tile < 2; ++tile) {
                        const int at = (tile * 2 + group) * 2 + (hand & 1);
                        if (ok) wait(s_operand[at], (hand >> 1) & 1);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t to = product_at(tile, group, turn), from = operand_at(at);
                        // 32 columns of x lie 64 bytes on, 64 a box; a group's step is kSteps of them
                        const uint64_t desc = x_desc + static_cast<uint64_t>(group) * (kSteps == 1 ? 4 : kSteps == 2 ? kXBox / 16 : 2 * kXBox / 16);
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < 2 * kHand; ++k) {      // 16 columns
                                constexpr int kStride = kSteps * 32;
                                const int column = q * kStride + part * kHand * 32 + k * 16;
                                mma_f16_from_tmem(to, from + 8 * k, desc + column / 64 * (kXBox / 16) + 2 * (column / 16 % 4), kProduct, part + k > 0);
                            }
                            mma_commit(smem_u32(&s_done[at]));
                            if (q + 2 >= kScales && part == kHands - 1 && tile == 1) mma_commit(smem_u32(&s_xfree[x]));
                        }
                        __syncwarp();
                    }
                    ++hand;
                }
                ++turn;
            }
            if (++x == kXUnits) {
                x = 0;
                ++x_round;
            }
        }
        if (elect_one()) mma_commit(smem_u32(&s_drain[group]));   // the operands' warps may have given up on what is still running
        __syncwarp();
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&s_drain[group]), 0, kDrainBudget)) && ok;
    } else {
        // ======== operands, then sums ========
        const int group = warp / kWarps, tile = row_tile >> 2;
        const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;
        float acc[kN];
#pragma unroll
        for (int r = 0; r < kN; ++r) acc[r] = 0.f;
        int stage = 0, round = 0, hand = 0, turn = 0;
        float scale = 0.f;                             // of the product that is still to be taken
        bool pending = false;
        // the product of a turn
        auto take = [&](int t) {
            tc_fence_after();
#pragma unroll
            for (int r0 = 0; r0 < kN; r0 += 16) {
                uint32_t v[16];
                tmem_ld_32x16(product_at(tile, group, t) + lanes + r0, v);
                tmem_ld_wait();
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[r0 + r] = fmaf(__uint_as_float(v[r]), scale, acc[r0 + r]);
            }
        };
        auto wait_done = [&](int h) { wait(s_done[(tile * 2 + group) * 2 + (h & 1)], (h >> 1) & 1); };
        grid_dependency_wait();
        for (int i = 0; i < count; ++i) {
            wait(s_full[stage], round & 1);
            const uint32_t block = ring + (stage * kWarps + row_tile) * a.block_bytes, scales = block + kCodeBytes, zeros = scales + kScales * kRowTile * 2;
            const bool work = ok && here.rb * kWarps + row_tile < a.row_tiles;
#pragma unroll 1
            for (int q = group; q < kScales; q += 2, ++turn) {
                float scale_here = 0.f;
                uint32_t z[2] = {0x0808u, 0x0808u};
                if (work) {
                    scale_here = qtz_dev::to_f32(bits16_as<T>(lds16(scales + 2 * (q * 32 + (lane >> 4) * 16 + (lane & 7) * 2 + ((lane >> 3) & 1)))));
                    if (kZero)
#pragma unroll
                        for (int j = 0; j < 2; ++j) z[j] = lds16(zeros + 2 * ((q * 2 + j) * 8 + (lane >> 2)));
                }
#pragma unroll
                for (int part = 0; part < kHands; ++part, ++hand) {
                    const int at = (tile * 2 + group) * 2 + (hand & 1);
                    if (hand >= 2) wait_done(hand - 2);        // the buffer's columns before have been multiplied
                    if (work) {
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const uint32_t z0 = (z[j] & 0xffu) * 0x00010001u, z1 = (z[j] >> 8) * 0x00010001u;
                            const uint32_t to = operand_at(at) + lanes + (static_cast<uint32_t>(16 * j) << 16);
#pragma unroll
                            for (int h = 0; h < kHand; ++h) {  // 32 columns: 16 of tensor memory
                                const int half = q * kSteps + part * kHand + h;
                                const uint2 w = lds64(block + ((half >> 1) * 2 + j) * 512 + lane * 16 + (half & 1) * 8);
                                uint32_t lo[4], hi[4];         // rows g, g + 8
                                unpack_codes<T>(w.x, z0, lo);
                                unpack_codes<T>(w.y, z1, hi);
                                tmem_st_16x256_x2(to + 16 * h, lo[0], lo[2], hi[0], hi[2], lo[1], lo[3], hi[1], hi[3]);
                            }
                        }
                        tmem_st_wait();
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(smem_u32(&s_operand[at]));
                        if (q + 2 >= kScales && part == kHands - 1) mbar_arrive(smem_u32(&s_empty[stage]));   // the unit's codes are taken
                    }
                }
                if (pending) {
                    // with two hands to a turn, the second has waited for the turn before already
                    if (kHands == 1) wait_done(hand - 2);
                    take(turn - 1);
                }
                scale = scale_here;
                pending = true;
            }
            if (++stage == a.stages) {
                stage = 0;
                ++round;
            }
            const bool ends = here.kb == a.k_blocks - 1;
            if (ends || i == count - 1) {              // the end of these rows, or of this CTA's columns of them
                if (pending) {
                    wait_done(hand - 1);
                    take(turn - 1);
                    pending = false;
                }
                // group 0 takes the first half of the activation rows, group 1 the second
                float sum[kN / 2];
#pragma unroll
                for (int r0 = 0; r0 < kN / 2; r0 += kExchange) {
#pragma unroll
                    for (int r = 0; r < kExchange; ++r)
                        exchange[(group * kExchange + r) * kThreads + row_tile * 32 + lane] = group ? acc[r0 + r] : acc[kN / 2 + r0 + r];
                    named_barrier(1, 2 * kThreads);
#pragma unroll
                    for (int r = 0; r < kExchange; ++r)
                        sum[r0 + r] = (group ? acc[kN / 2 + r0 + r] : acc[r0 + r]) + exchange[((1 - group) * kExchange + r) * kThreads + row_tile * 32 + lane];
                    named_barrier(1, 2 * kThreads);
                }
                const bool begins = i >= here.kb;
                if (begins && ends) {
                    const int o = (here.rb * kWarps + row_tile) * kRowTile + lane;
                    const float b = bias_of<T>(a, o);
#pragma unroll
                    for (int r = 0; r < kN / 2; ++r) put<T>(a, static_cast<int64_t>(here.pass) * kN + group * (kN / 2) + r, o, sum[r] + b);
                } else {
                    if (begins) open[1] = u0 + i;
                    else open[0] = u0 + i;
                    float* const part = part_of<kN>(a, blockIdx.x, begins ? 1 : 0) + group * (kN / 2) * kThreads + row_tile * 32 + lane;
#pragma unroll
                    for (int r = 0; r < kN / 2; ++r) part[r * kThreads] = sum[r];
                }
#pragma unroll
                for (int r = 0; r < kN; ++r) acc[r] = 0.f;
            }
            here.next(a);
        }
    }
    if (!ok) {
        timed_out(a);
        s_failed = 1;
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 2 * kWarps + 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    join_rows<T, kN, 2 * kThreads>(a, open, s_failed, s_last);
}

// ctas: of an SM; fixed: shared memory beside the rings; most_parts: that a row block is cut into (0: any number)
template <typename K, typename... X>
qtz_status launch(qtz_linear* p, LinearArgs& a, K kernel, int threads, int ctas, int fixed, int most_parts, cudaStream_t st, const X&... more)
{
    qtz_ctx* h = p->h;
    const int room = (kSmemLimit + 1024) / ctas - 1024 - 1024 - fixed;    // 1 KB: the kernels' static shared memory
    a.stages = room / (kWarps * p->block_bytes);
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    const int smem = fixed + kWarps * a.stages * p->block_bytes, grid = ctas * h->num_sms;
    // A share takes in at least 1 / most_parts of the columns: joining 16 or 32 rows costs more than it brings beyond that (1024 x 8192:
    // 9.7 and 12.5 us against 10.9 and 16.3 without a limit; with few rows the limit changes nothing and there is none).
    a.share = (a.units + grid - 1) / grid;
    if (most_parts && a.share < (a.k_blocks + most_parts - 1) / most_parts) a.share = (a.k_blocks + most_parts - 1) / most_parts;
    const qtz_status s = qtz_allow_smem(h, kernel);
    if (s != QTZ_OK) return s;
    QTZ_CUDA(h, qtz_launch_dependent(kernel, dim3((a.units + a.share - 1) / a.share), threads, smem, st, a, more...));
    return QTZ_OK;
}

template <typename T, int kTiles>
qtz_status launch_digits(qtz_linear* p, LinearArgs& a, bool zero, cudaStream_t st)
{
    constexpr int kFixed = kDigitBuffers * sizeof(Digits<kTiles>);
    auto go = [&](auto kernel) { return launch(p, a, kernel, kThreads, 2, kFixed, 0, st); };
    if (p->scales == 8) return zero ? go(linear_digits_kernel<T, kTiles, 1, true>) : go(linear_digits_kernel<T, kTiles, 1, false>);
    if (p->scales == 4) return zero ? go(linear_digits_kernel<T, kTiles, 2, true>) : go(linear_digits_kernel<T, kTiles, 2, false>);
    return zero ? go(linear_digits_kernel<T, kTiles, 4, true>) : go(linear_digits_kernel<T, kTiles, 4, false>);
}

template <typename T, int kN>
qtz_status launch_wide(qtz_linear* p, LinearArgs& a, bool zero, cudaStream_t st)
{
    constexpr int kFixed = 1024 + kXUnits * (kKBlock / 64) * kN * 128 + 2 * kThreads * kExchange * 4;
    CUtensorMap x_map;                                 // bytes: columns beyond k and rows beyond the last read as zero
    const uint64_t dims[2] = {2 * static_cast<uint64_t>(a.k), static_cast<uint64_t>(a.rows)}, strides[1] = {2 * static_cast<uint64_t>(a.x_stride)};
    const uint32_t box[2] = {128, kN};
    if (!qtz_encode_u8_map(&x_map, a.x, 2, dims, strides, box, 128)) return qtz_cuda_fail(p->h, cudaErrorInvalidValue, "tensor map of the activations");
    auto go = [&](auto kernel) { return launch(p, a, kernel, kWideThreads, 1, kFixed, kN == 16 ? 16 : 8, st, x_map); };
    if (p->scales == 8) return zero ? go(linear_wide_kernel<T, kN, 1, true>) : go(linear_wide_kernel<T, kN, 1, false>);
    if (p->scales == 4) return zero ? go(linear_wide_kernel<T, kN, 2, true>) : go(linear_wide_kernel<T, kN, 2, false>);
    return zero ? go(linear_wide_kernel<T, kN, 4, true>) : go(linear_wide_kernel<T, kN, 4, false>);
}

template <typename T>
qtz_status launch_rows(qtz_linear* p, LinearArgs& a, bool zero, cudaStream_t st)
{
    // us at 1, 2, 4 | 5 to 8, 12, 16 | 32 rows: 24.4, 26.2, 31.6 | 40.0, 40.1, 40.3 | 41.8 through 28672 x 8192, groups of 128; 6.2, 6.3, 7.3 |
    // 9.3, 9.4, 9.7 | 12.4 through 4096 x 4096, groups of 32; 4.7, 4.8, 5.2 | 6.4, 6.5, 6.9 | 8.4 through 1000 x 1024.  Digits for five to
    // eight rows would take 32 operand columns; with 24, three digits a row, eight rows took 42.8, 9.0 and 6.0.  More than 32 rows take
    // several passes over the weights, which then lie in L2: 64 rows at once left no second buffer for the products (69.9 us against
    // 30.3 for two passes through 5003 x 10001).
    if (a.rows <= 2) return launch_digits<T, 1>(p, a, zero, st);
    if (a.rows <= 4) return launch_digits<T, 2>(p, a, zero, st);
    if (a.rows <= 16) return launch_wide<T, 16>(p, a, zero, st);
    return launch_wide<T, 32>(p, a, zero, st);
}

// Scratch of the joining, shared by the layers of a handle: parts and counters of a full grid.
qtz_status ensure_scratch(qtz_ctx* h, cudaStream_t st)
{
    if (h->linear_dev) return QTZ_OK;
    const int ctas = 2 * h->num_sms;                   // of up to four rows; half as many with more
    const size_t parts = static_cast<size_t>(h->num_sms) * 2 * kWarps * kRowTile * kMaxTokens * sizeof(float);
    QTZ_CUDA(h, cudaMalloc(&h->linear_dev, parts + ctas * sizeof(int32_t)));
    QTZ_CUDA(h, cudaMemsetAsync(static_cast<uint8_t*>(h->linear_dev) + parts, 0, ctas * sizeof(int32_t), st));
    h->linear_counters = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(h->linear_dev) + parts);
    return QTZ_OK;
}

}  // namespace

extern "C" qtz_status qtz_linear_destroy(qtz_linear_plan p)
{
    if (!p) return QTZ_ERR_INVALID_ARG;
    qtz_device_guard guard(p->device);
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
    p->device = h->device;
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
    const int64_t passes = (rows + kMaxTokens - 1) / kMaxTokens;
    if (passes * row_blocks * p->k_blocks > 0x3fffffff) return QTZ_ERR_TOO_LARGE;
    qtz_device_guard guard(p->h->device);
    LinearArgs a{p->blocks, x_dev, x_stride, rows, p->bias, y_dev, y_stride, p->d.n, p->d.k, p->row_tiles, p->k_blocks, static_cast<int32_t>(passes),
                 static_cast<int32_t>(passes * row_blocks * p->k_blocks), 0, p->scales, p->block_bytes, 0, static_cast<float*>(p->h->linear_dev),
                 p->h->linear_counters, p->h->wait_budget, p->h->status_dev};
    const bool zero = p->d.wdtype == QTZ_U4_PACKED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (p->d.ftype == QTZ_F16) return launch_rows<__half>(p, a, zero, st);
    return launch_rows<__nv_bfloat16>(p, a, zero, st);
}

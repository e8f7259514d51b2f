// Linear layers with 4-bit weights and group scales on few rows of real activations (decoding).
//
// Mathematics.  y[r][o] = sum_g s[o][g] sum_{k in g} (q[o][k] - z[o][g]) x[r][k] + b[o].  The inner sum runs on the fp16 / bf16
// matrix instructions (m16n8k16: 16 output rows x 8 activation rows) with q - z as an exact 16-bit operand and fp32 sums; the
// scale multiplies the fp32 sum of its group, or of the 64 columns of it that are at hand.  Nothing is rounded before y.
//
// What bounds it: half a byte of weight is read for 2 flops an activation row, so up to some 16 rows HBM does (measured copy
// rate: 46 weights a clock and SM), beyond that the matrix instructions (1024 products a clock and SM: 32 weights at 32 rows).
// So the weights are read once, in the order of use, as contiguous blocks of 32 rows x 256 columns with their scales and zero
// points behind the codes; every warp streams its blocks through a ring of its own (bulk copies, several blocks ahead), and a
// code costs little more than one instruction: two are cut from a word by one logic operation that also writes the exponent
// (1024 + q in fp16, 128 + q in bf16), one packed operation takes the offset off.  Activations are few and come through L1: the
// eight warps of a CTA work on the same columns of 256 rows.
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
    int scales = 0;                    // scales of a row in a block of 256 columns: 1, 2, 4 or 8
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

// One thread per 32-bit word of codes: word (chunk of 64 columns, half of the 32 rows, lane, w) holds eight columns of one row,
// column pair p at bits 4 p and 16 + 4 p, in the order in which the lanes of a matrix instruction hold their operand.
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
            v |= q << (4 * (j >> 1) + 16 * (j & 1));
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

// (a & mask) | exponent in one operation
__device__ __forceinline__ uint32_t cut(uint32_t a, uint32_t mask, uint32_t exponent)
{
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(a), "r"(mask), "r"(exponent));
    return r;
}

template <typename H2> __device__ __forceinline__ H2 as(uint32_t v) { return *reinterpret_cast<const H2*>(&v); }
template <typename H2> __device__ __forceinline__ uint32_t bits(H2 v) { return *reinterpret_cast<const uint32_t*>(&v); }

// The four pairs of a word as q - z.  fp16: 1024 + q - (1024 + z), and (1024 + 16 q) / 16 - (64 + z) for the pairs at odd nibbles.
// bf16 has no room for the latter: 128 + q - (128 + z) after a shift each.  `zero`: z as two 16-bit values of T.
template <typename T>
__device__ __forceinline__ void unpack_codes(uint32_t w, uint32_t zero, uint32_t (&out)[4])
{
    if constexpr (std::is_same<T, __half>::value) {
        const __half2 even = __hadd2(as<__half2>(zero), as<__half2>(0x64006400u));
        const __half2 odd = __hneg2(__hadd2(as<__half2>(zero), as<__half2>(0x54005400u)));
        const uint32_t v = w >> 8;
        out[0] = bits(__hsub2(as<__half2>(cut(w, 0x000f000fu, 0x64006400u)), even));
        out[1] = bits(__hfma2(as<__half2>(cut(w, 0x00f000f0u, 0x64006400u)), as<__half2>(0x2c002c00u), odd));
        out[2] = bits(__hsub2(as<__half2>(cut(v, 0x000f000fu, 0x64006400u)), even));
        out[3] = bits(__hfma2(as<__half2>(cut(v, 0x00f000f0u, 0x64006400u)), as<__half2>(0x2c002c00u), odd));
    } else {
        const __nv_bfloat162 offset = __hadd2(as<__nv_bfloat162>(zero), as<__nv_bfloat162>(0x43004300u));
#pragma unroll
        for (int p = 0; p < 4; ++p) out[p] = bits(__hsub2(as<__nv_bfloat162>(cut(w >> (4 * p), 0x000f000fu, 0x43004300u)), offset));
    }
}

// z (0..15) as two equal values of T
template <typename T>
__device__ __forceinline__ uint32_t zero_pair(uint32_t z)
{
    if constexpr (std::is_same<T, __half>::value) return bits(__half2half2(__ushort2half_rn(static_cast<unsigned short>(z))));
    else return bits(__bfloat162bfloat162(__ushort2bfloat16_rn(static_cast<unsigned short>(z))));
}

__device__ __forceinline__ uint4 lds128(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
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

// kNt: blocks of eight activation rows; kFine: groups of 32 columns; kZero: with zero points
template <typename T, int kNt, bool kFine, bool kZero>
__global__ void __launch_bounds__(kThreads, kNt <= 2 ? 2 : 1)
linear_kernel(const __grid_constant__ LinearArgs a)
{
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t s_full[kWarps][kMaxStages];
    __shared__ int s_last[2], s_failed;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
    const uint32_t ring = smem_u32(smem) + warp * a.stages * a.block_bytes;
    if (lane < kMaxStages) mbar_init(smem_u32(&s_full[warp][lane]), 1);
    if (tid == 0) s_failed = 0;
    fence_barrier_init();
    __syncthreads();

    const int u0 = min(static_cast<int>(blockIdx.x) * a.share, a.units), u1 = min(u0 + a.share, a.units);
    // a unit: (rows of x, 256 rows of W, 256 columns), the columns fastest
    auto tile_of = [&](int unit) { return unit / a.k_blocks % a.row_blocks * kWarps + warp; };
    auto issue = [&](int unit, int stage) {            // lane 0 only
        const int tile = tile_of(unit);
        const uint32_t bar = smem_u32(&s_full[warp][stage]);
        if (tile >= a.row_tiles) {                     // no rows for this warp
            mbar_arrive(bar);
            return;
        }
        mbar_arrive_expect_tx(bar, a.block_bytes);
        bulk_load(ring + stage * a.block_bytes, a.blocks + (static_cast<int64_t>(tile) * a.k_blocks + unit % a.k_blocks) * a.block_bytes, a.block_bytes, bar);
    };
    int issued = min(a.stages, u1 - u0);
    if (lane == 0)
        for (int i = 0; i < issued; ++i) issue(u0 + i, i);

    float acc[2][kNt][4];
    auto clear = [&]() {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int nt = 0; nt < kNt; ++nt)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[j][nt][c] = 0.f;
    };
    clear();
    // rows of y: value c of acc[j][nt] belongs to output row g + 8 (c >> 1) of half j and activation row 2 t4 + (c & 1) of block nt
    auto write = [&](int unit) {
        const int o0 = tile_of(unit) * kRowTile + g;
        const int64_t r0 = static_cast<int64_t>(unit / (a.k_blocks * a.row_blocks)) * (8 * kNt) + 2 * t4;
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
                        if (r < a.rows) static_cast<T*>(a.y)[r * a.y_stride + o] = qtz_dev::from_f32<T>(acc[j][nt][2 * hi + c] + b);
                    }
            }
    };
    constexpr int kPart = kWarps * kRowTile * 8 * kNt;
    int open[2] = {-1, -1};                            // units whose rows are shared with an earlier / a later CTA
    bool failed = false;
    int stage = 0;
    uint32_t phase = 0;
    for (int unit = u0; unit < u1; ++unit) {
        const int kb = unit % a.k_blocks, i = unit - u0;
        // after a wait that gave up nothing more is issued, but what is in flight is still waited for (with the same limit)
        if (i < issued && !__all_sync(0xffffffffu, mbar_wait(smem_u32(&s_full[warp][stage]), phase, a.wait_budget))) {
            if (lane == 0 && atomicCAS(a.status, 0, QTZ_ERR_DEVICE_TIMEOUT) == 0) a.status[1] = QTZ_SITE_LINEAR;
            failed = true;
        }
        if (!failed && tile_of(unit) < a.row_tiles) {
            const uint32_t block = ring + stage * a.block_bytes, scales = block + kCodeBytes, zeros = scales + a.per_block * kRowTile * 2;
            const int64_t r0 = static_cast<int64_t>(unit / (a.k_blocks * a.row_blocks)) * (8 * kNt) + g;
            const uint16_t* xp[kNt];
#pragma unroll
            for (int nt = 0; nt < kNt; ++nt)
                xp[nt] = r0 + 8 * nt < a.rows ? static_cast<const uint16_t*>(a.x) + (r0 + 8 * nt) * a.x_stride + kb * kKBlock + 8 * t4 : nullptr;
            const int left = a.k - kb * kKBlock - 8 * t4;      // columns from this lane's first one on
#pragma unroll 1
            for (int chunk = 0; chunk < 4; ++chunk) {
                uint32_t w[2][2][2][4];                // [half of the rows][half of the columns][row g, g + 8][pair]
                float s[2][kFine ? 2 : 1][2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint4 q = lds128(block + (chunk * 2 + j) * 512 + lane * 16);
                    const uint32_t words[2][2] = {{q.x, q.y}, {q.z, q.w}};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int si = kFine ? 2 * chunk + h : chunk * a.per_block / 4, at = (si * 2 + j) * 8 + g;
                        uint32_t z0 = zero_pair<T>(8), z1 = z0;
                        if (kZero) {
                            const uint32_t z = lds16(zeros + 2 * at);
                            z0 = zero_pair<T>(z & 0xff);
                            z1 = zero_pair<T>(z >> 8);
                        }
                        if (kFine || h == 0) {
                            const float2 f = qtz_dev::unpack2(lds32(scales + 4 * at), T());
                            s[j][kFine ? h : 0][0] = f.x;
                            s[j][kFine ? h : 0][1] = f.y;
                        }
                        unpack_codes<T>(words[h][0], z0, w[j][h][0]);
                        unpack_codes<T>(words[h][1], z1, w[j][h][1]);
                    }
                }
#pragma unroll
                for (int nt = 0; nt < kNt; ++nt) {
                    uint32_t b[2][4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int k = chunk * 64 + h * 32, have = xp[nt] ? left - k : 0;
                        uint4 v = make_uint4(0, 0, 0, 0);
                        if (have > 0) v = __ldg(reinterpret_cast<const uint4*>(xp[nt] + k));
                        b[h][0] = v.x; b[h][1] = v.y; b[h][2] = v.z; b[h][3] = v.w;
                        if (have > 0 && have < 8)              // the last columns: what lies behind them is not data
#pragma unroll
                            for (int c = 0; c < 4; ++c) b[h][c] = have >= 2 * c + 2 ? b[h][c] : have == 2 * c + 1 ? b[h][c] & 0xffffu : 0u;
                    }
                    float part[2][4] = {};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int step = 0; step < 2; ++step)
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                const uint32_t op[4] = {w[j][h][0][2 * step], w[j][h][1][2 * step], w[j][h][0][2 * step + 1], w[j][h][1][2 * step + 1]};
                                mma<T>(part[j], op, b[h][2 * step], b[h][2 * step + 1]);
                            }
                        if (kFine || h == 1)
#pragma unroll
                            for (int j = 0; j < 2; ++j)
#pragma unroll
                                for (int c = 0; c < 4; ++c) {
                                    acc[j][nt][c] = fmaf(part[j][c], s[j][kFine ? h : 0][c >> 1], acc[j][nt][c]);
                                    part[j][c] = 0.f;
                                }
                    }
                }
            }
        }
        __syncwarp();                                  // every lane has read the stage
        if (!failed && i + a.stages < u1 - u0) {
            if (lane == 0) issue(unit + a.stages, stage);
            ++issued;
        }
        if (++stage == a.stages) {
            stage = 0;
            phase ^= 1;
        }
        if (kb == a.k_blocks - 1 || unit == u1 - 1) {  // the end of these rows, or of this CTA's columns of them
            const bool begins = unit - kb >= u0, ends = kb == a.k_blocks - 1;
            if (begins && ends) {
                if (tile_of(unit) < a.row_tiles) write(unit);
            } else {
                open[begins ? 1 : 0] = unit;
                float* part = a.parts + (static_cast<int64_t>(blockIdx.x) * 2 + (begins ? 1 : 0)) * kPart + warp * (kRowTile * 8 * kNt) + lane;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int nt = 0; nt < kNt; ++nt)
#pragma unroll
                        for (int c = 0; c < 4; ++c) part[((j * kNt + nt) * 4 + c) * 32] = acc[j][nt][c];
            }
            clear();
        }
    }
    if (failed) s_failed = 1;

    // ---- joining: rows whose columns lie in several CTAs, c0 .. c1 ----
    if (open[0] < 0 && open[1] < 0) return;            // the same for all warps
    __threadfence();
    __syncthreads();
    if (s_failed) return;                              // the results are void, and the counters have to be cleared
    auto first_cta = [&](int unit) { return (unit - unit % a.k_blocks) / a.share; };
    auto last_cta = [&](int unit) { return (unit - unit % a.k_blocks + a.k_blocks - 1) / a.share; };
    if (tid == 0 || tid == 32) {
        const int which = tid / 32;
        if (open[which] >= 0) {
            const int c0 = first_cta(open[which]), c1 = last_cta(open[which]);
            s_last[which] = atomicAdd(a.counters + c0, 1) == c1 - c0;
            if (s_last[which]) a.counters[c0] = 0;     // ready for the next call
        }
    }
    __syncthreads();
    for (int which = 0; which < 2; ++which) {
        if (open[which] < 0 || !s_last[which] || tile_of(open[which]) >= a.row_tiles) continue;
        __threadfence();
        const int c0 = first_cta(open[which]), c1 = last_cta(open[which]);
        clear();
#pragma unroll 4
        for (int c = c0; c <= c1; ++c) {
            const float* part = a.parts + (static_cast<int64_t>(c) * 2 + (c == c0 ? 1 : 0)) * kPart + warp * (kRowTile * 8 * kNt) + lane;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int nt = 0; nt < kNt; ++nt)
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[j][nt][v] += __ldcg(part + ((j * kNt + nt) * 4 + v) * 32);
        }
        write(open[which]);
    }
}

template <typename T, int kNt, bool kFine, bool kZero>
qtz_status launch(qtz_linear* p, LinearArgs& a, cudaStream_t st)
{
    qtz_ctx* h = p->h;
    const int ctas = kNt <= 2 ? 2 : 1;
    const int room = (kSmemLimit + 1024) / ctas - 1024 - 1024;     // 1 KB: the kernel's static shared memory
    a.stages = room / (kWarps * p->block_bytes);
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    const int smem = kWarps * a.stages * p->block_bytes;
    const int grid = h->num_sms * ctas;
    // A share takes in at least 1 / 32 of the columns (1 / 8 for many rows, whose parts are large): joining costs more than it
    // brings beyond that.
    const int most = kNt == 1 ? 32 : 8;
    a.share = (a.units + grid - 1) / grid;
    if (a.share < (a.k_blocks + most - 1) / most) a.share = (a.k_blocks + most - 1) / most;
    QTZ_CUDA(h, cudaFuncSetAttribute(linear_kernel<T, kNt, kFine, kZero>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    linear_kernel<T, kNt, kFine, kZero><<<(a.units + a.share - 1) / a.share, kThreads, smem, st>>>(a);
    QTZ_LAUNCH_CHECK(h, "linear_kernel");
    return QTZ_OK;
}

template <typename T, int kNt>
qtz_status launch_kind(qtz_linear* p, LinearArgs& a, bool zero, cudaStream_t st)
{
    if (p->scales == 8) return zero ? launch<T, kNt, true, true>(p, a, st) : launch<T, kNt, true, false>(p, a, st);
    return zero ? launch<T, kNt, false, true>(p, a, st) : launch<T, kNt, false, false>(p, a, st);
}

template <typename T>
qtz_status launch_rows(qtz_linear* p, LinearArgs& a, bool zero, cudaStream_t st)
{
    if (a.rows <= 8) return launch_kind<T, 1>(p, a, zero, st);
    if (a.rows <= 16) return launch_kind<T, 2>(p, a, zero, st);
    return launch_kind<T, 4>(p, a, zero, st);
}

// Scratch of the joining, shared by the layers of a handle: parts and counters of a full grid.
qtz_status ensure_scratch(qtz_ctx* h, cudaStream_t st)
{
    if (h->linear_dev) return QTZ_OK;
    const int ctas = 2 * h->num_sms;
    // 16 rows run with two CTAs an SM, 32 with one: the same size
    const size_t parts = static_cast<size_t>(ctas) * 2 * kWarps * kRowTile * (kMaxTokens / 2) * sizeof(float);
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
    p->scales = d.group == 32 ? 8 : d.group % 256 == 0 ? 1 : d.group % 128 == 0 ? 2 : 4;
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

// Linear layers in 8-bit floating point: e4m3 activations with a scale for each row and 128 columns, e4m3 weights with a scale for each
// block of 128 x 128.
//
// Mathematics.  y[r][o] = sum_b x_scale[r][b] w_scale[o / 128][b] sum_{k in b} x[r][k] w[o][k] + bias[o].
// The inner sums are products of the tensor cores (tcgen05 kind::f8f6f4: exact products, fp32 sums; of 32 columns taken together, what lies
// 2^-25 below the largest is cut off, as measured with products of 200704 and 2^-9).  Scales differ from block to block, so that each
// block's product leaves tensor memory and is added, times its factor, to fp32 sums in registers: 128 of them a thread, which owns a row
// of x and 128 weights and so needs one factor a block.
//
// What bounds it.  Few rows: the weights' bytes.  Many: the tensor cores take 512 cycles for a block of a pair's 256 x 256 tile, reading
// it from tensor memory and adding it takes the eight warps of a CTA about as long, half of the fp32 pipe's time, and the two work on
// alternate buffers.  Measured, in cycles a block: products and loads alone 520, with the reading 548, with the sums 700 to 800 (the
// buffer comes back after the first half has been added: registers hold no more); the tensor pipe is 68 % busy.  Steps
// that counted: arrivals at the other CTA without release order (the fence took 1000 cycles a block); one warp to load, one for scales,
// two for products, so that no wait stands behind another; scales counted on the product's own barrier; the next block's barrier polled
// and its first half asked for behind this block's sums; rows of y that leave shared memory by copies while the next tile begins (stores by
// the threads: 8192 rows 1585 us instead of 1535, 2048 rows through 8192 x 512 18.8 instead of 15.9); fp32 operations in pairs.  Tried and
// left: halves of 128 columns with four buffers (the same), single CTAs of 128 x 256 (1090 cycles: shared memory brings and reads 192
// bytes a clock), tiles dealt out block by block with parts in global memory (128 KB a part: 33 -> 55 us for 256 x 8192 -> 10240),
// a launch of clusters for the tiles beyond whole rounds (a launch and a join cost 10 us: 777 rows through 11008 x 4096 49.8 -> 53.0).
// Measured (the figures above: when the step they name was taken), device time of ten calls in a CUDA graph, layers in turn that
// do not fit the L2 together, bf16 y but as said: 8192 rows through 28672 x 8192 1.6 ms, 2.4 PFLOP/s,
// in the first calls and 1.8 ms under the power cap; 1777 rows through 6144 x 4096 47 us (three rounds of 74 pairs for 2.3 of tiles); 256
// rows through 10240 x 8192 28.6 us (54 tiles of 192 weights for 74 pairs); 45 rows through 5003 x 10001, fp16 with bias, 14.6 us (12.4
// with the weights in the L2); one row through 28672 x 8192 38 us, 6.2 TB/s; one row through 1000 x 1024, fp16 with bias, 4.4 us.  Rows of y
// that do not start on 16 bytes leave value by value: 2048 rows through 5003 x 4096 65 us, through 5008 x 4096 43.
#include <new>

#include "qtz_f8.cuh"
#include "qtz_plan.cuh"
#include "qtz_ptx.cuh"

struct qtz_f8_layer {
    qtz_ctx* h = nullptr;
    int device = 0;                    // a plan may be destroyed after its handle
    int32_t n = 0, k = 0;
    int32_t n_tiles = 0, k_blocks = 0; // of 128 rows, of 128 columns
    uint8_t* tiles = nullptr;          // [n_tiles / 2, rounded up][k_blocks][256][128] codes, zeros beyond k; what lies beyond n is not used
    float* scales = nullptr;           // [n_tiles][k_blocks], behind the tiles in the same allocation
    float* bias = nullptr;             // [n], behind the scales; null: none
    CUtensorMap w_map{}, w_map_32{};   // the tiles as rows of 128 bytes, 128 and 32 rows at a time
};

namespace {

using namespace qtz_ptx;
struct PackArgs {
    const uint8_t* codes;
    int64_t stride;
    int32_t n, k, k_blocks, vector;
    uint8_t* tiles;
};

// A CTA a block of 128 x 128; rows that start on 16 bytes (`vector`) are read so.
__global__ void __launch_bounds__(256) pack_kernel(const __grid_constant__ PackArgs a)
{
    const int64_t place = (static_cast<int64_t>(blockIdx.y / 2) * a.k_blocks + blockIdx.x) * 2 + blockIdx.y % 2;
    uint4* const tile = reinterpret_cast<uint4*>(a.tiles + place * (kF8Block * kF8Block));
    for (int i = threadIdx.x; i < kF8Block * kF8Block / 16; i += 256) {
        const int64_t row = static_cast<int64_t>(blockIdx.y) * kF8Block + i / 8;
        const int col = blockIdx.x * kF8Block + i % 8 * 16, valid = row < a.n ? a.k - col : 0;
        const uint8_t* const from = a.codes + row * a.stride + col;
        uint32_t w[4] = {};
        if (a.vector && valid >= 16) {
            tile[i] = *reinterpret_cast<const uint4*>(from);
            continue;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (e < valid) w[e / 4] |= static_cast<uint32_t>(from[e]) << (e % 4 * 8);
        tile[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

__global__ void bias_kernel(const void* bias, int32_t ftype, float* out, int32_t n)
{
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) out[i] = qtz_dev::load_real(bias, i, ftype);
}

struct LinearArgs {
    const float *w_scales, *bias, *x_scales;
    int64_t row_stride, block_stride, rows, y_stride;
    void* y;
    int32_t n, n_tiles, k_blocks, ftype;
    int32_t vector;            // rows of y start on 16 bytes
    int32_t row_tiles;         // tiles of activation rows
    int32_t tiles;             // in all
    int32_t split;             // CTAs or pairs of a cluster, which share the columns of a tile
    long long wait_budget;
    int32_t* status;
};

constexpr int kThreads = 384, kSumThreads = 256;         // loads, products (two warps), scales; eight warps for the sums
constexpr int kLaunchRegs = 168, kFew = 80, kMany = 208;   // registers of a thread: at launch, of the first four warps, of the others
static_assert(4 * 32 * kFew + 8 * 32 * kMany <= kThreads * kLaunchRegs, "more registers than the CTA was launched with");
constexpr int kTileBytes = kF8Block * kF8Block;
constexpr int kSmemLimit = 227 * 1024;
constexpr int kMaxStages = 12;
// Descriptor of the products: fp32 sums of e4m3 x e4m3, kN columns, kM rows.
template <int kM, int kN>
constexpr uint32_t kProduct = (1u << 4) | (static_cast<uint32_t>(kN >> 3) << 17) | (static_cast<uint32_t>(kM >> 4) << 24);

__device__ __forceinline__ void timed_out(const LinearArgs& a)
{
    if (atomicCAS(a.status, 0, QTZ_ERR_DEVICE_TIMEOUT) == 0) a.status[1] = QTZ_SITE_F8_LINEAR;
}

__device__ __forceinline__ void put(const LinearArgs& a, int64_t at, float v)
{
    if (a.ftype == QTZ_BF16) static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
    else if (a.ftype == QTZ_F16) static_cast<__half*>(a.y)[at] = __float2half_rn(v);
    else static_cast<float*>(a.y)[at] = v;
}

// (x, y) += (u, v) * (s, t), two fp32 sums in one operation.
__device__ __forceinline__ void fma2(float& x, float& y, float u, float v, float s, float t)
{
    unsigned long long sums, values, factors;
    asm("mov.b64 %0, {%1, %2};" : "=l"(sums) : "f"(x), "f"(y));
    asm("mov.b64 %0, {%1, %2};" : "=l"(values) : "f"(u), "f"(v));
    asm("mov.b64 %0, {%1, %2};" : "=l"(factors) : "f"(s), "f"(t));
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(sums) : "l"(values), "l"(factors));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(sums));
}

__device__ __forceinline__ float bias_of(const LinearArgs& a, int o) { return a.bias && o < a.n ? __ldg(a.bias + o) : 0.f; }

template <typename T>
__device__ __forceinline__ uint4 pack16(const float* v)
{
    if constexpr (sizeof(T) == 4) return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    else return make_uint4(qtz_dev::pack2(v[0], v[1], T()), qtz_dev::pack2(v[2], v[3], T()), qtz_dev::pack2(v[4], v[5], T()), qtz_dev::pack2(v[6], v[7], T()));
}

constexpr int kOutBytes = 2048;        // of a warp's values on their way out: 32 rows of 64 bytes

// A warp's `rows` (at most 32) rows of kCols columns, of which `cols` exist; lane l holds row l, row r goes to to + r * stride.  64 bytes of
// each row at a time cross through `out`, so that neighbouring lanes write neighbouring values; pieces of 16 bytes are shifted by row, for
// the banks.  vector: rows start on 16 bytes.
template <typename T, int kCols>
__device__ __forceinline__ void put_rows(T* to, int64_t stride, int rows, int cols, bool vector, uint4* out, const float (&acc)[kCols])
{
    constexpr int kPer = 16 / sizeof(T), kStep = 64 / sizeof(T);
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int c0 = 0; c0 < kCols; c0 += kStep) {
        const int here = min(kStep, cols - c0);
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 4; ++q) out[lane * 4 + (q ^ (lane >> 1 & 3))] = pack16<T>(acc + c0 + q * kPer);
        __syncwarp();
        if (vector) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = i * 8 + (lane >> 2), q = lane & 3;
                const uint4* const from = out + r * 4 + (q ^ (r >> 1 & 3));
                T* const at = to + r * stride + c0 + q * kPer;
                if (r < rows && q * kPer + kPer <= here) *reinterpret_cast<uint4*>(at) = *from;
                else if (r < rows)
                    for (int e = 0; e < here - q * kPer; ++e) at[e] = reinterpret_cast<const T*>(from)[e];
            }
        } else {
            for (int at = lane; at < rows * kStep; at += 32) {
                const int r = at / kStep, e = at % kStep;
                if (e < here) to[r * stride + c0 + e] = reinterpret_cast<const T*>(out + r * 4 + (e / kPer ^ (r >> 1 & 3)))[e % kPer];
            }
        }
    }
}

template <int kCols>
__device__ __forceinline__ void add_bias(const LinearArgs& a, int o, float (&acc)[kCols])
{
    if (!a.bias) return;
#pragma unroll
    for (int c = 0; c < kCols; ++c) acc[c] += bias_of(a, o + c);
}

// The same into y, from (row, o) on.
template <int kCols>
__device__ __forceinline__ void put_y(const LinearArgs& a, int64_t row, int o, uint4* out, const float (&acc)[kCols])
{
    const int rows = static_cast<int>(min(static_cast<int64_t>(32), a.rows - row)), cols = a.n - o;
    const int64_t at = row * a.y_stride + o;
    if (a.ftype == QTZ_BF16) put_rows(static_cast<__nv_bfloat16*>(a.y) + at, a.y_stride, rows, cols, a.vector, out, acc);
    else if (a.ftype == QTZ_F16) put_rows(static_cast<__half*>(a.y) + at, a.y_stride, rows, cols, a.vector, out, acc);
    else put_rows(static_cast<float*>(a.y) + at, a.y_stride, rows, cols, a.vector, out, acc);
}

// Rows leave by copies in `steps` steps each time, which fill two places in turn, the first one at the start.  How many of the last copies
// may still be reading when a step fills its place: the last but one had it before, or, at the start behind an odd number of steps,
// the last one.
__host__ __device__ constexpr int still_reading(int steps, int step) { return step == 0 && steps % 2 == 1 ? 0 : 1; }

// Whether no step, of two times in a row, fills a place that a copy may be reading.
__host__ __device__ constexpr bool places_are_free(int steps)
{
    for (int i = 0; i < 2 * steps; ++i)
        for (int j = i - 1; j >= 0 && j >= i - still_reading(steps, i % steps); --j)
            if (j % steps % 2 == i % steps % 2) return false;
    return true;
}

// 32 rows of kCols columns where rows of y start on 16 bytes, by copies that run on behind the caller: 64 bytes of each row at a time in the
// order of a 64-byte swizzle, in two places of `out` in turn.  Rows beyond the last the tensor map leaves out; of columns it would write whole
// pieces of 16 bytes.
template <typename T, int kCols>
__device__ __forceinline__ void send_rows(const CUtensorMap& y_map, int64_t row, int o, uint32_t out, const float (&acc)[kCols])
{
    constexpr int kPer = 16 / sizeof(T), kStep = 64 / sizeof(T), kSteps = kCols / kStep;
    static_assert(places_are_free(kSteps), "");
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int c0 = 0; c0 < kCols; c0 += kStep) {
        const uint32_t to = out + c0 / kStep % 2 * kOutBytes;
        if (lane == 0) {
            if (still_reading(kSteps, c0 / kStep) == 0) tma_store_wait_read();
            else tma_store_wait_read_n<1>();
        }
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 4; ++q) sts128(to + lane * 64 + (q ^ (lane >> 1 & 3)) * 16, pack16<T>(acc + c0 + q * kPer));
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            tma_store_2d(&y_map, to, (o + c0) * static_cast<int>(sizeof(T)), static_cast<int>(row));
            tma_store_commit();
        }
    }
}

// First row, among the packed tiles' rows, of half a tile of 256 weights.
__device__ __forceinline__ int w_row(const LinearArgs& a, int col, int kb, int half) { return ((col * a.k_blocks + kb) * 2 + half) * kF8Block; }

// The sums of a thread: a row of x and kCols weights.  Blocks' products are read from tensor memory as far as registers allow, 96 columns
// at once or 128 in halves, and added times the block's factor.  A block's buffer is given back when the last of them have been read, and the
// next block's first columns, whose barrier was polled meanwhile, are on their way before those are added.
template <int kCols>
struct Sums {
    static_assert(kCols == 96 || kCols == 128, "");
    static constexpr int kLate = kCols == 128 ? 64 : 0;                // the first columns that are added after the buffer was given back
    float acc[kCols];
    uint32_t v0[32], v1[32], v2[kCols == 96 ? 32 : 1];                 // columns on their way

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int c = 0; c < kCols; ++c) acc[c] = 0.f;
    }
    __device__ __forceinline__ void add(const uint32_t (&v)[32], int at, float s)
    {
#pragma unroll
        for (int c = 0; c < 32; c += 2) fma2(acc[at + c], acc[at + c + 1], __uint_as_float(v[c]), __uint_as_float(v[c + 1]), s, s);
    }
    __device__ __forceinline__ void landed()
    {
        tmem_ld_wait_for(v0);
        tmem_ld_tie(v1);
        if constexpr (kCols == 96) tmem_ld_tie(v2);
    }
    __device__ __forceinline__ void begin(uint32_t from)
    {
        tmem_ld_32x32(from, v0);
        tmem_ld_32x32(from + 32, v1);
        if constexpr (kCols == 96) tmem_ld_32x32(from + 64, v2);
    }
    // The block at `from`, whose first columns were asked for; factor(g): of columns 32 g on.  read() gives its buffer back; where `more`
    // holds, the next block's barrier is polled with poll() and waited for with wait(answer), and its first columns asked for at `next`.
    // False: that wait gave up.
    template <typename Factor, typename Read, typename Poll, typename Wait>
    __device__ __forceinline__ bool block(uint32_t from, Factor factor, bool more, uint32_t next, Read read, Poll poll, Wait wait)
    {
        landed();
        if constexpr (kLate > 0) {
            add(v0, 0, factor(0));
            tmem_ld_32x32(from + 64, v0);
            add(v1, 32, factor(1));
            tmem_ld_32x32(from + 96, v1);
            landed();
        }
        tc_fence_before();
        __syncwarp();
        read();
        const bool answer = more && poll();
        add(v0, kLate, factor(kLate / 32));
        if (more) {
            if (!wait(answer)) return false;
            tc_fence_after();
            tmem_ld_32x32(next, v0);
        }
        add(v1, kLate + 32, factor(kLate / 32 + 1));
        if (more) tmem_ld_32x32(next + 32, v1);
        if constexpr (kCols == 96) {
            add(v2, 64, factor(2));
            if (more) tmem_ld_32x32(next + 64, v2);
        }
        return true;
    }
};

// Places for the scales of blocks, and how many blocks ahead they are asked for.  A thread of the sums reads its block's factor a block
// early, so that the loads of a block's scales are counted with the product of the block before.
constexpr int kSlots = 8, kAhead = 4;

// ---- few rows: the weights stream past a tile of rows ----
// A tile is 128 rows of x, of which kRows are loaded (what the other rows of the product hold is not looked at), and 256 weights.  The CTAs
// of a cluster take equal parts of a tile's columns and join their sums through each other's shared memory.  A thread owns a row of x and
// half of the weights, which share a scale: one factor a thread and block of 128 columns.
constexpr int kMaxSplit = 8;           // CTAs of a cluster
constexpr int kTileCols = 256, kQuads = kTileCols / 4;

template <int kRows>
struct Stream {
    static constexpr int kStage = 2 * kTileBytes + kRows * kF8Block;
    static constexpr int kRoom = (kSmemLimit - 1024 - 8 * kOutBytes - kSlots * (kRows + 2) * 4 - 1024) / kStage, kStages = kRoom < kMaxStages ? kRoom : kMaxStages;
    static constexpr int kSmem = 1024 + kStages * kStage + 8 * kOutBytes;
};

// Four neighbouring sums.
__device__ __forceinline__ void put_quad(const LinearArgs& a, int64_t row, int o, float4 v)
{
    using qtz_dev::pack2;
    const int64_t to = row * a.y_stride + o;
    const float y[4] = {v.x + bias_of(a, o), v.y + bias_of(a, o + 1), v.z + bias_of(a, o + 2), v.w + bias_of(a, o + 3)};
    if (a.vector && o + 4 <= a.n) {
        if (a.ftype == QTZ_F32) *reinterpret_cast<float4*>(static_cast<float*>(a.y) + to) = make_float4(y[0], y[1], y[2], y[3]);
        else if (a.ftype == QTZ_F16) *reinterpret_cast<uint2*>(static_cast<__half*>(a.y) + to) = make_uint2(pack2(y[0], y[1], __half()), pack2(y[2], y[3], __half()));
        else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.y) + to) = make_uint2(pack2(y[0], y[1], __nv_bfloat16()), pack2(y[2], y[3], __nv_bfloat16()));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (o + e < a.n) put(a, to + e, y[e]);
    }
}

// Sums of a tile that the CTAs of a cluster hold in shared memory, [row][64 quads of columns], a quad at its number ^ (row % 32) (for the
// banks): each CTA takes an equal part of the quads and adds them up in the order of the columns.  Called by the warps of the sums.
__device__ __forceinline__ uint32_t quad_at(uint32_t base, int row, int quad) { return base + (row * kQuads + (quad ^ (row & 31))) * 16; }

__device__ __forceinline__ void join_cluster(const LinearArgs& a, int64_t row0, int col, uint32_t base, int part, int rank0, int rank_step)
{
    const int quads = static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(kF8Block), a.rows - row0))) * kQuads, end = (part + 1) * quads / a.split;
    // all of a quad's parts are on their way together
    for (int q = part * quads / a.split + static_cast<int>(threadIdx.x) - (kThreads - kSumThreads); q < end; q += kSumThreads) {
        const uint32_t at = quad_at(base, q / kQuads, q % kQuads);
        float4 p[kMaxSplit];
#pragma unroll
        for (int c = 0; c < kMaxSplit; ++c)
            if (c < a.split) p[c] = lds_cluster(mapa_shared(at, rank0 + c * rank_step));
        float4 v = p[0];
#pragma unroll
        for (int c = 1; c < kMaxSplit; ++c)
            if (c < a.split) v = make_float4(v.x + p[c].x, v.y + p[c].y, v.z + p[c].z, v.w + p[c].w);
        put_quad(a, row0 + q / kQuads, col * kTileCols + q % kQuads * 4, v);
    }
}

// A thread's 128 sums, of row `row` and columns half * 128 on, into that place.
__device__ __forceinline__ void keep_sums(const float (&acc)[128], uint32_t base, int row, int half)
{
#pragma unroll
    for (int c = 0; c < 128; c += 4) sts128(quad_at(base, row, half * 32 + c / 4), make_float4(acc[c], acc[c + 1], acc[c + 2], acc[c + 3]));
}

struct StreamTile {                    // row tiles of the same 256 weights follow each other
    int row, col;
    __device__ StreamTile(const LinearArgs& a, int tile) : row(tile % a.row_tiles), col(tile / a.row_tiles) {}
};

template <int kRows>
__global__ void __launch_bounds__(kThreads, 1)
stream_kernel(const __grid_constant__ LinearArgs a, const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map)
{
    using S = Stream<kRows>;
    extern __shared__ uint8_t smem_raw[];              // the ring: kRows rows of x, a tile of weights; then values on their way out
    __shared__ float s_x[kSlots][kRows], s_w[kSlots][2];               // scales
    __shared__ __align__(8) uint64_t s_full[kMaxStages], s_empty[kMaxStages], s_done[2], s_free[2], s_drain;
    __shared__ uint32_t s_tmem;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    // warps of the sums whose rows exist: those of a quarter of tensor memory take 32 rows
    const int quarters = static_cast<int>(min(static_cast<int64_t>(4), (a.rows + 31) / 32));
    if (tid == 0) {
        prefetch_tensormap(&w_map);
        prefetch_tensormap(&x_map);
        for (int i = 0; i < S::kStages; ++i) {
            mbar_init(smem_u32(&s_full[i]), 1);
            mbar_init(smem_u32(&s_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&s_done[i]), 2);        // the product; scales
            mbar_init(smem_u32(&s_free[i]), 2 * quarters);
        }
        mbar_init(smem_u32(&s_drain), 2);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(&s_tmem), 512);
        tmem_relinquish();
    }
    fence_barrier_init();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
    const int tile0 = blockIdx.x / a.split, step = gridDim.x / a.split, part = blockIdx.x % a.split;
    const int kb0 = part * a.k_blocks / a.split, kbs = (part + 1) * a.k_blocks / a.split - kb0, count = (a.tiles - 1 - tile0) / step * kbs + kbs;   // blocks
    bool ok = true;
    auto wait = [&](uint64_t& bar, int parity) { ok = mbar_wait_warp(smem_u32(&bar), parity, a.wait_budget, ok); };
    grid_launch_dependents();

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFew));
        if (warp == 0) {
            // ======== loads ========
            // Weights were there when the layer was made: a ring of them is asked for before all else is waited for.
            int stage = 0, round = 0, issued = 0;
            auto weights = [&](int col, int kb, int to_stage) {
                if (elect_one()) {
                    const uint32_t bar = smem_u32(&s_full[to_stage]), to = base + to_stage * S::kStage + kRows * kF8Block;
                    const bool both = 2 * col + 1 < a.n_tiles;
                    mbar_arrive_expect_tx(bar, both ? S::kStage : S::kStage - kTileBytes);
                    tma_load_2d(to, &w_map, bar, 0, w_row(a, col, kb, 0));
                    if (both) tma_load_2d(to + kTileBytes, &w_map, bar, 0, w_row(a, col, kb, 1));
                }
                __syncwarp();
            };
            const int early = min(S::kStages, kbs);
            for (int i = 0; i < early; ++i) weights(StreamTile(a, tile0).col, kb0 + i, i);
            grid_dependency_wait();
            for (int tile = tile0; ok && tile < a.tiles; tile += step) {
                const StreamTile at(a, tile);
                for (int kb = kb0; kb < kb0 + kbs; ++kb, ++issued) {
                    if (issued >= S::kStages) wait(s_empty[stage], (round & 1) ^ 1);
                    if (!ok) break;
                    if (issued >= early) weights(at.col, kb, stage);
                    if (elect_one()) tma_load_2d(base + stage * S::kStage, &x_map, smem_u32(&s_full[stage]), kb * kF8Block, at.row * kF8Block);
                    __syncwarp();
                    if (++stage == S::kStages) {
                        stage = 0;
                        ++round;
                    }
                }
            }
            // nothing may be in flight when the CTA ends, whatever has given up
            for (int j = max(0, issued - S::kStages); j < issued; ++j)
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&s_full[j % S::kStages]), (j / S::kStages) & 1, kDrainBudget)) && ok;
        } else if (warp == 1 || warp == 3) {
            // ======== products: a warp for the even blocks, one for the odd ones ========
            grid_dependency_wait();                        // no wait of this kernel begins to count before the kernel ahead of it has ended
            const int buffer = warp >> 1;
            int stage = buffer, round = 0;
            for (int i = buffer; i < count; i += 2) {
                wait(s_full[stage], round & 1);
                if (i >= 2) wait(s_free[buffer], (i >> 1 & 1) ^ 1);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t x = make_kmajor_desc(base + stage * S::kStage, 128), w = make_kmajor_desc(base + stage * S::kStage + kRows * kF8Block, 128);
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma_f8(tmem + buffer * 256, x + 2 * k, w + 2 * k, kProduct<128, 256>, k > 0);
                    mma_commit(smem_u32(&s_done[buffer]));
                    mma_commit(smem_u32(&s_empty[stage]));
                }
                __syncwarp();
                stage += 2;
                if (stage >= S::kStages) {
                    stage -= S::kStages;
                    ++round;
                }
            }
            if (elect_one()) mma_commit(smem_u32(&s_drain));   // the others may have given up on what is still running
            __syncwarp();
        } else if (warp == 2) {
            // ======== scales ========
            grid_dependency_wait();
            constexpr int kEach = (kRows + 31) / 32;
            int tile = tile0, kb = 0;
            const float* from[kEach + 1];              // rows of x; lanes 0 and 1: 128 weights
            for (int i = 0; i < count + kAhead; ++i) {
                const int now = i - kAhead;
                if (now >= 0) {
                    cp_async_wait<kAhead - 2>();       // the block's scales and the next one's
                    __syncwarp();
                    if (now >= 2) wait(s_done[now & 1], (now >> 1 & 1) ^ 1);
                    if (!ok) break;
                    if (lane == 0) mbar_arrive(smem_u32(&s_done[now & 1]));
                }
                if (i < count) {
                    if (kb == 0) {
                        const StreamTile at(a, tile);
                        const int64_t row0 = static_cast<int64_t>(at.row) * kF8Block + lane;
#pragma unroll
                        for (int j = 0; j < kEach; ++j) from[j] = a.x_scales + min(row0 + 32 * j, a.rows - 1) * a.row_stride + kb0 * a.block_stride;
                        from[kEach] = a.w_scales + static_cast<int64_t>(min(2 * at.col + (lane & 1), a.n_tiles - 1)) * a.k_blocks + kb0;
                    }
                    // The place held the scales of eight blocks ago, which have been used: the product of the block two behind that one, which
                    // waited for it, is done.
                    const int slot = i % kSlots;
#pragma unroll
                    for (int j = 0; j < kEach; ++j)
                        if (32 * j + lane < kRows) cp_async_4(smem_u32(&s_x[slot][32 * j + lane]), from[j] + kb * a.block_stride);
                    if (lane < 2) cp_async_4(smem_u32(&s_w[slot][lane]), from[kEach] + kb);
                    if (++kb == kbs) {
                        kb = 0;
                        tile += step;
                    }
                }
                cp_async_commit();
            }
            cp_async_wait<0>();
        }
        if (a.split > 1) {
            cluster_sync();
            cluster_sync();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kMany));
        if ((warp & 3) < quarters) {
            // ======== sums ========
            const int half = (warp - 4) >> 2, row_warp = (warp & 3) * 32, row_lane = min(row_warp + lane, kRows - 1);
            const uint32_t from = tmem + (static_cast<uint32_t>(warp & 3) << 21) + half * 128;
            uint4* const out = reinterpret_cast<uint4*>(smem_raw + (base - smem_u32(smem_raw)) + S::kStages * S::kStage + (warp - 4) * kOutBytes);
            grid_dependency_wait();                    // y may be what the kernel before reads
            Sums<128> sums;
            float s_next = 0.f;                        // the next block's factor: its scales are there with this block's
            int i = 0;
            for (int tile = tile0; ok && tile < a.tiles; tile += step) {
                wait(s_done[i & 1], i >> 1 & 1);
                if (!ok) break;
                tc_fence_after();
                sums.begin(from + (i & 1) * 256);
                sums.clear();
#pragma unroll 1
                for (int kb = 0; kb < kbs; ++kb, ++i) {
                    const float s = i ? s_next : s_x[0][row_lane] * s_w[0][half];
                    s_next = s_x[(i + 1) % kSlots][row_lane] * s_w[(i + 1) % kSlots][half];
                    const uint32_t next_done = smem_u32(&s_done[(i + 1) & 1]), next_parity = (i + 1) >> 1 & 1;
                    ok = sums.block(from + (i & 1) * 256, [&](int) { return s; }, kb + 1 < kbs, from + ((i + 1) & 1) * 256,
                                    [&]() { if (lane == 0) mbar_arrive(smem_u32(&s_free[i & 1])); },
                                    [&]() { return mbar_try_wait(next_done, next_parity); },
                                    [&](bool answer) { return mbar_wait_warp_polled(answer, next_done, next_parity, a.wait_budget, true); });
                    if (!ok) break;
                }
                if (!ok) break;
                const StreamTile at(a, tile);
                if (a.split == 1) {
                    const int o = at.col * kTileCols + half * 128;
                    add_bias(a, o, sums.acc);
                    put_y(a, static_cast<int64_t>(at.row) * kF8Block + row_warp, o, out, sums.acc);
                } else if (row_warp + lane < kRows) keep_sums(sums.acc, base, row_warp + lane, half);   // the ring is free: the cluster's only tile is done
            }
        }
        if (a.split > 1) {
            const StreamTile at(a, tile0);
            cluster_sync();                            // the cluster's sums are there
            join_cluster(a, static_cast<int64_t>(at.row) * kF8Block, at.col, base, part, 0, 1);
            cluster_sync();                            // and have been read
        }
    }
    if (!ok) timed_out(a);
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        (void)mbar_wait(smem_u32(&s_drain), 0, kDrainBudget);
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// ---- many rows: CTA pairs on tiles of 256 rows of x and kCols weights ----
// Each CTA of a pair holds 128 of the rows and half of the weights; its half of the product, 128 rows x kCols columns, lies in its own
// tensor memory, twice, so that one block of 128 columns is multiplied while the sums of the one before are taken.  A thread owns a row
// of x and half of the columns.  Of 256 these share a scale of the weights: one factor a thread and block.  A tile of 192 begins with a
// scale or in the middle of one, and meets two.
template <int kCols>
struct Pair {
    static constexpr int kHalf = kCols / 2, kStage = kTileBytes + kHalf * kF8Block;
    static constexpr int kStages = kCols == 256 ? 5 : 6;              // what the rows on their way to y leave room for
    static constexpr int kSmem = 1024 + kStages * kStage + 8 * 2 * kOutBytes;
    // Blocks that scales are asked for ahead, in a place whose factors have been used when the arrivals were made that the wait before rests
    // on: those arrivals say that tensor memory has been read, and are no order for reads of shared memory.  128 columns use a block's factors
    // before they give its buffer back, 96 behind that.
    static constexpr int kScalesAhead = kCols == 256 ? kAhead : kAhead - 1;
    // The wait is for the product two blocks before the one whose scales have landed, and that began when the block two before it was read.
    static_assert(kScalesAhead + 4 + (kCols == 256 ? 0 : 1) <= kSlots, "");
    // registers of a thread; those of 96 columns are all read at once
    static constexpr int kFewRegs = kCols == 256 ? kFew : 56, kManyRegs = kCols == 256 ? kMany : 224;
    static_assert(4 * 32 * kFewRegs + 8 * 32 * kManyRegs <= kThreads * kLaunchRegs, "more registers than the CTA was launched with");
};
constexpr int kBand = 16;              // row tiles that the pairs work on side by side, for the L2

struct PairTile {
    int row, col;                      // in tiles
    __device__ PairTile(const LinearArgs& a, int tile)
    {
        const int cols = a.tiles / a.row_tiles, band = tile / (kBand * cols), rest = tile - band * kBand * cols;
        const int tall = min(kBand, a.row_tiles - band * kBand);
        col = rest / tall;
        row = band * kBand + rest % tall;
    }
};

// Called by all threads of a cluster in which a wait has run out, when nothing else is left to do: no load may be on its way when the CTAs
// end.  `issued`, of the first thread: blocks whose loads its CTA has asked for.  All of a pair's are counted on the first CTA's barriers
// `full`.  One side may have asked for blocks that the other did not: for no more than there are stages, since a stage is filled
// again only behind the product of both sides' last loads.  Their barriers are given what they lack.  counts: two places in shared memory.
// Not inlined: between the last barrier and the end of pair_kernel it took 0.7 us of calls in which nothing runs out
// (256 x 8192 -> 10240, 28.6 -> 29.4 us).
__device__ __noinline__ void drain_pair(uint32_t full, uint32_t* counts, int issued, int stages, uint32_t stage_bytes)
{
    const uint32_t rank = cluster_ctarank(), side = rank & 1;
    if (threadIdx.x == 0) sts_cluster(mapa_shared(smem_u32(counts + side), rank & ~1u), static_cast<uint32_t>(issued));
    cluster_sync();
    if (side == 0 && threadIdx.x < 32) {
        const int mine = static_cast<int>(counts[0]), theirs = static_cast<int>(counts[1]), most = max(mine, theirs);
        if (threadIdx.x == 0)
            for (int j = min(mine, theirs); j < most; ++j) {
                if (mine < theirs) mbar_arrive_expect_tx(full + j % stages * 8, stage_bytes);
                else mbar_complete_tx(full + j % stages * 8, stage_bytes);
            }
        __syncwarp();
        for (int j = max(0, most - stages); j < most; ++j) (void)mbar_wait(full + j % stages * 8, (j / stages) & 1, kDrainBudget);
        __syncwarp();
    }
    cluster_sync();                                    // the other CTA's are waited for here too
}

template <int kCols>
__global__ void __launch_bounds__(kThreads, 1)
pair_kernel(const __grid_constant__ LinearArgs a, const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map,
            const __grid_constant__ CUtensorMap y_map)
{
    using P = Pair<kCols>;
    constexpr int kHalf = P::kHalf, kPairStage = P::kStage, kPairStages = P::kStages;
    extern __shared__ uint8_t smem_raw[];              // the ring: a tile of x, half a tile of weights; then values on their way out
    __shared__ float s_x[kSlots][kF8Block], s_w[kSlots][2];            // scales
    __shared__ __align__(8) uint64_t s_full[kPairStages], s_empty[kPairStages], s_done[2], s_free[2], s_drain;
    __shared__ uint32_t s_tmem, s_gave_up, s_issued[2];                // a wait of the cluster has run out; drain_pair
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u, rank = cluster_ctarank(), side = rank & 1, first = rank & ~1u;
    if (tid == 0) {
        s_gave_up = 0;
        prefetch_tensormap(&w_map);
        prefetch_tensormap(&x_map);
        if (a.vector) prefetch_tensormap(&y_map);
        for (int i = 0; i < kPairStages; ++i) {
            mbar_init(smem_u32(&s_full[i]), 1);
            mbar_init(smem_u32(&s_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&s_done[i]), 2);
            mbar_init(smem_u32(&s_free[i]), 16);
        }
        mbar_init(smem_u32(&s_drain), 2);
    }
    if (warp == 1) {
        tmem_alloc_pair(smem_u32(&s_tmem), 512);
        tmem_relinquish_pair();
    }
    fence_barrier_init();
    tc_fence_before();
    __syncthreads();
    cluster_sync();                                    // both CTAs' barriers are there
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
    // the pairs of a cluster share the columns of a tile
    const int tile0 = blockIdx.x / (2 * a.split), step = gridDim.x / (2 * a.split), part = rank >> 1;
    const int kb0 = part * a.k_blocks / a.split, kbs = (part + 1) * a.k_blocks / a.split - kb0;
    bool ok = true;
    int issued = 0;                                    // blocks whose loads this side has asked for
    grid_launch_dependents();

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(P::kFewRegs));
        if (warp == 0) {
            // ======== loads: both CTAs' are counted on the first one's barrier ========
            int stage = 0, round = 0;
            auto weights = [&](int col, int kb, int to_stage) {
                if (elect_one()) {
                    const uint32_t own = smem_u32(&s_full[to_stage]), bar = mapa_shared(own, first), to = base + to_stage * kPairStage + kTileBytes;
                    if (side == 0) mbar_arrive_expect_tx(own, 2 * kPairStage);
                    if constexpr (kCols == 256) {
                        tma_load_2d_pair(to, &w_map, bar, 0, w_row(a, col, kb, min(static_cast<int>(side), a.n_tiles - 1 - 2 * col)));
                    } else {                           // 32 weights lie in one packed tile; beyond the last tile they read as zero
#pragma unroll
                        for (int i = 0; i < kHalf; i += 32) {
                            const int o = col * kCols + static_cast<int>(side) * kHalf + i;
                            tma_load_2d_pair(to + i * kF8Block, &w_map, bar, 0, w_row(a, o / 256, kb, 0) + o % 256);
                        }
                    }
                }
                __syncwarp();
            };
            const int early = min(kPairStages, kbs);
            for (int i = 0; i < early; ++i) weights(PairTile(a, tile0).col, kb0 + i, i);
            grid_dependency_wait();
            for (int tile = tile0; ok && tile < a.tiles; tile += step) {
                const PairTile at(a, tile);
                const int x_row = (2 * at.row + static_cast<int>(side)) * kF8Block;
                for (int kb = kb0; kb < kb0 + kbs; ++kb, ++issued) {
                    if (issued >= kPairStages) ok = mbar_wait_warp(smem_u32(&s_empty[stage]), (round & 1) ^ 1, a.wait_budget, ok);
                    if (!ok) break;
                    if (issued >= early) weights(at.col, kb, stage);
                    if (elect_one()) tma_load_2d_pair(base + stage * kPairStage, &x_map, mapa_shared(smem_u32(&s_full[stage]), first), kb * kF8Block, x_row);
                    __syncwarp();
                    if (++stage == kPairStages) {
                        stage = 0;
                        ++round;
                    }
                }
            }
        } else if (warp != 2) {
            // ======== products: a warp for the even blocks, one for the odd ones ========
            grid_dependency_wait();                        // no wait of this kernel begins to count before the kernel ahead of it has ended
            const int blocks = side == 0 ? (a.tiles - 1 - tile0) / step * kbs + kbs : 0, buffer = warp >> 1;
            int stage = buffer, round = 0;
            for (int block = buffer; block < blocks; block += 2) {
                ok = mbar_wait_warp(smem_u32(&s_full[stage]), round & 1, a.wait_budget, ok);
                if (block >= 2) ok = mbar_wait_warp(smem_u32(&s_free[buffer]), (block >> 1 & 1) ^ 1, a.wait_budget, ok);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t x = make_kmajor_desc(base + stage * kPairStage, 128), w = make_kmajor_desc(base + stage * kPairStage + kTileBytes, 128);
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma_f8_pair(tmem + buffer * 256, x + 2 * k, w + 2 * k, kProduct<256, kCols>, k > 0);
                    mma_commit_pair(smem_u32(&s_done[buffer]), first);
                    mma_commit_pair(smem_u32(&s_empty[stage]), first);
                }
                __syncwarp();
                stage += 2;
                if (stage >= kPairStages) {
                    stage -= kPairStages;
                    ++round;
                }
            }
            if (side == 0 && elect_one()) mma_commit_pair(smem_u32(&s_drain), first);
            __syncwarp();
        } else if (warp == 2) {
            // ======== scales: on their way three or four blocks ahead, counted with the products of the block ========
            grid_dependency_wait();
            const int blocks = (a.tiles - 1 - tile0) / step * kbs + kbs;
            int tile = tile0, kb = 0;
            const float* from[5];                      // four rows of x; lanes 0 and 1: a tile of weights
            for (int block = 0; block < blocks + P::kScalesAhead; ++block) {
                const int now = block - P::kScalesAhead;
                if (now >= 0) {
                    cp_async_wait<P::kScalesAhead - 2>();
                    __syncwarp();
                    if (now >= 2) ok = mbar_wait_warp(smem_u32(&s_done[now & 1]), (now >> 1 & 1) ^ 1, a.wait_budget, ok);
                    if (!ok) break;
                    if (lane == 0) mbar_arrive(smem_u32(&s_done[now & 1]));
                }
                if (block < blocks) {
                    if (kb == 0) {
                        const PairTile at(a, tile);
                        const int64_t row0 = (2 * static_cast<int64_t>(at.row) + side) * kF8Block + lane;
#pragma unroll
                        for (int j = 0; j < 4; ++j) from[j] = a.x_scales + min(row0 + 32 * j, a.rows - 1) * a.row_stride + kb0 * a.block_stride;
                        from[4] = a.w_scales + static_cast<int64_t>(min(at.col * kCols / kF8Block + (lane & 1), a.n_tiles - 1)) * a.k_blocks + kb0;
                    }
                    const int slot = block % kSlots;   // of the block eight before, whose factors have been used
#pragma unroll
                    for (int j = 0; j < 4; ++j) cp_async_4(smem_u32(&s_x[slot][32 * j + lane]), from[j] + kb * a.block_stride);
                    if (lane < 2) cp_async_4(smem_u32(&s_w[slot][lane]), from[4] + kb);
                    if (++kb == kbs) {
                        kb = 0;
                        tile += step;
                    }
                }
                cp_async_commit();
            }
            cp_async_wait<0>();
        }
        if (kCols == 256 && a.split > 1) {
            cluster_sync();
            cluster_sync();
        }
    } else {
        // ======== sums ========
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(P::kManyRegs));
        const int half = (warp - 4) >> 2, row_lane = (warp & 3) * 32 + lane;
        const uint32_t from = tmem + (static_cast<uint32_t>(warp & 3) << 21) + half * kHalf;
        uint4* const out = reinterpret_cast<uint4*>(smem_raw + (base - smem_u32(smem_raw)) + kPairStages * kPairStage + (warp - 4) * 2 * kOutBytes);
        grid_dependency_wait();
        Sums<kHalf> sums;
        int block = 0;
        // the next block's factors, of the scales that this thread's weights may meet: they are there with this block's
        constexpr int kFactors = kCols == 256 ? 1 : 2;
        float next[kFactors] = {};
        auto ask = [&](int slot) {
            const float x = s_x[slot][row_lane];
            if constexpr (kCols == 256) next[0] = x * s_w[slot][half];
            else {
                next[0] = x * s_w[slot][0];
                next[1] = x * s_w[slot][1];
            }
        };
        for (int tile = tile0; ok && tile < a.tiles; tile += step) {
            ok = mbar_wait_warp(smem_u32(&s_done[block & 1]), block >> 1 & 1, a.wait_budget, ok);
            if (!ok) break;
            tc_fence_after();
            sums.begin(from + (block & 1) * 256);
            sums.clear();
            // which of 32 weights each: the second scale of a tile of 192 begins after 128 of an even tile and 64 of an odd one
            const int col = PairTile(a, tile).col, second = (kF8Block - col * kCols % kF8Block - half * kHalf) / 32;
            if (block == 0) ask(0);
#pragma unroll 1
            for (int kb = 0; kb < kbs; ++kb, ++block) {
                float s[kFactors];
#pragma unroll
                for (int f = 0; f < kFactors; ++f) s[f] = next[f];
                ask((block + 1) % kSlots);
                const uint32_t next_done = smem_u32(&s_done[(block + 1) & 1]), next_parity = (block + 1) >> 1 & 1;
                ok = sums.block(from + (block & 1) * 256, [&](int g) { return g < second ? s[0] : s[kFactors - 1]; }, kb + 1 < kbs, from + ((block + 1) & 1) * 256,
                                [&]() { if (lane == 0) mbar_arrive_remote_relaxed(smem_u32(&s_free[block & 1]), first); },
                                [&]() { return mbar_try_wait(next_done, next_parity); },
                                [&](bool answer) { return mbar_wait_warp_polled(answer, next_done, next_parity, a.wait_budget, true); });
                if (!ok) break;
            }
            if (!ok) break;
            const PairTile at(a, tile);
            if (kCols == 256 && a.split > 1) {
                if constexpr (kCols == 256) keep_sums(sums.acc, base, row_lane, half);   // the ring is free: the cluster's only tile is done
            } else {
                const int64_t row = (2 * static_cast<int64_t>(at.row) + side) * kF8Block + row_lane - lane;
                const int o = at.col * kCols + half * kHalf;
                if (row >= a.rows || o >= a.n) continue;
                add_bias(a, o, sums.acc);
                if (!a.vector || o + kHalf > a.n) {
                    if (lane == 0) tma_store_wait_read();
                    put_y(a, row, o, out, sums.acc);
                } else if (a.ftype == QTZ_BF16) {
                    send_rows<__nv_bfloat16>(y_map, row, o, smem_u32(out), sums.acc);
                } else if (a.ftype == QTZ_F16) {
                    send_rows<__half>(y_map, row, o, smem_u32(out), sums.acc);
                } else {
                    send_rows<float>(y_map, row, o, smem_u32(out), sums.acc);
                }
            }
        }
        if (lane == 0) tma_store_wait_all();
        __syncwarp();
        if (kCols == 256 && a.split > 1) {
            const PairTile at(a, tile0);
            cluster_sync();                            // the cluster's sums are there
            join_cluster(a, (2 * static_cast<int64_t>(at.row) + side) * kF8Block, at.col, base, part, side, 2);
            cluster_sync();                            // and have been read
        }
    }
    if (!ok) {
        timed_out(a);
        for (int c = 0; c < 2 * a.split; ++c) sts_cluster(mapa_shared(smem_u32(&s_gave_up), c), 1u);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) (void)mbar_wait(smem_u32(&s_drain), 0, kDrainBudget);   // the products that the first CTA issued are done
    __syncthreads();
    cluster_sync();                                    // and no arrival of the other CTA is under way
    // Where no wait ran out, each block's loads landed before its product; where one did, they are waited for.
    if (s_gave_up) drain_pair(smem_u32(s_full), s_issued, issued, kPairStages, kPairStage);
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem, 512);
    }
}

// Asked for once a handle: how many clusters run at once.
qtz_status learn_clusters(qtz_ctx* h)
{
    if (h->f8_clusters[1]) return QTZ_OK;
    for (const void* kernel : {reinterpret_cast<const void*>(pair_kernel<256>), reinterpret_cast<const void*>(pair_kernel<192>), reinterpret_cast<const void*>(stream_kernel<16>), reinterpret_cast<const void*>(stream_kernel<32>),
                               reinterpret_cast<const void*>(stream_kernel<64>), reinterpret_cast<const void*>(stream_kernel<128>)}) {
        cudaFuncAttributes at;
        QTZ_CUDA(h, cudaFuncGetAttributes(&at, kernel));
        if (at.numRegs < kLaunchRegs) return QTZ_ERR_UNSUPPORTED;  // its warps would wait for registers that nobody gives back
    }
    const qtz_status s = qtz_allow_smem(h, stream_kernel<kF8Block>);
    if (s != QTZ_OK) return s;
    for (int c = 2; c <= kMaxSplit; ++c) {             // an SM holds one CTA of any of these kernels
        cudaLaunchAttribute size;
        size.id = cudaLaunchAttributeClusterDimension;
        size.val.clusterDim.x = c;
        size.val.clusterDim.y = size.val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(c);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = Stream<kF8Block>::kSmem;
        cfg.attrs = &size;
        cfg.numAttrs = 1;
        QTZ_CUDA(h, cudaOccupancyMaxActiveClusters(&h->f8_clusters[c], stream_kernel<kF8Block>, &cfg));
    }
    h->f8_clusters[1] = h->num_sms;
    return QTZ_OK;
}

template <typename K, typename... M>
qtz_status launch(qtz_ctx* h, K* kernel, const LinearArgs& a, int cluster, int ctas, int smem, cudaStream_t st, const M&... maps)
{
    const qtz_status s = qtz_allow_smem(h, kernel);
    if (s != QTZ_OK) return s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    QTZ_CUDA(h, cudaLaunchKernelEx(&cfg, kernel, a, maps...));
    return QTZ_OK;
}

template <int kRows>
qtz_status launch_stream(qtz_f8_layer* p, LinearArgs& a, const CUtensorMap& x_map, cudaStream_t st)
{
    qtz_ctx* h = p->h;
    a.row_tiles = static_cast<int32_t>((a.rows + kF8Block - 1) / kF8Block);
    a.tiles = a.row_tiles * ((a.n_tiles + 1) / 2);
    return launch(h, stream_kernel<kRows>, a, a.split, a.split * (a.split > 1 || a.tiles < h->num_sms ? a.tiles : h->num_sms), Stream<kRows>::kSmem, st, p->w_map, x_map);
}

// How many CTAs (pairs, with each = 2) of a cluster can share a tile's columns with all tiles at work at once; 1 where there are more tiles.
int most_split(const qtz_ctx* h, int64_t tiles, int each, int k_blocks)
{
    int split = 1;
    for (int c = 2; c * each <= kMaxSplit && c <= k_blocks; ++c)
        if (tiles <= h->f8_clusters[c * each]) split = c;
    return split;
}

template <int kCols>
qtz_status launch_pair(qtz_f8_layer* p, LinearArgs& a, const CUtensorMap& x_map, cudaStream_t st)
{
    const int size = a.ftype == QTZ_F32 ? 4 : 2;
    const uint64_t dims[2] = {static_cast<uint64_t>(a.n) * size, static_cast<uint64_t>(a.rows)}, strides[1] = {static_cast<uint64_t>(a.y_stride) * size};
    const uint32_t box[2] = {64, 32};
    CUtensorMap y_map{};
    if (a.vector && !qtz_encode_u8_map(&y_map, a.y, 2, dims, strides, box, 64)) a.vector = 0;   // rows too far apart for one
    qtz_ctx* h = p->h;
    a.row_tiles = static_cast<int32_t>((a.rows + 255) / 256);
    a.tiles = a.row_tiles * ((a.n + kCols - 1) / kCols);
    const int pairs = h->num_sms / 2;
    return launch(h, pair_kernel<kCols>, a, 2 * a.split, 2 * a.split * (a.split > 1 || a.tiles < pairs ? a.tiles : pairs), Pair<kCols>::kSmem, st,
                  kCols == 256 ? p->w_map : p->w_map_32, x_map, y_map);
}

}  // namespace

extern "C" qtz_status qtz_f8_linear_destroy(qtz_f8_linear_plan p)
{
    if (!p) return QTZ_ERR_INVALID_ARG;
    qtz_device_guard guard(p->device);
    if (p->tiles) cudaFree(p->tiles);
    (void)cudaGetLastError();
    delete p;
    return QTZ_OK;
}

extern "C" qtz_status qtz_f8_linear_create(qtz_handle h, int32_t n, int32_t k, const uint8_t* codes_dev, int64_t codes_stride, const float* scales_dev,
                                           const void* bias_dev, int32_t bias_ftype, qtz_f8_linear_plan* out, void* stream)
{
    if (!out) return QTZ_ERR_INVALID_ARG;
    *out = nullptr;
    if (!h || !codes_dev || !scales_dev || n <= 0 || k <= 0 || (n > 1 && codes_stride < k) || (bias_dev && !qtz_is_real(bias_ftype))) return QTZ_ERR_INVALID_ARG;
    const int64_t n_tiles = (static_cast<int64_t>(n) + kF8Block - 1) / kF8Block, k_blocks = (static_cast<int64_t>(k) + kF8Block - 1) / kF8Block;
    if (n_tiles > 65535 || n_tiles * k_blocks > (1 << 23)) return QTZ_ERR_TOO_LARGE;
    qtz_device_guard guard(h->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const qtz_status s = learn_clusters(h);
    if (s != QTZ_OK) return s;
    qtz_f8_layer* p = new (std::nothrow) qtz_f8_layer();
    if (!p) return QTZ_ERR_INVALID_ARG;
    p->h = h;
    p->device = h->device;
    p->n = n;
    p->k = k;
    p->n_tiles = static_cast<int32_t>(n_tiles);
    p->k_blocks = static_cast<int32_t>(k_blocks);
    const size_t blocks = static_cast<size_t>(n_tiles) * k_blocks, places = (static_cast<size_t>(n_tiles) + 1) / 2 * 2 * k_blocks, tile_bytes = places * kF8Block * kF8Block;
    cudaError_t e = cudaMalloc(reinterpret_cast<void**>(&p->tiles), tile_bytes + (blocks + n) * sizeof(float));
    if (e == cudaSuccess) {
        p->scales = reinterpret_cast<float*>(p->tiles + tile_bytes);
        e = cudaMemcpyAsync(p->scales, scales_dev, blocks * sizeof(float), cudaMemcpyDeviceToDevice, st);
    }
    if (e == cudaSuccess && bias_dev) {
        p->bias = p->scales + blocks;
        bias_kernel<<<(n + 255) / 256, 256, 0, st>>>(bias_dev, bias_ftype, p->bias, n);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) {
        const PackArgs a{codes_dev, codes_stride, n, k, p->k_blocks, qtz_aligned16(codes_dev) && (n == 1 || codes_stride % 16 == 0), p->tiles};
        pack_kernel<<<dim3(static_cast<unsigned>(k_blocks), static_cast<unsigned>(n_tiles)), 256, 0, st>>>(a);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);   // later calls may fetch the tiles before they wait for the stream
    const uint64_t dims[2] = {kF8Block, places * kF8Block}, strides[1] = {kF8Block};
    const uint32_t box[2] = {kF8Block, kF8Block}, box_32[2] = {kF8Block, 32};
    if (e == cudaSuccess && !(qtz_encode_u8_map(&p->w_map, p->tiles, 2, dims, strides, box, 128) && qtz_encode_u8_map(&p->w_map_32, p->tiles, 2, dims, strides, box_32, 128)))
        e = cudaErrorInvalidValue;
    if (e != cudaSuccess) {
        qtz_cuda_fail(h, e, "qtz_f8_linear_create");
        qtz_f8_linear_destroy(p);
        return QTZ_ERR_CUDA;
    }
    *out = p;
    return QTZ_OK;
}

extern "C" qtz_status qtz_f8_linear(qtz_f8_linear_plan p, const uint8_t* codes_dev, int64_t codes_stride, const float* scales_dev,
                                    int64_t scales_row_stride, int64_t scales_block_stride, int64_t rows, void* y_dev, int64_t y_stride,
                                    int32_t ftype, void* stream)
{
    if (!p || rows < 0 || !qtz_is_real(ftype)) return QTZ_ERR_INVALID_ARG;
    if (rows == 0) return QTZ_OK;
    if (!codes_dev || !scales_dev || !y_dev || (rows > 1 && (codes_stride < p->k || y_stride < p->n))) return QTZ_ERR_INVALID_ARG;
    if (!qtz_aligned16(codes_dev) || (rows > 1 && codes_stride % 16 != 0)) return QTZ_ERR_MISALIGNED;
    if (rows > 0x7fffff00 || (rows + 127) / 128 * p->n_tiles * p->k_blocks > 0x3fffffff) return QTZ_ERR_TOO_LARGE;   // counted in 32 bits
    qtz_ctx* h = p->h;
    qtz_device_guard guard(h->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    LinearArgs a{p->scales, p->bias, scales_dev, scales_row_stride, scales_block_stride, rows, y_stride, y_dev, p->n, p->n_tiles, p->k_blocks, ftype,
                 qtz_aligned16(y_dev) && (rows <= 1 || y_stride * (ftype == QTZ_F32 ? 4 : 2) % 16 == 0), 0, 0, 0, h->wait_budget, h->status_dev};
    // Up to 128 rows single CTAs, whose tiles those are.  More: a tile's block of 128 columns takes a pair 10 and a CTA about 13 units of time,
    // and the longest of either has so many of them (us, CTAs | pairs: 160 x 4096 -> 4096 13.8 | 14.8, 160 x 8192 -> 10240 42 | 33,
    // 800 x 10001 -> 5003 51 | 82, 512 x 4096 -> 6144 23 | 20); CTAs that take several tiles are slower than that (1777 x 4096 -> 4096 63 | 35).
    // A pair's block of 192 weights takes 9 units, so that such tiles are taken where the pairs are through with them in no more rounds
    // (us, 256 | 192: 256 x 8192 -> 10240, one round of either, 32.2 | 28.2; 777 x 4096 -> 11008, three rounds or four, 45.5 | 53) and
    // there are blocks enough to make up for a later start (256 x 4096 -> 11008 18.7 | 17.2, 200 x 1000 -> 12000 8.6 | 9.0).
    const int64_t cols = (p->n_tiles + 1) / 2, pair_tiles = (rows + 255) / 256 * cols, tiles = (rows + 127) / 128 * cols, pairs = h->num_sms / 2;
    const int pair_split = most_split(h, pair_tiles, 2, p->k_blocks), split = most_split(h, tiles, 1, p->k_blocks);
    const int64_t rounds = (pair_tiles + pairs - 1) / pairs, narrow_tiles = (rows + 255) / 256 * ((p->n + 191) / 192);
    const bool narrow = pair_split == 1 && p->k_blocks >= 16 && (narrow_tiles + pairs - 1) / pairs == rounds;
    const int64_t pair_blocks = rounds * ((p->k_blocks + pair_split - 1) / pair_split), blocks = (p->k_blocks + split - 1) / split;
    const bool pair = rows > 128 && (tiles > h->num_sms || (narrow ? 9 : 10) * pair_blocks < 13 * blocks);
    a.split = pair ? pair_split : split;
    const int box_rows = pair ? 128 : rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
    CUtensorMap x_map;                                 // columns beyond k and rows beyond the last read as zero
    const int64_t pitch = rows > 1 ? codes_stride : (p->k + 15) / 16 * 16;
    const uint64_t dims[2] = {static_cast<uint64_t>(p->k), static_cast<uint64_t>(rows)}, strides[1] = {static_cast<uint64_t>(pitch)};
    const uint32_t box[2] = {kF8Block, static_cast<uint32_t>(box_rows)};
    if (!qtz_encode_u8_map(&x_map, codes_dev, 2, dims, strides, box, 128)) return qtz_cuda_fail(h, cudaErrorInvalidValue, "tensor map of the activations");
    if (pair) return narrow ? launch_pair<192>(p, a, x_map, st) : launch_pair<256>(p, a, x_map, st);
    switch (box_rows) {
    case 16: return launch_stream<16>(p, a, x_map, st);
    case 32: return launch_stream<32>(p, a, x_map, st);
    case 64: return launch_stream<64>(p, a, x_map, st);
    default: return launch_stream<128>(p, a, x_map, st);
    }
}

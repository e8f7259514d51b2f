// Attention of new tokens over the paged 8-bit key/value cache, on the integer tensor cores.
//
// Mathematics.  For one query row q and one block with key scale s_k and value scale s_v the kernel holds, per token p,
//   t_p = (q . k_p) c log2(e) s_k + log2(s_v),      w_p = 2^(t_p - m),     m = running maximum of t
// so that w_p = s_v exp(logit_p) 2^-m carries the block's value scale: the sum over values is sum w_p v_p on the codes
// themselves, and the softmax's denominator is sum w_p / s_v.
// Both products have 8-bit codes on one side, which the tensor cores (kind::i8) read straight from the bytes that TMA
// brings in: nothing is converted.  The other side is split into base-256 digits, one operand column each:
//   q_row = 2^(e - 29) (d_3 2^24 + d_2 2^16 + d_1 2^8 + d_0)     e = exponent of the row's largest value, d in [-128, 127]
//   w_p   = 2^(m' - 31) (b_3 2^24 + b_2 2^16 + b_1 2^8 + b_0)    b in [0, 255]; m' = maximum of t over the tile, not the running one
// Integer sums are exact; a query's values lose 2^-29 of the row's largest at most (fp16 and bf16 are exact down to 2^-19 and 2^-22 of
// it), a weight 2^-32 of its tile's largest, which is 2^-25 of it for a whole tile.  Three digits, 22 bits, were not enough: a strong
// value of a query can meet codes of zero, so that the others decide, and weights count by their sum: a token of large weight and no
// value took 10^5 others out of y.  The sums are joined in fp32, a tile's times 2^(m' - m).
//
// One tile is 128 tokens of one key/value head against kRows query rows (heads of the group x new tokens):
//   S^T [128 tokens x 4 kRows] = K [128 x D] Q^T        a thread owns a token: logits, maximum, weights
//   O^T [D x 4 kRows]          = V^T [D x 128] W        a thread owns a column of the head: fp32 running sum
// with V read as it lies (the depth of the product along its rows).
//
// What bounds it: one token reads 2 D bytes a head for 4 D flops a query head: HBM, by a factor of 4 to 100 over the tensor
// cores.  So every byte is read once, and the work is cut for an even stream: the tiles of all (request, key/value head, row
// tile) items form one sequence that is dealt out in equal contiguous shares to a grid that fills the GPU once, whatever the
// lengths.  A producer warp streams a CTA's share through a ring of TMA boxes, several tiles ahead and across items.  Items
// that lie in more than one share are joined by the last CTA to arrive, in the order of the tiles, so that results do not
// depend on timing.
// Measured: 64 requests of 300 to 32768 tokens, 8 heads of 128, 4 query heads each: 160 us for 1.03 GB, 6.4 TB/s, 0.99 of the copy
// rate.  One request over 262143 tokens, 4 heads: 54.7 us for 268 MB, 4.9 TB/s: 6 us until the first tile, 8 for the two joins.  16
// requests with 5 new tokens and a window of 1024: 22.0 us for 24 MB, four tiles a CTA: all of it start, first use and joins.  Many new
// tokens a request are not what it is made for: 16 rows a pass over the keys, and all row tiles of a request go over the same tiles,
// masked ones included (4 requests of 500 to 900 tokens, 100 of them new: 83 us).
#include <cuda.h>

#include <type_traits>

#include "qtz_half_util.cuh"
#include "qtz_kv.cuh"
#include "qtz_plan.cuh"
#include "qtz_ptx.cuh"

namespace {

using namespace qtz_ptx;

constexpr int kMaxRequests = 8192;
constexpr int kTile = 128;                 // tokens of a tile: the rows of one matrix instruction
constexpr int kComputeWarps = 4;
constexpr int kComputeThreads = 32 * kComputeWarps;
constexpr int kThreads = kComputeThreads + 64;   // + one warp for TMA, one for the matrix instructions
constexpr int kMaxRows = 16;
constexpr int kMaxStages = 6;
constexpr int kMaxBoxes = 8;
constexpr uint32_t kNoBox = 0xffffffffu;   // in the place of a scale: a NaN that no arithmetic gives
constexpr int kSmemLimit = 227 * 1024;     // most that a CTA may ask for; an SM has 1 KB more, and each CTA costs 1 KB more than it asks for

struct AttnArgs {
    qtz_kv_cache c;
    const void* q;
    int64_t q_token_stride, q_head_stride;
    int32_t q_heads, group;
    const int32_t *starts, *lens;
    int32_t requests, tokens;
    const int32_t* table;
    int32_t width;
    float scale_log2;                      // softmax scale * log2(e)
    int32_t window;
    void* y;
    int64_t y_token_stride, y_head_stride;
    float* lse;
    int32_t* counters;                     // [CTAs][2] arrivals of parts at a group, [CTAs] of groups at an item (see the joining)
    float* parts;                          // [CTAs][2][kMaxRows * D + 4 kMaxRows]: sums, maxima, denominators; those of the joined group
    int32_t stages, box_shift;             // tokens of a box: 1 << box_shift
    int64_t wait_budget;
    int32_t* status;
};

// The sequence is dealt out by cost: a tile counts two units and the end of an item five, for the last sums, the output rows, the
// next queries and the refill behind them.  us with 1, 3, 5, 8 units, measured with row tiles of 5: 168, 161, 161, 161 for 64 requests of
// 300 to 32768 tokens, 8 key/value heads, 128 columns; 87, 75, 71, 71 for 256 of 100 to 1000 (62 with tiles of 4); 35.3 to 35.1 for 8 of
// 4000 to 16000.
constexpr int kTileUnits = 2, kItemUnits = 5;

struct RequestShape {
    int first, added;                      // rows of q
    int len, limit;                        // tokens; those that the table can hold
    int row_tiles, lo, hi, tiles;          // items per head; tiles [lo, hi) of the cache; tiles per item (at least one)

    __device__ __forceinline__ int item_units() const { return kTileUnits * tiles + kItemUnits; }
    // Tiles of the request's items that begin before unit `off` of the request.
    __device__ __forceinline__ int tiles_before(int off) const
    {
        const int item = off / item_units(), rest = off - item * item_units();
        return item * tiles + min(tiles, (rest + kTileUnits - 1) / kTileUnits);
    }
};

template <int kRows>
__device__ __forceinline__ RequestShape shape_of(const AttnArgs& a, int r)
{
    RequestShape s;
    s.first = min(max(a.starts[r], 0), a.tokens);
    s.added = min(max(a.starts[r + 1], s.first), a.tokens) - s.first;
    s.len = min(max(a.lens[r], 0), 0x7fffff00);
    s.limit = static_cast<int>(min(static_cast<int64_t>(s.len), static_cast<int64_t>(a.width) * a.c.block_tokens));
    s.row_tiles = static_cast<int>((static_cast<int64_t>(s.added) * a.group + kRows - 1) / kRows);
    const int begin = s.len - s.added + 1 - a.window;
    s.lo = a.window > 0 && begin > 0 ? begin / kTile : 0;
    s.hi = (s.limit + kTile - 1) / kTile;
    s.tiles = max(1, s.hi - s.lo);
    return s;
}

// What the warps of a CTA look up again and again: the requests from the one that its share begins in.
constexpr int kKnown = 16;
struct KnownRequests {
    int first;
    RequestShape s[kKnown];
};

// A place in the sequence of tiles.
template <int kRows>
struct Cursor {
    RequestShape s;
    int request, item, k;                  // item: (head, row tile) within the request; k: tile within the item
    uint32_t begin;                        // unit that the item's first tile begins at

    // The first tile that begins at or after `unit`, in the first known request.
    __device__ __forceinline__ void seek(const AttnArgs& a, const uint32_t* prefix, const KnownRequests& known, uint32_t unit)
    {
        request = known.first;
        s = known.s[0];
        const int off = static_cast<int>(unit - prefix[request]);
        item = off / s.item_units();
        begin = prefix[request] + item * s.item_units();
        k = (off - item * s.item_units() + kTileUnits - 1) / kTileUnits;
        if (k >= s.tiles) {
            k = s.tiles - 1;
            next(a, prefix, known);
        }
    }
    __device__ __forceinline__ void next(const AttnArgs& a, const uint32_t* prefix, const KnownRequests& known)
    {
        if (++k < s.tiles) return;
        k = 0;
        begin += s.item_units();
        if (++item < a.c.kv_heads * s.row_tiles) return;
        item = 0;
        do ++request; while (request < a.requests && prefix[request + 1] == prefix[request]);
        if (request - known.first < kKnown) s = known.s[request - known.first];
        else if (request < a.requests) s = shape_of<kRows>(a, request);
    }
    __device__ __forceinline__ int head() const { return item / s.row_tiles; }
    __device__ __forceinline__ int pos() const { return (s.lo + k) * kTile; }
};

__device__ __forceinline__ float ex2(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float lg2(float v)
{
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

__device__ __forceinline__ void st_shared_u8(uint32_t addr, uint32_t v)
{
    asm volatile("st.shared.u8 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

// The four digits' sums over 128 codes, each below 2^22
__device__ __forceinline__ float join_digits(uint32_t d0, uint32_t d1, uint32_t d2, uint32_t d3)
{
    const int hi = static_cast<int>(d3) * 256 + static_cast<int>(d2), lo = static_cast<int>(d1) * 256 + static_cast<int>(d0);
    return fmaf(static_cast<float>(hi), 65536.f, static_cast<float>(lo));
}

// The digits' sums of rows r0 to r0 + 3, as far as there are any.
template <int kRows>
__device__ __forceinline__ void load_digits(uint32_t taddr, int r0, uint32_t (&v)[16])
{
    if (kRows % 4 == 1 && r0 + 4 > kRows) tmem_ld_32x4(taddr + 4 * r0, v);
    else if (kRows % 4 == 2 && r0 + 4 > kRows) tmem_ld_32x8(taddr + 4 * r0, v);
    else tmem_ld_32x16(taddr + 4 * r0, v);
}

// What the compute threads know of an item: two of them, for the one at work and the next.
struct ItemInfo {
    float factor[kMaxRows];                // from a digit sum to a logit in base 2
    int32_t begin[kMaxRows], end[kMaxRows];
    int64_t out[kMaxRows];                 // offset of the row in y, -1 beyond the request's rows
    int64_t lse[kMaxRows];
    int32_t full_lo, full_hi;              // tokens that every row sees
};

// An item that lies in CTAs c0 .. c1 (c1 < 0: there is none).
struct OpenItem {
    int64_t out[kMaxRows], lse[kMaxRows];
    int c0, c1;
};

// Shared memory of a CTA beside the ring, the operands and the prefix sums.
struct Shared {
    float max[2][kComputeWarps][kMaxRows], sum[kMaxRows][kComputeWarps];
    // of each row, for each warp: the tile's maximum (0 for none), and what the sums so far and the tile's are multiplied by
    float origin[kComputeWarps][kMaxRows], keep[2][kComputeWarps][kMaxRows], gain[2][kComputeWarps][kMaxRows];
    ItemInfo item[2];
    float2 scales[kMaxStages][kMaxBoxes];  // (k, v) of each box; kNoBox: there is none
    uint64_t full[kMaxStages], empty[kMaxStages], sfull[2], pfull[2], ofull[2], qfull, drain;
    KnownRequests known;
    OpenItem open[2];                      // begun in an earlier CTA; going on in the next
    uint32_t scan[kThreads / 32], tmem;
    int last[2], failed, tiles;
};

template <typename T, int D, int kRows>
__global__ void __launch_bounds__(kThreads, D == 256 ? 1 : 2)
attention_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map)
{
    constexpr int kHalves = D > 128 ? 2 : 1;           // boxes along a row of the cache
    constexpr int kRowBytes = D < 128 ? D : 128;
    constexpr int kN = (4 * kRows + 15) / 16 * 16;     // operand columns: 4 row + digit
    constexpr int kRowsUp = (kRows + 3) / 4 * 4;
    constexpr int kBox = kTile * kRowBytes;            // K or V of one tile and half
    constexpr int kStage = 2 * kHalves * kBox;
    constexpr int kColumns = kN == 48 ? 64 : kN;       // of tensor memory: two buffers of S, two of each half of O
    constexpr int kUsed = (2 + 2 * kHalves) * kColumns, kTmemColumns = kUsed <= 64 ? 64 : kUsed <= 128 ? 128 : kUsed <= 256 ? 256 : 512;
    constexpr int kPart = kMaxRows * D + 4 * kMaxRows;
    constexpr uint32_t kMulK = (2u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(kN >> 3) << 17) | (static_cast<uint32_t>(kTile >> 4) << 24);
    constexpr uint32_t kMulV = (2u << 4) | (1u << 7) | (0u << 10) | (1u << 15) | (static_cast<uint32_t>(kN >> 3) << 17) | (128u >> 4 << 24);

    extern __shared__ __align__(1024) uint8_t smem[];  // the swizzle counts from multiples of 1 KB; nothing static lies before it
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t base = smem_u32(smem);
    const uint32_t off_p = a.stages * kStage, off_q = off_p + kN * 128, off_shared = off_q + kN * D, off_prefix = off_shared + (sizeof(Shared) + 15) / 16 * 16;
    uint32_t* const prefix = reinterpret_cast<uint32_t*>(smem + off_prefix);
    Shared& sh = *reinterpret_cast<Shared*>(smem + off_shared);
    KnownRequests& known = sh.known;

    if (tid == 0) {
        sh.open[0].c1 = sh.open[1].c1 = -1;
        sh.failed = sh.tiles = 0;
        prefetch_tensormap(&k_map);
        prefetch_tensormap(&v_map);
        for (int i = 0; i < kMaxStages; ++i) {
            mbar_init(smem_u32(&sh.full[i]), 1 + kMaxBoxes);   // the boxes' bytes; the scales of each lane
            mbar_init(smem_u32(&sh.empty[i]), 1);
        }
        mbar_init(smem_u32(&sh.sfull[0]), 1);
        mbar_init(smem_u32(&sh.sfull[1]), 1);
        mbar_init(smem_u32(&sh.ofull[0]), 1);
        mbar_init(smem_u32(&sh.ofull[1]), 1);
        mbar_init(smem_u32(&sh.drain), 1);
        mbar_init(smem_u32(&sh.pfull[0]), kComputeWarps);
        mbar_init(smem_u32(&sh.pfull[1]), kComputeWarps);
        mbar_init(smem_u32(&sh.qfull), kComputeWarps);
        fence_barrier_init();
    }
    if (warp == kComputeWarps + 1) {
        tmem_alloc(smem_u32(&sh.tmem), kTmemColumns);
        tmem_relinquish();
    }

    grid_launch_dependents();
    grid_dependency_wait();                            // everything up to here was this CTA's own

    // ---- units before each request: an exclusive prefix sum over the requests ----
    const int per = (a.requests + kThreads - 1) / kThreads;
    const int r_lo = min(tid * per, a.requests), r_hi = min(r_lo + per, a.requests);
    uint32_t mine = 0;
    RequestShape shape = {};                           // of the last of them: the only one up to kThreads requests
    for (int r = r_lo; r < r_hi; ++r) {
        shape = shape_of<kRows>(a, r);
        const uint32_t n = static_cast<uint32_t>(a.c.kv_heads) * shape.row_tiles * shape.item_units();
        prefix[r] = n;
        mine += n;
    }
    uint32_t scan = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, scan, off);
        if (lane >= off) scan += u;
    }
    if (lane == 31) sh.scan[warp] = scan;
    __syncthreads();
    uint32_t before = scan - mine, total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) before += sh.scan[w];
        total += sh.scan[w];
    }
    for (int r = r_lo; r < r_hi; ++r) {
        const uint32_t n = prefix[r];
        prefix[r] = before;
        before += n;
    }
    if (tid == 0) prefix[a.requests] = total;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;

    // No share is smaller than a tile: every CTA between an item's first and last has a part of it.
    const int all = static_cast<int>(total);
    // Share c begins at floor(all c / sharing), so that equal items whose number divides the grid begin with a share and need no
    // change of item within one (one request of 262143 tokens and 4 heads: 58 us against 63 with shares rounded up).
    const uint32_t sharing = min(gridDim.x, max(total / kTileUnits, 1u)), least = total / sharing, left = total - least * sharing;
    auto share_begin = [&](uint32_t c) { return c >= sharing ? all : static_cast<int>(c * least + c * left / sharing); };
    auto share_of = [&](uint32_t unit) { return static_cast<int>((static_cast<uint64_t>(unit + 1) * sharing - 1) / total); };
    const int u0 = share_begin(blockIdx.x), u1 = share_begin(blockIdx.x + 1);
    auto timed_out = [&]() {
        if (lane == 0 && atomicCAS(a.status, 0, QTZ_ERR_DEVICE_TIMEOUT) == 0) a.status[1] = QTZ_SITE_KV_ATTENTION;
    };
    if (u1 > u0) {
        int u = 0, v = a.requests;                     // the last request that begins at or before the share
        while (v - u > 1) {
            const int mid = (u + v) >> 1;
            if (prefix[mid] <= static_cast<uint32_t>(u0)) u = mid; else v = mid;
        }
        if (tid == 0) known.first = u;
        int tiles = 0;                                 // that begin in [u0, u1)
        for (int r = max(r_lo, u); r < r_hi && prefix[r] < static_cast<uint32_t>(u1); ++r) {
            if (per > 1) shape = shape_of<kRows>(a, r);
            if (r - u < kKnown) known.s[r - u] = shape;
            if (shape.row_tiles == 0) continue;
            const int end = static_cast<int>(min(prefix[r + 1], static_cast<uint32_t>(u1)) - prefix[r]);
            tiles += shape.tiles_before(end) - (r == u ? shape.tiles_before(u0 - static_cast<int>(prefix[r])) : 0);
        }
        if (tiles) atomicAdd(&sh.tiles, tiles);
    }
    __syncthreads();
    const int count = sh.tiles;
    Cursor<kRows> cur;
    if (count > 0) cur.seek(a, prefix, known, u0);

    if (count > 0 && warp == kComputeWarps) {
        // ======== producer: lane j brings box j of the tile, and its scales ========
        // Table entries are requested kAhead tiles before they are needed, and the scales travel like the boxes, by asynchronous
        // copies that the tile's barrier counts: the producer waits for no look-up (under load one takes longer than a tile).
        const int box_rows = 1 << a.box_shift, boxes = kTile >> a.box_shift;
        constexpr int kAhead = 4;
        int id[kAhead], offset[kAhead], head[kAhead];  // offset: within the block, -1 where there is nothing to bring
        auto request_entry = [&](int& e, int& o, int& h) {
            const int pos = cur.pos() + lane * box_rows;
            e = o = -1;
            h = cur.head();
            if (lane >= boxes || pos >= cur.s.limit) return;
            const int j = pos / a.c.block_tokens;
            o = pos - j * a.c.block_tokens;
            e = a.table[static_cast<int64_t>(cur.request) * a.width + j];
        };
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            id[j] = offset[j] = -1;
            head[j] = 0;
            if (j >= count) continue;
            if (j > 0) cur.next(a, prefix, known);
            request_entry(id[j], offset[j], head[j]);
        }
        int i = 0, stage = 0, round = 0;
        for (; i < count; ++i) {
            int row = -1;
            int64_t bh = 0;
            if (offset[0] >= 0) {
                if (id[0] < 0 || id[0] >= a.c.blocks) {
                    qtz_dev::report_invalid(a.status, QTZ_SITE_KV_ATTENTION);
                } else {
                    bh = static_cast<int64_t>(id[0]) * a.c.kv_heads + head[0];
                    row = static_cast<int>(bh * a.c.block_tokens + offset[0]);
                }
            }
#pragma unroll
            for (int j = 0; j + 1 < kAhead; ++j) {
                id[j] = id[j + 1];
                offset[j] = offset[j + 1];
                head[j] = head[j + 1];
            }
            id[kAhead - 1] = offset[kAhead - 1] = -1;
            if (i + kAhead < count) {
                cur.next(a, prefix, known);
                request_entry(id[kAhead - 1], offset[kAhead - 1], head[kAhead - 1]);
            }
            if (round > 0 && !__all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.empty[stage]), (round - 1) & 1, a.wait_budget))) {
                timed_out();
                break;
            }
            const uint32_t bar = smem_u32(&sh.full[stage]), dst = base + stage * kStage;
            if (lane < kMaxBoxes && row < 0) sh.scales[stage][lane] = make_float2(__uint_as_float(kNoBox), 0.f);
            const int have = __popc(__ballot_sync(0xffffffffu, row >= 0));
            __syncwarp();
            if (lane == 0) mbar_arrive_expect_tx(bar, have * box_rows * 2 * D);
            __syncwarp();
            if (row >= 0) {
                const uint32_t at = dst + lane * box_rows * kRowBytes, sc = smem_u32(&sh.scales[stage][lane]);
#pragma unroll
                for (int hh = 0; hh < kHalves; ++hh) tma_load_2d(at + hh * kBox, &k_map, bar, hh * 128, row);
#pragma unroll
                for (int hh = 0; hh < kHalves; ++hh) tma_load_2d(at + (kHalves + hh) * kBox, &v_map, bar, hh * 128, row);
                cp_async_4(sc, a.c.k_scale_dev + bh);
                cp_async_4(sc + 4, a.c.v_scale_dev + bh);
            }
            if (lane < kMaxBoxes) cp_async_arrive(bar);
            if (++stage == a.stages) {
                stage = 0;
                ++round;
            }
        }
        // nothing may be in flight when the CTA ends
        for (int j = max(0, i - a.stages); j < i; ++j)
            if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.full[j % a.stages]), (j / a.stages) & 1, kDrainBudget))) timed_out();
    } else if (count > 0 && warp == kComputeWarps + 1) {
        // ======== matrix instructions: S of the next tile is issued before O of this one ========
        int items = 0;
        bool ok = true;
        auto multiply_keys = [&](int i, const Cursor<kRows>& c) {
            const int stage = i % a.stages;
            if (i == 0 || c.k == 0) {
                ok = ok && __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.qfull), items & 1, a.wait_budget));
                ++items;
            }
            ok = ok && __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.full[stage]), (i / a.stages) & 1, a.wait_budget));
            if (!ok) return;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int hh = 0; hh < kHalves; ++hh)
#pragma unroll
                    for (int j = 0; j < kRowBytes / 32; ++j)
                        mma_i8(tmem + (i & 1) * kColumns, make_kmajor_desc(base + stage * kStage + hh * kBox, kRowBytes) + 2 * j,
                               make_kmajor_desc(base + off_q + hh * kN * kRowBytes, kRowBytes) + 2 * j, kMulK, hh + j > 0);
                mma_commit(smem_u32(&sh.sfull[i & 1]));
            }
            __syncwarp();
        };
        multiply_keys(0, cur);
        for (int i = 0; i < count && ok; ++i) {
            // A new item's queries come after this tile's weights: its S may not keep O waiting.
            bool fresh = false;
            if (i + 1 < count) {
                cur.next(a, prefix, known);
                fresh = cur.k == 0;
                if (!fresh) multiply_keys(i + 1, cur);
            }
            ok = ok && __all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.pfull[i & 1]), (i >> 1) & 1, a.wait_budget));
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
                const uint32_t v = base + (i % a.stages) * kStage + kHalves * kBox;
#pragma unroll
                for (int hh = 0; hh < kHalves; ++hh)
#pragma unroll
                    for (int j = 0; j < kTile / 32; ++j)
                        mma_i8(tmem + (2 + (i & 1) * kHalves + hh) * kColumns, make_mnmajor_desc(v + hh * kBox + j * 32 * kRowBytes, kRowBytes),
                               make_kmajor_desc(base + off_p, 128) + 2 * j, kMulV, j > 0);
                mma_commit(smem_u32(&sh.ofull[i & 1]));
                mma_commit(smem_u32(&sh.empty[i % a.stages]));
            }
            __syncwarp();
            if (fresh) multiply_keys(i + 1, cur);
        }
        if (!ok) timed_out();
        if (elect_one()) mma_commit(smem_u32(&sh.drain));   // the compute warps may have given up on what is still running
        __syncwarp();
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.drain), 0, kDrainBudget))) timed_out();
    } else if (count > 0) {
        // ======== compute: thread = token of S^T, then column of O^T ========
        bool ok = true;
        auto wait = [&](uint64_t& bar, int parity) {   // the warp goes on together
            ok = mbar_wait_warp(smem_u32(&bar), parity, a.wait_budget, ok);
        };
        // An item's query rows: warp w takes rows w, w + 4, ..  They are fetched a tile before they become the digits of the
        // operand, which is when the products of the item before are done with its rows.
        constexpr int kPer = D / 32;                   // values of a row that a lane holds
        constexpr int kMine = (kRows + kComputeWarps - 1) / kComputeWarps;
        uint32_t raw[kMine][kPer / 2];
        struct Row {
            int64_t token;
            int head, local;
            bool has;
        };
        auto row_of_lane = [&](const Cursor<kRows>& c) {   // lane r finds row r
            Row w;
            const int h = c.head(), index = (c.item - h * c.s.row_tiles) * kRows + lane;
            w.local = index / a.group;
            w.head = h * a.group + (index - w.local * a.group);
            w.has = lane < kRows && w.local < c.s.added;
            w.token = c.s.first + w.local;
            return w;
        };
        auto fetch_queries = [&](const Cursor<kRows>& c) {
            const Row w = row_of_lane(c);
            const int64_t from = w.has ? w.token * a.q_token_stride + w.head * a.q_head_stride : -1;
#pragma unroll
            for (int j = 0; j < kMine; ++j) {
                const int64_t at = __shfl_sync(0xffffffffu, from, warp + j * kComputeWarps);
                const T* q = static_cast<const T*>(a.q) + at + lane * kPer;
#pragma unroll
                for (int k = 0; k < kPer / 2; ++k) raw[j][k] = 0;
                if (at < 0) continue;                  // no lane from kRows on holds a row
                if constexpr (kPer == 2) {
                    raw[j][0] = *reinterpret_cast<const uint32_t*>(q);
                } else if constexpr (kPer == 4) {
                    const uint2 u = *reinterpret_cast<const uint2*>(q);
                    raw[j][0] = u.x; raw[j][1] = u.y;
                } else {
                    const uint4 u = *reinterpret_cast<const uint4*>(q);
                    raw[j][0] = u.x; raw[j][1] = u.y; raw[j][2] = u.z; raw[j][3] = u.w;
                }
            }
        };
        auto convert_queries = [&](const Cursor<kRows>& c, int which) {
            ItemInfo& it = sh.item[which];
            if (warp == 0) {
                const Row w = row_of_lane(c);
                const int own = c.s.len - c.s.added + w.local + 1;   // tokens up to the row's own
                const int end = w.has ? min(own, c.s.limit) : 0x7fffffff, begin = w.has && a.window > 0 ? max(0, own - a.window) : 0;
                if (lane < kRows) {
                    it.begin[lane] = begin;
                    it.end[lane] = end;
                    it.out[lane] = w.has ? w.token * a.y_token_stride + w.head * a.y_head_stride : -1;
                    it.lse[lane] = w.token * a.q_heads + w.head;
                }
                const int lo = __reduce_max_sync(0xffffffffu, begin), hi = __reduce_min_sync(0xffffffffu, end);
                if (lane == 0) {
                    it.full_lo = lo;
                    it.full_hi = hi;
                }
            }
#pragma unroll
            for (int j = 0; j < kMine; ++j) {
                const int r = warp + j * kComputeWarps;
                if (r >= kRows) break;
                float v[kPer], top = 0.f;
                bool odd = false;
#pragma unroll
                for (int k = 0; k < kPer / 2; ++k) {
                    const float2 f = qtz_dev::unpack2(raw[j][k], T());
                    v[2 * k] = f.x;
                    v[2 * k + 1] = f.y;
                }
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    odd = odd || (__float_as_uint(v[k]) & 0x7f800000u) == 0x7f800000u;
                    top = fmaxf(top, fabsf(v[k]));
                }
                top = redux_max(top);
                odd = __any_sync(0xffffffffu, odd);
                // rows below 2^-97 count as 2^-97 (their logits are zero either way)
                const int ex = min(max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -97), 127);
                const float mult = __uint_as_float(static_cast<uint32_t>(127 + 29 - ex) << 23);
                uint32_t bytes[kPer];                  // of a number, the lower three as signed digits
#pragma unroll
                for (int k = 0; k < kPer; ++k) bytes[k] = (static_cast<uint32_t>(odd ? 0 : __float2int_rn(v[k] * mult)) + 0x00808080u) ^ 0x00808080u;
                const int d = lane * kPer, hh = d / 128, x = d % kRowBytes;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int n = 4 * r + g, swz = kRowBytes == 128 ? (n & 7) : ((n >> 1) & 3);
                    uint8_t* to = smem + off_q + hh * kN * kRowBytes + n * kRowBytes + (((x >> 4) ^ swz) << 4) + (x & 15);
                    auto pair = [&](int k) { return __byte_perm(bytes[k], bytes[k + 1], g | (4 + g) << 4); };
                    if constexpr (kPer == 2) *reinterpret_cast<uint16_t*>(to) = static_cast<uint16_t>(pair(0));
                    else if constexpr (kPer == 4) *reinterpret_cast<uint32_t*>(to) = __byte_perm(pair(0), pair(2), 0x5410);
                    else *reinterpret_cast<uint2*>(to) = make_uint2(__byte_perm(pair(0), pair(2), 0x5410), __byte_perm(pair(4), pair(6), 0x5410));
                }
                // a row that holds NaN or infinity gives NaN
                if (lane == 0) it.factor[r] = odd ? __uint_as_float(0x7fc00000u) : a.scale_log2 * __uint_as_float(static_cast<uint32_t>(127 - 29 + ex) << 23);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.qfull));
        };
        auto next_item = [&](Cursor<kRows> c) {
            c.k = c.s.tiles - 1;
            c.next(a, prefix, known);
            return c;
        };

        fetch_queries(cur);
        convert_queries(cur, 0);
        int items = 0;
        float m = -INFINITY, l[kRows], acc[kHalves][kRows];   // m: of row `lane`
        int seg_first = cur.k, stage = 0, round = 0;
        bool pending = false;                          // O of the tile before is still to be taken

        auto reset = [&]() {
            m = -INFINITY;
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                l[r] = 0.f;
#pragma unroll
                for (int hh = 0; hh < kHalves; ++hh) acc[hh][r] = 0.f;
            }
        };
        reset();
        auto write_row = [&](const ItemInfo& it, int r, float mm, float ll, const float (&v)[kHalves], int d) {
            if (it.out[r] < 0) return;
            const float inv = ll == 0.f ? 0.f : __fdiv_rn(1.f, ll);
            T* y = static_cast<T*>(a.y) + it.out[r] + d;
#pragma unroll
            for (int hh = 0; hh < kHalves; ++hh) y[hh * 128] = qtz_dev::from_f32<T>(v[hh] * inv);
            if (d == 0 && a.lse) a.lse[it.lse[r]] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * 0.693147181f;
        };

        auto take_sums = [&](int i) {
            wait(sh.ofull[i & 1], (i >> 1) & 1);
            tc_fence_after();
#pragma unroll
            for (int hh = 0; hh < kHalves; ++hh)
#pragma unroll
                for (int r0 = 0; r0 < kRows; r0 += 4) {
                    uint32_t o[16];
                    load_digits<kRows>(tmem + (2 + (i & 1) * kHalves + hh) * kColumns + (static_cast<uint32_t>(warp) << 21), r0, o);
                    const float4 keep = *reinterpret_cast<const float4*>(&sh.keep[i & 1][warp][r0]), gain = *reinterpret_cast<const float4*>(&sh.gain[i & 1][warp][r0]);
                    tmem_ld_wait();
#pragma unroll
                    for (int r = 0; r < 4 && r0 + r < kRows; ++r)
                        acc[hh][r0 + r] = fmaf(join_digits(o[4 * r], o[4 * r + 1], o[4 * r + 2], o[4 * r + 3]), (&gain.x)[r], acc[hh][r0 + r] * (&keep.x)[r]);
                }
        };

        for (int i = 0; i < count; ++i) {
            const ItemInfo& it = sh.item[items & 1];
            const int pos0 = cur.pos(), pos = pos0 + tid;
            const bool last = cur.k == cur.s.tiles - 1, more = i + 1 < count;
            // the next item's first tile is at most one tile after the next
            const int to_next = cur.s.tiles - cur.k;
            if (i + to_next < count && (to_next == 2 || (to_next == 1 && (i == 0 || cur.k == 0)))) fetch_queries(next_item(cur));
            if (i == 0 || cur.k == 0) wait(sh.qfull, items & 1);
            wait(sh.full[stage], round & 1);
            // Scales lie in [2^-100, 2^122] here (the least is QTZ_KV_MIN_SCALE; no 16-bit value gives more than 2^121), so
            // that their logarithms and inverses are ordinary numbers.
            const float2 scales = sh.scales[stage][tid >> a.box_shift];
            const float ks = fminf(fmaxf(scales.x, QTZ_KV_MIN_SCALE), 5.3169120e36f), vs = fminf(fmaxf(scales.y, QTZ_KV_MIN_SCALE), 5.3169120e36f);
            if (++stage == a.stages) {
                stage = 0;
                ++round;
            }
            wait(sh.sfull[i & 1], (i >> 1) & 1);
            tc_fence_after();
            float x[kRows];
            {
                const float lv = lg2(vs);
#pragma unroll
                for (int r0 = 0; r0 < kRows; r0 += 4) {
                    uint32_t s[16];
                    load_digits<kRows>(tmem + (i & 1) * kColumns + (static_cast<uint32_t>(warp) << 21), r0, s);
                    tmem_ld_wait();
#pragma unroll
                    for (int r = 0; r < 4 && r0 + r < kRows; ++r)
                        x[r0 + r] = fmaf(join_digits(s[4 * r], s[4 * r + 1], s[4 * r + 2], s[4 * r + 3]), it.factor[r0 + r] * ks, lv);
                }
            }
            if (__float_as_uint(scales.x) == kNoBox) {
#pragma unroll
                for (int r = 0; r < kRows; ++r) x[r] = -INFINITY;
            } else if (pos0 < it.full_lo || pos0 + kTile > it.full_hi) {
#pragma unroll
                for (int r = 0; r < kRows; ++r)
                    if (pos < it.begin[r] || pos >= it.end[r]) x[r] = -INFINITY;
            }
            float top[kRowsUp];
#pragma unroll
            for (int r = 0; r < kRowsUp; ++r) top[r] = r < kRows ? redux_max(x[r]) : -INFINITY;
            if (lane == 0)
#pragma unroll
                for (int r = 0; r < kRowsUp; r += 4)
                    *reinterpret_cast<float4*>(&sh.max[i & 1][warp][r]) = make_float4(top[r], top[r + 1], top[r + 2], top[r + 3]);
            ok = named_barrier_and(1, kComputeThreads, ok);
            if (!ok) break;
            // lane r finds what all threads need of row r
            if (lane < kRows) {
                float t = -INFINITY;
#pragma unroll
                for (int w = 0; w < kComputeWarps; ++w) t = fmaxf(t, sh.max[i & 1][w][lane]);
                const float now = fmaxf(m, t), origin = now == -INFINITY ? 0.f : now;   // subtracted from -inf without giving NaN
                sh.origin[warp][lane] = t == -INFINITY ? 0.f : t;
                sh.keep[i & 1][warp][lane] = ex2(m - origin);
                sh.gain[i & 1][warp][lane] = ex2(t - origin);
                m = now;
            }
            __syncwarp();
            // O of the tile before: its product ran beside this tile's logits; after it the weights' place is free
            if (pending) take_sums(i - 1);
            pending = true;
            const float inv = __fdividef(1.f, vs);
            uint32_t bits[kRows];
#pragma unroll
            for (int r0 = 0; r0 < kRows; r0 += 4) {
                const float4 origin = *reinterpret_cast<const float4*>(&sh.origin[warp][r0]), keep = *reinterpret_cast<const float4*>(&sh.keep[i & 1][warp][r0]),
                             gain = *reinterpret_cast<const float4*>(&sh.gain[i & 1][warp][r0]);
#pragma unroll
                for (int j = 0; j < 4 && r0 + j < kRows; ++j) {
                    const int r = r0 + j;
                    const float w = ex2(x[r] - (&origin.x)[j]);
                    l[r] = fmaf(w * (&gain.x)[j], inv, l[r] * (&keep.x)[j]);
                    bits[r] = __float2uint_rn(w * 2147483648.f);   // units of 2^-31
                }
            }
            const uint32_t to = base + off_p;
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int n = 4 * r + g;
                    st_shared_u8(to + n * 128 + (((tid >> 4) ^ (n & 7)) << 4) + (tid & 15), bits[r] >> (8 * g));
                }
            tc_fence_before();
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.pfull[i & 1]));
            if (last && more) convert_queries(next_item(cur), (items + 1) & 1);

            if (!last && more) {
                ++cur.k;
            } else {                                   // the end of the item, or of this CTA's part of it
                take_sums(i);
                pending = false;
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], off);
                    if (lane == 0) sh.sum[r][warp] = l[r];
                }
                ok = named_barrier_and(1, kComputeThreads, ok);
                if (!ok) break;
                const bool whole = seg_first == 0 && last;
                // slot 0: an item that began in an earlier CTA; slot 1: one that goes on in the next
                float* part = a.parts + (static_cast<int64_t>(blockIdx.x) * 2 + (seg_first == 0 ? 1 : 0)) * kPart;
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    const float4 t = *reinterpret_cast<const float4*>(sh.sum[r]);
                    const float sum = (t.x + t.y) + (t.z + t.w), top = __shfl_sync(0xffffffffu, m, r);
                    float v[kHalves];
#pragma unroll
                    for (int hh = 0; hh < kHalves; ++hh) v[hh] = acc[hh][r] * 4.656612873077393e-10f;   // 2^-31
                    if (D >= 128 || tid < D) {
                        if (whole) {
                            write_row(it, r, top, sum, v, tid);
                        } else {
#pragma unroll
                            for (int hh = 0; hh < kHalves; ++hh) part[r * D + hh * 128 + tid] = v[hh];
                        }
                    }
                    if (!whole && tid == 0) {
                        part[kMaxRows * D + r] = top;
                        part[kMaxRows * D + kMaxRows + r] = sum;
                    }
                }
                if (!whole) {                          // joined below
                    OpenItem& open = sh.open[seg_first == 0 ? 1 : 0];
                    if (tid < kRows) {
                        open.out[tid] = it.out[tid];
                        open.lse[tid] = it.lse[tid];
                    }
                    if (tid == 0) {
                        open.c0 = share_of(cur.begin);
                        open.c1 = share_of(cur.begin + kTileUnits * (cur.s.tiles - 1));
                    }
                }
                reset();
                seg_first = 0;
                ++items;
                if (more) cur.next(a, prefix, known);
            }
        }
        if (!ok) {
            timed_out();
            sh.failed = 1;
        }
    }

    tc_fence_before();
    __syncthreads();                                   // the parts, before they are counted
    if (warp == kComputeWarps + 1) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemColumns);
    }

    // ======== joining: items that lie in several CTAs, c0 .. c1 ========
    // The last CTA of each group of neighbours to arrive joins the group's parts into the place of its first; with several
    // groups, the last of those joins the groups.  Always in the order of the tiles.  (After a wait that gave up nothing is
    // joined: the results are void, and the counters have to be cleared.)
    if (sh.failed) return;
    const int me = static_cast<int>(blockIdx.x);
    auto group_size = [](int n) {                      // about the square root: both steps join about equally many parts
        int g = 4;
        while (g * g < n) ++g;
        return n <= 8 ? n : g;
    };
    if (lane == 0 && warp < 2 && sh.open[warp].c1 >= 0) {
        const OpenItem& open = sh.open[warp];
        const int size = group_size(open.c1 - open.c0 + 1), first = me - (me - open.c0) % size, others = min(size - 1, open.c1 - first);
        int32_t* counter = a.counters + 2 * first + (first == open.c0 ? 1 : 0);
        sh.last[warp] = arrive_acq_rel(counter) == others;
        if (sh.last[warp]) *counter = 0;               // ready for the next call
    }
    __syncthreads();
    // Half of the warps for each of the two items, all for one.
    const bool both = sh.open[0].c1 >= 0 && sh.last[0] && sh.open[1].c1 >= 0 && sh.last[1];
    const int crew = both ? kThreads / 2 : kThreads, slot = both ? tid / crew : sh.open[1].c1 >= 0 && sh.last[1] ? 1 : 0, ht = tid % crew;
    const OpenItem& open = sh.open[slot];
    auto sync_crew = [&]() { named_barrier(2 + slot, crew); };
    if (open.c1 >= 0 && sh.last[slot]) {
        const int c0 = open.c0, c1 = open.c1, size = group_size(c1 - c0 + 1), groups = (c1 - c0) / size + 1, first = me - (me - c0) % size;
        auto part_of = [&](int cta) { return a.parts + (static_cast<int64_t>(cta) * 2 + (cta == c0 ? 1 : 0)) * kPart; };
        constexpr int kQuads = kRows * D / 4;          // four neighbouring values of a row
        constexpr int kOwn = kMaxRows * D, kJoined = kOwn + 2 * kMaxRows;
        // Joins n parts, those of CTAs from, from + step, ..: into `to`, or into the output.  Each thread finds the weights of the rows
        // that it adds up itself: all loads of a round are under way together, and nothing is waited for in between.
        constexpr int kUp = (kQuads + kThreads - 1) / kThreads, kAtOnce = kUp < 4 ? kUp : 4, kFlight = 18 / kAtOnce;
        auto join = [&](int from, int step, int n, int scalars, float* to) {
#pragma unroll 1
            for (int q0 = ht; q0 < kQuads; q0 += kAtOnce * crew) {
                float4 v[kAtOnce];
                float top[kAtOnce], sum[kAtOnce];
                int quad[kAtOnce];
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
                    top[j] = -INFINITY;
                    sum[j] = 0.f;
                    quad[j] = min(q0 + j * crew, kQuads - 1);
                }
#pragma unroll 1
                for (int x0 = 0; x0 < n; x0 += kFlight) {
                    float4 p[kAtOnce][kFlight];
                    float pm[kAtOnce][kFlight], pl[kAtOnce][kFlight];
#pragma unroll
                    for (int x = 0; x < kFlight; ++x) {
                        const float* part = part_of(from + (x0 + x) * step);
#pragma unroll
                        for (int j = 0; j < kAtOnce; ++j) {
                            p[j][x] = make_float4(0.f, 0.f, 0.f, 0.f);
                            pm[j][x] = -INFINITY;
                            pl[j][x] = 0.f;
                            if (x0 + x < n) {
                                p[j][x] = __ldcg(reinterpret_cast<const float4*>(part) + quad[j]);
                                pm[j][x] = __ldcg(part + scalars + quad[j] / (D / 4));
                                pl[j][x] = __ldcg(part + scalars + kMaxRows + quad[j] / (D / 4));
                            }
                        }
                    }
#pragma unroll
                    for (int j = 0; j < kAtOnce; ++j) {
                        float t = top[j];
#pragma unroll
                        for (int x = 0; x < kFlight; ++x) t = fmaxf(t, pm[j][x]);
                        const float keep = top[j] == t ? 1.f : ex2(top[j] - t);
                        top[j] = t;
                        sum[j] *= keep;
                        v[j].x *= keep;
                        v[j].y *= keep;
                        v[j].z *= keep;
                        v[j].w *= keep;
#pragma unroll
                        for (int x = 0; x < kFlight; ++x) {
                            const float w = pm[j][x] == -INFINITY && pl[j][x] == 0.f ? 0.f : ex2(pm[j][x] - (t == -INFINITY ? 0.f : t));
                            sum[j] = fmaf(pl[j][x], w, sum[j]);
                            v[j].x = fmaf(p[j][x].x, w, v[j].x);
                            v[j].y = fmaf(p[j][x].y, w, v[j].y);
                            v[j].z = fmaf(p[j][x].z, w, v[j].z);
                            v[j].w = fmaf(p[j][x].w, w, v[j].w);
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    if (q0 + j * crew >= kQuads) break;
                    const int r = quad[j] / (D / 4), d = quad[j] % (D / 4) * 4;
                    if (to) {
                        *reinterpret_cast<float4*>(to + r * D + d) = v[j];
                        if (d == 0) {                  // beside those that other threads still read
                            to[kJoined + r] = top[j];
                            to[kJoined + kMaxRows + r] = sum[j];
                        }
                    } else if (open.out[r] >= 0) {
                        const float inv = sum[j] == 0.f ? 0.f : __fdiv_rn(1.f, sum[j]);
                        uint2 o;
                        o.x = qtz_dev::pack2(v[j].x * inv, v[j].y * inv, T());
                        o.y = qtz_dev::pack2(v[j].z * inv, v[j].w * inv, T());
                        *reinterpret_cast<uint2*>(static_cast<T*>(a.y) + open.out[r] + d) = o;
                        if (d == 0 && a.lse) a.lse[open.lse[r]] = sum[j] == 0.f ? -INFINITY : (top[j] + log2f(sum[j])) * 0.693147181f;
                    }
                }
            }
        };
        join(first, 1, min(size, c1 - first + 1), kOwn, groups > 1 ? part_of(first) : nullptr);
        if (groups > 1) {
            sync_crew();
            if (ht == 0) {
                int32_t* counter = a.counters + 2 * gridDim.x + c0;
                sh.last[slot] = arrive_acq_rel(counter) == groups - 1;
                if (sh.last[slot]) *counter = 0;
            }
            sync_crew();
            if (sh.last[slot]) join(c0, size, groups, kJoined, nullptr);
        }
    }
}

int ctas_per_sm(int head_dim) { return head_dim == 256 ? 1 : 2; }

template <typename T, int D, int kRows>
qtz_status launch(qtz_ctx* h, AttnArgs& a, const CUtensorMap& km, const CUtensorMap& vm, cudaStream_t st)
{
    constexpr int kN = (4 * kRows + 15) / 16 * 16, kStage = 2 * kTile * D;
    const int ctas = ctas_per_sm(D);
    const int fixed = kN * 128 + kN * D + static_cast<int>((sizeof(Shared) + 15) / 16 * 16 + sizeof(uint32_t) * (a.requests + 1));
    const int room = (kSmemLimit + 1024) / ctas - 1024 - fixed;
    a.stages = room / kStage < kMaxStages ? room / kStage : kMaxStages;
    if (a.stages < 2) return QTZ_ERR_TOO_LARGE;
    const int smem = fixed + a.stages * kStage;
    const qtz_status s = qtz_allow_smem(h, attention_kernel<T, D, kRows>);
    if (s != QTZ_OK) return s;
    QTZ_CUDA(h, qtz_launch_dependent(attention_kernel<T, D, kRows>, dim3(h->num_sms * ctas), kThreads, smem, st, a, km, vm));
    return QTZ_OK;
}

int rows_of_tile(int64_t group, int64_t tokens, int64_t requests)
{
    // Query rows of a (request, key/value head) if all requests bring equally many tokens: the smallest tile that takes them
    // reads the cache once; larger ones only compute unused columns.  16 requests of 1000 to 8000 tokens, us: 4 rows 34.5; 5 rows 35.4
    // in a tile of 5, 36.6 in one of 8 (heads of 64: 28.4, 32.0); 8 rows 36.7; 10 rows 38.1 in a tile of 10, 40.5 in one of 12, 48.7 in one
    // of 16; 12 rows 40.4 in a tile of 12, 48.9 in one of 16; 16 rows 49.3.
    const int64_t rows = group * ((tokens + requests - 1) / requests);
    return rows <= 4 ? 4 : rows <= 5 ? 5 : rows <= 8 ? 8 : rows <= 10 ? 10 : rows <= 12 ? 12 : 16;
}

template <typename T, int D>
qtz_status launch_rows(qtz_ctx* h, AttnArgs& a, int rows, const CUtensorMap& km, const CUtensorMap& vm, cudaStream_t st)
{
    switch (rows) {
        case 4: return launch<T, D, 4>(h, a, km, vm, st);
        case 5: return launch<T, D, 5>(h, a, km, vm, st);
        case 8: return launch<T, D, 8>(h, a, km, vm, st);
        case 10: return launch<T, D, 10>(h, a, km, vm, st);
        case 12: return launch<T, D, 12>(h, a, km, vm, st);
        default: return launch<T, D, 16>(h, a, km, vm, st);
    }
}

int64_t counters_bytes(const qtz_ctx* h, int head_dim) { return (static_cast<int64_t>(h->num_sms) * ctas_per_sm(head_dim) * 3 * 4 + 255) / 256 * 256; }

}  // namespace

extern "C" int64_t qtz_kv_attention_workspace_bytes(qtz_handle h, const qtz_kv_cache* cache)
{
    if (!h || qtz_kv_check(cache) != QTZ_OK) return 0;
    const int d = cache->head_dim;
    return counters_bytes(h, d) + static_cast<int64_t>(h->num_sms) * ctas_per_sm(d) * 2 * (kMaxRows * d + 4 * kMaxRows) * 4;
}

extern "C" qtz_status qtz_kv_attention(qtz_handle h, const qtz_kv_cache* cache, const void* q_dev, int64_t q_token_stride,
                                       int64_t q_head_stride, int32_t q_heads, int32_t ftype, const int32_t* starts_dev,
                                       const int32_t* lens_dev, int32_t requests, int64_t tokens, const int32_t* table_dev,
                                       int32_t table_width, float scale, int32_t window, void* y_dev, int64_t y_token_stride,
                                       int64_t y_head_stride, float* lse_dev, void* workspace_dev, void* stream)
{
    if (!h || requests <= 0 || tokens < 0 || table_width <= 0 || window < 0 || !isfinite(scale)) return QTZ_ERR_INVALID_ARG;
    qtz_status s = qtz_kv_check(cache);
    if (s != QTZ_OK) return s;
    if (ftype != QTZ_F16 && ftype != QTZ_BF16) return QTZ_ERR_INVALID_ARG;
    if (q_heads <= 0 || q_heads % cache->kv_heads != 0) return QTZ_ERR_INVALID_ARG;
    if (requests > kMaxRequests || tokens > 0x7fffffff || q_heads > 65535) return QTZ_ERR_TOO_LARGE;
    if (tokens == 0) return QTZ_OK;
    if (!q_dev || !y_dev || !starts_dev || !lens_dev || !table_dev || !workspace_dev) return QTZ_ERR_INVALID_ARG;
    if (!qtz_aligned16(q_dev) || !qtz_aligned16(y_dev) || !qtz_aligned16(workspace_dev) ||
        !qtz_kv_strides_ok(tokens, q_token_stride, q_heads, q_head_stride) || !qtz_kv_strides_ok(tokens, y_token_stride, q_heads, y_head_stride))
        return QTZ_ERR_MISALIGNED;
    // rows of the cache and units of the longest possible step are counted in 32 bits
    const int64_t rows = static_cast<int64_t>(cache->blocks) * cache->kv_heads * cache->block_tokens;
    const int64_t reach = static_cast<int64_t>(table_width) * cache->block_tokens, group = q_heads / cache->kv_heads;
    const int tile_rows = rows_of_tile(group, tokens, requests);
    const double items = static_cast<double>(cache->kv_heads) * (static_cast<double>(tokens) * group / tile_rows + requests);
    const double units = items * (kTileUnits * static_cast<double>(reach / kTile + 1) + kItemUnits);
    if (rows > 0x7fffffff || reach > 0x7fffffff || units > 2.0e9) return QTZ_ERR_TOO_LARGE;
    qtz_device_guard guard(h->device);
    int box_shift = 4;                         // the largest box that divides both a block and a tile
    while ((1 << box_shift) < kTile && cache->block_tokens % (2 << box_shift) == 0) ++box_shift;
    CUtensorMap km, vm;
    const uint32_t row_bytes = cache->head_dim < 128 ? cache->head_dim : 128;
    const uint64_t dims[2] = {static_cast<uint64_t>(cache->head_dim), static_cast<uint64_t>(rows)};
    const uint64_t strides[1] = {static_cast<uint64_t>(cache->head_dim)};
    const uint32_t box[2] = {row_bytes, 1u << box_shift};
    if (!qtz_encode_u8_map(&km, cache->k_dev, 2, dims, strides, box, static_cast<int>(row_bytes)) ||
        !qtz_encode_u8_map(&vm, cache->v_dev, 2, dims, strides, box, static_cast<int>(row_bytes)))
        return qtz_cuda_fail(h, cudaErrorInvalidValue, "tensor map of the cache");
    float* parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace_dev) + counters_bytes(h, cache->head_dim));
    AttnArgs a{*cache, q_dev, q_token_stride, q_head_stride, q_heads, static_cast<int32_t>(group), starts_dev, lens_dev, requests,
               static_cast<int32_t>(tokens), table_dev, table_width, scale * 1.44269504f, window < (1 << 30) ? window : 1 << 30, y_dev,
               y_token_stride, y_head_stride, lse_dev, static_cast<int32_t*>(workspace_dev), parts, 0, box_shift, h->wait_budget, h->status_dev};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (ftype == QTZ_F16) {
        if (cache->head_dim == 64) return launch_rows<__half, 64>(h, a, tile_rows, km, vm, st);
        if (cache->head_dim == 128) return launch_rows<__half, 128>(h, a, tile_rows, km, vm, st);
        return launch_rows<__half, 256>(h, a, tile_rows, km, vm, st);
    }
    if (cache->head_dim == 64) return launch_rows<__nv_bfloat16, 64>(h, a, tile_rows, km, vm, st);
    if (cache->head_dim == 128) return launch_rows<__nv_bfloat16, 128>(h, a, tile_rows, km, vm, st);
    return launch_rows<__nv_bfloat16, 256>(h, a, tile_rows, km, vm, st);
}

// Attention of new tokens over the paged 8-bit key/value cache.
//
// Mathematics.  For one query row q and one block with key scale s_k and value scale s_v the kernel holds, per token p,
//   t_p = (q . k_p) c log2(e) s_k + log2(s_v),      w_p = 2^(t_p - m),     m = running maximum of t
// so that w_p = s_v exp(logit_p) 2^-m carries the block's value scale: the sum over values is sum w_p v_p on the codes
// themselves, and the softmax's denominator is sum w_p / s_v.  Codes become fp16 exactly (a byte placed in the mantissa of
// 1024 + u, minus the offset), queries keep all their bits in fp16 after each row is scaled by a power of two, so logits are
// exact products summed in fp32; w_p, at most 1, is the only value rounded to 16 bits (fp16: 2^-11, finer than a bf16 output).
//
// What bounds it: one token reads 2 D bytes a head for 4 D flops a query head: HBM, by a factor of 4 to 100 over the tensor
// cores.  So every byte is read once, and the work is cut for an even stream: the 16-token tiles of all (request, key/value
// head, 16 query rows) items form one sequence that is dealt out in equal contiguous shares to the warps of a grid of one
// CTA per SM, whatever the lengths.  Each warp streams its share through a private ring in shared memory (TMA boxes of 16
// rows, issued by lane 0, several tiles ahead of use, across items).  An item that one warp finishes is written from
// registers; shares that meet in an item are joined in the CTA, and across CTAs by the last one to arrive, always in the
// order of the tiles, so that results do not depend on timing.
#include <cuda.h>

#include "qtz_half_util.cuh"
#include "qtz_kv.cuh"
#include "qtz_plan.cuh"
#include "qtz_ptx.cuh"

namespace {

using namespace qtz_ptx;

constexpr int kMaxRequests = 8192;
constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kTile = 16;          // tokens of a tile: the depth of one matrix instruction
constexpr int kMaxStages = 8;
constexpr int kBatch = 32;         // tiles whose addresses and scales a warp looks up together
constexpr int kMinShare = 8;       // tiles: shorter shares cost more in joining than they save in streaming
constexpr int kSmemLimit = 227 * 1024;

struct TileInfo {                  // what a warp needs to know about one tile
    int32_t row;                   // first row of the tile in the [blocks * heads * block_tokens] view
    float k_scale, v_scale;
    int32_t pos;                   // position of its first token
    int32_t request, item;         // item: index within the request (head, row tile)
    int32_t flags;
    int32_t pad;
};
enum { kValid = 1, kFirst = 2, kLast = 4 };

struct AttnArgs {
    qtz_kv_cache c;
    const void* q;
    int64_t q_token_stride, q_head_stride;
    int32_t q_heads, group;
    const int32_t *starts, *lens;
    int32_t requests, tokens;
    const int32_t* table;
    int32_t width;
    float scale_log2;              // softmax scale * log2(e)
    int32_t window;
    void* y;
    int64_t y_token_stride, y_head_stride;
    float* lse;
    int32_t* counters;             // [CTAs] arrivals at the item that begins in a CTA and ends in a later one
    float* warp_parts;             // [CTAs][warps][16 * D]
    float* cta_parts;              // [CTAs][2][16 * D + 32]
    int32_t stages;
    int64_t wait_budget;
    int32_t* status;
};

struct RequestShape {
    int first, added;              // rows of q
    int len, limit;                // tokens; those that the table can hold
    int row_tiles, lo, hi, tiles;  // items per head; tiles [lo, hi) of the cache; tiles per item (at least one)
};

__device__ __forceinline__ RequestShape shape_of(const AttnArgs& a, int r)
{
    RequestShape s;
    s.first = min(max(a.starts[r], 0), a.tokens);
    s.added = min(max(a.starts[r + 1], s.first), a.tokens) - s.first;
    s.len = min(max(a.lens[r], 0), 0x7ffffff0);
    s.limit = static_cast<int>(min(static_cast<int64_t>(s.len), static_cast<int64_t>(a.width) * a.c.block_tokens));
    s.row_tiles = static_cast<int>((static_cast<int64_t>(s.added) * a.group + 15) / 16);
    const int64_t begin = static_cast<int64_t>(s.len) - s.added + 1 - a.window;
    s.lo = a.window > 0 && begin > 0 ? static_cast<int>(begin / kTile) : 0;
    s.hi = (s.limit + kTile - 1) / kTile;
    s.tiles = max(1, s.hi - s.lo);
    return s;
}

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

// D (16 x 8, fp32) += A (16 x 16, fp16, row major) B (16 x 8, fp16, column major)
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Bytes (b0, b1) or (b2, b3) of a word of codes with the sign bit flipped, as two fp16 values: 1024 + (code + 128) - 1152.
template <int kPair>
__device__ __forceinline__ uint32_t codes_to_half2(uint32_t flipped)
{
    const uint32_t v = __byte_perm(flipped, 0x64646464u, kPair == 0 ? 0x4140 : 0x4342);
    const uint32_t offset = 0x64806480u;   // 1152
    const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&v), *reinterpret_cast<const __half2*>(&offset));
    return *reinterpret_cast<const uint32_t*>(&h);
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

struct WorkerParts {               // the partial results that a warp leaves for its CTA
    int head, tail;                // 0 / 1
    int head_begin, head_end, head_request, head_item;
    int tail_begin, tail_end, tail_request, tail_item;
};
struct Group {                     // an item's partial results within one CTA
    int begin, end, request, item, first, count;
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1)
attention_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map)
{
    constexpr int kHalves = D > 128 ? D / 128 : 1;     // boxes along a row
    constexpr int kRowBytes = D < 128 ? D : 128;
    constexpr int kChunks = kRowBytes / 64;            // 16-byte chunks of a key row that a lane holds, per box
    constexpr int kNt = D / 8;                         // 8-column tiles of the output
    constexpr int kNtBox = kNt / kHalves;
    constexpr int kKs = D / 16;                        // matrix instructions along a head
    constexpr int kBox = kTile * kRowBytes;
    constexpr int kStage = 2 * kHalves * kBox;

    extern __shared__ uint8_t smem_raw[];
    __shared__ float s_m[kWarps][2][16], s_l[kWarps][2][16];
    __shared__ WorkerParts s_parts[kWarps];
    __shared__ Group s_groups[2 * kWarps];
    __shared__ int s_members[2 * kWarps], s_group_count, s_last;
    __shared__ uint64_t s_bars[kWarps][kMaxStages];
    __shared__ uint32_t s_scan[kWarps];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
    const int ring_bytes = a.stages * kStage;
    TileInfo* info = reinterpret_cast<TileInfo*>(smem + kWarps * ring_bytes) + warp * 2 * kBatch;
    uint32_t* prefix = reinterpret_cast<uint32_t*>(smem + kWarps * ring_bytes + kWarps * 2 * kBatch * sizeof(TileInfo));
    const uint32_t ring = smem_base + warp * ring_bytes;
    const uint32_t bars = smem_u32(&s_bars[warp][0]);

    if (lane < kMaxStages) mbar_init(bars + 8 * lane, 1);
    if (tid == 0) {
        prefetch_tensormap(&k_map);
        prefetch_tensormap(&v_map);
    }
    fence_barrier_init();

    // ---- tiles before each request: an exclusive prefix sum over the requests ----
    const int per = (a.requests + kThreads - 1) / kThreads;
    const int r_lo = min(tid * per, a.requests), r_hi = min(r_lo + per, a.requests);
    uint32_t mine = 0;
    for (int r = r_lo; r < r_hi; ++r) {
        const RequestShape s = shape_of(a, r);
        const uint32_t n = static_cast<uint32_t>(a.c.kv_heads) * s.row_tiles * s.tiles;
        prefix[r] = n;
        mine += n;
    }
    uint32_t scan = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, scan, off);
        if (lane >= off) scan += u;
    }
    if (lane == 31) s_scan[warp] = scan;
    __syncthreads();
    uint32_t before = scan - mine, total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += s_scan[w];
        total += s_scan[w];
    }
    for (int r = r_lo; r < r_hi; ++r) {
        const uint32_t n = prefix[r];
        prefix[r] = before;
        before += n;
    }
    if (tid == 0) prefix[a.requests] = total;
    __syncthreads();

    const int all = static_cast<int>(total);
    const int workers = gridDim.x * kWarps;
    const int share = max((all + workers - 1) / workers, kMinShare);
    const int cta_share = share * kWarps;
    const int t0 = min((static_cast<int>(blockIdx.x) * kWarps + warp) * share, all);
    const int count = min(t0 + share, all) - t0;

    // ---- tile look-up, a batch at a time: lane i takes tile t0 + batch * kBatch + i ----
    const int64_t heads = a.c.kv_heads;
    auto look_up = [&](int batch) {                    // everything but the scales; returns block * heads + head, or -1
        const int i = batch * kBatch + lane;
        if (i >= count) return static_cast<int64_t>(-1);
        const uint32_t tile = t0 + i;
        int u = 0, v = a.requests;
        while (v - u > 1) {
            const int mid = (u + v) >> 1;
            if (prefix[mid] <= tile) u = mid; else v = mid;
        }
        const RequestShape s = shape_of(a, u);
        const int off = static_cast<int>(tile - prefix[u]);
        const int item = off / s.tiles, k = off - item * s.tiles;
        const int pos = (s.lo + k) * kTile, h = item / s.row_tiles;
        int flags = (k == 0 ? kFirst : 0) | (k == s.tiles - 1 ? kLast : 0);
        int64_t bh = -1;
        TileInfo& e = info[(batch & 1) * kBatch + lane];
        if (s.lo + k < s.hi) {
            const int id = a.table[static_cast<int64_t>(u) * a.width + pos / a.c.block_tokens];
            if (id >= 0 && id < a.c.blocks) {
                flags |= kValid;
                bh = id * heads + h;
                e.row = static_cast<int32_t>(bh * a.c.block_tokens + pos % a.c.block_tokens);
            } else {
                qtz_dev::report_invalid(a.status, QTZ_SITE_KV_ATTENTION);
            }
        }
        e.pos = pos;
        e.request = u;
        e.item = item;
        e.flags = flags;
        return bh;
    };
    // Scales lie in [2^-100, 2^122] here (the least is QTZ_KV_MIN_SCALE; no 16-bit value gives more than 2^121), so that their
    // logarithms and inverses are ordinary numbers.
    auto scale_of = [&](const float* p, int64_t bh) { return bh < 0 ? 1.f : fminf(fmaxf(p[bh], QTZ_KV_MIN_SCALE), 5.3169120e36f); };

    int64_t bh = look_up(0);
    float ks = scale_of(a.c.k_scale_dev, bh), vs = scale_of(a.c.v_scale_dev, bh);
    auto put_scales = [&](int batch) {
        info[(batch & 1) * kBatch + lane].k_scale = ks;
        info[(batch & 1) * kBatch + lane].v_scale = vs;
    };
    put_scales(0);
    __syncwarp();

    bool failed = false;
    auto issue = [&](int i, int stage) {               // lane 0 only
        const TileInfo& e = info[((i / kBatch) & 1) * kBatch + i % kBatch];
        const uint32_t bar = bars + 8 * stage, dst = ring + stage * kStage;
        if (!(e.flags & kValid)) {
            mbar_arrive(bar);
            return;
        }
        mbar_arrive_expect_tx(bar, kStage);
#pragma unroll
        for (int hh = 0; hh < kHalves; ++hh) {
            tma_load_2d(dst + hh * kBox, &k_map, bar, hh * 128, e.row);
            tma_load_2d(dst + (kHalves + hh) * kBox, &v_map, bar, hh * 128, e.row);
        }
    };
    int issued = min(a.stages, count);
    if (lane == 0)
        for (int i = 0; i < issued; ++i) issue(i, i);

    // ---- state of the current item ----
    uint32_t qf[kKs][4];
    float o[kNt][4], m0 = 0.f, m1 = 0.f, l0 = 0.f, l1 = 0.f, f0 = 0.f, f1 = 0.f;
    int end0 = 0, end1 = 0, begin0 = 0, begin1 = 0, full_lo = 0, full_hi = 0;
    int seg_begin = 0;                                 // index in the share where the item's part of this warp begins
    bool seg_whole = false;

    // A row of a 16-row tile: its token and head, or false beyond the request's rows.
    auto row_of = [&](const RequestShape& s, int item, int row, int64_t& token, int& head, int& local) {
        const int h = item / s.row_tiles, index = (item - h * s.row_tiles) * 16 + row;
        local = index / a.group;
        head = h * a.group + (index - local * a.group);
        token = s.first + local;
        return local < s.added;
    };
    auto write_lse = [&](int64_t token, int head, float m, float l) {
        if (a.lse) a.lse[token * a.q_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147181f;
    };

    int stage = 0;
    uint32_t phase = 0;
    for (int i = 0; i < count; ++i) {
        const int in_batch = i % kBatch, batch = i / kBatch;
        // the next batch's addresses and scales come in three steps, far apart, so that no load is waited for
        if (in_batch == 0) bh = look_up(batch + 1);
        else if (in_batch == 8) {
            ks = scale_of(a.c.k_scale_dev, bh);
            vs = scale_of(a.c.v_scale_dev, bh);
        } else if (in_batch == 16) {
            put_scales(batch + 1);
            __syncwarp();
        }
        const TileInfo e = info[(batch & 1) * kBatch + in_batch];

        if (i == 0 || (e.flags & kFirst)) {            // a new item: its query rows, converted once
            const RequestShape s = shape_of(a, e.request);
            seg_begin = i;
            seg_whole = (e.flags & kFirst) != 0;
            m0 = m1 = -INFINITY;
            l0 = l1 = 0.f;
#pragma unroll
            for (int n = 0; n < kNt; ++n)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[n][c] = 0.f;
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
                int64_t token;
                int head, local;
                const bool has = row_of(s, e.item, g + 8 * hi, token, head, local);
                const T* q = static_cast<const T*>(a.q) + token * a.q_token_stride + head * a.q_head_stride;
                // what the row sees; a row beyond the request's is never written and needs no mask
                const int own = s.len - s.added + local + 1;
                (hi ? end1 : end0) = has ? min(own, s.limit) : 0x7fffffff;
                (hi ? begin1 : begin0) = has && a.window > 0 ? max(0, own - a.window) : 0;
                uint32_t raw[kKs][2];
                float top = 0.f;
#pragma unroll
                for (int ch = 0; ch < kHalves * kChunks; ++ch) {
                    const int d0 = (ch / kChunks) * 128 + (kChunks * t4 + ch % kChunks) * 16;
                    uint4 u = {0, 0, 0, 0}, v = {0, 0, 0, 0};
                    if (has) {
                        u = __ldg(reinterpret_cast<const uint4*>(q + d0));
                        v = __ldg(reinterpret_cast<const uint4*>(q + d0) + 1);
                    }
                    const uint32_t w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        raw[ch * 4 + k / 2][k & 1] = w[k];
                        const float2 f = qtz_dev::unpack2(w[k], T());
                        top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
                    }
                }
                // bf16 rows are scaled by a power of two that takes their largest value to [2^14, 2^15): values down to
                // 2^-28 of it stay exact in fp16.  fp16 rows are taken as they are.
                float mult = 1.f, back = a.scale_log2;
                if constexpr (sizeof(T) == 2 && !std::is_same<T, __half>::value) {
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    const int ex = max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -100);
                    mult = __uint_as_float(static_cast<uint32_t>(127 + 14 - ex) << 23);
                    back *= __uint_as_float(static_cast<uint32_t>(127 - 14 + ex) << 23);
                }
                (hi ? f1 : f0) = back;
#pragma unroll
                for (int k = 0; k < kKs; ++k)
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        if constexpr (std::is_same<T, __half>::value) {
                            qf[k][2 * p + hi] = raw[k][p];
                        } else {
                            const float2 f = qtz_dev::unpack2(raw[k][p], T());
                            qf[k][2 * p + hi] = qtz_dev::pack2(f.x * mult, f.y * mult, __half());
                        }
                    }
            }
            // tiles inside [full_lo, full_hi) need no mask for any row
            full_lo = max(begin0, begin1);
            full_hi = min(end0, end1);
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) {
                full_lo = max(full_lo, __shfl_xor_sync(0xffffffffu, full_lo, off));
                full_hi = min(full_hi, __shfl_xor_sync(0xffffffffu, full_hi, off));
            }
        }

        // after a wait that gave up nothing more is issued, but what is in flight is still waited for (with the same limit)
        if (i < issued && !mbar_wait(bars + 8 * stage, phase, a.wait_budget)) {
            if (lane == 0 && atomicCAS(a.status, 0, QTZ_ERR_DEVICE_TIMEOUT) == 0) a.status[1] = QTZ_SITE_TMA_FULL;
            failed = true;
        }
        failed = __any_sync(0xffffffffu, failed);

        if ((e.flags & kValid) && !failed) {
            const uint32_t kb = ring + stage * kStage, vb = kb + kHalves * kBox;
            float sa[4] = {}, sb[4] = {};
#pragma unroll
            for (int ch = 0; ch < kHalves * kChunks; ++ch) {
                const int hh = ch / kChunks;
                // 16-byte chunk c of row r lies at chunk c ^ (r & 7) of a 128-byte row, c ^ ((r >> 1) & 3) of a 64-byte row
                const int chunk = kRowBytes == 128 ? ((2 * t4 + ch % kChunks) ^ g) : (t4 ^ (g >> 1));
                const uint32_t at = kb + hh * kBox + g * kRowBytes + chunk * 16;
                const uint4 ua = lds128(at), ub = lds128(at + 8 * kRowBytes);
                const uint32_t wa[4] = {ua.x, ua.y, ua.z, ua.w}, wb[4] = {ub.x, ub.y, ub.z, ub.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t xa = wa[k] ^ 0x80808080u, xb = wb[k] ^ 0x80808080u;
                    mma(sa, qf[ch * 4 + k], codes_to_half2<0>(xa), codes_to_half2<1>(xa));
                    mma(sb, qf[ch * 4 + k], codes_to_half2<0>(xb), codes_to_half2<1>(xb));
                }
            }
            const float lv = lg2(e.v_scale), k0 = f0 * e.k_scale, k1 = f1 * e.k_scale;
            float x0[4] = {fmaf(sa[0], k0, lv), fmaf(sa[1], k0, lv), fmaf(sb[0], k0, lv), fmaf(sb[1], k0, lv)};
            float x1[4] = {fmaf(sa[2], k1, lv), fmaf(sa[3], k1, lv), fmaf(sb[2], k1, lv), fmaf(sb[3], k1, lv)};
            if (e.pos < full_lo || e.pos + kTile > full_hi) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int p = e.pos + (c >> 1) * 8 + 2 * t4 + (c & 1);
                    if (p < begin0 || p >= end0) x0[c] = -INFINITY;
                    if (p < begin1 || p >= end1) x1[c] = -INFINITY;
                }
            }
            float n0 = fmaxf(fmaxf(x0[0], x0[1]), fmaxf(x0[2], x0[3])), n1 = fmaxf(fmaxf(x1[0], x1[1]), fmaxf(x1[2], x1[3]));
            n0 = fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, 1));
            n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, 1));
            n0 = fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, 2));
            n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, 2));
            n0 = fmaxf(n0, m0);
            n1 = fmaxf(n1, m1);
            if (__any_sync(0xffffffffu, n0 > m0 || n1 > m1)) {
                const float c0 = n0 > m0 ? ex2(m0 - n0) : 1.f, c1 = n1 > m1 ? ex2(m1 - n1) : 1.f;
                l0 *= c0;
                l1 *= c1;
#pragma unroll
                for (int n = 0; n < kNt; ++n) {
                    o[n][0] *= c0;
                    o[n][1] *= c0;
                    o[n][2] *= c1;
                    o[n][3] *= c1;
                }
                m0 = n0;
                m1 = n1;
            }
            const float b0 = m0 == -INFINITY ? 0.f : m0, b1 = m1 == -INFINITY ? 0.f : m1;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                x0[c] = ex2(x0[c] - b0);
                x1[c] = ex2(x1[c] - b1);
            }
            const float inv = __fdividef(1.f, e.v_scale);
            l0 = fmaf((x0[0] + x0[1]) + (x0[2] + x0[3]), inv, l0);
            l1 = fmaf((x1[0] + x1[1]) + (x1[2] + x1[3]), inv, l1);
            const uint32_t pf[4] = {qtz_dev::pack2(x0[0], x0[1], __half()), qtz_dev::pack2(x1[0], x1[1], __half()),
                                    qtz_dev::pack2(x0[2], x0[3], __half()), qtz_dev::pack2(x1[2], x1[3], __half())};
#pragma unroll
            for (int hh = 0; hh < kHalves; ++hh) {
                uint32_t w[4][4];                      // [token of this lane][word]: tokens 2 t4, 2 t4 + 1, 2 t4 + 8, 2 t4 + 9
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int row = 2 * t4 + (k & 1) + 8 * (k >> 1);
                    if constexpr (kRowBytes == 128) {
                        const uint4 u = lds128(vb + hh * kBox + row * 128 + ((g ^ (row & 7)) << 4));
                        w[k][0] = u.x; w[k][1] = u.y; w[k][2] = u.z; w[k][3] = u.w;
                    } else {
                        const uint2 u = lds64(vb + row * 64 + (((g >> 1) ^ ((row >> 1) & 3)) << 4) + (g & 1) * 8);
                        w[k][0] = u.x; w[k][1] = u.y; w[k][2] = 0; w[k][3] = 0;
                    }
                }
#pragma unroll
                for (int k = 0; k < kNtBox / 4; ++k) {
                    // two tokens' bytes side by side: (a0 b0 a1 b1), (a2 b2 a3 b3)
                    const uint32_t x = __byte_perm(w[0][k], w[1][k], 0x5140) ^ 0x80808080u, y = __byte_perm(w[0][k], w[1][k], 0x7362) ^ 0x80808080u;
                    const uint32_t u = __byte_perm(w[2][k], w[3][k], 0x5140) ^ 0x80808080u, v = __byte_perm(w[2][k], w[3][k], 0x7362) ^ 0x80808080u;
                    const int n = hh * kNtBox + 4 * k;
                    mma(o[n + 0], pf, codes_to_half2<0>(x), codes_to_half2<0>(u));
                    mma(o[n + 1], pf, codes_to_half2<1>(x), codes_to_half2<1>(u));
                    mma(o[n + 2], pf, codes_to_half2<0>(y), codes_to_half2<0>(v));
                    mma(o[n + 3], pf, codes_to_half2<1>(y), codes_to_half2<1>(v));
                }
            }
        }
        __syncwarp();                                  // every lane has read the stage
        if (!failed && issued < count) {
            if (lane == 0) issue(issued, stage);
            ++issued;
        }
        if (++stage == a.stages) {
            stage = 0;
            phase ^= 1;
        }

        if ((e.flags & kLast) || i == count - 1) {     // the end of the item, or of this warp's part of it
            l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
            l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
            l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
            l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
            if (seg_whole && (e.flags & kLast)) {
                const RequestShape s = shape_of(a, e.request);
#pragma unroll
                for (int hi = 0; hi < 2; ++hi) {
                    int64_t token;
                    int head, local;
                    if (!row_of(s, e.item, g + 8 * hi, token, head, local)) continue;
                    const float l = hi ? l1 : l0, r = l == 0.f ? 0.f : __fdiv_rn(1.f, l);
                    T* y = static_cast<T*>(a.y) + token * a.y_token_stride + head * a.y_head_stride;
#pragma unroll
                    for (int n = 0; n < kNt; n += 8)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            // column 2 t4 + c of the 8-column tiles n .. n + 7 holds eight neighbouring values
                            const int d = kRowBytes == 128 ? (n / 16) * 128 + 16 * (2 * t4 + c) + (n % 16) : 8 * (2 * t4 + c);
                            uint4 v;
                            v.x = qtz_dev::pack2(o[n + 0][2 * hi + c] * r, o[n + 1][2 * hi + c] * r, T());
                            v.y = qtz_dev::pack2(o[n + 2][2 * hi + c] * r, o[n + 3][2 * hi + c] * r, T());
                            v.z = qtz_dev::pack2(o[n + 4][2 * hi + c] * r, o[n + 5][2 * hi + c] * r, T());
                            v.w = qtz_dev::pack2(o[n + 6][2 * hi + c] * r, o[n + 7][2 * hi + c] * r, T());
                            *reinterpret_cast<uint4*>(y + d) = v;
                        }
                    if (t4 == 0) write_lse(token, head, hi ? m1 : m0, l);
                }
            } else {
                // A part that goes on in the next warp is this warp's last work: it may lie in the ring.  One that began in an
                // earlier warp may be followed by more items: it goes to the workspace.
                const int slot = seg_whole ? 1 : 0;
                float* to = slot ? reinterpret_cast<float*>(smem + warp * ring_bytes)
                                 : a.warp_parts + (static_cast<int64_t>(blockIdx.x) * kWarps + warp) * (16 * D);
#pragma unroll
                for (int n = 0; n < kNt; ++n)
#pragma unroll
                    for (int c = 0; c < 4; ++c) to[(n * 4 + c) * 32 + lane] = o[n][c];
                if (t4 == 0) {
                    s_m[warp][slot][g] = m0;
                    s_m[warp][slot][g + 8] = m1;
                    s_l[warp][slot][g] = l0;
                    s_l[warp][slot][g + 8] = l1;
                }
            }
            if (lane == 0) {
                const RequestShape s = shape_of(a, e.request);
                const int begin = static_cast<int>(prefix[e.request]) + e.item * s.tiles;
                WorkerParts& p = s_parts[warp];
                if (seg_begin == 0) p.head = p.tail = 0;
                if (!seg_whole) {
                    p.head = 1;
                    p.head_begin = begin; p.head_end = begin + s.tiles; p.head_request = e.request; p.head_item = e.item;
                } else if (!(e.flags & kLast)) {
                    p.tail = 1;
                    p.tail_begin = begin; p.tail_end = begin + s.tiles; p.tail_request = e.request; p.tail_item = e.item;
                }
            }
        }
    }
    if (count <= 0 && lane == 0) s_parts[warp].head = s_parts[warp].tail = 0;
    __syncthreads();

    // ---- joining: first the parts that the warps of this CTA left ----
    if (tid == 0) {
        int groups = 0, members = 0;
        for (int w = 0; w < kWarps; ++w) {
            const WorkerParts& p = s_parts[w];
            if (p.head) {
                if (groups == 0 || s_groups[groups - 1].begin != p.head_begin)
                    s_groups[groups++] = Group{p.head_begin, p.head_end, p.head_request, p.head_item, members, 0};
                s_members[members++] = 2 * w;
                ++s_groups[groups - 1].count;
            }
            if (p.tail) {
                s_groups[groups++] = Group{p.tail_begin, p.tail_end, p.tail_request, p.tail_item, members, 1};
                s_members[members++] = 2 * w + 1;
            }
        }
        s_group_count = groups;
    }
    __syncthreads();

    // A unit is eight neighbouring output values: register column c, tiles n .. n + 7, of one lane's position.
    constexpr int kUnits = 4 * (kNt / 8) * 32;
    auto finish = [&](const Group& gr, int unit, const float (&v)[8], float m, float l) {
        const int ln = unit & 31, c = (unit >> 5) & 3, n = (unit >> 7) * 8;
        const RequestShape s = shape_of(a, gr.request);
        int64_t token;
        int head, local;
        if (!row_of(s, gr.item, (ln >> 2) + 8 * (c >> 1), token, head, local)) return;
        const float r = l == 0.f ? 0.f : __fdiv_rn(1.f, l);
        const int column = 2 * (ln & 3) + (c & 1), d = kRowBytes == 128 ? (n / 16) * 128 + 16 * column + (n % 16) : 8 * column;
        uint4 u;
        u.x = qtz_dev::pack2(v[0] * r, v[1] * r, T());
        u.y = qtz_dev::pack2(v[2] * r, v[3] * r, T());
        u.z = qtz_dev::pack2(v[4] * r, v[5] * r, T());
        u.w = qtz_dev::pack2(v[6] * r, v[7] * r, T());
        *reinterpret_cast<uint4*>(static_cast<T*>(a.y) + token * a.y_token_stride + head * a.y_head_stride + d) = u;
        if (n == 0 && column == 0) write_lse(token, head, m, l);
    };
    auto weight = [](float m, float l, float top) { return m == -INFINITY && l == 0.f ? 0.f : ex2(m - top); };

    const int cta_begin = blockIdx.x * cta_share, cta_end = min(cta_begin + cta_share, all);
    constexpr int64_t kPart = 16 * D + 32;
    for (int k = 0; k < s_group_count; ++k) {
        const Group gr = s_groups[k];
        const bool complete = gr.begin >= cta_begin && gr.end <= cta_end;
        float* part = a.cta_parts + (static_cast<int64_t>(blockIdx.x) * 2 + (gr.begin >= cta_begin ? 1 : 0)) * kPart;
        for (int unit = tid; unit < kUnits; unit += kThreads) {
            const int ln = unit & 31, c = (unit >> 5) & 3, n = (unit >> 7) * 8, row = (ln >> 2) + 8 * (c >> 1);
            float top = -INFINITY, l = 0.f, v[8] = {};
            for (int j = 0; j < gr.count; ++j) {
                const int mb = s_members[gr.first + j];
                top = fmaxf(top, s_m[mb >> 1][mb & 1][row]);
            }
            const float base = top == -INFINITY ? 0.f : top;
            for (int j = 0; j < gr.count; ++j) {
                const int mb = s_members[gr.first + j], w = mb >> 1;
                const float* from = (mb & 1) ? reinterpret_cast<const float*>(smem + w * ring_bytes)
                                             : a.warp_parts + (static_cast<int64_t>(blockIdx.x) * kWarps + w) * (16 * D);
                const float wt = weight(s_m[w][mb & 1][row], s_l[w][mb & 1][row], base);
                l = fmaf(s_l[w][mb & 1][row], wt, l);
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] = fmaf(from[((n + x) * 4 + c) * 32 + ln], wt, v[x]);
            }
            if (complete) {
                finish(gr, unit, v, top, l);
            } else {
#pragma unroll
                for (int x = 0; x < 8; ++x) part[((n + x) * 4 + c) * 32 + ln] = v[x];
                if (n == 0 && (c & 1) == 0 && (ln & 3) == 0) {
                    part[16 * D + row] = top;
                    part[16 * D + 16 + row] = l;
                }
            }
        }
    }

    // ---- then the items that lie across CTAs: the last to arrive joins all their parts, in order ----
    for (int k = 0; k < s_group_count; ++k) {
        const Group gr = s_groups[k];
        if (gr.begin >= cta_begin && gr.end <= cta_end) continue;
        const int c0 = gr.begin / cta_share, c1 = (gr.end - 1) / cta_share;
        __threadfence();
        __syncthreads();
        if (tid == 0) {
            const int arrived = atomicAdd(&a.counters[c0], 1);
            s_last = arrived == c1 - c0;
            if (s_last) a.counters[c0] = 0;            // ready for the next call
        }
        __syncthreads();
        if (!s_last) continue;
        __threadfence();
        for (int unit = tid; unit < kUnits; unit += kThreads) {
            const int ln = unit & 31, c = (unit >> 5) & 3, n = (unit >> 7) * 8, row = (ln >> 2) + 8 * (c >> 1);
            auto part_of = [&](int cta) { return a.cta_parts + (static_cast<int64_t>(cta) * 2 + (cta == c0 ? 1 : 0)) * kPart; };
            float top = -INFINITY, l = 0.f, v[8] = {};
            for (int cta = c0; cta <= c1; ++cta) top = fmaxf(top, __ldcg(part_of(cta) + 16 * D + row));
            const float base = top == -INFINITY ? 0.f : top;
            for (int cta = c0; cta <= c1; ++cta) {
                const float* from = part_of(cta);
                const float pl = __ldcg(from + 16 * D + 16 + row), wt = weight(__ldcg(from + 16 * D + row), pl, base);
                l = fmaf(pl, wt, l);
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] = fmaf(__ldcg(from + ((n + x) * 4 + c) * 32 + ln), wt, v[x]);
            }
            finish(gr, unit, v, top, l);
        }
    }
}

int stage_bytes(int head_dim) { return 2 * kTile * head_dim; }

template <typename T, int D>
qtz_status launch(qtz_ctx* h, AttnArgs& a, const CUtensorMap& km, const CUtensorMap& vm, cudaStream_t st)
{
    const size_t fixed = 1024 + static_cast<size_t>(kWarps) * 2 * kBatch * sizeof(TileInfo) + sizeof(uint32_t) * (a.requests + 1);
    // static shared memory of the kernel is a few KB; what is left after the look-up tables goes to the rings
    const size_t room = kSmemLimit - 6 * 1024 - fixed;
    a.stages = static_cast<int32_t>(room / (kWarps * stage_bytes(D)));
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    const size_t smem = fixed + static_cast<size_t>(kWarps) * a.stages * stage_bytes(D);
    QTZ_CUDA(h, cudaFuncSetAttribute(attention_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
    attention_kernel<T, D><<<h->num_sms, kThreads, smem, st>>>(a, km, vm);
    QTZ_LAUNCH_CHECK(h, "attention_kernel");
    return QTZ_OK;
}

int64_t counters_bytes(const qtz_ctx* h) { return (static_cast<int64_t>(h->num_sms) * 4 + 255) / 256 * 256; }

}  // namespace

extern "C" int64_t qtz_kv_attention_workspace_bytes(qtz_handle h, const qtz_kv_cache* cache)
{
    if (!h || qtz_kv_check(cache) != QTZ_OK) return 0;
    const int64_t part = 16 * static_cast<int64_t>(cache->head_dim);
    return counters_bytes(h) + 4 * h->num_sms * (kWarps * part + 2 * (part + 32));
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
        (q_token_stride | q_head_stride | y_token_stride | y_head_stride) % 8 != 0)
        return QTZ_ERR_MISALIGNED;
    // rows of the cache and tiles of the longest possible step are counted in 32 bits
    const int64_t rows = static_cast<int64_t>(cache->blocks) * cache->kv_heads * cache->block_tokens;
    const int64_t group = q_heads / cache->kv_heads, tiles = static_cast<int64_t>(table_width) * cache->block_tokens / kTile;
    const double bound = static_cast<double>(cache->kv_heads) * static_cast<double>(tiles) * (static_cast<double>(tokens) * group / 16 + requests);
    if (rows > 0x7fffffff || bound > 2.0e9 || static_cast<int64_t>(table_width) * cache->block_tokens > 0x7fffffff) return QTZ_ERR_TOO_LARGE;
    qtz_device_guard guard(h->device);
    CUtensorMap km, vm;
    const uint32_t row_bytes = cache->head_dim < 128 ? cache->head_dim : 128;
    const uint64_t dims[2] = {static_cast<uint64_t>(cache->head_dim), static_cast<uint64_t>(rows)};
    const uint64_t strides[1] = {static_cast<uint64_t>(cache->head_dim)};
    const uint32_t box[2] = {row_bytes, kTile};
    if (!qtz_encode_u8_map(&km, cache->k_dev, 2, dims, strides, box, static_cast<int>(row_bytes)) ||
        !qtz_encode_u8_map(&vm, cache->v_dev, 2, dims, strides, box, static_cast<int>(row_bytes)))
        return qtz_cuda_fail(h, cudaErrorInvalidValue, "tensor map of the cache");
    const int64_t part = 16 * static_cast<int64_t>(cache->head_dim);
    float* parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace_dev) + counters_bytes(h));
    AttnArgs a{*cache, q_dev, q_token_stride, q_head_stride, q_heads, static_cast<int32_t>(group), starts_dev, lens_dev, requests,
               static_cast<int32_t>(tokens), table_dev, table_width, scale * 1.44269504f, window < (1 << 30) ? window : 1 << 30, y_dev, y_token_stride, y_head_stride, lse_dev,
               static_cast<int32_t*>(workspace_dev), parts, parts + h->num_sms * kWarps * part, 0, h->wait_budget, h->status_dev};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (ftype == QTZ_F16) {
        if (cache->head_dim == 64) return launch<__half, 64>(h, a, km, vm, st);
        if (cache->head_dim == 128) return launch<__half, 128>(h, a, km, vm, st);
        return launch<__half, 256>(h, a, km, vm, st);
    }
    if (cache->head_dim == 64) return launch<__nv_bfloat16, 64>(h, a, km, vm, st);
    if (cache->head_dim == 128) return launch<__nv_bfloat16, 128>(h, a, km, vm, st);
    return launch<__nv_bfloat16, 256>(h, a, km, vm, st);
}

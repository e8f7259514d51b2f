// The paged 8-bit key/value cache: admission of a step (block tables, slots), quantizing append, read-back.
#include "qtz_half_util.cuh"
#include "qtz_kv.cuh"
#include "qtz_ptx.cuh"

using qtz_ptx::grid_dependency_wait;
using qtz_ptx::grid_launch_dependents;
using qtz_ptx::redux_max;

namespace {

// ------------------------------------------------------------------------------------
// admission
// ------------------------------------------------------------------------------------
constexpr int kSchedThreads = 512;
constexpr int kMaxRequests = 8192;

struct ScheduleArgs {
    const int32_t *cached, *added;
    int32_t requests;
    uint32_t block;
    int32_t width;
    int32_t* table;
    const int32_t *free_ids, *free_count;
    int32_t *starts, *lens;
    int64_t* slots;
    int64_t capacity;
    int32_t* report;
};

// Exclusive prefix sums of (new tokens, new blocks) over the requests, recomputed by every CTA in shared memory: the lengths are a
// few KB that all CTAs read from L2, which is cheaper than a second launch or a grid barrier.  Bound by latency: 3.4 us for 96
// requests with a token each, 5.8 us for 1501 with 0 to 83 tokens, where 0.04 us would do for the 257 KB that have to move.  Each thread
// then finds the request of its token, or of its new block, by bisection, and writes the slot or the table entry.
__global__ void __launch_bounds__(kSchedThreads)
schedule_kernel(const __grid_constant__ ScheduleArgs a)
{
    extern __shared__ int32_t sm[];
    grid_launch_dependents();
    grid_dependency_wait();
    int32_t* const tok = sm;                  // [requests + 1]
    int32_t* const blk = sm + a.requests + 1; // [requests + 1]
    __shared__ int64_t w_tok[kSchedThreads / 32], w_blk[kSchedThreads / 32];
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int per = (a.requests + kSchedThreads - 1) / kSchedThreads;
    const int lo = min(t * per, a.requests), hi = min(lo + per, a.requests);
    auto blocks_of = [&](uint32_t tokens) { return tokens / a.block + (tokens % a.block != 0); };
    int64_t nt = 0, nb = 0;
    bool bad = false;
    for (int r = lo; r < hi; ++r) {
        const int c = a.cached[r], m = a.added[r];
        if (c < 0 || m < 0 || m > 0x7fffffff - c) {
            bad = true;
            continue;
        }
        const uint32_t need = blocks_of(c + m);
        if (need > static_cast<uint32_t>(a.width)) bad = true;
        nt += m;
        nb += need - blocks_of(c);
    }
    int64_t st = nt, sb = nb;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int64_t u = __shfl_up_sync(0xffffffffu, st, off), v = __shfl_up_sync(0xffffffffu, sb, off);
        if (lane >= off) {
            st += u;
            sb += v;
        }
    }
    if (lane == 31) {
        w_tok[warp] = st;
        w_blk[warp] = sb;
    }
    bad = __syncthreads_or(bad);
    int64_t bt = 0, bb = 0, total_t = 0, total_b = 0;
#pragma unroll
    for (int w = 0; w < kSchedThreads / 32; ++w) {
        if (w < warp) {
            bt += w_tok[w];
            bb += w_blk[w];
        }
        total_t += w_tok[w];
        total_b += w_blk[w];
    }
    const int count = *a.free_count;
    const bool refused = bad || total_t > a.capacity || total_t > 0x7fffffff || total_b > count;
    bt += st - nt;
    bb += sb - nb;
    if (!refused) {
        for (int r = lo; r < hi; ++r) {
            const int c = a.cached[r], m = a.added[r];
            tok[r] = static_cast<int32_t>(bt);
            blk[r] = static_cast<int32_t>(bb);
            bt += m;
            bb += blocks_of(c + m) - blocks_of(c);
        }
        if (t == 0) {
            tok[a.requests] = static_cast<int32_t>(total_t);
            blk[a.requests] = static_cast<int32_t>(total_b);
        }
    }
    __syncthreads();
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kSchedThreads + t, step = static_cast<int64_t>(gridDim.x) * kSchedThreads;
    for (int64_t r = first; r <= a.requests; r += step) {
        a.starts[r] = refused ? 0 : tok[r];
        if (r < a.requests) a.lens[r] = a.cached[r] + (refused ? 0 : a.added[r]);
    }
    if (first == 0) {
        a.report[0] = refused ? count : count - static_cast<int32_t>(total_b);
        a.report[1] = refused ? 0 : static_cast<int32_t>(total_t);
        a.report[2] = refused ? 0 : static_cast<int32_t>(total_b);
        a.report[3] = refused ? 1 : 0;
    }
    // request that owns entry i of an exclusive prefix array: the last one that starts at or before i
    auto owner = [&](const int32_t* pre, int i) {
        int u = 0, v = a.requests;
        while (v - u > 1) {
            const int mid = (u + v) >> 1;
            if (pre[mid] <= i) u = mid; else v = mid;
        }
        return u;
    };
    if (!refused)
        for (int64_t i = first; i < total_b; i += step) {
            const int r = owner(blk, static_cast<int>(i));
            a.table[static_cast<int64_t>(r) * a.width + blocks_of(a.cached[r]) + (i - blk[r])] = a.free_ids[count - 1 - i];
        }
    for (int64_t i = first; i < a.capacity; i += step) {
        int64_t slot = -1;
        if (!refused && i < total_t) {
            const int r = owner(tok, static_cast<int>(i));
            const uint32_t c = a.cached[r], pos = c + (static_cast<uint32_t>(i) - tok[r]), j = pos / a.block, have = blocks_of(c);
            const int id = j < have ? a.table[static_cast<int64_t>(r) * a.width + j] : a.free_ids[count - 1 - (blk[r] + static_cast<int>(j - have))];
            slot = static_cast<int64_t>(id) * a.block + (pos - j * a.block);
        }
        a.slots[i] = slot;
    }
}

// ------------------------------------------------------------------------------------
// append
// ------------------------------------------------------------------------------------
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxWindow = 256;
// Pieces (8 values) that a lane holds of a run that its warp takes, and the most that it takes; longer runs take the CTA.  Appending 7000
// prompt tokens (8 heads of 128) takes 23 us in blocks of 16, a run of 8 pieces, and 33 if a warp takes 4 at most; in blocks of 32
// 24, and 41 if it takes 16.  192 single tokens appended and read: 10.5 us, 18.9 with CTAs alone.
constexpr int kWarpHeld = 4, kWarpPieces = 8;
constexpr int kHeld = 4;                      // 16-byte pieces of a long run that a thread keeps in registers: 64 tokens of 128 values

struct AppendArgs {
    qtz_kv_cache c;
    const void* x[2];
    int64_t token_stride[2], head_stride[2];
    const int64_t* slots;
    int64_t tokens;
    int32_t window;                           // tokens whose runs a CTA looks after
    int32_t shift;                            // 16-byte pieces of a token: 1 << shift
    int32_t* status;
};

// Slots are below 2^36 (checked), block_tokens is a multiple of 16: both divide by 16 into 32 bits.
__device__ __forceinline__ uint32_t block_of(int64_t slot, uint32_t block_tokens)
{
    return static_cast<uint32_t>(slot >> 4) / (block_tokens >> 4);
}

// The definition: clamp(round(x / s)); NaN gives the lowest code.
__device__ __noinline__ int32_t quant_code(float x, float s)
{
    float t = rintf(__fdiv_rn(x, s));
    t = fminf(fmaxf(t, -127.f), 127.f);       // fmaxf(NaN, -127) is -127
    return static_cast<int32_t>(t);
}

// Two codes' 16-bit values -> |max| of both halves; NaN is passed over.
__device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b, __half)
{
    const __half2 m = __hmax2(*reinterpret_cast<const __half2*>(&a), __habs2(*reinterpret_cast<const __half2*>(&b)));
    return *reinterpret_cast<const uint32_t*>(&m);
}
__device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b, __nv_bfloat16)
{
    const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), __habs2(*reinterpret_cast<const __nv_bfloat162*>(&b)));
    return *reinterpret_cast<const uint32_t*>(&m);
}

// Largest finite magnitude of eight values, folded into `top`.
template <typename T>
__device__ __forceinline__ float max_abs8(uint4 v, float top)
{
    uint32_t m = max_abs2(max_abs2(max_abs2(max_abs2(0u, v.x, T()), v.y, T()), v.z, T()), v.w, T());
    float2 f = qtz_dev::unpack2(m, T());
    if (fmaxf(f.x, f.y) > 3.402823466e38f) {  // an infinity among them: leave those out
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        f = make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 u = qtz_dev::unpack2(w[k], T());
            if (fabsf(u.x) <= 3.402823466e38f) f.x = fmaxf(f.x, fabsf(u.x));
            if (fabsf(u.y) <= 3.402823466e38f) f.y = fmaxf(f.y, fabsf(u.y));
        }
    }
    return fmaxf(top, fmaxf(f.x, f.y));
}

// Codes of eight values.  x * (1/s) is off from the quotient that the definition rounds by three roundings, 1.5 * 2^-23 of it: 2.3 * 10^-5
// at a code of 127.  It rounds to the same integer unless it lies within 4 * 10^-5 of the middle between two; there, and for NaN and
// infinity, the definition itself is taken.  The integer is read from the mantissa after adding 1.5 * 2^23 (round half to even).
template <typename T>
__device__ __forceinline__ uint2 quantize8(uint4 v, float s, float r)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t q[8];
    bool near_tie = false;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 f = qtz_dev::unpack2(w[k], T());
        const float t0 = f.x * r, t1 = f.y * r, u0 = t0 + 12582912.f, u1 = t1 + 12582912.f;
        near_tie = near_tie || !(fabsf(t0 - (u0 - 12582912.f)) <= 0.49996f) || !(fabsf(t1 - (u1 - 12582912.f)) <= 0.49996f);
        q[2 * k] = __float_as_uint(u0);
        q[2 * k + 1] = __float_as_uint(u1);
    }
    if (near_tie)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 f = qtz_dev::unpack2(w[k], T());
            q[2 * k] = quant_code(f.x, s);
            q[2 * k + 1] = quant_code(f.y, s);
        }
    uint2 o;
    o.x = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
    o.y = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
    return o;
}

// Sixteen old codes under a larger scale: round(code * ratio).
__device__ __forceinline__ uint4 rescale16(uint4 v, float ratio)
{
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int code = static_cast<int>(w[k] << (24 - 8 * j)) >> 24;
            q[j] = __float_as_uint(static_cast<float>(code) * ratio + 12582912.f);
        }
        w[k] = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// What bounds it: each new value is read and its code written once; for a single token the latency of slot, value, old scale.
// A CTA looks after the runs (tokens of one block, neighbours in the list) that begin in its window of the list, for one head and
// tensor.  Short runs take a warp each, long ones the CTA, whose threads keep the run's values in registers between the maximum
// and the codes.  The window grows with the list, so that a step of single tokens spreads over the GPU and a prompt does not launch a
// CTA for each of its tokens.  Prompts of 10 800 tokens (8 heads of 128): 27 us for 66 MB, 2.5 TB/s, with the issue slots 59 % busy:
// loads, maxima and codes of a run follow one another with nothing of the next run under way (shared memory, which has the room for
// it, is not used), and four CTAs an SM fill the gaps only in part.  192 single tokens: about 6 us, of which 3 the chain slot, value,
// old scale, code.
template <typename T>
__global__ void __launch_bounds__(kThreads, 4)
append_kernel(const __grid_constant__ AppendArgs a)
{
    __shared__ int64_t s_slot[kMaxWindow + 1];
    __shared__ int s_start[kMaxWindow], s_len[kMaxWindow], s_count;
    __shared__ float s_top[2][kWarps];
    grid_dependency_wait();                            // the next kernel is not let in early: its waiting CTAs cost this one 3 us of 7
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, heads = a.c.kv_heads, dim = a.c.head_dim;
    const uint32_t block = a.c.block_tokens;
    const int h = blockIdx.y, which = blockIdx.z, shift = a.shift;
    const int64_t i0 = static_cast<int64_t>(blockIdx.x) * a.window;
    const int n = static_cast<int>(min(static_cast<int64_t>(a.window), a.tokens - i0));
    const int64_t limit = static_cast<int64_t>(a.c.blocks) * block;
    if (tid == 0) s_count = 0;
    for (int j = tid; j <= n; j += kThreads) s_slot[j] = i0 + j > 0 ? a.slots[i0 + j - 1] : -1;   // one before the window
    __syncthreads();
    // runs that begin here, in any order: they write different blocks
    for (int j = tid; j < n; j += kThreads) {
        const int64_t slot = s_slot[j + 1], before = s_slot[j];
        if (slot < 0) continue;
        if (slot >= limit) {
            qtz_dev::report_invalid(a.status, QTZ_SITE_KV_APPEND);
            continue;
        }
        if (before >= 0 && before < limit && block_of(before, block) == block_of(slot, block)) continue;
        s_start[atomicAdd(&s_count, 1)] = j;
    }
    __syncthreads();
    const int runs = s_count;
    const int64_t ts = a.token_stride[which];
    const T* const x = static_cast<const T*>(a.x[which]) + h * a.head_stride[which] + i0 * ts;
    const int mask = (1 << shift) - 1;
    // piece p of the run that begins at token j of the window
    auto value = [&](int j, int p) { return *reinterpret_cast<const uint4*>(x + (j + (p >> shift)) * ts + ((p & mask) << 3)); };
    // The scale of a block after its run, and what its old codes are multiplied by (1: nothing to do).
    auto new_scale = [&](float top, const float* scale, int offset, float& ratio) {
        float s = fmaxf(__fdiv_rn(top, 127.f), QTZ_KV_MIN_SCALE);
        ratio = 1.f;
        if (offset > 0) {
            const float old = fmaxf(*scale, QTZ_KV_MIN_SCALE);
            if (old < s) ratio = __fdiv_rn(old, s);
            s = fmaxf(s, old);
        }
        return s;
    };
    auto place = [&](uint32_t b, float*& scale, int8_t*& codes) {
        const int64_t bh = static_cast<int64_t>(b) * heads + h;
        scale = (which ? a.c.v_scale_dev : a.c.k_scale_dev) + bh;
        codes = (which ? a.c.v_dev : a.c.k_dev) + bh * block * dim;
    };
    // where piece p of that run goes, within its block
    auto target = [&](int j, int p, int64_t first) {
        const int t = j + (p >> shift);
        const int64_t slot = t < n ? s_slot[t + 1] : a.slots[i0 + t];
        return static_cast<int>(slot - first) * dim + ((p & mask) << 3);
    };

    bool long_runs = false;
    for (int k = warp; k < runs; k += kWarps) {
        const int j = s_start[k];
        const int64_t slot = s_slot[j + 1];
        const uint32_t b = block_of(slot, block);
        const int64_t first = static_cast<int64_t>(b) * block;
        int len = 0;
        for (bool more = true; more;) {
            const int t = j + len + lane;
            const int64_t other = i0 + t < a.tokens ? (t < n ? s_slot[t + 1] : a.slots[i0 + t]) : -1;
            const unsigned off = ~__ballot_sync(0xffffffffu, other >= first && other < first + block);
            more = off == 0;
            len = min(len + (more ? 32 : __ffs(off) - 1), static_cast<int>(block));
            more = more && len < static_cast<int>(block);
        }
        if (lane == 0) s_len[k] = len;
        if (len << shift > kWarpPieces * 32) {
            long_runs = true;
            continue;
        }
        float* scale;
        int8_t* codes;
        place(b, scale, codes);
        const int offset = static_cast<int>(slot - first), count = len << shift;
        uint4 v[kWarpHeld];
        float top = 0.f;
#pragma unroll
        for (int q = 0; q < kWarpHeld; ++q) {
            v[q] = make_uint4(0, 0, 0, 0);
            if (q * 32 + lane < count) v[q] = value(j, q * 32 + lane);
        }
#pragma unroll
        for (int q = 0; q < kWarpHeld; ++q) top = max_abs8<T>(v[q], top);
        for (int p = kWarpHeld * 32 + lane; p < count; p += 32) top = max_abs8<T>(value(j, p), top);   // read again below
        top = redux_max(top);
        float ratio;
        const float s = new_scale(top, scale, offset, ratio), r = __frcp_rn(s);
        __syncwarp();
        if (lane == 0) *scale = s;
        if (ratio != 1.f)
            for (int p = lane; p < offset * dim / 16; p += 32) reinterpret_cast<uint4*>(codes)[p] = rescale16(reinterpret_cast<uint4*>(codes)[p], ratio);
#pragma unroll
        for (int q = 0; q < kWarpHeld; ++q) {
            const int p = q * 32 + lane;
            if (p < count) *reinterpret_cast<uint2*>(codes + target(j, p, first)) = quantize8<T>(v[q], s, r);
        }
        for (int p = kWarpHeld * 32 + lane; p < count; p += 32)
            *reinterpret_cast<uint2*>(codes + target(j, p, first)) = quantize8<T>(value(j, p), s, r);
    }
    if (!__syncthreads_or(long_runs)) return;
    int turn = 0;
    for (int k = 0; k < runs; ++k) {
        const int len = s_len[k];
        if (len << shift <= kWarpPieces * 32) continue;
        const int j = s_start[k];
        const int64_t slot = s_slot[j + 1];
        const uint32_t b = block_of(slot, block);
        const int64_t first = static_cast<int64_t>(b) * block;
        float* scale;
        int8_t* codes;
        place(b, scale, codes);
        const int offset = static_cast<int>(slot - first), count = len << shift;
        const float before = offset > 0 ? *scale : 0.f;    // in flight beside the values
        uint4 held[kHeld];
        float top = 0.f;
#pragma unroll
        for (int q = 0; q < kHeld; ++q) {
            held[q] = make_uint4(0, 0, 0, 0);
            if (q * kThreads + tid < count) held[q] = value(j, q * kThreads + tid);
        }
#pragma unroll
        for (int q = 0; q < kHeld; ++q) top = max_abs8<T>(held[q], top);
        for (int p = kHeld * kThreads + tid; p < count; p += kThreads) top = max_abs8<T>(value(j, p), top);   // read again below
        top = redux_max(top);
        float* const tops = s_top[turn ^= 1];          // two places: a run's are read while the next one's are written
        if (lane == 0) tops[warp] = top;
        __syncthreads();                               // and every thread has read the old scale
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, tops[w]);
        float ratio;
        const float s = new_scale(top, &before, offset, ratio), r = __frcp_rn(s);
        if (tid == 0) *scale = s;
        if (ratio != 1.f)
            for (int p = tid; p < offset * dim / 16; p += kThreads) reinterpret_cast<uint4*>(codes)[p] = rescale16(reinterpret_cast<uint4*>(codes)[p], ratio);
#pragma unroll
        for (int q = 0; q < kHeld; ++q) {
            const int p = q * kThreads + tid;
            if (p < count) *reinterpret_cast<uint2*>(codes + target(j, p, first)) = quantize8<T>(held[q], s, r);
        }
        for (int p = kHeld * kThreads + tid; p < count; p += kThreads)
            *reinterpret_cast<uint2*>(codes + target(j, p, first)) = quantize8<T>(value(j, p), s, r);
    }
}

// ------------------------------------------------------------------------------------
// read
// ------------------------------------------------------------------------------------
struct ReadArgs {
    qtz_kv_cache c;
    const int64_t* slots;
    int64_t tokens;
    void* out[2];
    int32_t* status;
};

// One warp per token: lanes take sixteen codes at a time of all heads of both tensors.  One byte in, two or four out.  10 800 tokens of 8
// heads of 128 to bf16: 16 us for 66 MB, 4.1 TB/s, 0.64 of the copy rate: a warp has one token's loads under way, behind its look-up.
template <typename T>
__global__ void __launch_bounds__(kThreads)
read_kernel(const __grid_constant__ ReadArgs a)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (i >= a.tokens) return;
    grid_dependency_wait();
    const int64_t slot = a.slots[i];
    const uint32_t block = a.c.block_tokens;
    const bool bad = slot >= static_cast<int64_t>(a.c.blocks) * block, none = slot < 0 || bad;
    if (bad && lane == 0) qtz_dev::report_invalid(a.status, QTZ_SITE_KV_READ);
    const uint32_t b = none ? 0 : block_of(slot, block);
    const int offset = none ? 0 : static_cast<int>(slot - static_cast<int64_t>(b) * block);
    const int shift = a.c.head_dim == 64 ? 2 : a.c.head_dim == 128 ? 3 : 4, pieces = a.c.kv_heads << shift;   // of 16 codes
#pragma unroll 4
    for (int p = lane; p < 2 * pieces; p += 32) {
        const int which = p >= pieces, u = p - which * pieces, h = u >> shift, d = (u - (h << shift)) * 16;
        const int64_t bh = static_cast<int64_t>(b) * a.c.kv_heads + h;
        uint4 q = make_uint4(0, 0, 0, 0);
        float s = 0.f;
        if (!none) {
            q = *reinterpret_cast<const uint4*>((which ? a.c.v_dev : a.c.k_dev) + (bh * block + offset) * a.c.head_dim + d);
            s = fmaxf((which ? a.c.v_scale_dev : a.c.k_scale_dev)[bh], QTZ_KV_MIN_SCALE);
        }
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
        T* const out = static_cast<T*>(a.out[which]) + i * (pieces * 16) + u * 16;
        float f[16];
#pragma unroll
        for (int k = 0; k < 16; ++k)          // 1.5 * 2^23 + 128 + code, from the code's byte with its sign bit flipped
            f[k] = (__uint_as_float(__byte_perm(w[k / 4] ^ 0x80808080u, 0x4b400000u, 0x7650 | (k & 3))) - 12583040.f) * s;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int k = 0; k < 16; k += 4) *reinterpret_cast<float4*>(out + k) = make_float4(f[k], f[k + 1], f[k + 2], f[k + 3]);
        } else {
#pragma unroll
            for (int k = 0; k < 16; k += 8) {
                uint4 o;
                o.x = qtz_dev::pack2(f[k], f[k + 1], T());
                o.y = qtz_dev::pack2(f[k + 2], f[k + 3], T());
                o.z = qtz_dev::pack2(f[k + 4], f[k + 5], T());
                o.w = qtz_dev::pack2(f[k + 6], f[k + 7], T());
                *reinterpret_cast<uint4*>(out + k) = o;
            }
        }
    }
}

}  // namespace

qtz_status qtz_kv_check(const qtz_kv_cache* c)
{
    if (!c || !c->k_dev || !c->v_dev || !c->k_scale_dev || !c->v_scale_dev) return QTZ_ERR_INVALID_ARG;
    if (c->blocks <= 0 || c->kv_heads <= 0 || c->block_tokens <= 0 || c->head_dim <= 0) return QTZ_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return QTZ_ERR_UNSUPPORTED;
    if (c->block_tokens % 16 != 0 || c->block_tokens > 256) return QTZ_ERR_UNSUPPORTED;
    if (c->kv_heads > 65535) return QTZ_ERR_TOO_LARGE;
    if (static_cast<int64_t>(c->blocks) * c->block_tokens >= (1ll << 36)) return QTZ_ERR_TOO_LARGE;
    if (!qtz_aligned16(c->k_dev) || !qtz_aligned16(c->v_dev)) return QTZ_ERR_MISALIGNED;
    return QTZ_OK;
}

extern "C" qtz_status qtz_kv_schedule(qtz_handle h, const int32_t* cached_dev, const int32_t* added_dev, int32_t requests,
                                      int32_t block_tokens, int32_t* table_dev, int32_t table_width, const int32_t* free_dev,
                                      const int32_t* free_count_dev, int32_t* starts_dev, int32_t* lens_dev, int64_t* slots_dev,
                                      int64_t capacity, int32_t* report_dev, void* stream)
{
    if (!h || !cached_dev || !added_dev || !table_dev || !free_dev || !free_count_dev || !starts_dev || !lens_dev || !report_dev)
        return QTZ_ERR_INVALID_ARG;
    if (requests <= 0 || block_tokens <= 0 || table_width <= 0 || capacity < 0 || (capacity > 0 && !slots_dev)) return QTZ_ERR_INVALID_ARG;
    if (requests > kMaxRequests) return QTZ_ERR_TOO_LARGE;
    qtz_device_guard guard(h->device);
    const ScheduleArgs a{cached_dev, added_dev, requests, static_cast<uint32_t>(block_tokens), table_width, table_dev, free_dev, free_count_dev,
                         starts_dev, lens_dev, slots_dev, capacity, report_dev};
    const size_t smem = 2 * sizeof(int32_t) * (requests + 1);
    qtz_status s = qtz_allow_smem(h, schedule_kernel);
    if (s != QTZ_OK) return s;
    const int64_t work = capacity > requests + 1 ? capacity : requests + 1, ctas = (work + kSchedThreads - 1) / kSchedThreads;
    QTZ_CUDA(h, qtz_launch_dependent(schedule_kernel, dim3(static_cast<unsigned>(ctas < h->num_sms ? ctas : h->num_sms)), kSchedThreads, smem,
                                     static_cast<cudaStream_t>(stream), a));
    return QTZ_OK;
}

extern "C" qtz_status qtz_kv_append(qtz_handle h, const qtz_kv_cache* cache, const void* k_dev, int64_t k_token_stride,
                                    int64_t k_head_stride, const void* v_dev, int64_t v_token_stride, int64_t v_head_stride,
                                    int32_t ftype, const int64_t* slots_dev, int64_t tokens, void* stream)
{
    if (!h || tokens < 0) return QTZ_ERR_INVALID_ARG;
    qtz_status s = qtz_kv_check(cache);
    if (s != QTZ_OK) return s;
    if (ftype != QTZ_F16 && ftype != QTZ_BF16) return QTZ_ERR_INVALID_ARG;
    if (tokens == 0) return QTZ_OK;
    if (!k_dev || !v_dev || !slots_dev) return QTZ_ERR_INVALID_ARG;
    if (!qtz_aligned16(k_dev) || !qtz_aligned16(v_dev) || !qtz_kv_strides_ok(tokens, k_token_stride, cache->kv_heads, k_head_stride) ||
        !qtz_kv_strides_ok(tokens, v_token_stride, cache->kv_heads, v_head_stride))
        return QTZ_ERR_MISALIGNED;
    qtz_device_guard guard(h->device);
    // About 8 CTAs an SM, each with at least a token for every warp.  Prompts of 10 800 tokens, read-back included: 43 us, with 4 CTAs an SM
    // 46, with the smallest window throughout 73.  192 single tokens: 10.5, with the largest window 39.
    int64_t window = (tokens * 2 * cache->kv_heads + 8 * h->num_sms - 1) / (8 * h->num_sms);
    window = window < kWarps ? kWarps : window > kMaxWindow ? kMaxWindow : window;
    const int64_t ctas = (tokens + window - 1) / window;
    if (ctas > 0x7fffffff) return QTZ_ERR_TOO_LARGE;
    const AppendArgs a{*cache, {k_dev, v_dev}, {k_token_stride, v_token_stride}, {k_head_stride, v_head_stride}, slots_dev, tokens,
                       static_cast<int32_t>(window), cache->head_dim == 64 ? 3 : cache->head_dim == 128 ? 4 : 5, h->status_dev};
    const dim3 grid(static_cast<unsigned>(ctas), static_cast<unsigned>(cache->kv_heads), 2);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    QTZ_CUDA(h, qtz_launch_dependent(ftype == QTZ_F16 ? append_kernel<__half> : append_kernel<__nv_bfloat16>, grid, kThreads, 0, st, a));
    return QTZ_OK;
}

extern "C" qtz_status qtz_kv_read(qtz_handle h, const qtz_kv_cache* cache, const int64_t* slots_dev, int64_t tokens, int32_t ftype,
                                  void* k_out_dev, void* v_out_dev, void* stream)
{
    if (!h || tokens < 0) return QTZ_ERR_INVALID_ARG;
    qtz_status s = qtz_kv_check(cache);
    if (s != QTZ_OK) return s;
    if (ftype != QTZ_F16 && ftype != QTZ_BF16 && ftype != QTZ_F32) return QTZ_ERR_INVALID_ARG;
    if (tokens == 0) return QTZ_OK;
    if (!slots_dev || !k_out_dev || !v_out_dev) return QTZ_ERR_INVALID_ARG;
    if (!qtz_aligned16(k_out_dev) || !qtz_aligned16(v_out_dev)) return QTZ_ERR_MISALIGNED;
    const int64_t ctas = (tokens + kWarps - 1) / kWarps;
    if (ctas > 0x7fffffff) return QTZ_ERR_TOO_LARGE;
    qtz_device_guard guard(h->device);
    const ReadArgs a{*cache, slots_dev, tokens, {k_out_dev, v_out_dev}, h->status_dev};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    QTZ_CUDA(h, qtz_launch_dependent(ftype == QTZ_F16 ? read_kernel<__half> : ftype == QTZ_BF16 ? read_kernel<__nv_bfloat16> : read_kernel<float>,
                                     dim3(static_cast<unsigned>(ctas)), kThreads, 0, st, a));
    return QTZ_OK;
}

// The paged 8-bit key/value cache: admission of a step (block tables, slots), quantizing append, read-back.
#include "qtz_half_util.cuh"
#include "qtz_kv.cuh"

using qtz_dev::from_f32;
using qtz_dev::report_invalid;

namespace {

// ------------------------------------------------------------------------------------
// admission
// ------------------------------------------------------------------------------------
constexpr int kSchedThreads = 512;
constexpr int kMaxRequests = 8192;

struct ScheduleArgs {
    const int32_t *cached, *added;
    int32_t requests, block, width;
    int32_t* table;
    const int32_t *free_ids, *free_count;
    int32_t *starts, *lens;
    int64_t* slots;
    int64_t capacity;
    int32_t* report;
};

// Exclusive prefix sums of (new tokens, new blocks) over the requests, recomputed by every CTA in shared memory: the
// lengths are a few KB that all CTAs read from L2, which is cheaper than a second launch or a grid barrier.  Each CTA
// then writes its share of the slots and of the table.
__global__ void __launch_bounds__(kSchedThreads)
schedule_kernel(ScheduleArgs a)
{
    extern __shared__ int32_t sm[];
    int32_t* tok = sm;                        // [requests + 1]
    int32_t* blk = sm + a.requests + 1;       // [requests + 1]
    __shared__ int64_t w_tok[kSchedThreads / 32];
    __shared__ int32_t w_blk[kSchedThreads / 32];
    __shared__ int s_bad;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    if (t == 0) s_bad = 0;
    __syncthreads();
    const int per = (a.requests + kSchedThreads - 1) / kSchedThreads;
    const int lo = min(t * per, a.requests), hi = min(lo + per, a.requests);
    int64_t nt = 0, nb = 0;
    bool bad = false;
    for (int r = lo; r < hi; ++r) {
        const int64_t c = a.cached[r], m = a.added[r];
        if (c < 0 || m < 0) { bad = true; continue; }
        const int64_t need = (c + m + a.block - 1) / a.block;
        if (need > a.width || c + m > 0x7fffffff) bad = true;
        nt += m;
        nb += need - (c + a.block - 1) / a.block;
    }
    int64_t st = nt, sb = nb;
    for (int off = 1; off < 32; off <<= 1) {
        const int64_t u = __shfl_up_sync(0xffffffffu, st, off), v = __shfl_up_sync(0xffffffffu, sb, off);
        if (lane >= off) { st += u; sb += v; }
    }
    __shared__ int64_t w_b[kSchedThreads / 32];
    if (lane == 31) { w_tok[warp] = st; w_b[warp] = sb; }
    if (bad) s_bad = 1;
    __syncthreads();
    int64_t bt = 0, bb = 0, total_t = 0, total_b = 0;
    for (int w = 0; w < kSchedThreads / 32; ++w) {
        if (w < warp) { bt += w_tok[w]; bb += w_b[w]; }
        total_t += w_tok[w];
        total_b += w_b[w];
    }
    (void)w_blk;
    const int64_t count = *a.free_count;
    const bool refused = s_bad || total_t > a.capacity || total_t > 0x7fffffff || total_b > count;
    bt += st - nt;
    bb += sb - nb;
    if (!refused)
        for (int r = lo; r < hi; ++r) {
            const int c = a.cached[r], m = a.added[r];
            tok[r] = static_cast<int32_t>(bt);
            blk[r] = static_cast<int32_t>(bb);
            bt += m;
            bb += (static_cast<int64_t>(c) + m + a.block - 1) / a.block - (static_cast<int64_t>(c) + a.block - 1) / a.block;
        }
    if (t == 0 && !refused) {
        tok[a.requests] = static_cast<int32_t>(total_t);
        blk[a.requests] = static_cast<int32_t>(total_b);
    }
    __syncthreads();
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kSchedThreads + t, step = static_cast<int64_t>(gridDim.x) * kSchedThreads;
    for (int64_t r = first; r <= a.requests; r += step) {
        a.starts[r] = refused ? 0 : tok[r];
        if (r < a.requests) a.lens[r] = a.cached[r] + (refused ? 0 : a.added[r]);
    }
    if (first == 0) {
        a.report[0] = static_cast<int32_t>(refused ? count : count - total_b);
        a.report[1] = refused ? 0 : static_cast<int32_t>(total_t);
        a.report[2] = refused ? 0 : static_cast<int32_t>(total_b);
        a.report[3] = refused ? 1 : 0;
    }
    // request that owns entry i of an exclusive prefix array: the last one that starts at or before i
    auto owner = [&](const int32_t* pre, int64_t i) {
        int u = 0, v = a.requests;
        while (v - u > 1) {
            const int mid = (u + v) >> 1;
            if (pre[mid] <= i) u = mid; else v = mid;
        }
        return u;
    };
    if (!refused)
        for (int64_t i = first; i < total_b; i += step) {
            const int r = owner(blk, i);
            const int have = (a.cached[r] + a.block - 1) / a.block;
            a.table[static_cast<int64_t>(r) * a.width + have + (i - blk[r])] = a.free_ids[count - 1 - i];
        }
    for (int64_t i = first; i < a.capacity; i += step) {
        int64_t slot = -1;
        if (!refused && i < total_t) {
            const int r = owner(tok, i);
            const int c = a.cached[r];
            const int64_t pos = c + (i - tok[r]);
            const int j = static_cast<int>(pos / a.block), have = (c + a.block - 1) / a.block;
            const int64_t id = j < have ? a.table[static_cast<int64_t>(r) * a.width + j] : a.free_ids[count - 1 - (blk[r] + j - have)];
            slot = id * a.block + pos % a.block;
        }
        a.slots[i] = slot;
    }
}

// ------------------------------------------------------------------------------------
// append
// ------------------------------------------------------------------------------------
constexpr int kThreads = 256;

struct AppendArgs {
    qtz_kv_cache c;
    const void* x[2];
    int64_t token_stride[2], head_stride[2];
    const int64_t* slots;
    int64_t tokens;
    int32_t* status;
};

__device__ __forceinline__ int32_t quant_code(float x, float s)
{
    float t = rintf(__fdiv_rn(x, s));
    t = fminf(fmaxf(t, -127.f), 127.f);   // NaN: fmaxf returns the bound
    return static_cast<int32_t>(t);
}

// One warp per (token, head, tensor); the one whose token is the first of its block in the list does the whole run.
template <typename T>
__global__ void __launch_bounds__(kThreads)
append_kernel(AppendArgs a)
{
    const int64_t id = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31, heads = a.c.kv_heads, dim = a.c.head_dim, block = a.c.block_tokens;
    const int64_t i = id / (2 * heads);
    if (i >= a.tokens) return;
    const int rest = static_cast<int>(id - i * 2 * heads), h = rest >> 1, which = rest & 1;
    const int64_t slot = a.slots[i];
    if (slot < 0) return;
    const int64_t b = slot / block;
    if (b >= a.c.blocks) {
        if (lane == 0) report_invalid(a.status, QTZ_SITE_KV_APPEND);
        return;
    }
    if (i > 0 && a.slots[i - 1] >= 0 && a.slots[i - 1] / block == b) return;
    const T* x = static_cast<const T*>(a.x[which]) + h * a.head_stride[which];
    const int64_t ts = a.token_stride[which];
    float top = 0.f;
    int64_t end = i;
    for (; end < a.tokens && end - i < block; ++end) {
        const int64_t s = a.slots[end];
        if (s < 0 || s / block != b) break;
        for (int d = lane; d < dim; d += 32) {
            const float v = fabsf(qtz_dev::to_f32(x[end * ts + d]));
            if (v <= 3.402823466e38f) top = fmaxf(top, v);
        }
    }
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    float s = fmaxf(__fdiv_rn(top, 127.f), QTZ_KV_MIN_SCALE);
    float* scale = (which ? a.c.v_scale_dev : a.c.k_scale_dev) + b * heads + h;
    int8_t* codes = (which ? a.c.v_dev : a.c.k_dev) + (b * heads + h) * static_cast<int64_t>(block) * dim;
    const int o = static_cast<int>(slot - b * block);
    if (o > 0) {
        const float old = fmaxf(*scale, QTZ_KV_MIN_SCALE);
        if (old < s) {
            const float r = __fdiv_rn(old, s);
            for (int e = lane; e < o * dim; e += 32) codes[e] = static_cast<int8_t>(rintf(static_cast<float>(codes[e]) * r));
        }
        s = fmaxf(s, old);
    }
    __syncwarp();
    if (lane == 0) *scale = s;
    for (int64_t j = i; j < end; ++j) {
        int8_t* to = codes + (a.slots[j] - b * block) * dim;
        for (int d = lane; d < dim; d += 32) to[d] = static_cast<int8_t>(quant_code(qtz_dev::to_f32(x[j * ts + d]), s));
    }
}

// ------------------------------------------------------------------------------------
// read
// ------------------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(kThreads)
read_kernel(qtz_kv_cache c, const int64_t* __restrict__ slots, int64_t tokens, T* __restrict__ k_out, T* __restrict__ v_out, int32_t* status)
{
    const int per = c.kv_heads * c.head_dim / 8;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t i = id / per;
    if (i >= tokens) return;
    const int e = static_cast<int>(id - i * per) * 8, h = e / c.head_dim, d = e % c.head_dim;
    const int64_t slot = slots[i], b = slot / c.block_tokens;
    const bool bad = slot >= 0 && b >= c.blocks, none = slot < 0 || bad;
    if (bad && e == 0) report_invalid(status, QTZ_SITE_KV_READ);
    const int64_t at = none ? 0 : ((b * c.kv_heads + h) * c.block_tokens + slot % c.block_tokens) * c.head_dim + d;
    for (int which = 0; which < 2; ++which) {
        const float s = none ? 0.f : fmaxf((which ? c.v_scale_dev : c.k_scale_dev)[b * c.kv_heads + h], QTZ_KV_MIN_SCALE);
        T* out = (which ? v_out : k_out) + i * (c.kv_heads * c.head_dim) + e;
        const int8_t* q = (which ? c.v_dev : c.k_dev) + at;
        for (int j = 0; j < 8; ++j) out[j] = from_f32<T>(none ? 0.f : static_cast<float>(q[j]) * s);
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
    const ScheduleArgs a{cached_dev, added_dev, requests, block_tokens, table_width, table_dev, free_dev, free_count_dev,
                         starts_dev, lens_dev, slots_dev, capacity, report_dev};
    const size_t smem = 2 * sizeof(int32_t) * (requests + 1);
    QTZ_CUDA(h, cudaFuncSetAttribute(schedule_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * sizeof(int32_t) * (kMaxRequests + 1)));
    const int64_t work = capacity > requests + 1 ? capacity : requests + 1;
    const int64_t ctas = (work + 4 * kSchedThreads - 1) / (4 * kSchedThreads);
    schedule_kernel<<<static_cast<unsigned>(ctas < h->num_sms ? ctas : h->num_sms), kSchedThreads, smem, static_cast<cudaStream_t>(stream)>>>(a);
    QTZ_LAUNCH_CHECK(h, "schedule_kernel");
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
    if (!qtz_aligned16(k_dev) || !qtz_aligned16(v_dev) || (k_token_stride | k_head_stride | v_token_stride | v_head_stride) % 8 != 0)
        return QTZ_ERR_MISALIGNED;
    const int64_t warps = tokens * 2 * cache->kv_heads, ctas = (warps * 32 + kThreads - 1) / kThreads;
    if (ctas > 0x7fffffff) return QTZ_ERR_TOO_LARGE;
    qtz_device_guard guard(h->device);
    AppendArgs a{*cache, {k_dev, v_dev}, {k_token_stride, v_token_stride}, {k_head_stride, v_head_stride}, slots_dev, tokens, h->status_dev};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (ftype == QTZ_F16) append_kernel<__half><<<static_cast<unsigned>(ctas), kThreads, 0, st>>>(a);
    else append_kernel<__nv_bfloat16><<<static_cast<unsigned>(ctas), kThreads, 0, st>>>(a);
    QTZ_LAUNCH_CHECK(h, "append_kernel");
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
    const int64_t threads = tokens * (cache->kv_heads * cache->head_dim / 8), ctas = (threads + kThreads - 1) / kThreads;
    if (ctas > 0x7fffffff) return QTZ_ERR_TOO_LARGE;
    qtz_device_guard guard(h->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const unsigned g = static_cast<unsigned>(ctas);
    if (ftype == QTZ_F16) read_kernel<<<g, kThreads, 0, st>>>(*cache, slots_dev, tokens, static_cast<__half*>(k_out_dev), static_cast<__half*>(v_out_dev), h->status_dev);
    else if (ftype == QTZ_BF16) read_kernel<<<g, kThreads, 0, st>>>(*cache, slots_dev, tokens, static_cast<__nv_bfloat16*>(k_out_dev), static_cast<__nv_bfloat16*>(v_out_dev), h->status_dev);
    else read_kernel<<<g, kThreads, 0, st>>>(*cache, slots_dev, tokens, static_cast<float*>(k_out_dev), static_cast<float*>(v_out_dev), h->status_dev);
    QTZ_LAUNCH_CHECK(h, "read_kernel");
    return QTZ_OK;
}

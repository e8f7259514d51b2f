// Attention of new tokens over the paged 8-bit key/value cache.
#include "qtz_half_util.cuh"
#include "qtz_kv.cuh"

namespace {

constexpr int kMaxRequests = 8192;
constexpr int kWarps = 4;

struct AttnArgs {
    qtz_kv_cache c;
    const void* q;
    int64_t q_token_stride, q_head_stride;
    int32_t q_heads;
    const int32_t *starts, *lens;
    int32_t requests;
    const int32_t* table;
    int32_t width;
    float scale;
    int32_t window;
    void* y;
    int64_t y_token_stride, y_head_stride;
    float* lse;
    int32_t* status;
};

// One CTA per (row, head): warps take positions in turn, lanes share the head's dimensions; running maximum and sum.
template <typename T, int D>
__global__ void __launch_bounds__(kWarps * 32)
attention_kernel(AttnArgs a)
{
    constexpr int E = D / 32;
    const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int u = 0, v = a.requests;
    while (v - u > 1) {
        const int mid = (u + v) >> 1;
        if (a.starts[mid] <= t) u = mid; else v = mid;
    }
    if (t >= a.starts[a.requests]) return;
    const int g = h / (a.q_heads / a.c.kv_heads);
    const int end = min(a.lens[u] - (a.starts[u + 1] - t) + 1, a.width * a.c.block_tokens);
    const int begin = a.window > 0 ? max(0, end - a.window) : 0;
    const T* q = static_cast<const T*>(a.q) + t * a.q_token_stride + h * a.q_head_stride + lane * E;
    float qf[E], o[E] = {}, m = -INFINITY, l = 0.f;
    for (int e = 0; e < E; ++e) qf[e] = qtz_dev::to_f32(q[e]);
    for (int p = begin + warp; p < end; p += kWarps) {
        const int id = a.table[static_cast<int64_t>(u) * a.width + p / a.c.block_tokens];
        if (id < 0 || id >= a.c.blocks) {
            if (lane == 0) qtz_dev::report_invalid(a.status, QTZ_SITE_KV_ATTENTION);
            continue;
        }
        const int64_t bh = static_cast<int64_t>(id) * a.c.kv_heads + g;
        const int64_t at = (bh * a.c.block_tokens + p % a.c.block_tokens) * D + lane * E;
        float s = 0.f;
        for (int e = 0; e < E; ++e) s = fmaf(qf[e], static_cast<float>(a.c.k_dev[at + e]), s);
        for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        s *= fmaxf(a.c.k_scale_dev[bh], QTZ_KV_MIN_SCALE) * a.scale;
        const float mn = fmaxf(m, s), w = __expf(s - mn), keep = __expf(m - mn);
        l = fmaf(l, keep, w);
        const float ws = w * fmaxf(a.c.v_scale_dev[bh], QTZ_KV_MIN_SCALE);
        for (int e = 0; e < E; ++e) o[e] = fmaf(ws, static_cast<float>(a.c.v_dev[at + e]), o[e] * keep);
        m = mn;
    }
    __shared__ float sm[kWarps], sl[kWarps], so[kWarps][D];
    if (lane == 0) { sm[warp] = m; sl[warp] = l; }
    for (int e = 0; e < E; ++e) so[warp][lane * E + e] = o[e];
    __syncthreads();
    if (warp != 0) return;
    float top = -INFINITY, total = 0.f;
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sm[w]);
    float keep[kWarps];
    for (int w = 0; w < kWarps; ++w) {
        keep[w] = sm[w] == -INFINITY && sl[w] == 0.f ? 0.f : expf(sm[w] - top);
        total += sl[w] * keep[w];
    }
    T* y = static_cast<T*>(a.y) + t * a.y_token_stride + h * a.y_head_stride + lane * E;
    for (int e = 0; e < E; ++e) {
        float s = 0.f;
        for (int w = 0; w < kWarps; ++w) s = fmaf(so[w][lane * E + e], keep[w], s);
        y[e] = qtz_dev::from_f32<T>(total == 0.f ? 0.f : s / total);
    }
    if (a.lse && lane == 0) a.lse[static_cast<int64_t>(t) * a.q_heads + h] = top + logf(total);
}

template <typename T>
void launch(const AttnArgs& a, int64_t tokens, cudaStream_t st)
{
    const dim3 grid(static_cast<unsigned>(tokens), static_cast<unsigned>(a.q_heads));
    if (a.c.head_dim == 64) attention_kernel<T, 64><<<grid, kWarps * 32, 0, st>>>(a);
    else if (a.c.head_dim == 128) attention_kernel<T, 128><<<grid, kWarps * 32, 0, st>>>(a);
    else attention_kernel<T, 256><<<grid, kWarps * 32, 0, st>>>(a);
}

}  // namespace

extern "C" int64_t qtz_kv_attention_workspace_bytes(qtz_handle h, const qtz_kv_cache* cache)
{
    if (!h || qtz_kv_check(cache) != QTZ_OK) return 0;
    return 16;
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
    qtz_device_guard guard(h->device);
    const AttnArgs a{*cache, q_dev, q_token_stride, q_head_stride, q_heads, starts_dev, lens_dev, requests, table_dev, table_width,
                     scale, window, y_dev, y_token_stride, y_head_stride, lse_dev, h->status_dev};
    if (ftype == QTZ_F16) launch<__half>(a, tokens, static_cast<cudaStream_t>(stream));
    else launch<__nv_bfloat16>(a, tokens, static_cast<cudaStream_t>(stream));
    QTZ_LAUNCH_CHECK(h, "attention_kernel");
    return QTZ_OK;
}

// Linear layers with 4-bit weights and group scales on few rows of real activations (decoding).
#include <new>

#include "qtz_half_util.cuh"
#include "qtz_internal.cuh"

struct qtz_linear {
    qtz_ctx* h = nullptr;
    qtz_linear_desc d{};
    int groups = 0;
    uint8_t* codes = nullptr;
    void* scales = nullptr;
    uint8_t* zeros = nullptr;
    void* bias = nullptr;
};

namespace {

constexpr int kRows = 8;

// One warp per output column o: lanes stride over k, fp32 sums for up to kRows rows.
template <typename T>
__global__ void linear_kernel(const T* __restrict__ x, int64_t x_stride, int64_t rows, const uint8_t* __restrict__ codes,
                              const T* __restrict__ scales, const uint8_t* __restrict__ zeros, const T* __restrict__ bias, int n,
                              int k, int group, int groups, bool is_signed, T* __restrict__ y, int64_t y_stride)
{
    const int o = blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32, lane = threadIdx.x & 31;
    if (o >= n) return;
    const int64_t r0 = static_cast<int64_t>(blockIdx.y) * kRows;
    const int m = static_cast<int>(rows - r0 < kRows ? rows - r0 : kRows);
    float acc[kRows] = {};
    const uint8_t* row = codes + static_cast<int64_t>(o) * ((k + 1) / 2);
    for (int c = lane; c < k; c += 32) {
        int q = (c & 1) ? row[c >> 1] >> 4 : row[c >> 1] & 15;
        const int64_t g = static_cast<int64_t>(o) * groups + c / group;
        if (is_signed) q = (q ^ 8) - 8;
        else if (zeros) q -= min(static_cast<int>(zeros[g]), 15);
        const float w = static_cast<float>(q) * qtz_dev::to_f32(scales[g]);
#pragma unroll
        for (int j = 0; j < kRows; ++j)
            if (j < m) acc[j] = fmaf(w, qtz_dev::to_f32(x[(r0 + j) * x_stride + c]), acc[j]);
    }
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
        for (int off = 16; off > 0; off >>= 1) acc[j] += __shfl_xor_sync(0xffffffffu, acc[j], off);
        if (lane == 0 && j < m) y[(r0 + j) * y_stride + o] = qtz_dev::from_f32<T>(acc[j] + (bias ? qtz_dev::to_f32(bias[o]) : 0.f));
    }
}

}  // namespace

extern "C" qtz_status qtz_linear_destroy(qtz_linear_plan p)
{
    if (!p) return QTZ_ERR_INVALID_ARG;
    qtz_device_guard guard(p->h->device);
    cudaFree(p->codes);
    cudaFree(p->scales);
    cudaFree(p->zeros);
    cudaFree(p->bias);
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
    qtz_device_guard guard(h->device);
    qtz_linear* p = new (std::nothrow) qtz_linear();
    if (!p) return QTZ_ERR_INVALID_ARG;
    p->h = h;
    p->d = d;
    p->groups = (d.k + d.group - 1) / d.group;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const size_t nc = static_cast<size_t>(d.n) * ((d.k + 1) / 2), ng = static_cast<size_t>(d.n) * p->groups;
#define PLAN_COPY(dst, src, bytes)                                                                              \
    do {                                                                                                        \
        cudaError_t _e = cudaMalloc(reinterpret_cast<void**>(&(dst)), (bytes));                                 \
        if (_e == cudaSuccess) _e = cudaMemcpyAsync((dst), (src), (bytes), cudaMemcpyDeviceToDevice, st);       \
        if (_e != cudaSuccess) {                                                                                \
            qtz_cuda_fail(h, _e, "qtz_linear_create");                                                          \
            qtz_linear_destroy(p);                                                                              \
            return QTZ_ERR_CUDA;                                                                                \
        }                                                                                                       \
    } while (0)
    PLAN_COPY(p->codes, codes_dev, nc);
    PLAN_COPY(p->scales, scales_dev, ng * 2);
    if (zeros_dev) PLAN_COPY(p->zeros, zeros_dev, ng);
    if (bias_dev) PLAN_COPY(p->bias, bias_dev, static_cast<size_t>(d.n) * 2);
#undef PLAN_COPY
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
    if (rows > 65535 * kRows) return QTZ_ERR_TOO_LARGE;
    qtz_device_guard guard(p->h->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const dim3 grid((p->d.n + 7) / 8, static_cast<unsigned>((rows + kRows - 1) / kRows));
    const bool s4 = p->d.wdtype == QTZ_S4_PACKED;
    if (p->d.ftype == QTZ_F16)
        linear_kernel<__half><<<grid, 256, 0, st>>>(static_cast<const __half*>(x_dev), x_stride, rows, p->codes, static_cast<const __half*>(p->scales), p->zeros, static_cast<const __half*>(p->bias), p->d.n, p->d.k, p->d.group, p->groups, s4, static_cast<__half*>(y_dev), y_stride);
    else
        linear_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(static_cast<const __nv_bfloat16*>(x_dev), x_stride, rows, p->codes, static_cast<const __nv_bfloat16*>(p->scales), p->zeros, static_cast<const __nv_bfloat16*>(p->bias), p->d.n, p->d.k, p->d.group, p->groups, s4, static_cast<__nv_bfloat16*>(y_dev), y_stride);
    QTZ_LAUNCH_CHECK(p->h, "linear_kernel");
    return QTZ_OK;
}

// Linear layers in 8-bit floating point: e4m3 activations with a scale for each row and 128 columns, e4m3 weights with a scale for each
// block of 128 x 128.
//
// Mathematics.  y[r][o] = sum_b x_scale[r][b] w_scale[o / 128][b] sum_{k in b} x[r][k] w[o][k] + bias[o].
#include <cuda_fp8.h>

#include <new>

#include "qtz_f8.cuh"
#include "qtz_plan.cuh"
#include "qtz_ptx.cuh"

struct qtz_f8_layer {
    qtz_ctx* h = nullptr;
    int device = 0;                    // a plan may be destroyed after its handle
    int32_t n = 0, k = 0;
    int32_t n_tiles = 0, k_blocks = 0; // of 128 rows, of 128 columns
    uint8_t* tiles = nullptr;          // [n_tiles][k_blocks][128][128] codes, zeros beyond n and k
    float* scales = nullptr;           // [n_tiles][k_blocks], behind the tiles in the same allocation
    float* bias = nullptr;             // [n], behind the scales; null: none
};

namespace {

struct PackArgs {
    const uint8_t* codes;
    int64_t stride;
    int32_t n, k, k_blocks;
    uint8_t* tiles;
};

// A CTA a tile.
__global__ void __launch_bounds__(256) pack_kernel(const __grid_constant__ PackArgs a)
{
    uint8_t* const tile = a.tiles + (static_cast<int64_t>(blockIdx.y) * a.k_blocks + blockIdx.x) * (kF8Block * kF8Block);
    for (int i = threadIdx.x; i < kF8Block * kF8Block; i += 256) {
        const int64_t row = static_cast<int64_t>(blockIdx.y) * kF8Block + i / kF8Block;
        const int col = blockIdx.x * kF8Block + i % kF8Block;
        tile[i] = row < a.n && col < a.k ? a.codes[row * a.stride + col] : 0;
    }
}

__global__ void bias_kernel(const void* bias, int32_t ftype, float* out, int32_t n)
{
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) out[i] = qtz_dev::load_real(bias, i, ftype);
}

struct LinearArgs {
    const uint8_t *tiles, *x;
    const float *w_scales, *bias, *x_scales;
    int64_t x_stride, row_stride, block_stride, rows, y_stride;
    void* y;
    int32_t n, k, n_tiles, k_blocks;
    int32_t ftype;
};

__device__ __forceinline__ float e4m3_f32(uint8_t v)
{
    __nv_fp8_e4m3 t;
    t.__x = v;
    return static_cast<float>(t);
}

// 32 rows of x, 32 of W; a thread four sums of one row of x.
__global__ void __launch_bounds__(256) linear_kernel(const __grid_constant__ LinearArgs a)
{
    __shared__ float s_x[32][33], s_w[32][33];
    const int tid = threadIdx.x, tx = tid & 31, ty = tid >> 5;
    const int o0 = blockIdx.x * 32;
    for (int64_t r0 = static_cast<int64_t>(blockIdx.y) * 32; r0 < a.rows; r0 += static_cast<int64_t>(gridDim.y) * 32) {
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        for (int b = 0; b < a.k_blocks; ++b) {
            float part[4] = {0.f, 0.f, 0.f, 0.f};
            const uint8_t* tile = a.tiles + (static_cast<int64_t>(o0 / kF8Block) * a.k_blocks + b) * (kF8Block * kF8Block);
            for (int c = 0; c < kF8Block; c += 32) {
                __syncthreads();
                for (int i = ty; i < 32; i += 8) {
                    const int col = b * kF8Block + c + tx;
                    s_x[i][tx] = r0 + i < a.rows && col < a.k ? e4m3_f32(a.x[(r0 + i) * a.x_stride + col]) : 0.f;
                    s_w[i][tx] = e4m3_f32(tile[(o0 % kF8Block + i) * kF8Block + c + tx]);
                }
                __syncthreads();
                for (int i = 0; i < 32; ++i)
                    for (int j = 0; j < 4; ++j) part[j] = fmaf(s_x[ty * 4 + j][i], s_w[tx][i], part[j]);
            }
            const float ws = a.w_scales[static_cast<int64_t>(o0 / kF8Block) * a.k_blocks + b];
            for (int j = 0; j < 4; ++j)
                if (r0 + ty * 4 + j < a.rows) sum[j] = fmaf(part[j], a.x_scales[(r0 + ty * 4 + j) * a.row_stride + b * a.block_stride] * ws, sum[j]);
        }
        const int o = o0 + tx;
        for (int j = 0; j < 4; ++j) {
            const int64_t r = r0 + ty * 4 + j, at = r * a.y_stride + o;
            if (r >= a.rows || o >= a.n) continue;
            const float y = sum[j] + (a.bias ? a.bias[o] : 0.f);
            if (a.ftype == QTZ_F32) static_cast<float*>(a.y)[at] = y;
            else if (a.ftype == QTZ_F16) static_cast<__half*>(a.y)[at] = __float2half_rn(y);
            else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(y);
        }
    }
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
    qtz_f8_layer* p = new (std::nothrow) qtz_f8_layer();
    if (!p) return QTZ_ERR_INVALID_ARG;
    p->h = h;
    p->device = h->device;
    p->n = n;
    p->k = k;
    p->n_tiles = static_cast<int32_t>(n_tiles);
    p->k_blocks = static_cast<int32_t>(k_blocks);
    const size_t blocks = static_cast<size_t>(n_tiles) * k_blocks, tile_bytes = blocks * kF8Block * kF8Block;
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
        const PackArgs a{codes_dev, codes_stride, n, k, p->k_blocks, p->tiles};
        pack_kernel<<<dim3(static_cast<unsigned>(k_blocks), static_cast<unsigned>(n_tiles)), 256, 0, st>>>(a);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);   // later calls may fetch the tiles before they wait for the stream
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
    qtz_ctx* h = p->h;
    qtz_device_guard guard(h->device);
    const LinearArgs a{p->tiles, codes_dev, p->scales, p->bias, scales_dev, codes_stride, scales_row_stride, scales_block_stride, rows, y_stride,
                       y_dev, p->n, p->k, p->n_tiles, p->k_blocks, ftype};
    const int64_t down = (rows + 31) / 32;
    linear_kernel<<<dim3(static_cast<unsigned>((p->n + 31) / 32), static_cast<unsigned>(down < 65535 ? down : 65535)), 256, 0, static_cast<cudaStream_t>(stream)>>>(a);
    QTZ_LAUNCH_CHECK(h, "linear_kernel");
    return QTZ_OK;
}

// Rows of real values as e4m3 codes with one scale for each row and 128 columns: behind a root-mean-square norm, behind a gated
// activation, as they are; and weights with one scale for each 128 x 128 block.
//
// Mathematics.  s = max(max |v| / 448, 2^-100) over a block's finite values, code = e4m3(v * (1 / s)), rounded to nearest even.  The
// norm's values are v = h / sqrt(mean(h^2) + eps) * gain with h = x + residual, all in fp32; what is stored of h is rounded, what the
// norm goes on with is not.
//
// What bounds them: bytes.  Every value is read once, kept in registers between the row's sum of squares, the block's maximum and the
// code, and written once.  A thread holds eight neighbouring columns, so that the 16 lanes of a half warp hold a block and its maximum
// takes four shuffles.
#include "qtz_f8.cuh"
#include "qtz_ptx.cuh"

namespace {

using namespace qtz_ptx;

constexpr int kNormChunks = 4;             // of eight columns that a thread of the norm holds at most
constexpr int kNormThreads = 1024;
constexpr int kQuantThreads = 128;
constexpr int kQuantRows = 4;              // that a thread of the quantizer has under way

// Eight neighbouring values of a row of which `valid` exist; zeros behind them.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int valid, float (&v)[8])
{
    if (valid >= 8) {
        if constexpr (sizeof(T) == 2) {
            const uint4 w = *reinterpret_cast<const uint4*>(p);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = qtz_dev::unpack2(u[i], T());
                v[2 * i] = f.x;
                v[2 * i + 1] = f.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 f = reinterpret_cast<const float4*>(p)[i];
                v[4 * i] = f.x;
                v[4 * i + 1] = f.y;
                v[4 * i + 2] = f.z;
                v[4 * i + 3] = f.w;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < valid ? qtz_dev::to_f32(p[i]) : 0.f;
    }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, int valid, const float (&v)[8])
{
    if (valid >= 8) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4*>(p) = make_uint4(qtz_dev::pack2(v[0], v[1], T()), qtz_dev::pack2(v[2], v[3], T()),
                                                      qtz_dev::pack2(v[4], v[5], T()), qtz_dev::pack2(v[6], v[7], T()));
        } else {
            reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = qtz_dev::from_f32<T>(v[i]);
    }
}

__device__ __forceinline__ float finite_top(const float (&v)[8])
{
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float m = fabsf(v[i]);
        top = fmaxf(top, m < INFINITY ? m : 0.f);
    }
    return top;
}

// The codes and the scale of a block that the 16 lanes of a half warp hold; all lanes of the warp take part.  `codes` is where this
// lane's eight go, `valid` of them exist.
__device__ __forceinline__ void put_block(const float (&v)[8], int valid, uint8_t* codes, float* scale)
{
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(v[i]));
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    if (__any_sync(0xffffffffu, top == INFINITY)) {     // infinities do not count
        top = finite_top(v);
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    }
    if (valid <= 0) return;
    const float s = qtz_dev::f8_scale(top), inverse = 1.f / s;
    if ((threadIdx.x & 15) == 0) *scale = s;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = qtz_dev::e4m3x2(v[2 * i] * inverse, v[2 * i + 1] * inverse);
    if (valid >= 8) {
        *reinterpret_cast<uint2*>(codes) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) codes[i] = static_cast<uint8_t>(w[i >> 1] >> (8 * (i & 1)));
    }
}

struct NormArgs {
    const void *x, *residual, *gain;
    int64_t x_stride, residual_stride, sum_stride, values_stride, codes_stride, scales_stride;
    void *sum, *values;
    uint8_t* codes;
    float* scales;
    float eps;
    int32_t k;
};

// Sum of the squares of what the CTA's threads hold, in all threads.
template <int kChunks>
__device__ __forceinline__ float sum_of_squares(const float (&h)[kChunks][8], float* s_part)
{
    float v = 0.f;
#pragma unroll
    for (int j = 0; j < kChunks; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) v = fmaf(h[j][i], h[j][i], v);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();                                   // an earlier call's parts have been read
    if (lane == 0) s_part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = lane < warps ? s_part[lane] : 0.f;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}

// A CTA a row; thread t holds chunks t, t + blockDim, ... of eight columns.
template <typename T, int kChunks>
__global__ void __launch_bounds__(kNormThreads) norm_kernel(const __grid_constant__ NormArgs a)
{
    __shared__ float s_part[kNormThreads / 32];
    grid_dependency_wait();
    grid_launch_dependents();
    const int64_t row = blockIdx.x;
    const T* const x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* const residual = a.residual ? static_cast<const T*>(a.residual) + row * a.residual_stride : nullptr;
    float h[kChunks][8];
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
        const int col = (j * blockDim.x + threadIdx.x) * 8;
        load8<T>(x + col, a.k - col, h[j]);
    }
    if (residual) {
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const int col = (j * blockDim.x + threadIdx.x) * 8;
            float r[8];
            load8<T>(residual + col, a.k - col, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[j][i] += r[i];
        }
    }
    if (a.sum) {
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const int col = (j * blockDim.x + threadIdx.x) * 8;
            if (a.k > col) store8<T>(static_cast<T*>(a.sum) + row * a.sum_stride + col, a.k - col, h[j]);
        }
    }
    float squares = sum_of_squares(h, s_part), eps = a.eps;
    if (squares == INFINITY) {                         // too large to be squared in fp32 (eps is nothing beside it), or infinite
#pragma unroll
        for (int j = 0; j < kChunks; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) h[j][i] *= kF8MinScale;
        squares = sum_of_squares(h, s_part);
        eps = 0.f;
    }
    const float factor = 1.f / sqrtf(squares / static_cast<float>(a.k) + eps);
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
        const int col = (j * blockDim.x + threadIdx.x) * 8, valid = a.k - col;
        float g[8], v[8];
        load8<T>(static_cast<const T*>(a.gain) + col, valid, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = h[j][i] * factor * g[i];
        if (a.values && valid > 0) store8<T>(static_cast<T*>(a.values) + row * a.values_stride + col, valid, v);
        if (a.codes) put_block(v, valid, a.codes + row * a.codes_stride + col, a.scales + row * a.scales_stride + col / kF8Block);
    }
}

struct QuantArgs {
    const void *x, *gate;
    int64_t x_stride, gate_stride, rows, codes_stride, scales_stride;
    uint8_t* codes;
    float* scales;
    int32_t k;
};

// gate / (1 + exp(-gate)).  The fast division takes divisors below 2^126 only: a sixteenth of it is, wherever the exponential is finite.
__device__ __forceinline__ float silu(float g) { return __fdividef(g, (1.f + __expf(-g)) * 0.0625f) * 0.0625f; }

// A CTA takes 1024 columns of kQuantRows rows at a time, gridDim.y rows apart.
template <typename T, bool kGate>
__global__ void __launch_bounds__(kQuantThreads) quantize_kernel(const __grid_constant__ QuantArgs a)
{
    grid_dependency_wait();
    grid_launch_dependents();
    const int col = (blockIdx.x * kQuantThreads + threadIdx.x) * 8, valid = a.k - col;
    for (int64_t row0 = blockIdx.y; row0 < a.rows; row0 += static_cast<int64_t>(gridDim.y) * kQuantRows) {
        float v[kQuantRows][8], g[kQuantRows][8];
#pragma unroll
        for (int r = 0; r < kQuantRows; ++r) {
            const int64_t row = row0 + static_cast<int64_t>(r) * gridDim.y;
            load8<T>(static_cast<const T*>(a.x) + row * a.x_stride + col, row < a.rows ? valid : 0, v[r]);
            if constexpr (kGate) load8<T>(static_cast<const T*>(a.gate) + row * a.gate_stride + col, row < a.rows ? valid : 0, g[r]);
        }
#pragma unroll
        for (int r = 0; r < kQuantRows; ++r) {
            const int64_t row = row0 + static_cast<int64_t>(r) * gridDim.y;
            if (row >= a.rows) break;
            if constexpr (kGate)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[r][i] *= silu(g[r][i]);
            put_block(v[r], valid, a.codes + row * a.codes_stride + col, a.scales + row * a.scales_stride + col / kF8Block);
        }
    }
}

struct WeightArgs {
    const void* w;
    int64_t w_stride;
    uint8_t* codes;
    float* scales;
    int32_t n, k, ftype;
};

// A CTA a block of 128 x 128.  Weights are quantized once: one value a load, no alignment asked for.
__global__ void __launch_bounds__(256) weight_kernel(const __grid_constant__ WeightArgs a)
{
    __shared__ float s_top[8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row0 = static_cast<int64_t>(blockIdx.y) * kF8Block;
    const int col0 = blockIdx.x * kF8Block;
    float top = 0.f;
    for (int i = threadIdx.x; i < kF8Block * kF8Block; i += 256) {
        const int64_t row = row0 + i / kF8Block;
        const int col = col0 + i % kF8Block;
        if (row >= a.n || col >= a.k) continue;
        const float m = fabsf(qtz_dev::load_real(a.w, row * a.w_stride + col, a.ftype));
        if (m < INFINITY) top = fmaxf(top, m);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    if (lane == 0) s_top[warp] = top;
    __syncthreads();
    for (int i = 0; i < 8; ++i) top = fmaxf(top, s_top[i]);
    const float s = qtz_dev::f8_scale(top), inverse = 1.f / s;
    if (threadIdx.x == 0) a.scales[static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x] = s;
    for (int i = threadIdx.x; i < kF8Block * kF8Block; i += 256) {
        const int64_t row = row0 + i / kF8Block;
        const int col = col0 + i % kF8Block;
        if (row >= a.n || col >= a.k) continue;
        a.codes[row * a.k + col] = static_cast<uint8_t>(qtz_dev::e4m3x2(qtz_dev::load_real(a.w, row * a.w_stride + col, a.ftype) * inverse, 0.f));
    }
}

// Rows of `k` values in a type of `size` bytes that start on 16 bytes; a single row has no stride to keep.
qtz_status check_rows(const void* p, int64_t stride, int64_t rows, int32_t k, int size)
{
    if (!p || (rows > 1 && stride < k)) return QTZ_ERR_INVALID_ARG;
    return qtz_aligned16(p) && (rows <= 1 || stride * size % 16 == 0) ? QTZ_OK : QTZ_ERR_MISALIGNED;
}

qtz_status check_codes(const uint8_t* codes, int64_t codes_stride, const float* scales, int64_t scales_stride, int64_t rows, int32_t k)
{
    if (!scales || (rows > 1 && scales_stride < (k + kF8Block - 1) / kF8Block)) return QTZ_ERR_INVALID_ARG;
    return check_rows(codes, codes_stride, rows, k, 1);
}

template <typename T>
cudaError_t launch_norm(const NormArgs& a, int64_t rows, int num_sms, cudaStream_t st)
{
    // Few rows: a chunk a thread, since the row's latency counts.  Many: four, so that each thread has 64 or 128 bytes under way.
    const int chunks = (a.k + 7) / 8, least = (chunks + kNormThreads - 1) / kNormThreads;
    const int want = rows <= 2 * num_sms ? least : kNormChunks, per = want < least ? least : want;
    int threads = ((chunks + per - 1) / per + 31) / 32 * 32;
    const int hold = (chunks + threads - 1) / threads;
    auto go = [&](auto kernel) { return qtz_launch_dependent(kernel, dim3(static_cast<unsigned>(rows)), threads, 0, st, a); };
    switch (hold) {
    case 1: return go(norm_kernel<T, 1>);
    case 2: return go(norm_kernel<T, 2>);
    case 3: return go(norm_kernel<T, 3>);
    default: return go(norm_kernel<T, 4>);
    }
}

template <typename T>
cudaError_t launch_quantize(const QuantArgs& a, int num_sms, cudaStream_t st)
{
    const unsigned slabs = static_cast<unsigned>((a.k + kQuantThreads * 8 - 1) / (kQuantThreads * 8));
    int64_t groups = (a.rows + kQuantRows - 1) / kQuantRows;
    if (a.rows * slabs <= 8 * num_sms) groups = a.rows;          // few rows: one each, for the least latency
    const dim3 grid(slabs, static_cast<unsigned>(groups < 65535 ? groups : 65535));
    if (a.gate) return qtz_launch_dependent(quantize_kernel<T, true>, grid, kQuantThreads, 0, st, a);
    return qtz_launch_dependent(quantize_kernel<T, false>, grid, kQuantThreads, 0, st, a);
}

}  // namespace

extern "C" qtz_status qtz_f8_rmsnorm(qtz_handle h, const void* x_dev, int64_t x_stride, const void* residual_dev, int64_t residual_stride,
                                     const void* gain_dev, float eps, int64_t rows, int32_t k, int32_t ftype, void* sum_dev, int64_t sum_stride,
                                     void* values_dev, int64_t values_stride, uint8_t* codes_dev, int64_t codes_stride, float* scales_dev,
                                     int64_t scales_stride, void* stream)
{
    if (!h || rows < 0 || k <= 0 || !qtz_is_real(ftype) || !(eps >= 1e-30f && eps < INFINITY)) return QTZ_ERR_INVALID_ARG;
    if (k > kNormThreads * kNormChunks * 8 || rows > 0x7fffffff) return QTZ_ERR_TOO_LARGE;
    if (rows == 0) return QTZ_OK;
    if (!codes_dev && !values_dev) return QTZ_ERR_INVALID_ARG;
    const int size = ftype == QTZ_F32 ? 4 : 2;
    qtz_status s = check_rows(x_dev, x_stride, rows, k, size);
    if (s == QTZ_OK) s = check_rows(gain_dev, k, 1, k, size);
    if (s == QTZ_OK && residual_dev) s = check_rows(residual_dev, residual_stride, rows, k, size);
    if (s == QTZ_OK && sum_dev) s = check_rows(sum_dev, sum_stride, rows, k, size);
    if (s == QTZ_OK && values_dev) s = check_rows(values_dev, values_stride, rows, k, size);
    if (s == QTZ_OK && codes_dev) s = check_codes(codes_dev, codes_stride, scales_dev, scales_stride, rows, k);
    if (s != QTZ_OK) return s;
    qtz_device_guard guard(h->device);
    const NormArgs a{x_dev, residual_dev, gain_dev, x_stride, residual_stride, sum_stride, values_stride, codes_stride, scales_stride,
                     sum_dev, values_dev, codes_dev, scales_dev, eps, k};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    QTZ_CUDA(h, ftype == QTZ_F32 ? launch_norm<float>(a, rows, h->num_sms, st)
              : ftype == QTZ_F16 ? launch_norm<__half>(a, rows, h->num_sms, st) : launch_norm<__nv_bfloat16>(a, rows, h->num_sms, st));
    return QTZ_OK;
}

extern "C" qtz_status qtz_f8_quantize(qtz_handle h, const void* x_dev, int64_t x_stride, const void* gate_dev, int64_t gate_stride, int64_t rows,
                                      int32_t k, int32_t ftype, uint8_t* codes_dev, int64_t codes_stride, float* scales_dev, int64_t scales_stride,
                                      void* stream)
{
    if (!h || rows < 0 || k <= 0 || !qtz_is_real(ftype)) return QTZ_ERR_INVALID_ARG;
    if (k > (1 << 30)) return QTZ_ERR_TOO_LARGE;
    if (rows == 0) return QTZ_OK;
    const int size = ftype == QTZ_F32 ? 4 : 2;
    qtz_status s = check_rows(x_dev, x_stride, rows, k, size);
    if (s == QTZ_OK && gate_dev) s = check_rows(gate_dev, gate_stride, rows, k, size);
    if (s == QTZ_OK) s = check_codes(codes_dev, codes_stride, scales_dev, scales_stride, rows, k);
    if (s != QTZ_OK) return s;
    qtz_device_guard guard(h->device);
    const QuantArgs a{x_dev, gate_dev, x_stride, gate_stride, rows, codes_stride, scales_stride, codes_dev, scales_dev, k};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    QTZ_CUDA(h, ftype == QTZ_F32 ? launch_quantize<float>(a, h->num_sms, st)
              : ftype == QTZ_F16 ? launch_quantize<__half>(a, h->num_sms, st) : launch_quantize<__nv_bfloat16>(a, h->num_sms, st));
    return QTZ_OK;
}

extern "C" qtz_status qtz_f8_quantize_weights(qtz_handle h, const void* w_dev, int64_t w_stride, int32_t n, int32_t k, int32_t ftype,
                                              uint8_t* codes_dev, float* scales_dev, void* stream)
{
    if (!h || !w_dev || !codes_dev || !scales_dev || n <= 0 || k <= 0 || !qtz_is_real(ftype) || (n > 1 && w_stride < k)) return QTZ_ERR_INVALID_ARG;
    const int64_t down = (static_cast<int64_t>(n) + kF8Block - 1) / kF8Block, across = (static_cast<int64_t>(k) + kF8Block - 1) / kF8Block;
    if (down > 65535 || across > 65535) return QTZ_ERR_TOO_LARGE;
    qtz_device_guard guard(h->device);
    const WeightArgs a{w_dev, w_stride, codes_dev, scales_dev, n, k, ftype};
    weight_kernel<<<dim3(static_cast<unsigned>(across), static_cast<unsigned>(down)), 256, 0, static_cast<cudaStream_t>(stream)>>>(a);
    QTZ_LAUNCH_CHECK(h, "weight_kernel");
    return QTZ_OK;
}

// Rows of real values as e4m3 codes with one scale for each row and 128 columns: behind a root-mean-square norm, behind a gated
// activation, as they are; and weights with one scale for each 128 x 128 block.
//
// Mathematics.  s = max(max |v| / 448, 2^-100) over a block's finite values, code = e4m3(v * (1 / s)), rounded to nearest even.  The
// norm's values are v = h / sqrt(mean(h^2) + eps) * gain with h = x + residual, all in fp32; what is stored of h is rounded, what the
// norm goes on with is not.
//
// What bounds them: bytes.  Every value is read once, kept in registers between the row's sum of squares, the block's maximum and the
// code, and written once.  A thread holds 32 bytes of neighbouring columns, so that 8 or 16 lanes hold a block and its maximum takes three or
// four shuffles; warps and CTAs go over several rows and have the next row's values on their way while they work on one.
// Measured, device time of ten calls in a CUDA graph, inputs in turn: norm of 16384 rows of 8192 with residual, bf16, 148 us, 6.4 TB/s, the
// copy rate (with nothing on its way behind the row at work 248); gated quantizer 8192 x 28672 180 us, 6.6 TB/s (with 32 instructions a
// value instead of about 16 409), plain 111; 8192 x 10001 gated 71 us, 5.8 TB/s; one row of 2048 2.2 us.  Rows that take a thread more than
// 32 bytes (above 16384 columns of 16 bits, 8192 of fp32) have nothing on its way: 4096 x 32768 bf16 217 to 290 us where its bytes take
// 146, 4096 x 12288 fp32 142 to 149 where they take 102, both with residual.
#include "qtz_f8.cuh"
#include "qtz_ptx.cuh"

namespace {

using namespace qtz_ptx;

// Neighbouring columns of a thread: two loads of 16 bytes.
template <typename T>
constexpr int kColsOf = 32 / sizeof(T);
constexpr int kNormThreads = 1024, kWideThreads = 512; // of the norm: with 32 bytes of a row each, with more
constexpr int kMostColumns = 32768;
constexpr int kQuantWarps = 4, kQuantWarpsPerSm = 32;  // of a CTA of the quantizer; at work at once

// The columns of a thread, of which `valid` exist, as they are stored: words, and half a word at the end of a row of an odd number of
// 16-bit values.
template <typename T>
struct Raw {
    static constexpr int kCols = kColsOf<T>, kPer = 4 / sizeof(T);   // values of a word
    uint32_t w[8];

    // zeros behind the last
    __device__ __forceinline__ void load(const T* p, int valid)
    {
        if (valid >= kCols) {
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const uint4 v = *reinterpret_cast<const uint4*>(p + i * kPer);
                w[i] = v.x;
                w[i + 1] = v.y;
                w[i + 2] = v.z;
                w[i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = 0;
                if (i * kPer + kPer <= valid) w[i] = *reinterpret_cast<const uint32_t*>(p + i * kPer);
                else if (i * kPer < valid) w[i] = *reinterpret_cast<const uint16_t*>(p + i * kPer);
            }
        }
    }
    __device__ __forceinline__ void store(T* p, int valid) const
    {
        if (valid >= kCols) {
#pragma unroll
            for (int i = 0; i < 8; i += 4) *reinterpret_cast<uint4*>(p + i * kPer) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i * kPer + kPer <= valid) *reinterpret_cast<uint32_t*>(p + i * kPer) = w[i];
                else if (i * kPer < valid) *reinterpret_cast<uint16_t*>(p + i * kPer) = static_cast<uint16_t>(w[i]);
            }
        }
    }
    __device__ __forceinline__ void get(float (&v)[kCols]) const
    {
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
            if constexpr (sizeof(T) == 4) {
                v[i] = __uint_as_float(w[i]);
            } else {
                const float2 f = qtz_dev::unpack2(w[i / 2], T());
                v[i] = i % 2 ? f.y : f.x;
            }
        }
    }
    __device__ __forceinline__ void set(const float (&v)[kCols])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v[i]);
            else w[i] = qtz_dev::pack2(v[2 * i], v[2 * i + 1], T());
        }
    }
};

// Largest of the neighbouring lanes that share a block.
template <int kLanes>
__device__ __forceinline__ float block_max(float top)
{
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    return top;
}

// The codes and the scale of a block that 128 / kCols lanes hold; all lanes of the warp take part.  `codes` is where this lane's go, `valid`
// of them exist.
template <int kCols>
__device__ __forceinline__ void put_block(const float (&v)[kCols], int valid, uint8_t* codes, float* scale)
{
    constexpr int kLanes = kF8Block / kCols;
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < kCols; ++i) top = fmaxf(top, fabsf(v[i]));
    top = block_max<kLanes>(top);
    if (__any_sync(0xffffffffu, top == INFINITY)) {     // infinities do not count
        top = 0.f;
#pragma unroll
        for (int i = 0; i < kCols; ++i) top = fmaxf(top, fabsf(v[i]) < INFINITY ? fabsf(v[i]) : 0.f);
        top = block_max<kLanes>(top);
    }
    if (valid <= 0) return;
    const float s = qtz_dev::f8_scale(top), inverse = 1.f / s;
    if (threadIdx.x % kLanes == 0) *scale = s;
    uint32_t w[kCols / 4];
#pragma unroll
    for (int i = 0; i < kCols / 4; ++i)
        w[i] = qtz_dev::e4m3x2(v[4 * i] * inverse, v[4 * i + 1] * inverse) | qtz_dev::e4m3x2(v[4 * i + 2] * inverse, v[4 * i + 3] * inverse) << 16;
    if (valid >= kCols) {
        if constexpr (kCols == 16) *reinterpret_cast<uint4*>(codes) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2*>(codes) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < kCols / 4; ++i) {
            if (4 * i + 4 <= valid) *reinterpret_cast<uint32_t*>(codes + 4 * i) = w[i];
            else
#pragma unroll
                for (int j = 0; j < 3; ++j)
                    if (4 * i + j < valid) codes[4 * i + j] = static_cast<uint8_t>(w[i] >> (8 * j));
        }
    }
}

struct NormArgs {
    const void *x, *residual, *gain;
    int64_t x_stride, residual_stride, sum_stride, values_stride, codes_stride, scales_stride, rows;
    void *sum, *values;
    uint8_t* codes;
    float* scales;
    float eps;
    int32_t k;
};

// Sum of the squares of what the CTA's threads hold, in all threads.  `part`: a place for each warp, not the one of the call before.
template <int kChunks, int kCols>
__device__ __forceinline__ float sum_of_squares(const float (&h)[kChunks][kCols], float* part)
{
    float v = 0.f;
#pragma unroll
    for (int j = 0; j < kChunks; ++j)
#pragma unroll
        for (int i = 0; i < kCols; ++i) v = fmaf(h[j][i], h[j][i], v);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = lane < warps ? part[lane] : 0.f;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}

// A CTA goes over rows blockIdx.x, blockIdx.x + gridDim.x, ...; thread t holds chunks t, t + blockDim, ... of their columns.
template <typename T, int kChunks>
__global__ void __launch_bounds__(kChunks == 1 ? kNormThreads : kWideThreads) norm_kernel(const __grid_constant__ NormArgs a)
{
    __shared__ float s_part[2][kNormThreads / 32];
    constexpr int kCols = kColsOf<T>;
    constexpr bool kEarly = kChunks == 1;              // the next row's values are asked for before this row's are used: as registers allow
    grid_dependency_wait();
    grid_launch_dependents();
    Raw<T> x, residual;
    auto load = [&](int64_t row, int j) {
        const int col = (j * blockDim.x + threadIdx.x) * kCols;
        x.load(static_cast<const T*>(a.x) + row * a.x_stride + col, a.k - col);
        if (a.residual) residual.load(static_cast<const T*>(a.residual) + row * a.residual_stride + col, a.k - col);
    };
    if (kEarly) load(blockIdx.x, 0);
    int turn = 0;
#pragma unroll 1
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        float h[kChunks][kCols];
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            if (!kEarly) load(row, j);
            x.get(h[j]);
            if (a.residual) {
                float r[kCols];
                residual.get(r);
#pragma unroll
                for (int i = 0; i < kCols; ++i) h[j][i] += r[i];
            }
        }
        if (kEarly && row + gridDim.x < a.rows) load(row + gridDim.x, 0);
        if (a.sum) {
#pragma unroll
            for (int j = 0; j < kChunks; ++j) {
                const int col = (j * blockDim.x + threadIdx.x) * kCols;
                Raw<T> sum;
                sum.set(h[j]);
                sum.store(static_cast<T*>(a.sum) + row * a.sum_stride + col, a.k - col);
            }
        }
        float mean, eps = a.eps;                       // of the squares, with eps
#pragma unroll 1
        for (int again = 3;; --again) {
            mean = sum_of_squares(h, s_part[turn]) / static_cast<float>(a.k) + eps;
            turn ^= 1;
            if (mean != INFINITY || again == 0) break;
            // Too large to be squared in fp32, or infinite: 2^-24 of it, three times at most, since 32768 squares of less than 2^56 are finite.
            // The largest, or the root of eps, is above 2^32 then, so that what falls below fp32 here would do so in v as well.
            eps *= 3.5527136788005009e-15f;            // 2^-48
#pragma unroll
            for (int j = 0; j < kChunks; ++j)
#pragma unroll
                for (int i = 0; i < kCols; ++i) h[j][i] *= 5.9604644775390625e-8f;
        }
        const float factor = 1.f / sqrtf(mean);
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const int col = (j * blockDim.x + threadIdx.x) * kCols, valid = a.k - col;
            Raw<T> gain;
            float v[kCols];
            gain.load(static_cast<const T*>(a.gain) + col, valid);
            gain.get(v);
#pragma unroll
            for (int i = 0; i < kCols; ++i) v[i] *= h[j][i] * factor;
            if (a.values) {
                gain.set(v);
                gain.store(static_cast<T*>(a.values) + row * a.values_stride + col, valid);
            }
            if (a.codes) put_block(v, valid, a.codes + row * a.codes_stride + col, a.scales + row * a.scales_stride + col / kF8Block);
        }
    }
}

struct QuantArgs {
    const void *x, *gate;
    int64_t x_stride, gate_stride, rows, codes_stride, scales_stride;
    uint8_t* codes;
    float* scales;
    int32_t k;
    int32_t pieces, per;       // of a row; rows that a warp takes together
};

// gate / (1 + exp(-gate)).  A sixteenth of the divisor is inverted, so that the result is not below fp32 wherever the exponential is finite;
// the exponential is off by 2^-17 of itself at a gate of -88 and by less nearer to 0.
__device__ __forceinline__ float silu(float g)
{
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(fmaf(e, 0.0625f, 0.0625f)));
    return g * (r * 0.0625f);
}

// A warp takes a piece (1 KB) of one or two rows at a time.  Pieces are dealt out so that each warp meets all places of a row: the last
// one may be slower.
template <typename T, bool kGate>
__global__ void __launch_bounds__(kQuantWarps * 32) quantize_kernel(const __grid_constant__ QuantArgs a)
{
    constexpr int kCols = kColsOf<T>;
    grid_dependency_wait();
    grid_launch_dependents();
    const int warps = gridDim.x * kQuantWarps, unit = blockIdx.x * kQuantWarps + threadIdx.x / 32;
    int64_t row = unit / a.pieces;
    int piece = unit % a.pieces;
    const int rows_on = warps / a.pieces, pieces_on = warps % a.pieces;
#pragma unroll 1
    for (row *= a.per; row < a.rows;) {
        const int col = (piece * 32 + (threadIdx.x & 31)) * kCols, valid = a.k - col;
        const int count = static_cast<int>(min(static_cast<int64_t>(a.per), a.rows - row));
        const T* const x = static_cast<const T*>(a.x) + row * a.x_stride + col;
        const T* const gate = kGate ? static_cast<const T*>(a.gate) + row * a.gate_stride + col : nullptr;
        Raw<T> v[2], g[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (r >= count) break;
            v[r].load(x + r * a.x_stride, valid);
            if constexpr (kGate) g[r].load(gate + r * a.gate_stride, valid);
        }
        uint8_t* const codes = a.codes + row * a.codes_stride + col;
        float* const scales = a.scales + row * a.scales_stride + col / kF8Block;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (r >= count) break;
            float f[kCols];
            v[r].get(f);
            if constexpr (kGate) {
                float s[kCols];
                g[r].get(s);
#pragma unroll
                for (int i = 0; i < kCols; ++i) f[i] *= silu(s[i]);
            }
            put_block(f, valid, codes + r * a.codes_stride, scales + r * a.scales_stride);
        }
        row += static_cast<int64_t>(rows_on) * a.per;
        piece += pieces_on;
        if (piece >= a.pieces) {
            piece -= a.pieces;
            row += a.per;
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
cudaError_t launch_norm(const NormArgs& a, int num_sms, cudaStream_t st)
{
    constexpr int kMost = kMostColumns / kWideThreads / kColsOf<T>;
    const int chunks = (a.k + kColsOf<T> - 1) / kColsOf<T>, per = chunks <= kNormThreads ? 1 : chunks <= 4 * kWideThreads ? 4 : kMost;
    const int threads = ((chunks + per - 1) / per + 31) / 32 * 32;
    // A thousand threads an SM, what their registers allow, each CTA with a row at work and a row on its way.
    const int64_t at_once = static_cast<int64_t>(num_sms) * (threads >= 1024 ? 1 : 1024 / threads);
    const dim3 grid(static_cast<unsigned>(a.rows < at_once ? a.rows : at_once));
    auto go = [&](auto kernel) { return qtz_launch_dependent(kernel, grid, threads, 0, st, a); };
    if (per == 1) return go(norm_kernel<T, 1>);
    if (per == 4) return go(norm_kernel<T, 4>);
    return go(norm_kernel<T, kMost>);
}

template <typename T>
cudaError_t launch_quantize(QuantArgs& a, int num_sms, cudaStream_t st)
{
    a.pieces = (a.k + 32 * kColsOf<T> - 1) / (32 * kColsOf<T>);
    // Two rows a warp where the warps that the registers allow at once have enough to do, one for the least latency where they do not.
    const int64_t most = static_cast<int64_t>(num_sms) * kQuantWarpsPerSm;
    a.per = a.rows * a.pieces <= 4 * most ? 1 : 2;
    const int64_t units = (a.rows + a.per - 1) / a.per * a.pieces, warps = units < most ? units : most;
    const dim3 grid(static_cast<unsigned>((warps + kQuantWarps - 1) / kQuantWarps));
    if (a.gate) return qtz_launch_dependent(quantize_kernel<T, true>, grid, kQuantWarps * 32, 0, st, a);
    return qtz_launch_dependent(quantize_kernel<T, false>, grid, kQuantWarps * 32, 0, st, a);
}

}  // namespace

extern "C" qtz_status qtz_f8_rmsnorm(qtz_handle h, const void* x_dev, int64_t x_stride, const void* residual_dev, int64_t residual_stride,
                                     const void* gain_dev, float eps, int64_t rows, int32_t k, int32_t ftype, void* sum_dev, int64_t sum_stride,
                                     void* values_dev, int64_t values_stride, uint8_t* codes_dev, int64_t codes_stride, float* scales_dev,
                                     int64_t scales_stride, void* stream)
{
    if (!h || rows < 0 || k <= 0 || !qtz_is_real(ftype) || !(eps >= 1e-30f && eps < INFINITY)) return QTZ_ERR_INVALID_ARG;
    if (k > kMostColumns || rows > 0x7fffffff) return QTZ_ERR_TOO_LARGE;
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
    const NormArgs a{x_dev, residual_dev, gain_dev, x_stride, residual_stride, sum_stride, values_stride, codes_stride, scales_stride, rows,
                     sum_dev, values_dev, codes_dev, scales_dev, eps, k};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    QTZ_CUDA(h, ftype == QTZ_F32 ? launch_norm<float>(a, h->num_sms, st)
              : ftype == QTZ_F16 ? launch_norm<__half>(a, h->num_sms, st) : launch_norm<__nv_bfloat16>(a, h->num_sms, st));
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
    QuantArgs a{x_dev, gate_dev, x_stride, gate_stride, rows, codes_stride, scales_stride, codes_dev, scales_dev, k, 0, 0};
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

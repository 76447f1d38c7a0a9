// Rows of 8-bit integers with a scale each, and the fully connected layer on them (sparse_conv_int8_quantize,
// sparse_conv_int8_linear).
#include <hip/hip_runtime.h>

#include "text_ops.h"

namespace sc {

namespace {

enum { kF32 = 0, kF16 = 1, kBF16 = 2, kI8 = 3 };   // SC_F32, SC_F16, SC_BF16, SC_I8

constexpr int kThreads = 256;
constexpr float kTiny = 0x1p-100f;   // a row whose largest size is below this counts as zeros (127 / a would overflow from 2^-121)

// One row a workgroup.  The largest |x| is found on the bit patterns: they order as the sizes do, and a NaN lies above all.
template <class T>
__global__ __launch_bounds__(kThreads) void quantize_kernel(const T* x, int8_t* q, float* scale, int K, int pitch, long long ldx)
{
    __shared__ unsigned largest;
    const size_t row = blockIdx.x;
    x += row * ldx;
    q += row * pitch;
    if (threadIdx.x == 0) largest = 0;
    __syncthreads();
    unsigned most = 0;
    for (int k = threadIdx.x; k < K; k += kThreads) most = max(most, __float_as_uint((float)x[k]) & 0x7fffffffu);
    atomicMax(&largest, most);
    __syncthreads();
    const float a = __uint_as_float(largest);
    const bool counts = a >= kTiny && a < INFINITY;
    const float inv = counts ? 127.f / a : 0.f;
    if (threadIdx.x == 0) scale[row] = counts ? a / 127.f : a < kTiny ? 0.f : NAN;
    for (int k = threadIdx.x; k < pitch; k += kThreads) q[k] = counts && k < K ? (int8_t)(int)rintf((float)x[k] * inv) : 0;
}

// One output a thread.
template <class T>
__global__ __launch_bounds__(kThreads) void product_kernel(Int8Args a, const int8_t* x, const float* x_scale)
{
    const int across = (a.N + 15) / 16;
    const int n = (int)(blockIdx.x % across) * 16 + (threadIdx.x & 15), m = (int)(blockIdx.x / across) * 16 + (threadIdx.x >> 4);
    if (n >= a.N || m >= a.M) return;
    const int* xr = reinterpret_cast<const int*>(x + (size_t)m * a.pitch);
    const int* wr = reinterpret_cast<const int*>(a.w + (size_t)n * a.pitch);
    int sum = 0;
    for (int k = 0; k < a.pitch / 4; ++k) sum = __builtin_amdgcn_sdot4(xr[k], wr[k], sum, false);
    float y = (float)sum * x_scale[m] * a.w_scale[n] + (a.bias ? a.bias[n] : 0.f);
    if (a.relu && y < 0.f) y = 0.f;
    static_cast<T*>(a.out)[m * a.ldo + n] = (T)y;
}

}  // namespace

int launch_int8_quantize(int dtype, const void* x, int8_t* q, float* scale, int rows, int K, long long ldx, void* stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int pitch = (K + 127) / 128 * 128;
    if (dtype == kF32)
        hipLaunchKernelGGL(quantize_kernel<float>, dim3(rows), dim3(kThreads), 0, s, static_cast<const float*>(x), q, scale, K, pitch, ldx);
    else if (dtype == kF16)
        hipLaunchKernelGGL(quantize_kernel<_Float16>, dim3(rows), dim3(kThreads), 0, s, static_cast<const _Float16*>(x), q, scale, K, pitch, ldx);
    else
        hipLaunchKernelGGL(quantize_kernel<__bf16>, dim3(rows), dim3(kThreads), 0, s, static_cast<const __bf16*>(x), q, scale, K, pitch, ldx);
    return (int)hipGetLastError();
}

// The quantised input, then its scales.
long long int8_workspace(int M, int, int K, int in_dtype, int)
{
    return in_dtype == kI8 ? 0 : (long long)M * ((K + 127) / 128 * 128) + (M * 4ll + 15) / 16 * 16;
}

int launch_int8_linear(int in_dtype, int out_dtype, const Int8Args& a, void* stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int8_t* x = static_cast<const int8_t*>(a.x);
    const float* x_scale = a.x_scale;
    if (in_dtype != kI8) {
        int8_t* q = reinterpret_cast<int8_t*>(a.workspace);
        float* scale = reinterpret_cast<float*>(a.workspace + (size_t)a.M * a.pitch);
        const int e = launch_int8_quantize(in_dtype, a.x, q, scale, a.M, a.K, a.ldx, stream);
        if (e != 0) return e;
        x = q;
        x_scale = scale;
    }
    const long long tiles = ((a.N + 15ll) / 16) * ((a.M + 15) / 16);
    if (tiles >= (1ll << 31)) return (int)hipErrorInvalidValue;
    const dim3 grid((unsigned)tiles);
    if (out_dtype == kF32) hipLaunchKernelGGL(product_kernel<float>, grid, dim3(kThreads), 0, s, a, x, x_scale);
    else if (out_dtype == kF16) hipLaunchKernelGGL(product_kernel<_Float16>, grid, dim3(kThreads), 0, s, a, x, x_scale);
    else hipLaunchKernelGGL(product_kernel<__bf16>, grid, dim3(kThreads), 0, s, a, x, x_scale);
    return (int)hipGetLastError();
}

}  // namespace sc

// What the kernels of the fully connected layer share (linear.hip, and for each type linear_laid.h): activations, what happens to a finished sum,
// and what the launches of products take.
#pragma once

#include <hip/hip_runtime.h>

#include "text_ops.h"
#include "tiles.h"

namespace sc {

enum { kNone = 0, kRelu = 1, kGelu = 2, kSilu = 3 };   // SC_ACT_*

// What a launch multiplies.  (Arguments past 112 bytes cost the host 0.75 us more.)
struct ProductArgs {
    const void *x, *w;              // rows along the sum, whole pieces of 16 bytes, x_pitch and w_pitch bytes apart; turned: see the tile kernel
    const float* bias;              // or null
    const void* residual;           // or null
    void *out, *z;                  // z: what goes into the activation, or null
    float* partial;                 // or null.  Else a part of k each: sums [part][M][N], and nothing of the above
    int M, N, terms, x_pitch, w_pitch;      // terms: of a sum
    int act;
    int steps;                      // of 128 bytes, a part
    int parts;
    long long ldr, ldo;             // elements; z has N
};

// Kernels for operands that are laid out: few rows of x, tiles.
enum Kernel { kRow11, kRow21, kRow22, kRow41, kRow42, kTile22, kTile44, kTile88, kDeep22, kDeep42, kDeep44, kKernels };
constexpr int kStepsToWalk = 3;      // that a tile of kTile88 needs

// Which operands are turned.
enum Turned { kRows, kTurnedW, kTurnedBoth };

// Enqueues one of them (linear_laid.h); kTooLarge, or the HIP error.
int launch_laid_f32(Kernel kernel, Turned turned, const ProductArgs& a, hipStream_t s);
int launch_laid_f16(Kernel kernel, Turned turned, const ProductArgs& a, hipStream_t s);
int launch_laid_bf16(Kernel kernel, Turned turned, const ProductArgs& a, hipStream_t s);

namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef int int2v __attribute__((ext_vector_type(2)));

// Elements of 16 bytes, as the matrix instructions take them.
template <class T>
using Eight = T __attribute__((ext_vector_type(16 / sizeof(T))));

// ---------------------------------------------------------------- activations

constexpr float kLog2e = 1.4426950408889634f;

constexpr float kNormal[7] = {-2.302209377e+00f, -1.048351228e-01f, 9.404921002e-05f, 1.595799404e-04f, -1.143983536e-05f, 3.816313949e-07f, -5.067239961e-09f};

// The normal distribution's Phi.  log(Phi(z) / Phi(-z)) is odd and smooth: z times a polynomial of z^2, fitted here up to |z| = 5.5 for
// the least error of Phi, 1.3e-7 (beyond, Phi is within 1e-7 of 0 or 1, and the polynomial goes on towards infinity).  Two transcendental
// instructions, where erff takes the longest part of an epilogue.
__device__ __forceinline__ float normal(float z)
{
    const float u = z * z;
    float p = kNormal[6];
#pragma unroll
    for (int i = 5; i >= 0; --i) p = fmaf(p, u, kNormal[i]);
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(p * z));
}

__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z)); }

template <int kAct>
__device__ __forceinline__ float activate(float z)
{
    if (kAct == kRelu) return z < 0.f ? 0.f : z;
    if (kAct == kGelu) return z * normal(z);
    if (kAct == kSilu) return z * logistic(z);
    return z;
}

// The derivative.  It is 0 or 1 to fp32 long before 128: infinities, which a z that is kept in 16 bits may have become, count as that (they would give 0 times
// infinity).
template <int kAct>
__device__ __forceinline__ float slope(float z)
{
    z = z < -128.f ? -128.f : z > 128.f ? 128.f : z;
    if (kAct == kGelu) return fmaf(z * 0.39894228040143268f, __builtin_amdgcn_exp2f(-0.5f * kLog2e * z * z), normal(z));
    if (kAct == kSilu) {
        const float s = logistic(z);
        return s * fmaf(z, 1.f - s, 1.f);
    }
    return 1.f;
}

// A gradient g behind the activation.  ReLU passes it on or does not: a product with 0 would make a NaN of an infinite one.
template <int kAct>
__device__ __forceinline__ float behind(float g, float z)
{
    if (kAct == kRelu) return z > 0.f ? g : z == z ? 0.f : z;
    return g * slope<kAct>(z);
}

// f with the activation as a constant: one branch for all the elements that it takes.
template <class F>
__device__ __forceinline__ void with_activation(int act, F&& f)
{
    if (act == kRelu) f(std::integral_constant<int, kRelu>{});
    else if (act == kGelu) f(std::integral_constant<int, kGelu>{});
    else if (act == kSilu) f(std::integral_constant<int, kSilu>{});
}

// ---------------------------------------------------------------- products

// The same by the compiler's builtins, for kernels whose sums take few registers.
template <class T>
__device__ __forceinline__ float4v multiplied(float4v c, int4v w, int4v x)
{
    if constexpr (std::is_same<T, float>::value) {
        const float4v a = __builtin_bit_cast(float4v, w), b = __builtin_bit_cast(float4v, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    } else if constexpr (std::is_same<T, _Float16>::value) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Eight<_Float16>, w), __builtin_bit_cast(Eight<_Float16>, x), c, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Eight<__bf16>, w), __builtin_bit_cast(Eight<__bf16>, x), c, 0, 0, 0);
    }
}

// C sums of a row (n .. n + C - 1 of row m, of which `count` are there) to the output: bias, activation, residual, in fp32 and rounded once.
// kInside: all are there; kPlain: there is no activation, no residual and no z.
template <class T, int C, bool kInside = false, bool kPlain = false>
__device__ __forceinline__ void finish(const ProductArgs& a, const float (&sum)[C], const float (&bias)[C], int m, int n, int count)
{
    typedef T V __attribute__((ext_vector_type(C), aligned(sizeof(T))));
    float v[C];
#pragma unroll
    for (int e = 0; e < C; ++e) v[e] = sum[e] + bias[e];
    auto store = [&](T* to) {
        V y;
#pragma unroll
        for (int e = 0; e < C; ++e) y[e] = (T)v[e];
        if (kInside || count >= C) *reinterpret_cast<V*>(to) = y;
        else
#pragma unroll
            for (int e = 0; e < C; ++e)
                if (e < count) to[e] = y[e];
    };
    if constexpr (!kPlain) {
        if (a.z) store(static_cast<T*>(a.z) + (size_t)m * a.N + n);
        with_activation(a.act, [&](auto act) {
#pragma unroll
            for (int e = 0; e < C; ++e) v[e] = activate<act>(v[e]);
        });
        if (a.residual) {
            const T* from = static_cast<const T*>(a.residual) + (size_t)m * a.ldr + n;
            if (kInside || count >= C) {
                const V r = *reinterpret_cast<const V*>(from);
#pragma unroll
                for (int e = 0; e < C; ++e) v[e] += (float)r[e];
            } else {
#pragma unroll
                for (int e = 0; e < C; ++e)
                    if (e < count) v[e] += (float)from[e];
            }
        }
    }
    store(static_cast<T*>(a.out) + (size_t)m * a.ldo + n);
}

// Four elements of each of 16 rows that lie along i, as four elements along c of each of 16 i's: lane l of 16 gives the address of elements
// 4 (l % 4) .. + 3 of row l / 4, and gets rows 0 .. 3 of element l.
__device__ __forceinline__ int2v read_turned(const char* at)
{
    typedef short short4v __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(int2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((SC_LDS short4v*)(SC_LDS char*)at));
}

// What the number of a turned row's piece of 16 bytes is combined with (by exclusive or), row c of a tile of `length` i's.
template <class T>
__device__ __forceinline__ int swizzle_of(int c, int length)
{
    if (sizeof(T) == 4) return ((c >> 2) & (length == 32 ? 1 : 3)) << 2;
    if (length == 32) return ((c >> 3) & 1) << 1;
    return length == 64 ? (((c >> 1) & 1) | ((c >> 3) & 1) << 1) << 1 : ((c & 3) | ((c >> 3) & 1) << 2) << 1;
}

// Where a lane reads the i's of a block of 16 of a turned tile of `length` i's, whose rows lie in LDS as in memory but for that permutation; further blocks of
// a wavefront by exclusive or of 16 sizeof(T) times their number.
template <class T>
__device__ __forceinline__ int turned_address(int lane, int block, int length)
{
    const int r = lane & 15, q = lane >> 4, c = sizeof(T) == 2 ? 8 * q + (r >> 2) : 4 * q;
    return c * length * (int)sizeof(T) + ((block * (int)sizeof(T)) ^ swizzle_of<T>(c, length)) * 16 + (sizeof(T) == 2 ? (r & 3) * 8 : r * 4);
}

// A lane's 16 bytes along c of its i there: four c's of 16 bits at once, or one of fp32.
template <class T>
__device__ __forceinline__ int4v read_block(const char* at, int row_length)
{
    if constexpr (sizeof(T) == 2) {
        const int2v low = read_turned(at), high = read_turned(at + 4 * row_length);
        return int4v{low[0], low[1], high[0], high[1]};
    } else {
        int4v v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const int*>(at + e * row_length);
        return v;
    }
}

}  // namespace

}  // namespace sc

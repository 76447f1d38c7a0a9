// AdamW steps over many tensors at once, states in 32 bits or in 8 (sparse_conv_adamw, sparse_conv_adamw_count).
//
// m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2, p = p - (rate decay p + rate (m c1) / (sqrt(v) c2 + eps)), with c1 = 1 / (1 - b1^t)
// and c2 = 1 / sqrt(1 - b2^t); all in fp32.  Decay and update are added before p is rounded: a factor 1 - rate decay would itself be rounded to 2^-24,
// which is all of the decay from a rate decay of 3e-8 down.  The bytes bound it: each array once in and once out.
// 6.1 million fp32 parameters take 27.6 us (170 MB, which the caches hold in part), 33 million of float16 with 32-bit weights beside 191 (927 MB,
// 4.85 TB/s, four launches), 336 million of bfloat16 with states of 8 bits 719 (3.38 GB, 4.7 TB/s).
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>

#include "text_ops.h"
#include "tiles.h"

namespace sc {

namespace {

constexpr int kBlock = 256;           // elements that share a scale, a wavefront's four a lane
constexpr int kBlocks = 2;            // that a wavefront loads at once
constexpr int kChunk = kBlock * kBlocks * 4;      // elements of a workgroup

// Tensors of one launch: a launch's arguments are 4096 bytes at most.
constexpr int kMost = 48;
struct AdamwLaunch {
    AdamwTensor tensor[kMost];
    unsigned first[kMost];            // chunk that a tensor begins with
    int count;
    AdamwRule rule;
};
static_assert(sizeof(AdamwLaunch) <= 4096, "arguments of a launch");

// A number that an element's place in its tensor and the step give, 0 <= . < 1: the products and shifts spread every bit of them.
__device__ __forceinline__ float noise_of(unsigned place, unsigned step)
{
    unsigned h = place * 0x9e3779b9u + step * 0xbb67ae85u;
    h = (h ^ (h >> 16)) * 0x6a09e667u;
    h = (h ^ (h >> 15)) * 0xbb67ae85u;
    return (float)((h ^ (h >> 16)) >> 8) * 0x1p-24f;
}

__device__ __forceinline__ float largest_in_wavefront(float most)
{
#pragma unroll
    for (int d = 32; d > 0; d /= 2) most = fmaxf(most, __shfl_xor(most, d));
    return most;
}

// The factor that takes a block to numbers of 8 bits, and its scale, from its largest size.  (Below 2^-100 a block counts as zeros: 448 / largest
// would overflow soon after.)
__device__ __forceinline__ float factor_of(float largest, float& scale)
{
    const bool zeros = largest < 0x1p-100f;
    scale = zeros ? 0.f : largest * (1.f / 448.f);
    return zeros ? 0.f : 448.f * (1.f / largest);
}

// y >= 0 to four binary digits, up or down by chance, so that what the steps add up to stays right on average: with the nearest number
// a state that changes by a thousandth a step would stay where it is.  What is there stays above zero (a step divides by its root),
// so that below the smallest number the average is too large: it is the smallest number.
__device__ __forceinline__ float by_chance(float y, float noise)
{
    const int exponent = max((int)(__float_as_uint(y) >> 23) - 127 - 3, -9);
    const float step = __uint_as_float((unsigned)(127 + exponent) << 23), inverse = __uint_as_float((unsigned)(127 - exponent) << 23);
    const float whole = floorf(fmaf(y, inverse, noise)) * step;
    return y > 0.f ? fminf(fmaxf(whole, 0x1p-9f), 448.f) : 0.f;
}

// The moments, every operation rounded by itself: the numbers of 8 bits are those of the definition done in fp32 step by step, also where a value lies next to
// the border between two of them.
__device__ __forceinline__ void update(const AdamwRule& rule, float g, float& m, float& v)
{
#pragma clang fp contract(off)
    m = rule.beta1 * m + rule.rest1 * g;
    v = rule.beta2 * v + rule.rest2 * (g * g);
}

template <class T>
using Quad = T __attribute__((ext_vector_type(4), aligned(sizeof(T))));

template <class T>
__device__ __forceinline__ void load_quad(const T* p, int left, float (&v)[4])
{
    if (left >= 4) {
        const Quad<T> q = *reinterpret_cast<const Quad<T>*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)q[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = e < left ? (float)p[e] : 0.f;
    }
}

template <class T>
__device__ __forceinline__ void store_quad(T* p, int left, const float (&v)[4])
{
    if (left >= 4) {
        Quad<T> q;
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = (T)v[e];
        *reinterpret_cast<Quad<T>*>(p) = q;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = (T)v[e];
    }
}

typedef unsigned word_at __attribute__((aligned(1)));

__device__ __forceinline__ unsigned load_codes(const unsigned char* p, int left)
{
    if (left >= 4) return *reinterpret_cast<const word_at*>(p);
    unsigned w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) w |= (unsigned)p[e] << (8 * e);
    return w;
}

__device__ __forceinline__ void store_codes(unsigned char* p, int left, unsigned w)
{
    if (left >= 4) *reinterpret_cast<word_at*>(p) = w;
    else
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = (unsigned char)(w >> (8 * e));
}

__device__ __forceinline__ void decode(unsigned w, float scale, float (&v)[4])
{
    const auto low = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), high = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    v[0] = low[0] * scale;
    v[1] = low[1] * scale;
    v[2] = high[0] * scale;
    v[3] = high[1] * scale;
}

__device__ __forceinline__ unsigned encode(const float (&y)[4])
{
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], low, true);
}

template <class P, class G, bool kSmall, bool kMaster>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwLaunch a)
{
    int t = 0;      // the last tensor that begins at this chunk or before
    for (int step = 32; step > 0; step /= 2)
        if (t + step < a.count && a.first[t + step] <= blockIdx.x) t += step;
    const AdamwTensor& x = a.tensor[t];
    const long long count = x.count, begin = (long long)(blockIdx.x - a.first[t]) * kChunk;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    AdamwRule rule = a.rule;
    if (rule.counted) {
        rule.c1 = rule.counted->c1;
        rule.c2 = rule.counted->c2;
        rule.step = rule.counted->step;
    }
    float p[kBlocks][4], g[kBlocks][4], m[kBlocks][4], v[kBlocks][4];
    int left[kBlocks];
    long long at[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
        at[b] = begin + (b * 4 + wave) * kBlock + lane * 4;
        left[b] = (int)min(count - at[b], 4ll);
        load_quad<G>(static_cast<const G*>(x.grad) + at[b], left[b], g[b]);
        if (kMaster) load_quad<float>(x.master + at[b], left[b], p[b]);
        else load_quad<P>(static_cast<const P*>(x.param) + at[b], left[b], p[b]);
        if constexpr (kSmall) {
            const long long block = (at[b] - lane * 4) / kBlock;
            const bool there = block * kBlock < count;
            decode(load_codes(static_cast<const unsigned char*>(x.m) + at[b], left[b]), there ? x.m_scale[block] : 0.f, m[b]);
            decode(load_codes(static_cast<const unsigned char*>(x.v) + at[b], left[b]), there ? x.v_scale[block] : 0.f, v[b]);
        } else {
            load_quad<float>(static_cast<const float*>(x.m) + at[b], left[b], m[b]);
            load_quad<float>(static_cast<const float*>(x.v) + at[b], left[b], v[b]);
        }
    }
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
        if (at[b] - lane * 4 >= count) break;      // (a whole wavefront)
        float most_m = 0.f, most_v = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            update(rule, g[b][e] * rule.grad_scale, m[b][e], v[b][e]);
            const float root = __builtin_amdgcn_sqrtf(v[b][e]) * rule.c2 + rule.eps;
            const float change = rule.rate * rule.c1 * m[b][e] * __builtin_amdgcn_rcpf(root);
            p[b][e] -= fmaf(rule.decay, __builtin_amdgcn_fmed3f(p[b][e], -FLT_MAX, FLT_MAX), change);      // (an infinite weight stays what it is)
            if (kSmall) {
                most_m = fmaxf(most_m, fabsf(m[b][e]));
                most_v = fmaxf(most_v, v[b][e]);
                if (!(fabsf(m[b][e]) < INFINITY)) most_m = INFINITY;      // (infinity and NaN: the block's scales say so)
                if (!(v[b][e] < INFINITY)) most_v = INFINITY;
            }
        }
        if (kMaster) store_quad<float>(x.master + at[b], left[b], p[b]);
        store_quad<P>(static_cast<P*>(x.param) + at[b], left[b], p[b]);
        if constexpr (kSmall) {
            const long long block = (at[b] - lane * 4) / kBlock;
            float scale_m, scale_v, y[4];
            const float to_m = factor_of(largest_in_wavefront(most_m), scale_m), to_v = factor_of(largest_in_wavefront(most_v), scale_v);
            if (lane == 0) {
                x.m_scale[block] = scale_m;
                x.v_scale[block] = scale_v;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = fminf(fmaxf(m[b][e] * to_m, -448.f), 448.f);
            store_codes(static_cast<unsigned char*>(x.m) + at[b], left[b], encode(y));
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = by_chance(v[b][e] * to_v, noise_of((unsigned)(at[b] + e), rule.step));
            store_codes(static_cast<unsigned char*>(x.v) + at[b], left[b], encode(y));
        } else {
            store_quad<float>(static_cast<float*>(x.m) + at[b], left[b], m[b]);
            store_quad<float>(static_cast<float*>(x.v) + at[b], left[b], v[b]);
        }
    }
}

__global__ void adamw_count_kernel(long long* count, AdamwCounted* counted, double log_beta1, double log_beta2)
{
    const long long t = *count + 1;
    *count = t;
    counted->c1 = (float)(-1.0 / expm1((double)t * log_beta1));
    counted->c2 = (float)(1.0 / sqrt(-expm1((double)t * log_beta2)));
    counted->step = (unsigned)t;
}

template <class P, class G>
int launch(bool small, bool master, unsigned chunks, const AdamwLaunch& a, hipStream_t s)
{
    const dim3 grid(chunks), block(256);
    if (small && master) hipLaunchKernelGGL((adamw_kernel<P, G, true, true>), grid, block, 0, s, a);
    else if (small) hipLaunchKernelGGL((adamw_kernel<P, G, true, false>), grid, block, 0, s, a);
    else if (master) hipLaunchKernelGGL((adamw_kernel<P, G, false, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((adamw_kernel<P, G, false, false>), grid, block, 0, s, a);
    return (int)hipGetLastError();
}

int launch(int param, int grad, bool small, bool master, unsigned chunks, const AdamwLaunch& a, hipStream_t s)
{
    if (param == kF32) return grad == kF32 ? launch<float, float>(small, master, chunks, a, s) : grad == kF16 ? launch<float, _Float16>(small, master, chunks, a, s)
                                                                                                               : launch<float, __bf16>(small, master, chunks, a, s);
    if (param == kF16) return grad == kF32 ? launch<_Float16, float>(small, master, chunks, a, s) : launch<_Float16, _Float16>(small, master, chunks, a, s);
    return grad == kF32 ? launch<__bf16, float>(small, master, chunks, a, s) : launch<__bf16, __bf16>(small, master, chunks, a, s);
}

}  // namespace

int launch_adamw(const AdamwTensor* tensors, int count, int param_dtype, int grad_dtype, bool small, const AdamwRule& rule, void* stream)
{
    AdamwLaunch a;
    a.rule = rule;
    for (int i = 0; i < count;) {
        unsigned long long chunks = 0;
        a.count = 0;
        for (; i < count && a.count < kMost; ++i) {
            const unsigned long long own = (unsigned long long)((tensors[i].count + kChunk - 1) / kChunk);
            if (own == 0) continue;
            if (a.count > 0 && chunks + own > most_groups(256)) break;
            a.tensor[a.count] = tensors[i];
            a.first[a.count++] = (unsigned)chunks;
            chunks += own;
        }
        if (a.count == 0) continue;
        const int e = launch(param_dtype, grad_dtype, small, tensors[0].master != nullptr, (unsigned)chunks, a, static_cast<hipStream_t>(stream));
        if (e != 0) return e;
    }
    return 0;
}

int launch_adamw_count(long long* count, AdamwCounted* counted, double log_beta1, double log_beta2, void* stream)
{
    hipLaunchKernelGGL(adamw_count_kernel, dim3(1), dim3(1), 0, static_cast<hipStream_t>(stream), count, counted, log_beta1, log_beta2);
    return (int)hipGetLastError();
}

}  // namespace sc

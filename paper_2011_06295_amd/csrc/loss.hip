// The loss of a classifier with the gradient of its logits (sparse_conv_cross_entropy).
//
// loss = w (log sum_c exp z_c - z_label), gradient = w (exp(z_c - log sum exp z) - [c = label]).  The bytes bound it: logits once in, gradient
// once out.  A row stays in registers between the two, where two workgroups of a CU still fit (65536 classes of 16 bits, 32768 of fp32); longer
// rows are read twice.  Each thread keeps the largest of its logits and the sum of exponentials over that largest, the threads of a row
// join these pairs once, and every thread turns what it holds into the gradient.  4096 x 65536 bfloat16 with masked classes and rows takes 230 us (1.07 GB,
// 4.7 TB/s; 209 at the rate of a large copy); 128 x 6 fp32 5.9, of which the GPU works 2.3 and the host the rest.
#include <hip/hip_runtime.h>

#include "text_ops.h"
#include "tiles.h"

namespace sc {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct Pair {      // the largest logit and the sum of exp(z - largest)
    float most, sum;
};

// exp(z - most); 0 for any finite or infinitely small z where nothing is above minus infinity.
__device__ __forceinline__ float exp_over(float z, float most) { return __expf(z - (most == -INFINITY ? 0.f : most)); }

__device__ __forceinline__ Pair join(Pair a, Pair b)
{
    const float most = fmaxf(a.most, b.most);
    return {most, a.sum * exp_over(a.most, most) + b.sum * exp_over(b.most, most)};
}

// What a row's label and weight say: a row that counts for nothing has loss and gradient zero, and its logits are not read.
struct Row {
    int label;
    float weight;
    bool counts;
};

__device__ __forceinline__ Row row_of(const LossArgs& a, int row)
{
    const long long label = a.wide ? static_cast<const long long*>(a.labels)[row] : static_cast<const int*>(a.labels)[row];
    const float weight = a.weights ? a.weights[row] * a.scale : a.scale;
    const bool inside = label >= 0 && label < a.classes;
    return {inside ? (int)label : -1, weight, inside && weight != 0.f};
}

// Elements c .. c + kCount - 1 of a row; what lies past its end counts as minus infinity.
template <class T>
__device__ __forceinline__ typename Piece<T>::type load_logits(const T* row, int c, int classes)
{
    typedef typename Piece<T>::type V;
    if (c + Piece<T>::kCount <= classes) return *reinterpret_cast<const V*>(row + c);
    V v;
#pragma unroll
    for (int e = 0; e < Piece<T>::kCount; ++e) v[e] = c + e < classes ? row[c + e] : (T)(-INFINITY);
    return v;
}

template <class T>
__device__ __forceinline__ Pair add(Pair p, typename Piece<T>::type v)
{
    float z[Piece<T>::kCount], most = p.most;
#pragma unroll
    for (int e = 0; e < Piece<T>::kCount; ++e) {
        z[e] = (float)v[e];
        most = fmaxf(most, z[e]);
    }
    if (most != p.most) p.sum *= exp_over(p.most, most);
    const float base = most == -INFINITY ? 0.f : most;
#pragma unroll
    for (int e = 0; e < Piece<T>::kCount; ++e) p.sum += __expf(z[e] - base);
    return {most, p.sum};
}

template <class T>
__device__ __forceinline__ void store_gradient(T* row, int c, int classes, typename Piece<T>::type v, float most, float log2_sum, const Row& r)
{
    typedef typename Piece<T>::type V;
    V y;
#pragma unroll
    for (int e = 0; e < Piece<T>::kCount; ++e) {
        const float p = __builtin_amdgcn_exp2f(fmaf((float)v[e] - most, kLog2e, -log2_sum));      // (far from zero most + log_sum would lose the logarithm's digits)
        y[e] = (T)(r.weight * (c + e == r.label ? p - 1.f : p));
    }
    if (c + Piece<T>::kCount <= classes) *reinterpret_cast<V*>(row + c) = y;
    else
#pragma unroll
        for (int e = 0; e < Piece<T>::kCount; ++e)
            if (c + e < classes) row[c + e] = y[e];
}

template <class T>
__device__ __forceinline__ void store_zeros(T* row, int c, int classes)
{
    typename Piece<T>::type y;
#pragma unroll
    for (int e = 0; e < Piece<T>::kCount; ++e) y[e] = (T)0.f;
    if (c + Piece<T>::kCount <= classes) *reinterpret_cast<typename Piece<T>::type*>(row + c) = y;
    else
#pragma unroll
        for (int e = 0; e < Piece<T>::kCount; ++e)
            if (c + e < classes) row[c + e] = y[e];
}

// Few classes: kLanes lanes a row with kPieces pieces of 16 bytes each.
template <class T, int kLanes, int kPieces>
__global__ __launch_bounds__(256) void loss_lanes_kernel(LossArgs a)
{
    typedef typename Piece<T>::type V;
    constexpr int kCount = Piece<T>::kCount;
    const int lane = threadIdx.x % kLanes;
    const long long at = (blockIdx.x * 256ll + threadIdx.x) / kLanes;
    const int row = (int)min(at, a.rows - 1ll);      // (lanes past the last row go along with it, and store nothing)
    const Row r = row_of(a, row);
    const T* from = static_cast<const T*>(a.logits) + (size_t)row * a.ldl;
    T* to = static_cast<T*>(a.grad) + (size_t)row * a.ldg;
    V kept[kPieces];
    Pair p{-INFINITY, 0.f};
    float labelled = 0.f;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int c = (i * kLanes + lane) * kCount;
        kept[i] = load_logits<T>(from, c, r.counts ? a.classes : 0);
#pragma unroll
        for (int e = 0; e < kCount; ++e)
            if (c + e == r.label) labelled = (float)kept[i][e];
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) p = add<T>(p, kept[i]);
#pragma unroll
    for (int d = kLanes / 2; d > 0; d /= 2) p = join(p, {__shfl_xor(p.most, d), __shfl_xor(p.sum, d)});
    labelled = __shfl(labelled, max(r.label, 0) / kCount % kLanes, kLanes);
    const float log_sum = logf(p.sum), log2_sum = log_sum * kLog2e;
    if (at >= a.rows) return;
    if (lane == 0) a.loss[row] = r.counts ? r.weight * ((p.most - labelled) + log_sum) : 0.f;
    if (!a.grad) return;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int c = (i * kLanes + lane) * kCount;
        if (c >= a.classes) break;
        if (r.counts) store_gradient<T>(to, c, a.classes, kept[i], p.most, log2_sum, r);
        else store_zeros<T>(to, c, a.classes);
    }
}

// A workgroup a row, kPieces pieces a thread in registers; kPieces = 0: any number, read again for the gradient.
template <class T, int kThreads, int kPieces>
__global__ __launch_bounds__(kThreads) void loss_row_kernel(LossArgs a)
{
    typedef typename Piece<T>::type V;
    constexpr int kCount = Piece<T>::kCount, kWaves = kThreads / 64, kKept = kPieces > 0 ? kPieces : 1;
    __shared__ Pair of_wave[kWaves];
    __shared__ float labelled;
    const int row = (int)blockIdx.x, first = threadIdx.x * kCount;
    const Row r = row_of(a, row);
    const T* from = static_cast<const T*>(a.logits) + (size_t)row * a.ldl;
    T* to = static_cast<T*>(a.grad) + (size_t)row * a.ldg;
    constexpr long long kStep = (long long)kThreads * kCount;
    if (!r.counts) {
        if (threadIdx.x == 0) a.loss[row] = 0.f;
        if (a.grad)
            for (long long c = first; c < a.classes; c += kStep) store_zeros<T>(to, (int)c, a.classes);
        return;
    }
    V kept[kKept];
    Pair p{-INFINITY, 0.f};
    auto look = [&](V v, int c) {
        if (r.label >= c && r.label < c + kCount) {
#pragma unroll
            for (int e = 0; e < kCount; ++e)
                if (c + e == r.label) labelled = (float)v[e];
        }
    };
    if constexpr (kPieces > 0) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) kept[i] = load_logits<T>(from, first + i * (int)kStep, a.classes);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            look(kept[i], first + i * (int)kStep);
            p = add<T>(p, kept[i]);
        }
    } else {
        for (long long c = first; c < a.classes; c += kStep) {
            const V v = load_logits<T>(from, (int)c, a.classes);
            look(v, (int)c);
            p = add<T>(p, v);
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d /= 2) p = join(p, {__shfl_xor(p.most, d), __shfl_xor(p.sum, d)});
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = p;
    __syncthreads();
    p = of_wave[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) p = join(p, of_wave[w]);
    const float log_sum = logf(p.sum), log2_sum = log_sum * kLog2e;
    if (threadIdx.x == 0) a.loss[row] = r.weight * ((p.most - labelled) + log_sum);
    if (!a.grad) return;
    if constexpr (kPieces > 0) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            if (first + i * (int)kStep < a.classes) store_gradient<T>(to, first + i * (int)kStep, a.classes, kept[i], p.most, log2_sum, r);
    } else {
        for (long long c = first; c < a.classes; c += kStep) store_gradient<T>(to, (int)c, a.classes, load_logits<T>(from, (int)c, a.classes), p.most, log2_sum, r);
    }
}

template <class T, int kLanes, int kPieces>
int by_lanes(const LossArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL((loss_lanes_kernel<T, kLanes, kPieces>), dim3((unsigned)((a.rows * (long long)kLanes + 255) / 256)), dim3(256), 0, s, a);
    return (int)hipGetLastError();
}

template <class T, int kThreads, int kPieces>
int by_row(const LossArgs& a, hipStream_t s)
{
    if ((unsigned long long)a.rows > most_groups(kThreads)) return kTooLarge;
    hipLaunchKernelGGL((loss_row_kernel<T, kThreads, kPieces>), dim3((unsigned)a.rows), dim3(kThreads), 0, s, a);
    return (int)hipGetLastError();
}

template <class T>
int launch(const LossArgs& a, hipStream_t s)
{
    const int pieces = (int)((a.classes + (long long)Piece<T>::kCount - 1) / Piece<T>::kCount);
    if (pieces <= 256 && (unsigned long long)a.rows > most_groups(64)) return kTooLarge;
    if (pieces <= 4) return by_lanes<T, 4, 1>(a, s);
    if (pieces <= 16) return by_lanes<T, 16, 1>(a, s);
    if (pieces <= 64) return by_lanes<T, 64, 1>(a, s);
    if (pieces <= 128) return by_lanes<T, 64, 2>(a, s);
    if (pieces <= 256) return by_lanes<T, 64, 4>(a, s);
    if (pieces <= 1024) return by_row<T, 256, 4>(a, s);
    if (pieces <= 2048) return by_row<T, 512, 4>(a, s);
    if (pieces <= 4096) return by_row<T, 1024, 4>(a, s);
    if (pieces <= 8192) return by_row<T, 1024, 8>(a, s);
    return by_row<T, 1024, 0>(a, s);
}

}  // namespace

int launch_loss(int dtype, const LossArgs& a, void* stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == kF32) return launch<float>(a, s);
    if (dtype == kF16) return launch<_Float16>(a, s);
    return launch<__bf16>(a, s);
}

}  // namespace sc

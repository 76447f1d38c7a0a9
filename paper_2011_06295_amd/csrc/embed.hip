// Word vectors and their gradient (sparse_conv_embed, sparse_conv_embed_backward).
#include <hip/hip_runtime.h>

#include "text_ops.h"

namespace sc {

namespace {

constexpr int kThreads = 256;

enum { kF32 = 0, kF16 = 1, kBF16 = 2 };   // SC_F32, SC_F16, SC_BF16

__device__ __forceinline__ long long token_at(const void* tokens, bool wide, size_t i)
{
    return wide ? static_cast<const long long*>(tokens)[i] : static_cast<const int*>(tokens)[i];
}

// One output element a thread.
template <class T>
__global__ __launch_bounds__(kThreads) void embed_kernel(EmbedArgs a)
{
    const T* table = static_cast<const T*>(a.table);
    T* out = static_cast<T*>(a.out);
    const size_t total = (size_t)a.sentences * a.words * a.dim;
    for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (size_t)gridDim.x * kThreads) {
        size_t place, d;
        if (a.channels_first) {
            const size_t n = i / ((size_t)a.dim * a.words), in = i % ((size_t)a.dim * a.words);
            d = in / a.words;
            place = n * a.words + in % a.words;
        } else {
            place = i / a.dim;
            d = i % a.dim;
        }
        const long long v = token_at(a.tokens, a.wide, place);
        const bool known = v >= 0 && v < a.vocab;
        out[i] = known ? (T)((float)table[(size_t)v * a.dim + d] * a.scale) : (T)0.f;
    }
}

// One element of the table's gradient a thread; a workgroup looks through all tokens for its row.
template <class G, class W>
__global__ __launch_bounds__(kThreads) void embed_grad_kernel(EmbedGradArgs a)
{
    const G* grad = static_cast<const G*>(a.grad);
    W* table_grad = static_cast<W*>(a.table_grad);
    const int count = a.sentences * a.words;
    const int d = blockIdx.y * kThreads + threadIdx.x;
    __shared__ int token[kThreads];
    for (long long v = blockIdx.x; v < a.vocab; v += gridDim.x) {
        float sum = 0.f;
        bool named = false;
        for (int at = 0; at < count; at += kThreads) {
            __syncthreads();
            const long long t = at + (int)threadIdx.x < count ? token_at(a.tokens, a.wide, at + threadIdx.x) : -1;
            token[threadIdx.x] = t == v && v != a.padding;
            if (__syncthreads_or(token[threadIdx.x])) {
                for (int i = 0; i < kThreads; ++i)
                    if (token[i]) {
                        const size_t place = at + i, n = place / a.words, t = place % a.words;
                        named = true;
                        if (d < a.dim) sum += (float)grad[a.channels_first ? (n * a.dim + d) * a.words + t : place * a.dim + d];
                    }
            }
        }
        if (d < a.dim) {
            W* out = table_grad + (size_t)v * a.dim + d;
            if (!a.accumulate)
                *out = (W)(sum * a.scale);
            else if (named)
                *out = (W)((float)*out + sum * a.scale);
        }
    }
}

template <class G, class W>
int launch_grad(const EmbedGradArgs& a, hipStream_t s)
{
    const long long rows = a.vocab < 16384 ? a.vocab : 16384;
    hipLaunchKernelGGL((embed_grad_kernel<G, W>), dim3((unsigned)rows, (a.dim + kThreads - 1) / kThreads), dim3(kThreads), 0, s, a);
    return (int)hipGetLastError();
}

}  // namespace

int launch_embed(int dtype, const EmbedArgs& a, void* stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const size_t blocks = ((size_t)a.sentences * a.words * a.dim + kThreads - 1) / kThreads;
    const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536));
    if (dtype == kF32) hipLaunchKernelGGL(embed_kernel<float>, grid, dim3(kThreads), 0, s, a);
    else if (dtype == kF16) hipLaunchKernelGGL(embed_kernel<_Float16>, grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL(embed_kernel<__bf16>, grid, dim3(kThreads), 0, s, a);
    return (int)hipGetLastError();
}

long long embed_grad_workspace(const EmbedGradArgs&, int) { return 0; }

int launch_embed_grad(int grad_dtype, int table_dtype, const EmbedGradArgs& a, void* stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (grad_dtype == kF32) return launch_grad<float, float>(a, s);
    if (grad_dtype == kF16) return table_dtype == kF32 ? launch_grad<_Float16, float>(a, s) : launch_grad<_Float16, _Float16>(a, s);
    return table_dtype == kF32 ? launch_grad<__bf16, float>(a, s) : launch_grad<__bf16, __bf16>(a, s);
}

}  // namespace sc

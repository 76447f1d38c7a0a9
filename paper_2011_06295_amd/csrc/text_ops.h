// Internal declarations of the text model's operators: word vectors, their gradient, products in 8-bit integers.
// Nothing here is part of the public ABI.
#pragma once

#include <cstdint>

namespace sc {

// (A launch whose arguments take more than 112 bytes, the block counts of the grid among them where a kernel asks for them, keeps the
// host 3.5 us instead of 2.75: the structures below hold what the kernels need and nothing else.)

// A launch counts its threads in 32 bits, and cuts off what is above that without an error: the workgroups that it can have.
constexpr unsigned long long most_groups(int threads) { return 0xffffffffull / (unsigned)threads; }
// What a launch function returns, with nothing enqueued, for sizes past that (else 0, or the HIP error).
constexpr int kTooLarge = -1;

struct EmbedArgs {
    const void* table;     // [vocab][dim]
    const void* tokens;    // [sentences][words]
    void* out;             // [sentences][words][dim] or [sentences][dim][words]
    long long vocab;
    int dim, sentences, words;
    float scale;
    bool channels_first, wide;   // wide: 64-bit tokens
};
int launch_embed(int dtype, const EmbedArgs& a, void* stream);

struct EmbedGradArgs {
    const void* grad;      // as EmbedArgs::out
    const void* tokens;
    void* table_grad;      // [vocab][dim]
    long long vocab, padding;
    int dim, sentences, words;
    float scale;
    bool channels_first, wide, accumulate;
};
long long embed_grad_workspace(const EmbedGradArgs& a, int grad_dtype);
int launch_embed_grad(int grad_dtype, int table_dtype, const EmbedGradArgs& a, char* workspace, void* stream);

int launch_int8_quantize(int dtype, const void* x, int8_t* q, float* scale, int rows, int K, long long ldx, void* stream);

struct Int8Args {
    const void* x;         // [M][ldx], of in_dtype
    const float* x_scale;
    const int8_t* w;       // [N][pitch]
    const float* w_scale;
    const float* bias;     // or null
    void* out;             // [M][ldo]
    int M, N, K;
    int pitch;             // bytes of a row of w (and of x, where it is 8-bit)
    long long ldx, ldo;
    bool relu;
};
int int8_kernel(int M, int N, int K);      // number of the kernel that multiplies (for tests: all are to be reached)
int int8_own_kernel(int M, int N, int K, int in_dtype);      // of the kernel that quantises its input itself, or -1: a launch does that before
long long int8_workspace(int M, int N, int K, int in_dtype, int out_dtype);
int launch_int8_linear(int in_dtype, int out_dtype, const Int8Args& a, char* workspace, void* stream);

}  // namespace sc

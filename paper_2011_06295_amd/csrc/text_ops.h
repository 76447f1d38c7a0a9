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


struct LinearArgs {
    const void *x, *w;     // [M][ldx], [N][ldw]
    const float* bias;     // or null
    const void* residual;  // [M][ldr] or null
    void *out, *z;         // [M][ldo]; [M][N] or null
    long long ldx, ldw, ldr, ldo;
    int M, N, K, act;
};
long long linear_workspace(const LinearArgs& a, int dtype);
int launch_linear(int dtype, const LinearArgs& a, char* workspace, void* stream);

// (For tests: every kernel is to be reached.)  Of operands without gaps at multiples of 16 bytes: the number of the kernel, 100 for very few rows, 101 for
// arrays as they lie (103: in tiles of 32 x 32); of the gradients 101, 102 where d is formed before, else 1000 * grad_x's + grad_w's.
int linear_kernel(int dtype, int M, int N, int K);
int linear_grad_kernel(int dtype, int M, int N, int K, int act);
// Their forms: 1 tiles of 32 x 32, 2 rows of less than 16 bytes (both of one launch alone), 4 the slope is worked out as d is loaded, 8 the sums of the layer or
// of grad_x are split, 16 those of grad_w are.
int linear_form(int dtype, int M, int N, int K);
int linear_grad_form(int dtype, int M, int N, int K, int act);

struct LinearGradArgs {
    const void *grad, *z, *x, *w;      // [M][ldg], [M][N] or null, [M][ldx], [N][ldw]
    void *grad_x, *grad_w;             // [M][K], [N][K], either or null
    float* grad_bias;                  // [N] or null
    long long ldg, ldx, ldw;
    int M, N, K, act;
    bool accumulate;
};
long long linear_grad_workspace(const LinearGradArgs& a, int dtype);
int launch_linear_grad(int dtype, const LinearGradArgs& a, char* workspace, void* stream);

struct LossArgs {
    const void *logits, *labels;       // [rows][ldl], [rows]
    const float* weights;              // [rows] or null
    float* loss;                       // [rows]
    void* grad;                        // [rows][ldg] or null
    long long ldl, ldg;
    int rows, classes;
    float scale;
    bool wide;                         // 64-bit labels
};
int launch_loss(int dtype, const LossArgs& a, void* stream);

// Exactly sparse_conv_adamw_tensor of the public header.
struct AdamwTensor {
    void* param;
    const void* grad;
    void *m, *v;
    float *m_scale, *v_scale, *master;
    long long count;
};
struct AdamwCounted {      // what a step on a count in device memory reads
    float c1, c2;
    unsigned step, unused;
};
struct AdamwRule {
    float rate, decay, beta1, rest1, beta2, rest2, eps, grad_scale, c1, c2;      // decay: times the rate; rest = 1 - beta
    unsigned step;
    const AdamwCounted* counted;       // or null; else c1, c2 and step are there
};
int launch_adamw(const AdamwTensor* tensors, int count, int param_dtype, int grad_dtype, bool small, const AdamwRule& rule, void* stream);
int launch_adamw_count(long long* count, AdamwCounted* counted, double log_beta1, double log_beta2, void* stream);

}  // namespace sc

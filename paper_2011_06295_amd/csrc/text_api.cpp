// C entry points of the text model's operators (declared in include/sparse_conv.h): arguments are checked here, kernels are
// chosen and enqueued in embed.hip and int8.hip.  No C++ object that could throw is made on these paths.
#include <cmath>
#include <cstddef>
#include <cstdint>

#include "../../include/sparse_conv.h"
#include "text_ops.h"

namespace {

int type_bytes(int dtype)
{
    return dtype == SC_F32 ? 4 : dtype == SC_F16 || dtype == SC_BF16 ? 2 : dtype == SC_I8 ? 1 : 0;
}
bool is_float(int dtype) { return dtype == SC_F32 || dtype == SC_F16 || dtype == SC_BF16; }
bool aligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % (unsigned)bytes == 0; }

// The bytes [a, a + na) and [b, b + nb) have some in common.
bool overlap(const void* a, long long na, const void* b, long long nb)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return na > 0 && nb > 0 && x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

constexpr long long kMaxCount = 1ll << 31;
constexpr long long kMaxElements = 1ll << 46;      // of an array: past any memory, and numbers of bytes stay within 64 bits

// `rows` rows, `apart` elements from one to the next, are more than an array can be.
bool too_many(long long rows, long long apart) { return rows > 1 && apart > kMaxElements / rows; }

// Sizes that both directions of the lookup share.
int check_embed(long long vocab, int dim, int sentences, int words, int dtype, unsigned flags, unsigned known)
{
    if (vocab < 1 || dim < 1 || sentences < 0 || words < 0 || !is_float(dtype) || (flags & ~known)) return SC_EINVAL;
    const long long count = (long long)sentences * words;
    if (vocab >= kMaxCount || count >= kMaxCount || too_many(vocab, dim) || too_many(count, dim)) return SC_EUNSUPPORTED;
    return SC_OK;
}

constexpr unsigned kLookupFlags = SC_EMBED_CHANNELS_FIRST | SC_EMBED_TOKENS_64;
constexpr unsigned kGradientFlags = kLookupFlags | SC_EMBED_ACCUMULATE;

int check_int8(int M, int N, int K, int in_dtype, int out_dtype)
{
    if (M < 0 || N < 1 || K < 1 || !is_float(out_dtype) || !(is_float(in_dtype) || in_dtype == SC_I8)) return SC_EINVAL;
    if (K > 131071 || M >= (1 << 24) || N >= (1 << 24)) return SC_EUNSUPPORTED;
    return SC_OK;
}

constexpr int kMostLinear = 1 << 20;
constexpr long long kMostTiles = (1ll << 24) - 1;
constexpr long long kMostStep = 1ll << 34;      // elements of a tensor: workgroups of 2048 each
constexpr long long kMostApart = 1ll << 31;
// First moments of 8 bits: (1 - beta1) times the moment has to be more than half a step between its numbers, a 18th at most, or it never changes; 0.9 leaves a
// steady gradient's moment within a factor of 2.25.
constexpr double kMostBeta1OfSmall = 0.9;

// An array: `bytes` from p on, whose elements have `element` bytes.
struct Array {
    const void* p;
    long long bytes;
    int element;
};
bool missing(const Array& a) { return !a.p || !aligned(a.p, a.element); }
bool overlap(const Array& a, const Array& b) { return a.p && b.p && overlap(a.p, a.bytes, b.p, b.bytes); }

long long rows_bytes(long long rows, long long cols, long long ld, int b) { return rows > 0 ? ((rows - 1) * ld + cols) * b : 0; }

// Sizes that both directions of the layer share; ld: distances between rows of x, w, and of the output or its gradient.
int check_linear(int M, int N, int K, long long ldx, long long ldw, long long ldo, int dtype, int activation)
{
    if (M < 0 || N < 1 || K < 1 || ldx < K || ldw < K || ldo < N || !is_float(dtype) || activation < SC_ACT_NONE || activation > SC_ACT_SILU) return SC_EINVAL;
    if (M > kMostLinear || N > kMostLinear || K > kMostLinear || ldx >= kMostApart || ldw >= kMostApart || ldo >= kMostApart) return SC_EUNSUPPORTED;
    // (Tiles of 64 x 64 of each array: what a launch of 256 threads a tile can count.)
    const long long m = (M + 63) / 64, n = (N + 63) / 64, k = (K + 63) / 64;
    if (m * n >= kMostTiles || m * k >= kMostTiles || n * k >= kMostTiles) return SC_EUNSUPPORTED;
    return SC_OK;
}

static_assert(sizeof(sc::AdamwTensor) == sizeof(sparse_conv_adamw_tensor) && offsetof(sc::AdamwTensor, count) == offsetof(sparse_conv_adamw_tensor, count) &&
                  offsetof(sc::AdamwTensor, v_scale) == offsetof(sparse_conv_adamw_tensor, v_scale),
              "the same structure");
static_assert(sizeof(sc::AdamwCounted) == SC_ADAMW_COUNTED_BYTES, "what the header says");

bool is_beta(double b) { return b >= 0.0 && b < 1.0; }
bool is_amount(double a) { return a >= 0.0 && a <= 3.4e38; }

int status(int launched) { return launched == 0 ? SC_OK : launched == sc::kTooLarge ? SC_EUNSUPPORTED : SC_EHIP; }

}  // namespace

extern "C" {

int sparse_conv_embed(const void* table, const void* tokens, void* out, long long vocab, int dim, int sentences, int words,
                      int dtype, float scale, unsigned flags, void* stream)
{
    const int rc = check_embed(vocab, dim, sentences, words, dtype, flags, kLookupFlags);
    if (rc != SC_OK) return rc;
    const long long count = (long long)sentences * words;
    if (count == 0) return SC_OK;
    const int b = type_bytes(dtype), tb = (flags & SC_EMBED_TOKENS_64) ? 8 : 4;
    if (!table || !tokens || !out || !aligned(table, b) || !aligned(out, b) || !aligned(tokens, tb)) return SC_EINVAL;
    const long long out_bytes = count * dim * b;
    if (overlap(out, out_bytes, table, vocab * dim * b) || overlap(out, out_bytes, tokens, count * tb)) return SC_EINVAL;
    const sc::EmbedArgs a{table, tokens, out, vocab, dim, sentences, words, scale,
                          (flags & SC_EMBED_CHANNELS_FIRST) != 0, (flags & SC_EMBED_TOKENS_64) != 0};
    return status(sc::launch_embed(dtype, a, stream));
}

int sparse_conv_embed_backward_workspace(long long vocab, int dim, int sentences, int words, int grad_dtype, unsigned flags,
                                         long long* bytes)
{
    if (!bytes) return SC_EINVAL;
    const int rc = check_embed(vocab, dim, sentences, words, grad_dtype, flags, kGradientFlags);
    if (rc != SC_OK) return rc;
    sc::EmbedGradArgs a{};
    a.vocab = vocab; a.dim = dim; a.sentences = sentences; a.words = words;
    a.channels_first = (flags & SC_EMBED_CHANNELS_FIRST) != 0;
    a.wide = (flags & SC_EMBED_TOKENS_64) != 0;
    *bytes = sc::embed_grad_workspace(a, grad_dtype);
    return SC_OK;
}

int sparse_conv_embed_backward(const void* grad, const void* tokens, void* table_grad, long long vocab, int dim, int sentences,
                               int words, int grad_dtype, int table_dtype, float scale, long long padding, unsigned flags,
                               void* workspace, long long workspace_bytes, void* stream)
{
    const int rc = check_embed(vocab, dim, sentences, words, grad_dtype, flags, kGradientFlags);
    if (rc != SC_OK) return rc;
    if ((table_dtype != SC_F32 && table_dtype != grad_dtype) || padding < -1 || padding >= vocab) return SC_EINVAL;
    const long long count = (long long)sentences * words;
    const int b = type_bytes(grad_dtype), b2 = type_bytes(table_dtype), tb = (flags & SC_EMBED_TOKENS_64) ? 8 : 4;
    if (!table_grad || !aligned(table_grad, b2)) return SC_EINVAL;
    sc::EmbedGradArgs a{grad, tokens, table_grad, vocab, padding, dim, sentences, words, scale,
                        (flags & SC_EMBED_CHANNELS_FIRST) != 0, (flags & SC_EMBED_TOKENS_64) != 0,
                        (flags & SC_EMBED_ACCUMULATE) != 0};
    if (count > 0) {
        if (!grad || !tokens || !aligned(grad, b) || !aligned(tokens, tb)) return SC_EINVAL;
        const long long need = sc::embed_grad_workspace(a, grad_dtype), table_bytes = vocab * dim * b2;
        if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return SC_EINVAL;
        if (overlap(table_grad, table_bytes, grad, count * dim * b) || overlap(table_grad, table_bytes, tokens, count * tb)) return SC_EINVAL;
        if (need > 0 && (overlap(workspace, need, grad, count * dim * b) || overlap(workspace, need, tokens, count * tb) ||
                         overlap(workspace, need, table_grad, table_bytes))) return SC_EINVAL;
    } else if (flags & SC_EMBED_ACCUMULATE) {
        return SC_OK;
    }
    return status(sc::launch_embed_grad(grad_dtype, table_dtype, a, static_cast<char*>(workspace), stream));
}

int sparse_conv_int8_quantize(const void* x, signed char* q, float* scale, int rows, int K, long long ldx, int dtype, void* stream)
{
    if (rows < 0 || K < 1 || ldx < K || !is_float(dtype)) return SC_EINVAL;
    if (rows >= (1 << 24) || K > (1 << 24) || too_many(rows, ldx)) return SC_EUNSUPPORTED;
    if (rows == 0) return SC_OK;
    const int b = type_bytes(dtype);
    if (!x || !q || !scale || !aligned(x, b) || !aligned(q, 16) || !aligned(scale, 4)) return SC_EINVAL;
    const long long x_bytes = ((rows - 1ll) * ldx + K) * b, q_bytes = rows * SC_INT8_PITCH(K);
    if (overlap(x, x_bytes, q, q_bytes) || overlap(x, x_bytes, scale, rows * 4ll) || overlap(q, q_bytes, scale, rows * 4ll)) return SC_EINVAL;
    return status(sc::launch_int8_quantize(dtype, x, reinterpret_cast<int8_t*>(q), scale, rows, K, ldx, stream));
}

int sparse_conv_int8_linear_workspace(int M, int N, int K, int in_dtype, int out_dtype, long long* bytes)
{
    if (!bytes) return SC_EINVAL;
    const int rc = check_int8(M, N, K, in_dtype, out_dtype);
    if (rc != SC_OK) return rc;
    *bytes = sc::int8_workspace(M, N, K, in_dtype, out_dtype);
    return SC_OK;
}

int sparse_conv_int8_linear(const void* x, const float* x_scale, const signed char* w, const float* w_scale, const float* bias,
                            void* out, int M, int N, int K, long long ldx, long long ldo, int in_dtype, int out_dtype,
                            unsigned flags, void* workspace, long long workspace_bytes, void* stream)
{
    const int rc = check_int8(M, N, K, in_dtype, out_dtype);
    if (rc != SC_OK) return rc;
    const long long pitch = SC_INT8_PITCH(K);
    if ((flags & ~static_cast<unsigned>(SC_EPILOGUE_RELU)) || ldo < N || (in_dtype == SC_I8 ? ldx != pitch : ldx < K)) return SC_EINVAL;
    if (too_many(M, ldx) || too_many(M, ldo)) return SC_EUNSUPPORTED;
    if (M == 0) return SC_OK;
    const int b = type_bytes(in_dtype), b2 = type_bytes(out_dtype);
    if (!x || !w || !w_scale || !out || !aligned(x, in_dtype == SC_I8 ? 16 : b) || !aligned(w, 16) || !aligned(w_scale, 4) || !aligned(out, b2))
        return SC_EINVAL;
    if ((in_dtype == SC_I8 && (!x_scale || !aligned(x_scale, 4))) || (bias && !aligned(bias, 4))) return SC_EINVAL;
    const long long need = sc::int8_workspace(M, N, K, in_dtype, out_dtype);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return SC_EINVAL;
    const long long out_bytes = ((M - 1ll) * ldo + N) * b2, x_bytes = ((M - 1ll) * ldx + K) * b;
    if (overlap(out, out_bytes, x, x_bytes) || overlap(out, out_bytes, w, N * pitch) || overlap(out, out_bytes, w_scale, N * 4ll) ||
        (bias && overlap(out, out_bytes, bias, N * 4ll)) || (in_dtype == SC_I8 && overlap(out, out_bytes, x_scale, M * 4ll))) return SC_EINVAL;
    if (need > 0 && (overlap(workspace, need, x, x_bytes) || overlap(workspace, need, w, N * pitch) || overlap(workspace, need, w_scale, N * 4ll) ||
                     (bias && overlap(workspace, need, bias, N * 4ll)) || overlap(workspace, need, out, out_bytes))) return SC_EINVAL;
    const sc::Int8Args a{x, x_scale, reinterpret_cast<const int8_t*>(w), w_scale, bias, out, M, N, K, (int)pitch, ldx, ldo,
                         (flags & SC_EPILOGUE_RELU) != 0};
    return status(sc::launch_int8_linear(in_dtype, out_dtype, a, static_cast<char*>(workspace), stream));
}

int sparse_conv_linear_workspace(const void* x, const void* w, int M, int N, int K, long long ldx, long long ldw, int dtype, long long* bytes)
{
    if (!bytes) return SC_EINVAL;
    const int rc = check_linear(M, N, K, ldx, ldw, N, dtype, SC_ACT_NONE);
    if (rc != SC_OK) return rc;
    *bytes = 0;
    if (M == 0) return SC_OK;
    sc::LinearArgs a{};
    a.x = x; a.w = w; a.M = M; a.N = N; a.K = K; a.ldx = ldx; a.ldw = ldw;
    *bytes = sc::linear_workspace(a, dtype);
    return SC_OK;
}

int sparse_conv_linear(const void* x, const void* w, const float* bias, const void* residual, void* out, void* z, int M, int N, int K,
                       long long ldx, long long ldw, long long ldr, long long ldo, int dtype, int activation, void* workspace,
                       long long workspace_bytes, void* stream)
{
    int rc = check_linear(M, N, K, ldx, ldw, ldo, dtype, activation);
    if (rc == SC_OK && residual) rc = check_linear(M, N, K, ldx, ldw, ldr, dtype, activation);
    if (rc != SC_OK) return rc;
    if (M == 0) return SC_OK;
    const int b = type_bytes(dtype);
    const Array ax{x, rows_bytes(M, K, ldx, b), b}, aw{w, rows_bytes(N, K, ldw, b), b}, ab{bias, 4ll * N, 4}, ar{residual, residual ? rows_bytes(M, N, ldr, b) : 0, b},
        ao{out, rows_bytes(M, N, ldo, b), b}, az{z, rows_bytes(M, N, N, b), b};
    if (missing(ax) || missing(aw) || missing(ao) || (bias && missing(ab)) || (residual && missing(ar)) || (z && missing(az))) return SC_EINVAL;
    if (overlap(ao, ax) || overlap(ao, aw) || overlap(ao, ab) || overlap(ao, az) || (overlap(ao, ar) && !(residual == out && ldr == ldo)) ||
        overlap(az, ax) || overlap(az, aw) || overlap(az, ab) || overlap(az, ar)) return SC_EINVAL;
    const sc::LinearArgs a{x, w, bias, residual, out, z, ldx, ldw, ldr, ldo, M, N, K, activation};
    const long long need = sc::linear_workspace(a, dtype);
    const Array work{workspace, need, 16};
    if (need > 0 && (missing(work) || workspace_bytes < need || overlap(work, ax) || overlap(work, aw) || overlap(work, ab) || overlap(work, ar) ||
                     overlap(work, ao) || overlap(work, az))) return SC_EINVAL;
    return status(sc::launch_linear(dtype, a, static_cast<char*>(workspace), stream));
}

int sparse_conv_linear_backward_workspace(const void* grad, const void* x, const void* w, const void* grad_x, const void* grad_w,
                                          const void* grad_bias, int M, int N, int K, long long ldg, long long ldx, long long ldw,
                                          int dtype, int activation, long long* bytes)
{
    if (!bytes) return SC_EINVAL;
    const int rc = check_linear(M, N, K, ldx, ldw, ldg, dtype, activation);
    if (rc != SC_OK) return rc;
    *bytes = 0;
    if (M == 0) return SC_OK;
    sc::LinearGradArgs a{};
    a.grad = grad; a.x = x; a.w = w; a.M = M; a.N = N; a.K = K; a.ldg = ldg; a.ldx = ldx; a.ldw = ldw; a.act = activation;
    a.grad_x = const_cast<void*>(grad_x);
    a.grad_w = const_cast<void*>(grad_w);
    a.grad_bias = static_cast<float*>(const_cast<void*>(grad_bias));
    *bytes = sc::linear_grad_workspace(a, dtype);
    return SC_OK;
}

int sparse_conv_linear_backward(const void* grad, const void* z, const void* x, const void* w, void* grad_x, void* grad_w,
                                float* grad_bias, int M, int N, int K, long long ldg, long long ldx, long long ldw, int dtype,
                                int activation, unsigned flags, void* workspace, long long workspace_bytes, void* stream)
{
    const int rc = check_linear(M, N, K, ldx, ldw, ldg, dtype, activation);
    if (rc != SC_OK) return rc;
    if (flags & ~static_cast<unsigned>(SC_LINEAR_ACCUMULATE)) return SC_EINVAL;
    const int b = type_bytes(dtype);
    if (activation == SC_ACT_NONE) z = nullptr;
    if (!grad_w) x = nullptr;
    if (!grad_x) w = nullptr;
    const Array ag{grad, rows_bytes(M, N, ldg, b), b}, az{z, rows_bytes(M, N, N, b), b}, ax{x, rows_bytes(M, K, ldx, b), b}, aw{w, rows_bytes(N, K, ldw, b), b},
        gx{grad_x, rows_bytes(M, K, K, b), b}, gw{grad_w, rows_bytes(N, K, K, b), b}, gb{grad_bias, 4ll * N, 4};
    if ((grad_x && missing(gx)) || (grad_w && missing(gw)) || (grad_bias && missing(gb))) return SC_EINVAL;
    if (M > 0 && ((missing(ag) && (grad_x || grad_w || grad_bias)) || (activation != SC_ACT_NONE && missing(az)) || (grad_w && missing(ax)) || (grad_x && missing(aw)))) return SC_EINVAL;
    const Array written[] = {gx, gw, gb}, read[] = {ag, az, ax, aw};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < i; ++j)
            if (overlap(written[i], written[j])) return SC_EINVAL;
        for (const Array& r : read)
            if (overlap(written[i], r)) return SC_EINVAL;
    }
    sc::LinearGradArgs a{grad, z, x, w, grad_x, grad_w, grad_bias, ldg, ldx, ldw, M, N, K, activation, (flags & SC_LINEAR_ACCUMULATE) != 0};
    if (M == 0) {
        if (a.accumulate) return SC_OK;
        return status(sc::launch_linear_grad(dtype, a, nullptr, stream));
    }
    const long long need = sc::linear_grad_workspace(a, dtype);
    const Array work{workspace, need, 16};
    if (need > 0) {
        if (missing(work) || workspace_bytes < need) return SC_EINVAL;
        for (const Array& r : read)
            if (overlap(work, r)) return SC_EINVAL;
        for (const Array& r : written)
            if (overlap(work, r)) return SC_EINVAL;
    }
    return status(sc::launch_linear_grad(dtype, a, static_cast<char*>(workspace), stream));
}

int sparse_conv_cross_entropy(const void* logits, const void* labels, const float* weights, float* loss, void* grad, int rows,
                              int classes, long long ldl, long long ldg, int dtype, float scale, unsigned flags, void* stream)
{
    if (rows < 0 || classes < 1 || ldl < classes || (grad && ldg < classes) || !is_float(dtype) || (flags & ~static_cast<unsigned>(SC_LOSS_LABELS_64))) return SC_EINVAL;
    constexpr int kMostClasses = 0x7fffffff - (1 << 20);
    if (classes > kMostClasses || rows > kMostClasses || too_many(rows, ldl) || (grad && too_many(rows, ldg))) return SC_EUNSUPPORTED;
    if (rows == 0) return SC_OK;
    const int b = type_bytes(dtype), lb = (flags & SC_LOSS_LABELS_64) ? 8 : 4;
    const Array al{logits, rows_bytes(rows, classes, ldl, b), b}, an{labels, (long long)rows * lb, lb}, aw{weights, rows * 4ll, 4}, as{loss, rows * 4ll, 4},
        ag{grad, grad ? rows_bytes(rows, classes, ldg, b) : 0, b};
    if (missing(al) || missing(an) || missing(as) || (weights && missing(aw)) || (grad && missing(ag))) return SC_EINVAL;
    if (overlap(as, al) || overlap(as, an) || overlap(as, aw) || overlap(as, ag) || overlap(ag, an) || overlap(ag, aw) ||
        (overlap(ag, al) && !(grad == logits && ldg == ldl))) return SC_EINVAL;
    const sc::LossArgs a{logits, labels, weights, loss, grad, ldl, ldg, rows, classes, scale, (flags & SC_LOSS_LABELS_64) != 0};
    return status(sc::launch_loss(dtype, a, stream));
}

int sparse_conv_adamw(const sparse_conv_adamw_tensor* tensors, int count, int param_dtype, int grad_dtype, int state_dtype, double rate,
                      double beta1, double beta2, double eps, double decay, double grad_scale, long long step, const void* counted,
                      void* stream)
{
    if (count < 0 || (count > 0 && !tensors) || !is_float(param_dtype) || !is_float(grad_dtype) || (state_dtype != SC_F32 && state_dtype != SC_E4M3)) return SC_EINVAL;
    if (param_dtype != SC_F32 && grad_dtype != SC_F32 && grad_dtype != param_dtype) return SC_EINVAL;
    if (!is_amount(rate) || !is_amount(eps) || !is_amount(decay) || !is_beta(beta1) || !is_beta(beta2) || !std::isfinite(grad_scale)) return SC_EINVAL;
    if (counted ? !aligned(counted, 16) : step < 1) return SC_EINVAL;
    const bool small = state_dtype == SC_E4M3;
    if (small && beta1 > kMostBeta1OfSmall) return SC_EUNSUPPORTED;
    for (int i = 0; i < count; ++i) {
        const sparse_conv_adamw_tensor& t = tensors[i];
        if (t.count < 0 || (t.master != nullptr) != (tensors[0].master != nullptr)) return SC_EINVAL;
        if (t.count > kMostStep) return SC_EUNSUPPORTED;
        if (t.count == 0) continue;
        const int pb = type_bytes(param_dtype), gb = type_bytes(grad_dtype), sb = small ? 1 : 4;
        const long long scales = (t.count + SC_ADAMW_BLOCK - 1) / SC_ADAMW_BLOCK * 4;
        const Array arrays[] = {{t.param, t.count * pb, pb}, {t.grad, t.count * gb, gb}, {t.m, t.count * sb, sb}, {t.v, t.count * sb, sb},
                                {t.master, t.count * 4, 4}, {small ? t.m_scale : nullptr, scales, 4}, {small ? t.v_scale : nullptr, scales, 4}};
        for (int j = 0; j < 7; ++j) {
            if (j == 4 ? t.master && missing(arrays[j]) : (j < 4 || small) && missing(arrays[j])) return SC_EINVAL;
            for (int k = 0; k < j; ++k)
                if (overlap(arrays[j], arrays[k])) return SC_EINVAL;
        }
    }
    if (count == 0) return SC_OK;
    sc::AdamwRule rule{(float)rate, (float)(rate * decay), (float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps,
                       (float)grad_scale, 1.f, 1.f, (unsigned)step, static_cast<const sc::AdamwCounted*>(counted)};
    if (!counted) {
        rule.c1 = (float)(1.0 / (1.0 - std::pow(beta1, (double)step)));
        rule.c2 = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    }
    return status(sc::launch_adamw(reinterpret_cast<const sc::AdamwTensor*>(tensors), count, param_dtype, grad_dtype, small, rule, stream));
}

int sparse_conv_adamw_count(long long* steps, void* counted, double beta1, double beta2, void* stream)
{
    if (!steps || !counted || !aligned(steps, 8) || !aligned(counted, 16) || overlap(steps, 8, counted, SC_ADAMW_COUNTED_BYTES) || !is_beta(beta1) || !is_beta(beta2)) return SC_EINVAL;
    return status(sc::launch_adamw_count(steps, static_cast<sc::AdamwCounted*>(counted), std::log(beta1), std::log(beta2), stream));
}

}  // extern "C"

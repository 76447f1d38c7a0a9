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

}  // extern "C"

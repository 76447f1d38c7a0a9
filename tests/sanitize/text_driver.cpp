// Host-side sanitizer driver of the text model's entry points (test infrastructure): text_api.cpp, linked without any kernel and
// built with -fsanitize=address,undefined.  Random sizes up to the ends of their types, addresses that touch and overlap,
// strides, types and flags go through every call, and each status is compared with that of the documented rules in 128 bits.
// Any sanitizer report or mismatch ends the run with a non-zero status.  No memory is read and no GPU call is made.
#include <cstdint>
#include <cstdio>
#include <vector>

#include "../../include/sparse_conv.h"

namespace {

typedef __int128 wide;

uint64_t state = 0x9E3779B97F4A7C15ull;
uint64_t rnd()
{
    state ^= state << 13;
    state ^= state >> 7;
    state ^= state << 17;
    return state >> 8;
}
bool one_in(int n) { return rnd() % (uint64_t)n == 0; }

// -1, 0, small ones, and up to 2^bits - 1 by the logarithm.
long long size(int bits)
{
    if (one_in(24)) return -(long long)(rnd() % 2);
    if (one_in(12)) return (1ll << bits) - 1 - (long long)(rnd() % 3);
    return 1 + (long long)(rnd() & ((1ull << (rnd() % (uint64_t)bits)) - 1));
}

struct Array {
    uintptr_t at;
    wide bytes;
    int element, alignment;
};

bool refused(const Array& a) { return !a.at || a.at % (unsigned)a.alignment; }
bool overlap(const Array& a, const Array& b) { return a.bytes > 0 && b.bytes > 0 && a.at < b.at + b.bytes && b.at < a.at + a.bytes; }

// An address: mostly far from all others, now and then within or right behind one, null or at an odd place.
uintptr_t address(int number, const std::vector<Array>& earlier)
{
    if (one_in(40)) return 0;
    uintptr_t at = (uintptr_t)(number + 1) << 52;
    if (!earlier.empty() && one_in(6)) {
        const Array& other = earlier[rnd() % earlier.size()];
        if (other.at && other.bytes > 0) at = other.at + (uintptr_t)(one_in(2) ? other.bytes : (wide)(rnd() % (uint64_t)(other.bytes < (1ll << 50) ? other.bytes : 1ll << 50)));
        at &= ~(uintptr_t)15;
    }
    return one_in(30) ? at + rnd() % 16 : at;
}

int bytes_of(int dtype) { return dtype == SC_F32 ? 4 : dtype == SC_I8 ? 1 : 2; }
bool is_float(int dtype) { return dtype == SC_F32 || dtype == SC_F16 || dtype == SC_BF16; }
const wide kMost = (wide)1 << 46;
bool too_many(wide rows, wide apart) { return rows > 1 && rows * apart > kMost; }
void* at(const Array& a) { return reinterpret_cast<void*>(a.at); }

int wrong = 0, calls = 0;
long long seen[8];
void check(const char* what, int t, int got, int want)
{
    ++calls;
    ++seen[-got & 7];
    if (got != want && ++wrong < 10) std::fprintf(stderr, "text driver: %s, case %d: status %d, expected %d\n", what, t, got, want);
}

int type() { return (int)(rnd() % 5) - (one_in(20) ? 1 : 0); }

void lookup(int t)
{
    const long long vocab = one_in(30) ? 1ll << 31 : size(31);
    const int dim = (int)size(31), n = (int)size(16), words = (int)size(31), dtype = type();
    const unsigned flags = (unsigned)(rnd() % 4) | (one_in(20) ? 4u : 0u);
    const int b = bytes_of(dtype), tb = flags & SC_EMBED_TOKENS_64 ? 8 : 4;
    const wide count = (wide)n * words;
    std::vector<Array> a;
    a.push_back({address(0, a), (wide)vocab * dim * b, b, b});
    a.push_back({address(1, a), count * tb, tb, tb});
    a.push_back({address(2, a), count * dim * b, b, b});
    int want = SC_EHIP;
    if (vocab < 1 || dim < 1 || n < 0 || words < 0 || !is_float(dtype) || (flags & 4)) want = SC_EINVAL;
    else if (vocab >= 1ll << 31 || count >= (1ll << 31) || too_many(vocab, dim) || too_many(count, dim)) want = SC_EUNSUPPORTED;
    else if (count == 0) want = SC_OK;
    else if (refused(a[0]) || refused(a[1]) || refused(a[2]) || overlap(a[2], a[0]) || overlap(a[2], a[1])) want = SC_EINVAL;
    check("lookup", t, sparse_conv_embed(at(a[0]), at(a[1]), at(a[2]), vocab, dim, n, words, dtype, 1.f, flags, nullptr), want);
}

void gradient(int t)
{
    const long long vocab = one_in(30) ? 1ll << 31 : size(31), padding = one_in(3) ? -1 : (long long)(rnd() % (uint64_t)(vocab > 0 ? vocab + 2 : 3)) - 1;
    const int dim = (int)size(31), n = (int)size(16), words = (int)size(31), g = type(), w = one_in(3) ? SC_F32 : one_in(6) ? type() : g;
    const unsigned flags = (unsigned)(rnd() % 8) | (one_in(20) ? 8u : 0u);
    const int b = bytes_of(g), b2 = bytes_of(w), tb = flags & SC_EMBED_TOKENS_64 ? 8 : 4;
    const wide count = (wide)n * words;
    long long need = -1;
    int want = SC_OK;
    if (vocab < 1 || dim < 1 || n < 0 || words < 0 || !is_float(g) || (flags & 8)) want = SC_EINVAL;
    else if (vocab >= 1ll << 31 || count >= (1ll << 31) || too_many(vocab, dim) || too_many(count, dim)) want = SC_EUNSUPPORTED;
    check("gradient's workspace", t, sparse_conv_embed_backward_workspace(vocab, dim, n, words, g, flags, &need), want);
    const long long given = one_in(8) ? need - 1 : need;
    std::vector<Array> a;
    a.push_back({address(0, a), count * dim * b, b, b});
    a.push_back({address(1, a), count * tb, tb, tb});
    a.push_back({address(2, a), (wide)vocab * dim * b2, b2, b2});
    a.push_back({address(3, a), need > 0 ? need : 0, 1, 16});
    if (want == SC_OK) {
        want = SC_EHIP;
        if ((w != SC_F32 && w != g) || padding < -1 || padding >= vocab || refused(a[2])) want = SC_EINVAL;
        else if (count == 0) want = flags & SC_EMBED_ACCUMULATE ? SC_OK : SC_EHIP;
        else if (refused(a[0]) || refused(a[1]) || overlap(a[2], a[0]) || overlap(a[2], a[1])) want = SC_EINVAL;
        else if (need > 0 && (refused(a[3]) || given < need || overlap(a[3], a[0]) || overlap(a[3], a[1]) || overlap(a[3], a[2]))) want = SC_EINVAL;
    }
    check("gradient", t, sparse_conv_embed_backward(at(a[0]), at(a[1]), at(a[2]), vocab, dim, n, words, g, w, 1.f, padding, flags, at(a[3]), given, nullptr), want);
}

void quantize(int t)
{
    const int rows = (int)size(25), K = (int)size(25), dtype = type();
    const long long ldx = one_in(3) ? size(62) : K + (long long)(rnd() % 9) - (one_in(12) ? 1 : 0);
    const int b = bytes_of(dtype);
    std::vector<Array> a;
    a.push_back({address(0, a), ((wide)rows - 1) * ldx * b + (wide)K * b, b, b});
    a.push_back({address(1, a), (wide)rows * SC_INT8_PITCH(K), 1, 16});
    a.push_back({address(2, a), (wide)rows * 4, 4, 4});
    int want = SC_EHIP;
    if (rows < 0 || K < 1 || ldx < K || !is_float(dtype)) want = SC_EINVAL;
    else if (rows >= 1 << 24 || K > 1 << 24 || too_many(rows, ldx)) want = SC_EUNSUPPORTED;
    else if (rows == 0) want = SC_OK;
    else if (refused(a[0]) || refused(a[1]) || refused(a[2]) || overlap(a[0], a[1]) || overlap(a[0], a[2]) || overlap(a[1], a[2])) want = SC_EINVAL;
    check("quantize", t, sparse_conv_int8_quantize(at(a[0]), static_cast<signed char*>(at(a[1])), static_cast<float*>(at(a[2])), rows, K, ldx, dtype, nullptr), want);
}

void layer(int t)
{
    const int M = (int)size(25), N = (int)size(25), K = (int)size(17) + (one_in(20) ? 1 : 0), in = type(), out = one_in(10) ? type() : (int)(rnd() % 3);
    const long long pitch = SC_INT8_PITCH(K), ldx = in == SC_I8 && !one_in(8) ? pitch : one_in(4) ? size(62) : K + (long long)(rnd() % 9),
                    ldo = one_in(4) ? size(62) : N + (long long)(rnd() % 9) - (one_in(12) ? 1 : 0);
    const unsigned flags = one_in(12) ? 2u : (unsigned)(rnd() % 2);
    const int b = bytes_of(in), b2 = bytes_of(out);
    long long need = -1;
    int want = SC_OK;
    if (M < 0 || N < 1 || K < 1 || !is_float(out) || !(is_float(in) || in == SC_I8)) want = SC_EINVAL;
    else if (K > 131071 || M >= 1 << 24 || N >= 1 << 24) want = SC_EUNSUPPORTED;
    check("layer's workspace", t, sparse_conv_int8_linear_workspace(M, N, K, in, out, &need), want);
    const long long given = one_in(8) ? need - 1 : need;
    std::vector<Array> a;
    a.push_back({address(0, a), ((wide)M - 1) * ldx * b + (wide)K * b, b, in == SC_I8 ? 16 : b});
    a.push_back({address(1, a), (wide)M * 4, 4, 4});
    a.push_back({address(2, a), (wide)N * pitch, 1, 16});
    a.push_back({address(3, a), (wide)N * 4, 4, 4});
    a.push_back({one_in(3) ? 0 : address(4, a), (wide)N * 4, 4, 4});
    a.push_back({address(5, a), ((wide)M - 1) * ldo * b2 + (wide)N * b2, b2, b2});
    a.push_back({address(6, a), need > 0 ? need : 0, 1, 16});
    const Array &x = a[0], &xs = a[1], &w = a[2], &ws = a[3], &bias = a[4], &y = a[5], &work = a[6];
    if (want == SC_OK) {
        want = SC_EHIP;
        if ((flags & 2) || ldo < N || (in == SC_I8 ? ldx != pitch : ldx < K)) want = SC_EINVAL;
        else if (too_many(M, ldx) || too_many(M, ldo)) want = SC_EUNSUPPORTED;
        else if (M == 0) want = SC_OK;
        else if (refused(x) || refused(w) || refused(ws) || refused(y) || (in == SC_I8 && refused(xs)) || (bias.at && refused(bias))) want = SC_EINVAL;
        else if (overlap(y, x) || overlap(y, w) || overlap(y, ws) || (bias.at && overlap(y, bias)) || (in == SC_I8 && overlap(y, xs))) want = SC_EINVAL;
        else if (need > 0 && (refused(work) || given < need || overlap(work, x) || overlap(work, w) || overlap(work, ws) ||
                              (bias.at && overlap(work, bias)) || overlap(work, y))) want = SC_EINVAL;
    }
    check("layer", t, sparse_conv_int8_linear(at(x), static_cast<const float*>(at(xs)), static_cast<const signed char*>(at(w)), static_cast<const float*>(at(ws)),
                                              static_cast<const float*>(at(bias)), at(y), M, N, K, ldx, ldo, in, out, flags, at(work), given, nullptr), want);
}

}  // namespace

int main()
{
    for (int t = 0; t < 60000; ++t) {
        lookup(t);
        gradient(t);
        quantize(t);
        layer(t);
    }
    if (wrong) return 1;
    for (int status : {SC_OK, SC_EINVAL, SC_EUNSUPPORTED, SC_EHIP})
        if (seen[-status] < 1000) {
            std::fprintf(stderr, "text driver: status %d came %lld times only\n", status, seen[-status]);
            return 1;
        }
    std::printf("text driver: ok, %d calls\n", calls);
    return 0;
}

// Host-side sanitizer driver of the layer's, the loss's and the AdamW step's entry points (test infrastructure): text_api.cpp, linked without
// any kernel and built with -fsanitize=address,undefined.  Random sizes up to the ends of their types, addresses that touch and overlap, strides,
// types and flags go through every call, and each status is compared with that of the documented rules in 128 bits.  Any sanitizer report
// or mismatch ends the run with a non-zero status.  No memory is read but the list of tensors, and no GPU call is made.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "../../include/sparse_conv.h"

namespace {

typedef __int128 wide;

uint64_t state = 0xD1B54A32D192ED03ull;
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
    int alignment;
};

bool refused(const Array& a) { return !a.at || a.at % (unsigned)a.alignment; }
bool overlap(const Array& a, const Array& b) { return a.at && b.at && a.bytes > 0 && b.bytes > 0 && a.at < b.at + b.bytes && b.at < a.at + a.bytes; }

// The next array: mostly far from all others, now and then within or right behind one, null or at an odd place.
Array& add(std::vector<Array>& a, wide bytes, int alignment, bool absent = false)
{
    uintptr_t at = (uintptr_t)(a.size() + 1) << 56;
    if (one_in(50)) at = 0;
    else if (!a.empty() && one_in(9)) {
        const Array& other = a[rnd() % a.size()];
        if (other.at && other.bytes > 0) at = other.at + (uintptr_t)(one_in(2) ? other.bytes : (wide)(rnd() % (uint64_t)(other.bytes < (1ll << 50) ? other.bytes : 1ll << 50)));
        at &= ~(uintptr_t)15;
    }
    if (at && one_in(40)) at += rnd() % 16;
    a.push_back({absent ? 0 : at, bytes > 0 ? bytes : 0, alignment});
    return a.back();
}

int bytes_of(int dtype) { return dtype == SC_F32 ? 4 : 2; }
bool is_float(int dtype) { return dtype == SC_F32 || dtype == SC_F16 || dtype == SC_BF16; }
void* at(const Array& a) { return reinterpret_cast<void*>(a.at); }
float* floats(const Array& a) { return reinterpret_cast<float*>(a.at); }
int type() { return one_in(20) ? (int)(rnd() % 7) - 1 : (int)(rnd() % 3); }
wide rows_bytes(wide rows, wide cols, wide ld, int b) { return rows > 0 ? ((rows - 1) * ld + cols) * b : 0; }
long long apart(long long cols) { return one_in(6) ? size(33) : cols + (long long)(rnd() % 9) - (one_in(14) ? 1 : 0); }

int wrong = 0, calls = 0;
long long seen[8];
void check(const char* what, int t, int got, int want)
{
    ++calls;
    ++seen[-got & 7];
    if (got != want && ++wrong < 10) std::fprintf(stderr, "train driver: %s, case %d: status %d, expected %d\n", what, t, got, want);
}

const long long kMost = 1 << 20, kApart = 1ll << 31;

int sizes(long long M, long long N, long long K, long long ldx, long long ldw, long long ldo, int dtype, int act)
{
    if (M < 0 || N < 1 || K < 1 || ldx < K || ldw < K || ldo < N || !is_float(dtype) || act < 0 || act > 3) return SC_EINVAL;
    if (M > kMost || N > kMost || K > kMost || ldx >= kApart || ldw >= kApart || ldo >= kApart) return SC_EUNSUPPORTED;
    const wide m = (M + 63) / 64, n = (N + 63) / 64, k = (K + 63) / 64, most = (1 << 24) - 1;
    return m * n >= most || m * k >= most || n * k >= most ? SC_EUNSUPPORTED : SC_OK;
}

void layer(int t)
{
    const int M = (int)size(21), N = (int)size(21), K = (int)size(21), dtype = type(), act = one_in(20) ? (int)(rnd() % 9) - 2 : (int)(rnd() % 4), b = bytes_of(dtype);
    const bool with_bias = one_in(2), with_residual = one_in(2), with_z = one_in(2), in_place = one_in(4);
    const long long ldx = apart(K), ldw = apart(K), ldo = apart(N), ldr = in_place && !one_in(6) ? ldo : apart(N);
    std::vector<Array> a;
    a.reserve(16);
    const Array &x = add(a, rows_bytes(M, K, ldx, b), b), &w = add(a, rows_bytes(N, K, ldw, b), b), &bias = add(a, (wide)N * 4, 4, !with_bias),
                &y = add(a, rows_bytes(M, N, ldo, b), b), &z = add(a, (wide)M * N * b, b, !with_z);
    Array& r = add(a, rows_bytes(M, N, ldr, b), b, !with_residual);
    if (with_residual && in_place) r.at = y.at;
    long long need = -1;
    int want = sizes(M, N, K, ldx, ldw, N, dtype, 0);
    check("layer's workspace", t, sparse_conv_linear_workspace(at(x), at(w), M, N, K, ldx, ldw, dtype, &need), want);
    const long long given = one_in(8) ? need - 1 : need;
    const Array& work = add(a, need, 16);
    want = sizes(M, N, K, ldx, ldw, ldo, dtype, act);
    if (want == SC_OK && r.at) want = sizes(M, N, K, ldx, ldw, ldr, dtype, act);
    if (want == SC_OK && M > 0) {
        want = SC_EHIP;
        if (refused(x) || refused(w) || refused(y) || (bias.at && refused(bias)) || (r.at && refused(r)) || (z.at && refused(z))) want = SC_EINVAL;
        else if (overlap(y, x) || overlap(y, w) || overlap(y, bias) || overlap(y, z) || (overlap(y, r) && !(r.at == y.at && ldr == ldo)) || overlap(z, x) || overlap(z, w) ||
                 overlap(z, bias) || overlap(z, r)) want = SC_EINVAL;
        else if (need > 0 && (refused(work) || given < need)) want = SC_EINVAL;
        else if (need > 0)
            for (const Array* o : {&x, &w, &bias, &y, &z, (const Array*)&r})
                if (overlap(work, *o)) want = SC_EINVAL;
    }
    check("layer", t, sparse_conv_linear(at(x), at(w), floats(bias), at(r), at(y), at(z), M, N, K, ldx, ldw, ldr, ldo, dtype, act, at(work), given, nullptr), want);
}

void gradients(int t)
{
    const int M = (int)size(21), N = (int)size(21), K = (int)size(21), dtype = type(), act = one_in(20) ? (int)(rnd() % 9) - 2 : (int)(rnd() % 4), b = bytes_of(dtype);
    const long long ldg = apart(N), ldx = apart(K), ldw = apart(K);
    const unsigned flags = one_in(20) ? 2u : (unsigned)(rnd() % 2);
    std::vector<Array> a;
    a.reserve(16);
    const Array &g = add(a, rows_bytes(M, N, ldg, b), b), z = act == SC_ACT_NONE ? Array{0, 0, 1} : add(a, (wide)M * N * b, b), &gx = add(a, (wide)M * K * b, b, one_in(3)),
                &gw = add(a, (wide)N * K * b, b, one_in(3)), &gb = add(a, (wide)N * 4, 4, one_in(3)), x = gw.at ? add(a, rows_bytes(M, K, ldx, b), b) : Array{0, 0, 1},
                w = gx.at ? add(a, rows_bytes(N, K, ldw, b), b) : Array{0, 0, 1};
    long long need = -1;
    int want = sizes(M, N, K, ldx, ldw, ldg, dtype, act);
    check("gradients' workspace", t, sparse_conv_linear_backward_workspace(at(g), at(x), at(w), at(gx), at(gw), at(gb), M, N, K, ldg, ldx, ldw, dtype, act, &need), want);
    const long long given = one_in(8) ? need - 1 : need;
    const Array& work = add(a, need, 16);
    if (want == SC_OK) {
        want = M == 0 && (flags & 1) ? SC_OK : SC_EHIP;
        if (flags & 2) want = SC_EINVAL;
        for (const Array* o : {&gx, &gw, &gb})
            if (o->at && refused(*o)) want = SC_EINVAL;
        if (M > 0 && ((refused(g) && (gx.at || gw.at || gb.at)) || (act != SC_ACT_NONE && refused(z)) || (gw.at && refused(x)) || (gx.at && refused(w)))) want = SC_EINVAL;
        const Array* written[] = {&gx, &gw, &gb};
        for (int i = 0; i < 3; ++i) {
            for (int j = 0; j < i; ++j)
                if (overlap(*written[i], *written[j])) want = SC_EINVAL;
            for (const Array* o : {&g, &z, &x, &w})
                if (overlap(*written[i], *o)) want = SC_EINVAL;
        }
        if (M > 0 && need > 0) {
            if (refused(work) || given < need) want = SC_EINVAL;
            for (const Array* o : {&gx, &gw, &gb, &g, &z, &x, &w})
                if (overlap(work, *o)) want = SC_EINVAL;
        }
    }
    check("gradients", t, sparse_conv_linear_backward(at(g), at(z), at(x), at(w), at(gx), at(gw), floats(gb), M, N, K, ldg, ldx, ldw, dtype, act, flags, at(work), given, nullptr), want);
}

void loss(int t)
{
    const int rows = (int)size(31), classes = (int)size(31), dtype = type(), b = bytes_of(dtype);
    const long long ldl = apart(classes), ldg = apart(classes);
    const unsigned flags = one_in(20) ? 2u : (unsigned)(rnd() % 2);
    const int lb = flags & 1 ? 8 : 4;
    std::vector<Array> a;
    a.reserve(8);
    const Array &z = add(a, rows_bytes(rows, classes, ldl, b), b), &n = add(a, (wide)rows * lb, lb), &w = add(a, (wide)rows * 4, 4, one_in(2)), &l = add(a, (wide)rows * 4, 4);
    Array& g = add(a, rows_bytes(rows, classes, ldg, b), b, one_in(3));
    if (g.at && one_in(3)) g.at = z.at;
    const long long most = 0x7fffffff - (1 << 20);
    int want = SC_EHIP;
    if (rows < 0 || classes < 1 || ldl < classes || (g.at && ldg < classes) || !is_float(dtype) || (flags & 2)) want = SC_EINVAL;
    else if (classes > most || rows > most || (rows > 1 && ((wide)rows * ldl > (wide)1 << 46 || (g.at && (wide)rows * ldg > (wide)1 << 46)))) want = SC_EUNSUPPORTED;
    else if (rows == 0) want = SC_OK;
    else if (refused(z) || refused(n) || refused(l) || (w.at && refused(w)) || (g.at && refused(g))) want = SC_EINVAL;
    else if (overlap(l, z) || overlap(l, n) || overlap(l, w) || overlap(l, g) || overlap(g, n) || overlap(g, w) || (overlap(g, z) && !(g.at == z.at && ldg == ldl))) want = SC_EINVAL;
    check("loss", t, sparse_conv_cross_entropy(at(z), at(n), floats(w), floats(l), at(g), rows, classes, ldl, ldg, dtype, 1.f, flags, nullptr), want);
}

void step(int t)
{
    const int count = (int)(rnd() % 5) - (one_in(30) ? 1 : 0), p = type(), g = one_in(3) ? SC_F32 : one_in(6) ? type() : p, s = one_in(20) ? (int)(rnd() % 6) : one_in(2) ? (int)SC_F32 : (int)SC_E4M3;
    const bool small = s == SC_E4M3, master = one_in(3);
    const double rate = one_in(30) ? -1.0 : 1e-3, beta1 = one_in(30) ? 1.0 : one_in(10) ? 0.0 : 0.9, eps = one_in(30) ? NAN : 1e-8, scale = one_in(30) ? INFINITY : 1.0;
    const long long number = one_in(15) ? 0 : (long long)(rnd() % 100000) + 1;
    const uintptr_t counted = one_in(3) ? (one_in(5) ? 8 : 1ull << 40) : 0;
    std::vector<sparse_conv_adamw_tensor> list(count > 0 ? (size_t)count : 1);
    int want = count == 0 ? SC_OK : SC_EHIP;
    bool stop = false;          // at the first tensor that is refused, as the call does
    if (count < 0 || !is_float(p) || !is_float(g) || (s != SC_F32 && s != SC_E4M3) || (p != SC_F32 && g != SC_F32 && g != p) || rate < 0 || beta1 >= 1.0 || !(eps >= 0) || !std::isfinite(scale) ||
        (counted ? counted % 16 != 0 : number < 1)) {
        want = SC_EINVAL;
        stop = true;
    }
    for (int i = 0; i < count; ++i) {
        const long long n = one_in(20) ? (1ll << 34) + (long long)(rnd() % 3) : size(34);
        const wide elements = n > 0 ? n : 0, scales = (elements + 255) / 256 * 4;
        std::vector<Array> a;
        a.reserve(8);
        add(a, elements * bytes_of(p), bytes_of(p));
        add(a, elements * bytes_of(g), bytes_of(g));
        add(a, elements * (small ? 1 : 4), small ? 1 : 4);
        add(a, elements * (small ? 1 : 4), small ? 1 : 4);
        add(a, elements * 4, 4, !master && !one_in(40));
        add(a, scales, 4, !small);
        add(a, scales, 4, !small);
        list[(size_t)i] = {at(a[0]), at(a[1]), at(a[2]), at(a[3]), floats(a[5]), floats(a[6]), floats(a[4]), n};
        if (stop) continue;
        if (n < 0 || (a[4].at != 0) != (list[0].master != nullptr)) want = SC_EINVAL;
        else if (n > 1ll << 34) want = SC_EUNSUPPORTED;
        else if (n > 0) {
            for (int j = 0; j < 7; ++j) {
                if (j == 4 ? a[4].at && refused(a[4]) : (j < 4 || small) && refused(a[(size_t)j])) want = SC_EINVAL;
                for (int k = 0; k < j; ++k)
                    if (overlap(a[(size_t)j], a[(size_t)k])) want = SC_EINVAL;
            }
        }
        stop = want != SC_EHIP;
    }
    check("step", t, sparse_conv_adamw(list.data(), count, p, g, s, rate, beta1, 0.999, eps, 0.01, scale, number, reinterpret_cast<void*>(counted), nullptr), want);
    const uintptr_t steps = one_in(10) ? 0 : (one_in(10) ? 4 : 1ull << 40), room = one_in(6) ? steps : one_in(10) ? 8 : 1ull << 41;
    want = !steps || !room || steps % 8 || room % 16 || steps == room || beta1 >= 1.0 ? SC_EINVAL : SC_EHIP;
    check("count", t, sparse_conv_adamw_count(reinterpret_cast<long long*>(steps), reinterpret_cast<void*>(room), beta1, 0.999, nullptr), want);
}

}  // namespace

int main()
{
    for (int t = 0; t < 60000; ++t) {
        layer(t);
        gradients(t);
        loss(t);
        step(t);
    }
    if (wrong) return 1;
    for (int status : {SC_OK, SC_EINVAL, SC_EUNSUPPORTED, SC_EHIP})
        if (seen[-status] < 1000) {
            std::fprintf(stderr, "train driver: status %d came %lld times only\n", status, seen[-status]);
            return 1;
        }
    std::printf("train driver: ok, %d calls\n", calls);
    return 0;
}

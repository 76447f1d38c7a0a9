// Fully connected layer with bias, activation and residual, and its gradients (sparse_conv_linear, sparse_conv_linear_backward).
//
// z = x w^T + bias, out = act(z) + residual; with d = grad act'(z): grad_x = d w, grad_w = d^T x, grad_bias = sum_m d.  So every product is
// out[m][n] = sum_k a[m][k] b[n][k] of operands whose rows lie along the sum, or the other way round ("turned").  Products of 16-bit numbers are
// summed in fp32 by the matrix cores, fp32 is multiplied in fp32 (at most 152 TFLOP/s here).  d is rounded to the type of the operands once, since
// the matrix cores take nothing else; the bias' sums take it before that.
//
// Four ways, chosen by what each is estimated to take (below).  Times here and there: one call after another in a graph, three sets of arrays in turn.
//   very few rows     linear_dot_kernel: the weights once from memory at 4.7 TB/s (1 x 4096 -> 4096 bfloat16 7.2 us);
//   arrays as they lie  linear_direct_kernel, linear_direct_grad_kernel: one launch, tiles of 32 x 32 or 64 x 64, any address and either way round
//                     (203 x 1001 -> 1111 fp32 11.2 us; both gradients of 128 x 200 -> 256 with relu 5.2 us);
//   few rows          linear_row_kernel (linear_laid.h): the weights from memory (24 x 4096 -> 8192 float16 14.6 us; 17.3 where the caches hold none of them);
//   tiles             linear_tile_kernel (linear_laid.h): the matrix cores (8192 x 4096 -> 8192 bfloat16 with gelu and z kept 450 us, 1.22 PFLOP/s).
// The last two load straight to LDS, which takes rows at multiples of 16 bytes; others are laid out in scratch memory first (linear_lay_kernel).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "linear.h"

namespace sc {

namespace {

// The parts of a product added up, in their order, then as in the kernels that do all of a sum.  Four outputs of a row a thread; bytes and a launch
// bound it (about 3.5 us and 1 TB/s of partial sums on top of the product, with which the choice reckons).
template <class T>
__global__ __launch_bounds__(256) void linear_join_kernel(ProductArgs a)
{
    typedef float four __attribute__((ext_vector_type(4), aligned(4)));
    const int per_row = (a.N + 3) / 4;
    const long long at = blockIdx.x * 256ll + threadIdx.x;
    if (at >= (long long)per_row * a.M) return;
    const int m = (int)(at / per_row), n = (int)(at % per_row) * 4;
    float sum[4] = {0.f, 0.f, 0.f, 0.f}, bias[4];
    for (int part = 0; part < a.parts; ++part) {
        const float* from = a.partial + ((size_t)part * a.M + m) * a.N + n;
        if (n + 4 <= a.N) {
            const four v = *reinterpret_cast<const four*>(from);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += v[e];
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < a.N) sum[e] += from[e];
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) bias[e] = a.bias && n + e < a.N ? a.bias[n + e] : 0.f;
    finish<T, 4>(a, sum, bias, m, n, a.N - n);
}

// ---------------------------------------------------------------- products of arrays as they lie

// One operand: element (i, c) at p[i * ld + c] (its rows lie along the sum) or, "turned", at p[c * ld + i].  z: or null, else the element is
// p's times the activation's slope at z's, rounded; z has no gaps.
struct Side {
    const void *p, *z;
    long long ld, ldz;
    int count;                          // of i
};

// kRows i by U units of 128 bytes of c of an operand, a thread's share: pieces of 16 bytes, from any element on.  Loads are issued by no branch at all, so that
// those of several steps can be in flight (after one the compiler waits for all that came before): a piece that would reach outside is the nearest
// one inside, and `put` moves it into place, with zeros for c past the sum's end.  Outputs of i's that are not there are never stored.
// kFew: the operand has rows of less than a piece, which are loaded one by one.
template <class T, int kRows, int U, bool kTurned, bool kSlope, bool kFew>
struct Share {
    static constexpr int kCount = 16 / sizeof(T), kC = 128 * U / sizeof(T), kPieces = kRows * 8 * U / 256;
    static constexpr int kAcross = kTurned ? kRows / kCount : 8 * U, kLength = kTurned ? kRows * (int)sizeof(T) : 128 * U;      // pieces, bytes of a row in LDS
    typedef typename Piece<T>::type V;
    V v[kPieces], z[kSlope ? kPieces : 1];

    // The first i and c of piece t.  (Turned, all pieces of a thread are of the same i's.)
    static __device__ __forceinline__ void place(int t, int& i, int& c)
    {
        const int piece = t * 256 + (int)threadIdx.x, along = piece % kAcross * kCount, row = piece / kAcross;
        i = kTurned ? along : row;
        c = kTurned ? row : along;
    }

    // Element `along` on of a row of `length`.
    static __device__ __forceinline__ V load(const T* row, int along, int length)
    {
        V v;
        if constexpr (kFew) {
#pragma unroll
            for (int e = 0; e < kCount; ++e) v[e] = row[min(along + e, length - 1)];
        } else {
            v = *reinterpret_cast<const V*>(row + min(along, length - kCount));
        }
        return v;
    }

    __device__ __forceinline__ void fetch(const Side& s, int i0, int c0, int c_end)
    {
#pragma unroll
        for (int t = 0; t < kPieces; ++t) {
            int i, c;
            place(t, i, c);
            i += i0;
            c += c0;
            const size_t row = kTurned ? min(c, c_end - 1) : min(i, s.count - 1);
            const int along = kTurned ? i : c, length = kTurned ? s.count : c_end;
            v[t] = load(static_cast<const T*>(s.p) + row * s.ld, along, length);
            if constexpr (kSlope) z[t] = load(static_cast<const T*>(s.z) + row * s.ldz, along, length);
        }
    }

    // A piece that was loaded from before its place moves there; zeros behind the row's end (kFew: what was loaded there becomes zero).
    static __device__ __forceinline__ void move(V& v, int along, int length)
    {
        if constexpr (kFew) {
#pragma unroll
            for (int e = 0; e < kCount; ++e) v[e] = along + e < length ? v[e] : (T)0.f;
        } else {
            const int moved = max(along - (length - kCount), 0);
            const unsigned __int128 bits = __builtin_bit_cast(unsigned __int128, v);
            v = __builtin_bit_cast(V, moved < kCount ? bits >> (moved * 8 * (int)sizeof(T)) : (unsigned __int128)0);
        }
    }

    __device__ __forceinline__ void end(const Side& s, int i0, int c0, int c_end)
    {
        const bool last = c0 + kC > c_end, edge = kTurned && i0 + kRows > s.count;
        if (!last && !edge) return;
#pragma unroll
        for (int t = 0; t < kPieces; ++t) {
            int i, c;
            place(t, i, c);
            auto all = [&](V& v) {
                if (kTurned ? edge : last) move(v, kTurned ? i0 + i : c0 + c, kTurned ? s.count : c_end);
                if (kTurned && last)
#pragma unroll
                    for (int e = 0; e < kCount; ++e) v[e] = c0 + c < c_end ? v[e] : (T)0.f;
            };
            all(v[t]);
            if constexpr (kSlope) all(z[t]);
        }
    }

    // Multiplies by the slope; what is not rounded yet is added to `sums`, an element of the thread's pieces each (turned alone).
    __device__ __forceinline__ void apply(int act, float* sums)
    {
        auto all = [&](auto act) {
#pragma unroll
            for (int t = 0; t < kPieces; ++t)
#pragma unroll
                for (int e = 0; e < kCount; ++e) {
                    float g = (float)v[t][e];
                    if constexpr (act != kNone) {
                        g = behind<act>(g, (float)z[t][e]);
                        v[t][e] = (T)g;
                    }
                    if constexpr (kTurned) sums[e] += g;
                }
        };
        if constexpr (kSlope) with_activation(act, all);
        else all(std::integral_constant<int, kNone>{});
    }

    // kSums: the sums of what goes to LDS are wanted.  Rows lie along c there, U units, their pieces permuted by the row, or as they do in memory.
    template <bool kSums>
    __device__ __forceinline__ void put(const Side& s, int act, int i0, int c0, int c_end, char* to, float* sums)
    {
        end(s, i0, c0, c_end);
        if constexpr (kSlope || kSums) apply(act, sums);
        typedef T A __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
        for (int t = 0; t < kPieces; ++t) {
            int i, c;
            place(t, i, c);
            const int row = kTurned ? c : i, piece = (kTurned ? i : c) / kCount, turn = kTurned ? swizzle_of<T>(c, kRows) : U == 1 ? (i >> 1) & 7 : i & 15;
            *reinterpret_cast<A*>(to + row * kLength + ((piece ^ turn) << 4)) = v[t];
        }
    }
};

// 32 I by 32 J sums of a workgroup of four wavefronts, over c of c_begin .. c_end - 1.  The bytes of the kAhead steps that follow are on their way to
// registers while one is multiplied from LDS (two buffers, a barrier a step): a step takes 0.2 us of work, its loads 1 us and more.  Latency bounds it where
// a CU has one tile, so tiles are small (I = J = 1) while there are few: 24 x 1001 -> 1001 bfloat16 5.2 us in tiles of 32 x 32, 9.6 in 64 x 64.  Their steps are
// of two units of 128 bytes, for half of the barriers: 203 x 1001 -> 1111 fp32 11.2 us, 12.9 in steps of one unit; fp32 gradients of 300 x 300 -> 300 with relu
// 8.5 and 9.8 (in bfloat16 7.3 and 6.5), of 128 x 1024 -> 1024 12.5 and 17.5.  (One step of those ahead or three, and steps of four units, were 16 to 48 %
// slower at the first.  64 x 64: the same either way.)
constexpr int units_of(int I, int J) { return I * J == 1 ? 2 : 1; }
constexpr int ahead_of(int U) { return U == 1 ? 3 : 2; }

template <class T, int I, int J, bool kTurnedA, bool kTurnedB, bool kSlope, bool kFew>
__device__ __forceinline__ void direct_tile(const Side& a, const Side& b, int act, int i0, int j0, int c_begin, int c_end, char* lds, float4v (&acc)[I][J], float* sums)
{
    constexpr int U = units_of(I, J), kAhead = ahead_of(U), kRow = 128 * U, kA = 32 * I * kRow, kBuffer = kA + 32 * J * kRow, kC = kRow / sizeof(T);
    typedef Share<T, 32 * I, U, kTurnedA, kSlope, kFew> A;
    typedef Share<T, 32 * J, U, kTurnedB, false, kFew> B;
    A of_a[kAhead];
    B of_b[kAhead];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4, wi = wave & 1, wj = wave >> 1;
    const int turn = U == 1 ? r >> 1 : r, a_at = kTurnedA ? turned_address<T>(lane, wi * I, 32 * I) : (wi * I * 16 + r) * kRow + ((q ^ turn) << 4);
    const int b_at = kA + (kTurnedB ? turned_address<T>(lane, wj * J, 32 * J) : (wj * J * 16 + r) * kRow + ((q ^ turn) << 4));
    each<kAhead>([&](auto d) {
        of_a[d].fetch(a, i0, c_begin + d * kC, c_end);
        of_b[d].fetch(b, j0, c_begin + d * kC, c_end);
    });
    int buffer = 0;
    for (int first = c_begin; first < c_end; first += kAhead * kC)
        each<kAhead>([&](auto d) {      // (what lies past the end is zeros: the steps of a round are not skipped, whose loads would have to be waited for)
            const int c = first + d * kC;
            of_a[d].template put<kTurnedA>(a, act, i0, c, c_end, lds + buffer, sums);
            of_b[d].template put<false>(b, act, j0, c, c_end, lds + buffer + kA, nullptr);
            __syncthreads();
            of_a[d].fetch(a, i0, c + kAhead * kC, c_end);
            of_b[d].fetch(b, j0, c + kAhead * kC, c_end);
            auto read = [&](auto turned, int at, int h, int block, int length) {
                if constexpr (turned) return read_block<T>(lds + buffer + ((at + h * (64 / (int)sizeof(T)) * length) ^ (block * 16 * (int)sizeof(T))), length);
                else return *reinterpret_cast<const int4v*>(lds + buffer + (at ^ (h * 64)) + block * 16 * kRow);
            };
#pragma unroll
            for (int h = 0; h < 2 * U; ++h) {
                int4v fa[I], fb[J];
#pragma unroll
                for (int i = 0; i < I; ++i) fa[i] = read(std::integral_constant<bool, kTurnedA>{}, a_at, h, i, A::kLength);
#pragma unroll
                for (int j = 0; j < J; ++j) fb[j] = read(std::integral_constant<bool, kTurnedB>{}, b_at, h, j, B::kLength);
#pragma unroll
                for (int i = 0; i < I; ++i)
#pragma unroll
                    for (int j = 0; j < J; ++j) acc[i][j] = multiplied<T>(acc[i][j], fb[j], fa[i]);
            }
            buffer = kBuffer - buffer;
        });
}

// A tile's sums to the output (or to its part's sums): lane l holds row l % 16 of a's block and rows 4 (l / 16) .. + 3 of b's.
template <class T, int I, int J>
__device__ __forceinline__ void direct_store(const ProductArgs& a, int part, int m0, int n0, const float4v (&acc)[I][J])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4, wi = wave & 1, wj = wave >> 1;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int n = n0 + (wj * J + j) * 16 + q * 4;
        if (n >= a.N) continue;
        float bias[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) bias[e] = a.bias && n + e < a.N ? a.bias[n + e] : 0.f;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int m = m0 + (wi * I + i) * 16 + r;
            if (m >= a.M) continue;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = acc[i][j][e];
            if (a.partial) {
                float* to = a.partial + ((size_t)part * a.M + m) * a.N + n;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n + e < a.N) to[e] = v[e];
            } else {
                finish<T, 4>(a, v, bias, m, n, a.N - n);
            }
        }
    }
}

template <int I, int J>
__device__ __forceinline__ void zero(float4v (&acc)[I][J])
{
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};
}

// The layer on rows at any address, a part of the sum a workgroup.  `a` says where the output goes; a.steps: of 128 bytes, a part.
template <class T, int I, int J, bool kFew>
__global__ __launch_bounds__(256) void linear_direct_kernel(ProductArgs a, int K, long long ldx, long long ldw)
{
    __shared__ __attribute__((aligned(256))) char lds[2 * 32 * (I + J) * 128 * units_of(I, J)];
    const int across = (a.N + 32 * J - 1) / (32 * J), down = (a.M + 32 * I - 1) / (32 * I), tile = (int)(blockIdx.x % (unsigned)(across * down)), part = (int)(blockIdx.x / (unsigned)(across * down));
    const int m0 = tile % down * 32 * I, n0 = tile / down * 32 * J;
    constexpr int kC = 128 / sizeof(T);
    float4v acc[I][J];
    zero(acc);
    direct_tile<T, I, J, false, false, false, kFew>(Side{a.x, nullptr, ldx, 0, a.M}, Side{a.w, nullptr, ldw, 0, a.N}, kNone, m0, n0, part * a.steps * kC,
                                              min(K, (part + 1) * a.steps * kC), lds, acc, nullptr);
    direct_store<T, I, J>(a, part, m0, n0, acc);
}

// Both gradients in one launch: the first `tiles_x` workgroups take grad_x = d w (sum over N), the others grad_w = d^T x (over M) and, in the
// tiles of the first columns, the sums of d for the bias.  One launch instead of up to six (d, two products, joins, sums): 128 x 200 -> 256 fp32
// 4.5 us without an activation against 15.6 laid out, 5.2 with relu against 16.5.  Past about 2000 x 1000 -> 2000 (46 to 48 us either way) what the tiles read again
// from L2 costs more than that.
struct DirectGradArgs {
    const void *grad, *z, *x, *w;
    void *grad_x, *grad_w;
    float *grad_bias, *partial_x, *partial_w, *partial_bias;      // partial: of parts, or null
    long long ldg, ldx, ldw;
    const float* sums;                                            // or null: of d over 64 rows each, [(M + 63) / 64][N] (d itself is then `grad`)
    int M, N, K, act, accumulate, steps_x, steps_w;               // steps of 128 bytes, a part
    unsigned tiles_x;
};

template <class T, int I, int J, bool kSlope, bool kFew>
__global__ __launch_bounds__(256) void linear_direct_grad_kernel(DirectGradArgs a)
{
    __shared__ __attribute__((aligned(256))) char lds[2 * 32 * (I + J) * 128 * units_of(I, J)];
    constexpr int kC = 128 / sizeof(T), kCount = 16 / sizeof(T);
    const int across = (a.K + 32 * J - 1) / (32 * J);
    const Side d_rows{a.grad, a.z, a.ldg, a.N, a.M}, d_turned{a.grad, a.z, a.ldg, a.N, a.N};
    float4v acc[I][J];
    zero(acc);
    ProductArgs out{};
    if (blockIdx.x < a.tiles_x) {
        const int down = (a.M + 32 * I - 1) / (32 * I), tile = (int)(blockIdx.x % (unsigned)(across * down)), part = (int)(blockIdx.x / (unsigned)(across * down));
        const int m0 = tile % down * 32 * I, k0 = tile / down * 32 * J;
        direct_tile<T, I, J, false, true, kSlope, kFew>(d_rows, Side{a.w, nullptr, a.ldw, 0, a.K}, a.act, m0, k0, part * a.steps_x * kC, min(a.N, (part + 1) * a.steps_x * kC), lds, acc, nullptr);
        out.out = a.grad_x;
        out.partial = a.partial_x;
        out.M = a.M;
        out.N = a.K;
        out.ldo = a.K;
        direct_store<T, I, J>(out, part, m0, k0, acc);
        return;
    }
    const unsigned block = blockIdx.x - a.tiles_x;
    const int down = (a.N + 32 * I - 1) / (32 * I), tiles_w = down * (a.grad_w ? across : 1), tile = (int)(block % (unsigned)tiles_w), part = (int)(block / (unsigned)tiles_w);
    const int n0 = tile % down * 32 * I, k0 = tile / down * 32 * J;
    float sums[kCount] = {};
    direct_tile<T, I, J, true, true, kSlope, kFew>(d_turned, a.grad_w ? Side{a.x, nullptr, a.ldx, 0, a.K} : d_turned, a.act, n0, k0, part * a.steps_w * kC, min(a.M, (part + 1) * a.steps_w * kC), lds, acc, sums);
    out.out = a.grad_w;
    out.residual = a.accumulate ? a.grad_w : nullptr;
    out.partial = a.partial_w;
    out.M = a.N;
    out.N = a.K;
    out.ldo = out.ldr = a.K;
    if (a.grad_w) direct_store<T, I, J>(out, part, n0, k0, acc);
    if (!a.grad_bias || k0 != 0) return;
    if (a.sums) {
        constexpr int kGroups = 256 / (32 * I);
        if (part != 0) return;
        const int column = threadIdx.x % (32 * I), group = threadIdx.x / (32 * I), n = n0 + column, count = (a.M + 63) / 64;
        float* of = reinterpret_cast<float*>(lds);
        float total = 0.f;
        if (n < a.N)
#pragma unroll 8
            for (int i = group; i < count; i += kGroups) total += a.sums[(size_t)i * a.N + n];
        __syncthreads();
        of[threadIdx.x] = total;
        __syncthreads();
        if (group != 0 || n >= a.N) return;
        total = 0.f;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) total += of[g * 32 * I + column];
        a.grad_bias[n] = a.accumulate ? a.grad_bias[n] + total : total;
        return;
    }
    // The threads that hold the same i's lie kAcross apart; their sums are added in order.
    constexpr int kAcross = 32 * I / kCount;
    static_assert(256 % kAcross == 0, "a thread's pieces are of the same i's");
    float* of = reinterpret_cast<float*>(lds);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kCount; ++e) of[threadIdx.x / kAcross * (32 * I) + threadIdx.x % kAcross * kCount + e] = sums[e];
    __syncthreads();
    if ((int)threadIdx.x >= 32 * I || n0 + (int)threadIdx.x >= a.N) return;
    float total = 0.f;
#pragma unroll
    for (int p = 0; p < 256 / kAcross; ++p) total += of[p * 32 * I + threadIdx.x];
    const int n = n0 + threadIdx.x;
    if (a.partial_bias) a.partial_bias[(size_t)part * a.N + n] = total;
    else a.grad_bias[n] = a.accumulate ? a.grad_bias[n] + total : total;
}

// Very few rows of x: a wavefront (S wavefronts, that share the sum) takes C rows of w and all R of x, 16 bytes a lane of each at a time.  The weights'
// bytes bound it, and the latency of the first: 1 x 4096 -> 4096 bfloat16 7.2 us (33.6 MB, 6.55 at the rate of a large copy).
template <class T, int R, int C, int S>
__global__ __launch_bounds__(256) void linear_dot_kernel(ProductArgs a, int K, long long ldx, long long ldw)
{
    typedef typename Piece<T>::type V;
    constexpr int kCount = 16 / sizeof(T), kAhead = R * C <= 2 ? 4 : 2;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n0 = (int)(blockIdx.x * (4 / S) + wave / S) * C;
    const T* x = static_cast<const T*>(a.x);
    const T* w = static_cast<const T*>(a.w);
    float sum[R][C] = {};
    auto add = [&](const V (&xv)[R], const V (&wv)[C]) {
#pragma unroll
        for (int e = 0; e < kCount; ++e)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int c = 0; c < C; ++c) sum[r][c] = fmaf((float)xv[r][e], (float)wv[c][e], sum[r][c]);
    };
    const T* row[C];
#pragma unroll
    for (int c = 0; c < C; ++c) row[c] = w + (size_t)min(n0 + c, a.N - 1) * ldw;
    constexpr int kStep = 64 * kCount * S;
    int k = ((wave % S) * 64 + lane) * kCount;
    for (; k + (kAhead - 1) * kStep + kCount <= K; k += kAhead * kStep) {
        V xv[kAhead][R], wv[kAhead][C];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
#pragma unroll
            for (int c = 0; c < C; ++c) wv[u][c] = *reinterpret_cast<const V*>(row[c] + k + u * kStep);
#pragma unroll
            for (int r = 0; r < R; ++r) xv[u][r] = *reinterpret_cast<const V*>(x + (size_t)min(r, a.M - 1) * ldx + k + u * kStep);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) add(xv[u], wv[u]);
    }
    for (; k < K; k += kStep) {
        V xv[R], wv[C];
#pragma unroll
        for (int c = 0; c < C; ++c) wv[c] = load_piece<T>(row[c], k, K);
#pragma unroll
        for (int r = 0; r < R; ++r) xv[r] = load_piece<T>(x + (size_t)min(r, a.M - 1) * ldx, k, K);
        add(xv, wv);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int d = 32; d > 0; d /= 2) sum[r][c] += __shfl_xor(sum[r][c], d);
    if constexpr (S > 1) {
        __shared__ float of[4][R * C];
        if (lane == 0)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int c = 0; c < C; ++c) of[wave][r * C + c] = sum[r][c];
        __syncthreads();
        if (wave % S != 0) return;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                sum[r][c] = 0.f;
#pragma unroll
                for (int i = 0; i < S; ++i) sum[r][c] += of[wave + i][r * C + c];
            }
    }
    // Lane r finishes row r.
    float v[C], bias[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        v[c] = sum[0][c];
#pragma unroll
        for (int r = 1; r < R; ++r) v[c] = lane == r ? sum[r][c] : v[c];
        bias[c] = a.bias && n0 + c < a.N ? a.bias[n0 + c] : 0.f;
    }
    if (lane < min(R, a.M) && n0 < a.N) finish<T, C>(a, v, bias, lane, n0, a.N - n0);
}

// ---------------------------------------------------------------- which kernel

double pieces_of(int n, int size) { return (double)((n + size - 1) / size); }

// Microseconds that a product of rows of `bytes` is estimated to take.  The constants are fitted, for 16-bit types and for fp32, to what each kernel near the fastest
// took at 159 sizes (4 to 8192 rows of x, 64 to 8192 of w and of terms), on three sets of arrays in turn; those of the 2 x 2 row kernel of 16 bits
// at 98 more, of 5 to 128 rows, there also with weights that all come from HBM.  Without an activation, what the estimates choose took more than the fastest
// by: at 147 sizes of 5 to 128 rows, the 98 among them, 2.3 % on average on three sets in turn, 2.6 % from HBM, at most 43 % (5 x 256 -> 4544 bfloat16 4.7 us, 3.3 in
// tiles of 32 x 32); at others of 160 to 8192 rows 1.5 % in 16 bits (60), at most 17 %, and 6 % in fp32 (56), at most 43 % (1024 x 2304 -> 1088 85 us, 59 by
// the 4 x 1 row kernel).  What the epilogue does is not in the estimates.

// Row kernel: a launch, the sums of the wavefronts and the further workgroups of a CU, then the largest of what all workgroups load,
// what those of one CU load, both operands from memory, and the products.
struct RowRule {
    int MB, NB;
    double join, more;                        // us
    double all, one, arrays, products;        // MB/us of all, KB/us of one, MB/us of the arrays; us for 1000 bytes of a block
};
constexpr RowRule kRowRules[2][5] = {
    {{1, 1, 1.22, 0.603, 17.9, 137.0, 6.23, 0.0547}, {2, 1, 0.746, 0.317, 21.6, 129.0, 5.98, 0.0479}, {2, 2, 1.5, 1.01, 13.2, 120.0, 5.22, 0.0478},
     {4, 1, 0.899, 0.344, 21.1, 139.0, 4.77, 0.05}, {4, 2, 2.04, 0.601, 16.1, 121.0, 6.32, 0.0499}},
    {{1, 1, 1.15, 0.769, 16.3, 174.0, 4.99, 0.356}, {2, 1, 0.66, 0.317, 14.9, 66.9, 4.09, 0.358}, {2, 2, 1.56, 1.54, 28.8, 182.0, 4.61, 0.287},
     {4, 1, 0.829, 0.344, 48.2, 119.0, 4.34, 0.331}, {4, 2, 2.13, 1.37, 10.0, 166.0, 6.05, 0.289}}};

double row_estimate(const RowRule& r, int M, int N, double bytes)
{
    const double groups = pieces_of(M, 16 * r.MB) * pieces_of(N, 16 * r.NB), loaded = 16.0 * (r.MB + r.NB) * bytes, on_a_cu = std::ceil(groups / 256.0);
    return 3.0 + r.join * on_a_cu + r.more * (on_a_cu - 1.0) +
           std::max({groups * loaded / (r.all * 1e6), on_a_cu * loaded / (r.one * 1e3), ((double)M + N) * bytes / (r.arrays * 1e6), on_a_cu * r.MB * r.NB * bytes * r.products * 1e-3});
}

// Tile kernel: steps of `least` us while a workgroup has the CU to itself, `each` times the workgroups that share it beyond; the operands
// from memory at least; the output.
struct TileRule {
    int MB, NB, share;                        // blocks of a wavefront; workgroups that a CU holds
    double least, each, start, finish;
    double arrays, output;                    // MB/us
};
constexpr TileRule kTileRules[2][6] = {
    {{2, 2, 4, 0.223, 0.176, 1.25, 2.34, 1.58, 8.54}, {4, 4, 2, 0.063, 0.438, 1.79, 3.18, 4.61, 20.3}, {8, 8, 1, 0.00878, 1.15, 7.83, 2.04, 5.5, 6.17},
     {2, 2, 2, 0.043, 0.203, 2.63, 1.29, 5.17, 15.3}, {4, 2, 1, 0.0104, 0.297, 2.55, 1.58, 9.4, 5.15}, {4, 4, 1, 0.01, 0.429, 2.87, 2.09, 5.56, 7.34}},
    {{2, 2, 4, 0.268, 0.535, 1.25, 2.51, 1.72, 26.0}, {4, 4, 2, 0.0675, 1.91, 1.79, 3.91, 2.04, 6.97}, {8, 8, 1, 0.0, 7.7, 1.55, 8.19, 5.0, 12.3},
     {2, 2, 2, 0.043, 0.56, 2.35, 1.82, 29.1, 89.6}, {4, 2, 1, 0.015, 1.02, 2.82, 1.52, 4.47, 4.46}, {4, 4, 1, 0.01, 1.91, 1.57, 4.43, 2.0, 13.1}}};

double tile_estimate(const TileRule& r, int M, int N, int parts, double bytes, int element)
{
    const double groups = pieces_of(M, 32 * r.MB) * pieces_of(N, 32 * r.NB) * parts, steps = std::ceil(bytes / 128.0 / parts), held = 256.0 * r.share;
    const double rounds = std::floor(groups / held), rest = groups - rounds * held;
    double us = r.start + rounds * (steps * r.each * r.share + r.finish);
    if (rest > 0.0) us += steps * std::max(r.least, r.each * std::ceil(rest / 256.0)) + r.finish;
    return std::max(us, 3.0 + ((double)M + N) * bytes / (r.arrays * 1e6)) + (double)M * N * element / (r.output * 1e6);
}

// Parts of a sum, and the launch that adds them up.
double join_estimate(int parts, double outputs) { return parts > 1 ? 3.5 + 4.0 * outputs * (parts + 1) / 4e6 : 0.0; }

struct Choice {
    Kernel kernel;
    int parts, steps;
    double us;
};

// turned: both operands or w alone (tile kernels take those).
Choice choose(int dtype, int M, int N, int terms, bool turned)
{
    const int wide = dtype == kF32;
    const int row_bytes = (terms * (dtype == kF32 ? 4 : 2) + 15) / 16 * 16, all = (row_bytes + 127) / 128;
    const double bytes = row_bytes;
    Choice best{kKernels, 1, all, 0.0};
    for (int k = turned ? kTile22 : 0; k < kKernels; ++k) {
        if (k == kTile88 && dtype == kF32) continue;
        if (k == kDeep42 && turned) continue;
        for (int parts = 1; parts <= (k < kTile22 ? 1 : 64); parts *= 2) {
            const int steps = (all + parts - 1) / parts;
            if (parts > 1 && (steps < 8 || (double)M * N * parts > 1.6e7)) break;
            if (k == kTile88 && steps < kStepsToWalk) break;
            const double us = k < kTile22 ? row_estimate(kRowRules[wide][k], M, N, bytes)
                                          : tile_estimate(kTileRules[wide][k - kTile22], M, N, parts, bytes, wide ? 4 : 2) + join_estimate(parts, (double)M * N);
            if (best.kernel == kKernels || us < best.us) best = Choice{(Kernel)k, (all + steps - 1) / steps, steps, us};
        }
    }
    return best;
}

template <class T>
int launch_join(const ProductArgs& a, hipStream_t s)
{
    const long long groups = ((a.N + 3ll) / 4 * a.M + 255) / 256;
    if ((unsigned long long)groups > most_groups(256)) return kTooLarge;
    hipLaunchKernelGGL(linear_join_kernel<T>, dim3((unsigned)groups), dim3(256), 0, s, a);
    return (int)hipGetLastError();
}

long long round_up(long long n, long long to) { return (n + to - 1) / to * to; }

long long partial_bytes(int parts, int M, int N) { return parts > 1 ? round_up(4ll * parts * M * N, 256) : 0; }

// The product of operands that are laid out; partial: scratch memory of partial_bytes.
int product(int dtype, const Choice& c, Turned turned, ProductArgs a, char* partial, hipStream_t s)
{
    a.parts = c.parts;
    a.steps = c.steps;
    a.partial = c.parts > 1 ? reinterpret_cast<float*>(partial) : nullptr;
    int e = dtype == kF32 ? launch_laid_f32(c.kernel, turned, a, s) : dtype == kF16 ? launch_laid_f16(c.kernel, turned, a, s) : launch_laid_bf16(c.kernel, turned, a, s);
    if (e != 0 || c.parts == 1) return e;
    return dtype == kF32 ? launch_join<float>(a, s) : dtype == kF16 ? launch_join<_Float16>(a, s) : launch_join<__bf16>(a, s);
}

// ---------------------------------------------------------------- rows laid out

// Tiles of 64 x 64 elements of [rows][cols] (ld elements from one row to the next) to `copy` (or null), rows of copy_pitch elements with zeros behind
// what is there.  With an activation the elements are first multiplied by its slope at z (no gaps), in fp32, and rounded once; column_sums
// [tiles down][cols] (or null) receives the sums over the tile's rows of what was not rounded.  Bytes bound it: 8192 x 8192 bfloat16 with the slope
// of gelu, 403 MB, 77 us (5.2 TB/s).
struct LayArgs {
    const void *from, *z;
    void* copy;
    float* column_sums;
    long long ld;
    int rows, cols, copy_pitch, act;
};

template <class T>
__global__ __launch_bounds__(256) void linear_lay_kernel(LayArgs a)
{
    constexpr int kCount = 16 / sizeof(T), kPer = 64 / kCount, kTurns = 64 * kPer / 256;      // pieces a row of the tile; a thread's pieces
    typedef typename Piece<T>::type V;
    __shared__ float sums[256 / kPer][64];
    const int across = (max(a.cols, a.copy_pitch) + 63) / 64, tr = (int)(blockIdx.x / (unsigned)across), tc = (int)(blockIdx.x % (unsigned)across);
    const int piece = threadIdx.x % kPer, first = threadIdx.x / kPer, col = tc * 64 + piece * kCount;
    float total[kCount] = {};
    V v[kTurns], z[kTurns];
    // (All loads first.  A piece that ends past its row is the last one within it, moved down.)
    const int from = min(col, a.cols - kCount), moved = col - from;
    auto whole = [&](const T* row) {
        if (a.cols < kCount) return load_piece<T>(row, col, a.cols);
        return *reinterpret_cast<const V*>(row + from);
    };
    auto place = [&](V& v) {
        if (a.cols < kCount || moved <= 0) return;
        const unsigned __int128 bits = __builtin_bit_cast(unsigned __int128, v);
        v = __builtin_bit_cast(V, moved < kCount ? bits >> (moved * 8 * (int)sizeof(T)) : (unsigned __int128)0);
    };
#pragma unroll
    for (int t = 0; t < kTurns; ++t) v[t] = whole(static_cast<const T*>(a.from) + (size_t)min(tr * 64 + first + t * (256 / kPer), a.rows - 1) * a.ld);
    if (a.z)
#pragma unroll
        for (int t = 0; t < kTurns; ++t) z[t] = whole(static_cast<const T*>(a.z) + (size_t)min(tr * 64 + first + t * (256 / kPer), a.rows - 1) * a.cols);
    auto all = [&](auto act) {
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            const int row = tr * 64 + first + t * (256 / kPer);
            if (row >= a.rows) break;
            place(v[t]);
            if constexpr (act != kNone) place(z[t]);
#pragma unroll
            for (int e = 0; e < kCount; ++e) {
                float g = (float)v[t][e];
                if constexpr (act != kNone) {
                    g = col + e < a.cols ? behind<act>(g, (float)z[t][e]) : 0.f;
                    v[t][e] = (T)g;
                }
                total[e] += g;
            }
            if (a.copy && col < a.copy_pitch) {
                T* const to = static_cast<T*>(a.copy) + (size_t)row * a.copy_pitch + col;
                if (col + kCount <= a.copy_pitch) *reinterpret_cast<V*>(to) = v[t];
                else
#pragma unroll
                    for (int e = 0; e < kCount; ++e)
                        if (col + e < a.copy_pitch) to[e] = v[t][e];
            }
        }
    };
    if (a.z) with_activation(a.act, all);
    else all(std::integral_constant<int, kNone>{});
    if (!a.column_sums) return;
#pragma unroll
    for (int e = 0; e < kCount; ++e) sums[first][piece * kCount + e] = total[e];
    __syncthreads();
    if (threadIdx.x < 64 && tc * 64 + (int)threadIdx.x < a.cols) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 256 / kPer; ++i) s += sums[i][threadIdx.x];
        a.column_sums[(size_t)tr * a.cols + tc * 64 + threadIdx.x] = s;
    }
}

// out[n] = (accumulate: out[n] +) the sum of sums[i][n], in order.
__global__ __launch_bounds__(256) void linear_bias_kernel(const float* sums, float* out, int count, int N, int accumulate)
{
    constexpr int kRows = 16;
    __shared__ float of[kRows][16];
    const int c = threadIdx.x % 16, r = threadIdx.x / 16, n = blockIdx.x * 16 + c;
    float total = 0.f;
    if (n < N)
        for (int i = r; i < count; i += kRows) total += sums[(size_t)i * N + n];
    of[r][c] = total;
    __syncthreads();
    if (r != 0 || n >= N) return;
    total = 0.f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) total += of[i][c];
    out[n] = accumulate ? out[n] + total : total;
}

// Zeros in both arrays (either or null), whose bytes are a multiple of 2.
__global__ __launch_bounds__(256) void linear_zeros_kernel(unsigned short* a, long long na, unsigned short* b, long long nb)
{
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < max(na, nb); i += gridDim.x * 256ll) {
        if (i < na) a[i] = 0;
        if (i < nb) b[i] = 0;
    }
}

int launch_zeros(void* a, long long a_bytes, void* b, long long b_bytes, hipStream_t s)
{
    hipLaunchKernelGGL(linear_zeros_kernel, dim3(1024), dim3(256), 0, s, static_cast<unsigned short*>(a), a ? a_bytes / 2 : 0, static_cast<unsigned short*>(b), b ? b_bytes / 2 : 0);
    return (int)hipGetLastError();
}

template <class T>
int launch_lay_of(const LayArgs& a, hipStream_t s)
{
    const long long groups = ((a.rows + 63ll) / 64) * ((std::max(a.cols, a.copy_pitch) + 63ll) / 64);
    if ((unsigned long long)groups > most_groups(256)) return kTooLarge;
    hipLaunchKernelGGL(linear_lay_kernel<T>, dim3((unsigned)groups), dim3(256), 0, s, a);
    return (int)hipGetLastError();
}

int launch_lay(int dtype, const LayArgs& a, hipStream_t s)
{
    return dtype == kF32 ? launch_lay_of<float>(a, s) : dtype == kF16 ? launch_lay_of<_Float16>(a, s) : launch_lay_of<__bf16>(a, s);
}

int bytes_of(int dtype) { return dtype == kF32 ? 4 : 2; }

constexpr long long kMostPitch = 1 << 23;      // bytes: 256 rows of them are what a descriptor describes

// Rows that the products can read as they are: whole pieces of 16 bytes at multiples of 16.
bool laid_out(const void* p, long long ld, int rows, int cols, int b)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && cols * b % 16 == 0 && (rows == 1 || (ld * b % 16 == 0 && ld * b <= kMostPitch));
}

long long pitch_of(long long cols, int b) { return round_up(cols, 16 / b); }
long long laid_bytes(long long rows, long long cols, int b) { return round_up(rows * pitch_of(cols, b) * b, 256); }

// How the layer is computed: very few rows by linear_dot_kernel; rows at odd addresses, or too few steps to pay for laying them out, by
// linear_direct_kernel; else from rows that are laid out.
enum Way { kDot, kDirect, kLaid };

struct LinearPlan {
    Way way;
    Choice laid;            // of kLaid
    bool small;             // kDirect: tiles of 32 x 32
    int parts, steps;
    bool lay_x, lay_w;
    long long x, w, end;    // bytes of scratch memory: where w's copy and the parts begin, and all
};

double lay_estimate(double bytes) { return 3.0 + bytes / 4e6; }

// A direct launch of `tiles` that take `work` steps in all, `longest` of them one after another at most, of arrays of `bytes`.  turned: the gradients'
// operands; small: tiles of 32 x 32 instead of 64 x 64 (faster until they are several for each CU: gradients of 128 x 200 -> 256 fp32 4.5 us against
// 9.3, of 1024 x 1024 -> 1024 bfloat16 21.7 against 15.2).  Outputs, z and residuals are not in `bytes`, and rows at odd addresses count as others do (gradients of
// 1021 x 1001 -> 777 float16 with silu: 20 us estimated, 25.8 taken).
double direct_estimate(int dtype, bool turned, bool small, double tiles, double work, int longest, double bytes)
{
    const bool wide = dtype == kF32;
    const double alone = small ? (wide ? 0.24 : 0.20) : wide ? 0.74 : 0.34;
    const double shared = small ? (wide ? 0.20 : turned ? 0.15 : 0.20) : wide ? (turned ? 0.60 : 0.63) : turned ? 0.28 : 0.25;
    return (small ? 3.7 : 4.5) + std::max({longest * alone, work / 256.0 * shared, bytes / 5.2e6}) + tiles / 256.0 * (turned ? 1.2 : 0.9) * (small ? 0.5 : 1.0);
}

// Parts of a sum of `all` steps, one for each workgroup: their number is a power of two but where the last would be empty.
int parts_of(int all, int wanted)
{
    const int steps = (all + wanted - 1) / wanted;
    return (all + steps - 1) / steps;
}

// f(small, parts) for both tiles and all parts of a sum that are looked at: `all` steps, `tiles(size)` of them a part.
template <class Tiles, class F>
void each_split(int all, Tiles&& tiles, F&& f)
{
    for (int small = 0; small < 2; ++small)
        for (int parts = 1; parts <= 64 && (parts == 1 || (all >= 8 * parts && tiles(small ? 32 : 64) * parts <= 512.0)); parts *= 2) f(small != 0, parts_of(all, parts));
}

LinearPlan plan_of(const LinearArgs& a, int dtype)
{
    const int b = bytes_of(dtype), row_bytes = (int)pitch_of(a.K, b) * b, all = (row_bytes + 127) / 128;
    LinearPlan p{};
    p.lay_x = !laid_out(a.x, a.ldx, a.M, a.K, b);
    p.lay_w = !laid_out(a.w, a.ldw, a.N, a.K, b);
    // (Two rows that are laid out, or four of fp32: 4096 -> 4096 8.1 us and 8.4 by the other kernels in bfloat16, 13.1 and 14.6 in fp32; four in bfloat16 9.2 and
    // 8.5.  Eight that are not: 1001 -> 1001 6.3 and 5.3 in bfloat16, 5.5 and 8.2 in fp32.)
    if (a.M <= (p.lay_x || p.lay_w ? 8 : dtype == kF32 ? 4 : 2)) {
        p.way = kDot;
        return p;
    }
    double direct = -1.0;
    auto tiles = [&](int size) { return pieces_of(a.M, size) * pieces_of(a.N, size); };
    each_split(all, tiles, [&](bool small, int parts) {
        const int steps = (all + parts - 1) / parts;
        const double count = tiles(small ? 32 : 64), us = direct_estimate(dtype, false, small, count * parts, count * all, steps, ((double)a.M + a.N) * row_bytes) + join_estimate(parts, (double)a.M * a.N);
        if (direct >= 0.0 && us >= direct) return;
        direct = us;
        p.small = small;
        p.parts = parts;
        p.steps = steps;
    });
    p.laid = choose(dtype, a.M, a.N, a.K, false);
    const double laid = p.laid.us + (p.lay_x ? lay_estimate(2.0 * a.M * row_bytes) : 0.0) + (p.lay_w ? lay_estimate(2.0 * a.N * row_bytes) : 0.0);
    if (direct < laid) {
        p.way = kDirect;
        p.end = partial_bytes(p.parts, a.M, a.N);
        return p;
    }
    p.way = kLaid;
    p.x = p.lay_x ? laid_bytes(a.M, a.K, b) : 0;
    p.w = p.x + (p.lay_w ? laid_bytes(a.N, a.K, b) : 0);
    p.end = p.w + partial_bytes(p.laid.parts, a.M, a.N);
    return p;
}

template <class T, int R, int C>
int launch_dot(const ProductArgs& a, const LinearArgs& l, hipStream_t s)
{
    // (wavefronts that share a sum where there are too few rows of w for every SIMD to have some)
    const long long groups = (a.N + C - 1ll) / C;
    if (groups <= 512) hipLaunchKernelGGL((linear_dot_kernel<T, R, C, 4>), dim3((unsigned)groups), dim3(256), 0, s, a, l.K, l.ldx, l.ldw);
    else hipLaunchKernelGGL((linear_dot_kernel<T, R, C, 1>), dim3((unsigned)((groups + 3) / 4)), dim3(256), 0, s, a, l.K, l.ldx, l.ldw);
    return (int)hipGetLastError();
}

template <class T>
int launch_way(const LinearPlan& p, ProductArgs a, const LinearArgs& l, char* workspace, hipStream_t s)
{
    if (p.way == kDot) {
        if (l.M == 1) return launch_dot<T, 1, 2>(a, l, s);
        if (l.M == 2) return launch_dot<T, 2, 2>(a, l, s);
        if (l.M <= 4) return launch_dot<T, 4, 2>(a, l, s);
        return launch_dot<T, 8, 2>(a, l, s);
    }
    a.parts = p.parts;
    a.steps = p.steps;
    a.partial = p.parts > 1 ? reinterpret_cast<float*>(workspace) : nullptr;
    const long long tile = p.small ? 32 : 64, groups = (a.M + tile - 1) / tile * ((a.N + tile - 1) / tile) * p.parts;
    if ((unsigned long long)groups > most_groups(256)) return kTooLarge;
    const dim3 grid((unsigned)groups), block(256);
    const bool few = l.K < (int)(16 / sizeof(T));
    if (p.small && few) hipLaunchKernelGGL((linear_direct_kernel<T, 1, 1, true>), grid, block, 0, s, a, l.K, l.ldx, l.ldw);
    else if (p.small) hipLaunchKernelGGL((linear_direct_kernel<T, 1, 1, false>), grid, block, 0, s, a, l.K, l.ldx, l.ldw);
    else if (few) hipLaunchKernelGGL((linear_direct_kernel<T, 2, 2, true>), grid, block, 0, s, a, l.K, l.ldx, l.ldw);
    else hipLaunchKernelGGL((linear_direct_kernel<T, 2, 2, false>), grid, block, 0, s, a, l.K, l.ldx, l.ldw);
    const int e = (int)hipGetLastError();
    return e != 0 || p.parts == 1 ? e : launch_join<T>(a, s);
}

}  // namespace

long long linear_workspace(const LinearArgs& a, int dtype) { return plan_of(a, dtype).end; }

namespace {

// Operands without gaps at multiples of 16 bytes.
LinearPlan plan_of(int dtype, int M, int N, int K)
{
    LinearArgs a{};
    a.M = M;
    a.N = N;
    a.K = K;
    a.ldx = a.ldw = K;
    return plan_of(a, dtype);
}

bool few_of(int dtype, int terms) { return terms * bytes_of(dtype) < 16; }

}  // namespace

int linear_kernel(int dtype, int M, int N, int K)
{
    const LinearPlan p = plan_of(dtype, M, N, K);
    return p.way == kDot ? 100 : p.way == kDirect ? (p.small ? 103 : 101) : p.laid.kernel;
}

int linear_form(int dtype, int M, int N, int K)
{
    const LinearPlan p = plan_of(dtype, M, N, K);
    if (p.way == kDot) return 0;
    if (p.way == kLaid) return p.laid.parts > 1 ? 8 : 0;
    return p.small + 2 * few_of(dtype, K) + 8 * (p.parts > 1);
}

int launch_linear(int dtype, const LinearArgs& a, char* workspace, void* stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int b = bytes_of(dtype), row_bytes = (int)pitch_of(a.K, b) * b;
    const LinearPlan plan = plan_of(a, dtype);
    ProductArgs p{a.x, a.w, a.bias, a.residual, a.out, a.z, nullptr, a.M, a.N, a.K, (int)(a.M > 1 ? a.ldx * b : row_bytes), (int)(a.N > 1 ? a.ldw * b : row_bytes),
                  a.act, 0, 1, a.ldr, a.ldo};
    if (plan.way != kLaid)
        return dtype == kF32 ? launch_way<float>(plan, p, a, workspace, s) : dtype == kF16 ? launch_way<_Float16>(plan, p, a, workspace, s) : launch_way<__bf16>(plan, p, a, workspace, s);
    if (plan.lay_x) {
        const int e = launch_lay(dtype, LayArgs{a.x, nullptr, workspace, nullptr, a.ldx, a.M, a.K, row_bytes / b, kNone}, s);
        if (e != 0) return e;
        p.x = workspace;
        p.x_pitch = row_bytes;
    }
    if (plan.lay_w) {
        const int e = launch_lay(dtype, LayArgs{a.w, nullptr, workspace + plan.x, nullptr, a.ldw, a.N, a.K, row_bytes / b, kNone}, s);
        if (e != 0) return e;
        p.w = workspace + plan.x;
        p.w_pitch = row_bytes;
    }
    return product(dtype, plan.laid, kRows, p, workspace + plan.w, s);
}

namespace {

// How the gradients are computed, and where the pieces of a pass lie in its scratch memory.
struct GradPlan {
    bool direct, formed, small;                              // direct; the gradient behind the activation is formed by a launch before; tiles of 32 x 32
    int parts_x, parts_w, steps_x, steps_w;
    long long sums_x, sums_w, sums_bias;
    // laid out
    bool own_dz, lay_x, lay_w;                               // the gradient behind the activation is formed (else grad is it); x, w are copied
    Choice x, w;
    long long dz, x_at, w_at, sums, partial;
    long long end;
};

GradPlan plan_of(const LinearGradArgs& a, int dtype)
{
    const int b = bytes_of(dtype), count = 128 / b;
    GradPlan l{};
    l.own_dz = a.act != kNone || !laid_out(a.grad, a.ldg, a.M, a.N, b);
    l.lay_x = a.grad_w && !laid_out(a.x, a.ldx, a.M, a.K, b);
    l.lay_w = a.grad_x && !laid_out(a.w, a.ldw, a.N, a.K, b);
    long long at = 0;
    auto take = [&](bool wanted, long long bytes) {
        const long long here = at;
        if (wanted) at += round_up(bytes, 256);
        return here;
    };
    double laid = 0.0, direct = -1.0;
    // (Chosen as if all three were wanted: a gradient's bits do not depend on which others are.)
    l.x = choose(dtype, a.M, a.K, a.N, true);
    l.w = choose(dtype, a.N, a.K, a.M, true);
    laid = l.x.us + l.w.us + lay_estimate((l.own_dz ? 3.0 : 1.0) * a.M * a.N * b) + 3.0;
    // (Copies that an address or a distance alone makes necessary are not priced: x's and w's are not known where their gradients are not wanted.)
    if (a.K * b % 16 != 0) laid += lay_estimate(2.0 * a.N * a.K * b) + lay_estimate(2.0 * a.M * a.K * b);
    const int all_x = (a.N + count - 1) / count, all_w = (a.M + count - 1) / count;
    const double form = lay_estimate(3.0 * a.M * a.N * b) + 1.5;
    auto tiles_x = [&](int size) { return pieces_of(a.M, size) * pieces_of(a.K, size); };
    auto tiles_w = [&](int size) { return pieces_of(a.N, size) * pieces_of(a.K, size); };
    const double bytes = ((double)a.M * a.N * (a.act == kNone ? 1 : 2) + (double)a.M * a.K + (double)a.N * a.K) * b;
    each_split(all_x, tiles_x, [&](bool small, int parts_x) {
        each_split(all_w, tiles_w, [&](bool small_w, int parts_w) {
            if (small != small_w) return;
            const double x = tiles_x(small ? 32 : 64), w = tiles_w(small ? 32 : 64), work = x * all_x + w * all_w;
            const int steps_x = (all_x + parts_x - 1) / parts_x, steps_w = (all_w + parts_w - 1) / parts_w, longest = std::max(steps_x, steps_w);
            // (Where the slope is worked out as the tiles are loaded, every tile along K does it anew.)
            const double anew = a.act == kNone ? 0.0 : std::max(work / 256.0, (double)longest) * (a.act == kRelu ? 0.42 : 0.50) * (dtype == kF32 ? 0.5 : 1.0) * (small ? 0.8 : 1.0);
            const double us = direct_estimate(dtype, true, small, x * parts_x + w * parts_w, work, longest, bytes) + join_estimate(parts_x, (double)a.M * a.K) +
                              join_estimate(parts_w, (double)a.N * a.K) + 2.0 * ((parts_x > 1) + (parts_w > 1)) + std::min(anew, form);
            if (direct >= 0.0 && us >= direct) return;
            direct = us;
            l.small = small;
            l.formed = anew > form;
            l.parts_x = parts_x;
            l.parts_w = parts_w;
            l.steps_x = steps_x;
            l.steps_w = steps_w;
        });
    });
    if (direct < laid) {
        l.direct = true;
        l.dz = take(l.formed, (long long)a.M * a.N * b);
        l.sums = take(l.formed && a.grad_bias, (a.M + 63ll) / 64 * a.N * 4);
        l.sums_x = take(a.grad_x, partial_bytes(l.parts_x, a.M, a.K));
        l.sums_w = take(a.grad_w, partial_bytes(l.parts_w, a.N, a.K));
        l.sums_bias = take(a.grad_bias && l.parts_w > 1 && !l.formed, 4ll * l.parts_w * a.N);
        l.end = at;
        return l;
    }
    l.dz = take(l.own_dz && (a.grad_x || a.grad_w), laid_bytes(a.M, a.N, b));
    l.x_at = take(l.lay_x, laid_bytes(a.M, a.K, b));
    l.w_at = take(l.lay_w, laid_bytes(a.N, a.K, b));
    l.sums = take(a.grad_bias, (a.M + 63ll) / 64 * a.N * 4);
    l.partial = take(true, std::max(a.grad_x ? partial_bytes(l.x.parts, a.M, a.K) : 0, a.grad_w ? partial_bytes(l.w.parts, a.N, a.K) : 0));
    l.end = at;
    return l;
}

int launch_bias(const float* sums, float* out, int count, int N, bool accumulate, hipStream_t s)
{
    hipLaunchKernelGGL(linear_bias_kernel, dim3((unsigned)((N + 15) / 16)), dim3(256), 0, s, sums, out, count, N, (int)accumulate);
    return (int)hipGetLastError();
}

template <class T>
int launch_direct_grad(const GradPlan& l, const LinearGradArgs& a, char* workspace, hipStream_t s)
{
    const unsigned long long tile = l.small ? 32 : 64, across = (a.K + tile - 1) / tile;
    const unsigned long long x = a.grad_x ? (a.M + tile - 1) / tile * across * l.parts_x : 0;
    const unsigned long long w = a.grad_w || a.grad_bias ? (a.N + tile - 1) / tile * (a.grad_w ? across : 1ull) * l.parts_w : 0;
    if (x + w > most_groups(256)) return kTooLarge;
    if (x + w == 0) return 0;
    float* const px = a.grad_x && l.parts_x > 1 ? reinterpret_cast<float*>(workspace + l.sums_x) : nullptr;
    float* const pw = a.grad_w && l.parts_w > 1 ? reinterpret_cast<float*>(workspace + l.sums_w) : nullptr;
    float* const pb = a.grad_bias && l.parts_w > 1 && !l.formed ? reinterpret_cast<float*>(workspace + l.sums_bias) : nullptr;
    DirectGradArgs d{a.grad, a.act != kNone ? a.z : nullptr, a.x, a.w, a.grad_x, a.grad_w, a.grad_bias, px, pw, pb, a.ldg, a.ldx, a.ldw, nullptr, a.M, a.N, a.K, a.act,
                     a.accumulate, l.steps_x, l.steps_w, (unsigned)x};
    int e = 0;
    if (l.formed) {
        float* const sums = a.grad_bias ? reinterpret_cast<float*>(workspace + l.sums) : nullptr;
        e = launch_lay_of<T>(LayArgs{a.grad, a.z, workspace + l.dz, sums, a.ldg, a.M, a.N, a.N, a.act}, s);
        if (e != 0) return e;
        d.grad = workspace + l.dz;
        d.z = nullptr;
        d.ldg = a.N;
        d.sums = sums;
        d.act = kNone;
    }
    const dim3 grid((unsigned)(x + w)), block(256);
    const bool few = std::min(a.N, a.K) < (int)(16 / sizeof(T));
    auto enqueue = [&](auto slope, auto few_of) {
        if (l.small) hipLaunchKernelGGL((linear_direct_grad_kernel<T, 1, 1, decltype(slope)::value, decltype(few_of)::value>), grid, block, 0, s, d);
        else hipLaunchKernelGGL((linear_direct_grad_kernel<T, 2, 2, decltype(slope)::value, decltype(few_of)::value>), grid, block, 0, s, d);
    };
    if (d.z && few) enqueue(std::true_type{}, std::true_type{});
    else if (d.z) enqueue(std::true_type{}, std::false_type{});
    else if (few) enqueue(std::false_type{}, std::true_type{});
    else enqueue(std::false_type{}, std::false_type{});
    e = (int)hipGetLastError();
    ProductArgs p{};
    if (e == 0 && px) {
        p.out = a.grad_x;
        p.partial = px;
        p.M = a.M;
        p.N = a.K;
        p.parts = l.parts_x;
        p.ldo = a.K;
        e = launch_join<T>(p, s);
    }
    if (e == 0 && pw) {
        p.out = a.grad_w;
        p.residual = a.accumulate ? a.grad_w : nullptr;
        p.partial = pw;
        p.M = a.N;
        p.N = a.K;
        p.parts = l.parts_w;
        p.ldo = p.ldr = a.K;
        e = launch_join<T>(p, s);
    }
    if (e == 0 && pb) e = launch_bias(pb, a.grad_bias, l.parts_w, a.N, a.accumulate, s);
    return e;
}

}  // namespace

long long linear_grad_workspace(const LinearGradArgs& a, int dtype) { return plan_of(a, dtype).end; }

namespace {

GradPlan plan_of(int dtype, int M, int N, int K, int act)
{
    LinearGradArgs a{};
    a.M = M;
    a.N = a.ldg = N;
    a.K = a.ldx = a.ldw = K;
    a.act = act;
    return plan_of(a, dtype);
}

}  // namespace

int linear_grad_kernel(int dtype, int M, int N, int K, int act)
{
    const GradPlan p = plan_of(dtype, M, N, K, act);
    return p.direct ? 101 + p.formed : 1000 * p.x.kernel + p.w.kernel;
}

int linear_grad_form(int dtype, int M, int N, int K, int act)
{
    const GradPlan p = plan_of(dtype, M, N, K, act);
    if (!p.direct) return 8 * (p.x.parts > 1) + 16 * (p.w.parts > 1);
    return p.small + 2 * few_of(dtype, std::min(N, K)) + 4 * (act != kNone && !p.formed) + 8 * (p.parts_x > 1) + 16 * (p.parts_w > 1);
}

int launch_linear_grad(int dtype, const LinearGradArgs& a, char* workspace, void* stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int b = bytes_of(dtype);
    if (a.M == 0) return launch_zeros(a.grad_w, (long long)a.N * a.K * b, a.grad_bias, a.N * 4ll, s);      // sums of nothing
    const GradPlan l = plan_of(a, dtype);
    if (l.direct)
        return dtype == kF32 ? launch_direct_grad<float>(l, a, workspace, s) : dtype == kF16 ? launch_direct_grad<_Float16>(l, a, workspace, s) : launch_direct_grad<__bf16>(l, a, workspace, s);
    const int k_pitch = (int)pitch_of(a.K, b), n_pitch = (int)pitch_of(a.N, b);
    int e = 0;
    const void *d = a.grad, *x = a.x, *w = a.w;
    int d_bytes = (int)(a.M > 1 ? a.ldg * b : n_pitch * b), x_bytes = (int)(a.M > 1 ? a.ldx * b : k_pitch * b), w_bytes = (int)(a.N > 1 ? a.ldw * b : k_pitch * b);
    const bool form = l.own_dz && (a.grad_x || a.grad_w);
    if (form || a.grad_bias) {
        e = launch_lay(dtype, LayArgs{a.grad, a.act != kNone ? a.z : nullptr, form ? workspace + l.dz : nullptr, a.grad_bias ? reinterpret_cast<float*>(workspace + l.sums) : nullptr,
                                      a.ldg, a.M, a.N, n_pitch, a.act}, s);
        if (e != 0) return e;
        if (form) {
            d = workspace + l.dz;
            d_bytes = n_pitch * b;
        }
    }
    if (a.grad_bias && (e = launch_bias(reinterpret_cast<const float*>(workspace + l.sums), a.grad_bias, (a.M + 63) / 64, a.N, a.accumulate, s)) != 0) return e;
    if (l.lay_x) {
        if ((e = launch_lay(dtype, LayArgs{a.x, nullptr, workspace + l.x_at, nullptr, a.ldx, a.M, a.K, k_pitch, kNone}, s)) != 0) return e;
        x = workspace + l.x_at;
        x_bytes = k_pitch * b;
    }
    if (l.lay_w) {
        if ((e = launch_lay(dtype, LayArgs{a.w, nullptr, workspace + l.w_at, nullptr, a.ldw, a.N, a.K, k_pitch, kNone}, s)) != 0) return e;
        w = workspace + l.w_at;
        w_bytes = k_pitch * b;
    }
    if (a.grad_x) {
        const ProductArgs p{d, w, nullptr, nullptr, a.grad_x, nullptr, nullptr, a.M, a.K, a.N, d_bytes, w_bytes, kNone, 0, 1, 0, a.K};
        if ((e = product(dtype, l.x, kTurnedW, p, workspace + l.partial, s)) != 0) return e;
    }
    if (a.grad_w) {
        const ProductArgs p{d, x, nullptr, a.accumulate ? a.grad_w : nullptr, a.grad_w, nullptr, nullptr, a.N, a.K, a.M, d_bytes, x_bytes, kNone, 0, 1, a.K, a.K};
        if ((e = product(dtype, l.w, kTurnedBoth, p, workspace + l.partial, s)) != 0) return e;
    }
    return 0;
}

}  // namespace sc

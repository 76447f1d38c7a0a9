// Fully connected layer with bias, activation and residual, and its gradients (sparse_conv_linear, sparse_conv_linear_backward).
//
// Every product here is out[m][n] = sum_k x[m][k] w[n][k] of two arrays whose rows lie along k, at multiples of 16 bytes.  What does
// not come like that (odd rows; the transposes that the gradients need) is laid out in scratch memory first.  Products of 16-bit
// numbers are summed in fp32 by the matrix cores, fp32 is multiplied in fp32.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "text_ops.h"
#include "tiles.h"

namespace sc {

namespace {

enum { kNone = 0, kRelu = 1, kGelu = 2, kSilu = 3 };   // SC_ACT_*

typedef float float4v __attribute__((ext_vector_type(4)));

// Elements of 16 bytes, as the matrix instructions take them.
template <class T>
using Eight = T __attribute__((ext_vector_type(16 / sizeof(T))));

// What a launch multiplies.  (Arguments past 112 bytes cost the host 0.75 us more.)
struct ProductArgs {
    const void *x, *w;              // rows of row_bytes bytes (a multiple of 16), x_pitch and w_pitch apart
    const float* bias;              // or null
    const void* residual;           // or null
    void *out, *z;                  // z: what goes into the activation, or null
    float* partial;                 // or null.  Else a part of k each: sums [part][M][N], and nothing of the above
    int M, N, row_bytes, x_pitch, w_pitch;
    int act;
    int steps;                      // of 128 bytes, a part
    int parts;
    long long ldr, ldo;             // elements; z has N
};

// ---------------------------------------------------------------- activations

__device__ __forceinline__ float activate(float z, int act)
{
    if (act == kRelu) return z < 0.f ? 0.f : z;
    if (act == kGelu) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    if (act == kSilu) return z / (1.f + __expf(-z));
    return z;
}

// The derivative.
__device__ __forceinline__ float slope(float z, int act)
{
    if (act == kRelu) return z > 0.f ? 1.f : z == z ? 0.f : z;
    if (act == kGelu) return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * __expf(-0.5f * z * z) * 0.39894228040143268f;
    if (act == kSilu) {
        const float s = 1.f / (1.f + __expf(-z));
        return s * (1.f + z * (1.f - s));
    }
    return 1.f;
}

// ---------------------------------------------------------------- products

// A piece of 16 bytes of x and of w: lane l holds k = its share l / 16 of row l % 16 of each, and rows 4 (l / 16) .. + 3 of w's 16 at
// column l % 16 (of x) of the sums.  fp32 pieces take four instructions, e = 0 .. 3.  The sums stay in accumulation registers.
template <class T>
constexpr int kSub = sizeof(T) == 4 ? 4 : 1;

template <class T, int e>
__device__ __forceinline__ void multiply(float4v& c, int4v w, int4v x)
{
    if constexpr (std::is_same<T, float>::value) asm volatile("v_mfma_f32_16x16x4_f32 %0, %1, %2, %0" : "+a"(c) : "v"(w[e]), "v"(x[e]));
    else if constexpr (std::is_same<T, _Float16>::value) asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(w), "v"(x));
    else asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(w), "v"(x));
}

// The same by the compiler's builtins, for kernels whose sums take few registers.
template <class T>
__device__ __forceinline__ float4v multiplied(float4v c, int4v w, int4v x)
{
    if constexpr (std::is_same<T, float>::value) {
        const float4v a = __builtin_bit_cast(float4v, w), b = __builtin_bit_cast(float4v, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    } else if constexpr (std::is_same<T, _Float16>::value) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Eight<_Float16>, w), __builtin_bit_cast(Eight<_Float16>, x), c, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Eight<__bf16>, w), __builtin_bit_cast(Eight<__bf16>, x), c, 0, 0, 0);
    }
}

// C sums of a row (n .. n + C - 1 of row m, of which `count` are there) to the output: bias, activation, residual, in fp32 and rounded once.
template <class T, int C>
__device__ __forceinline__ void finish(const ProductArgs& a, const float (&sum)[C], const float (&bias)[C], int m, int n, int count)
{
    typedef T V __attribute__((ext_vector_type(C), aligned(sizeof(T))));
    float v[C];
#pragma unroll
    for (int e = 0; e < C; ++e) v[e] = sum[e] + bias[e];
    auto store = [&](T* to) {
        V y;
#pragma unroll
        for (int e = 0; e < C; ++e) y[e] = (T)v[e];
        if (count >= C) *reinterpret_cast<V*>(to) = y;
        else
#pragma unroll
            for (int e = 0; e < C; ++e)
                if (e < count) to[e] = y[e];
    };
    if (a.z) store(static_cast<T*>(a.z) + (size_t)m * a.N + n);
    if (a.act != kNone)
#pragma unroll
        for (int e = 0; e < C; ++e) v[e] = activate(v[e], a.act);
    if (a.residual) {
        const T* from = static_cast<const T*>(a.residual) + (size_t)m * a.ldr + n;
        if (count >= C) {
            const V r = *reinterpret_cast<const V*>(from);
#pragma unroll
            for (int e = 0; e < C; ++e) v[e] += (float)r[e];
        } else {
#pragma unroll
            for (int e = 0; e < C; ++e)
                if (e < count) v[e] += (float)from[e];
        }
    }
    store(static_cast<T*>(a.out) + (size_t)m * a.ldo + n);
}

// A load of a piece that lies past the rows' end: an offset that no descriptor reaches (they describe 2^31 bytes at most).
__device__ __forceinline__ unsigned past(unsigned offset, unsigned beyond, int i) { return offset | ((beyond >> i) & 1u) << 31; }

// Large tiles: a workgroup has a CU to itself, so it walks over tiles, `stride` apart, and loads the next one's first steps before it
// finishes one.  (Three steps a tile at least: a barrier lies between what reads a tile's biases and what loads over them.)
template <int MB, int NB>
constexpr bool kWalksOver = MB * NB >= 64;
constexpr int kStepsToWalk = 3;

// A tile of 16 MB WM rows of x by 16 NB WN rows of w, 128 bytes of each a step; WM x WN wavefronts with MB x NB blocks of 16 x 16 sums.
// S steps are in LDS or on their way there.
template <class T, int MB, int NB, int WM, int WN, int S>
__global__ __launch_bounds__(64 * WM * WN, MB * NB >= 64 || S > 2 ? 1 : 2) void linear_tile_kernel(ProductArgs a, unsigned tiles, unsigned stride)
{
    constexpr int TM = 16 * MB * WM, TN = 16 * NB * WN, W = WM * WN;
    constexpr int kLoadsX = TM / 8 / W, kLoadsW = TN / 8 / W, kLoads = kLoadsX + kLoadsW;
    constexpr int kX = TM * 128, kW = TN * 128, kHalf = MB / 2;
    static_assert(MB % 2 == 0 && NB % 2 == 0, "blocks come in pairs");
    static_assert(TN % 64 == 0 && TN <= 64 * W, "a bias a thread");
    __shared__ __attribute__((aligned(256))) char lds[S * (kX + kW)];
    constexpr int kSets = kWalksOver<MB, NB> ? 2 : 1;      // the tile that is finished, and the next one
    __shared__ __attribute__((aligned(16))) float channel_bias[kSets][TN];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int down = (a.M + TM - 1) / TM, across = (a.N + TN - 1) / TN, steps = a.steps, all_steps = (a.row_bytes + 127) / 128;
    // A row of LDS is the 128 bytes of a row's step; its eight pieces of 16 bytes are permuted by the row, so that the 16 rows that a
    // read takes one piece of lie in 16 different groups of four banks.  A lane's load fetches the piece that belongs where it lands.
    unsigned offset[kLoads], behind = 0;      // behind: bit i, load i's piece of the last step lies past the end of its row
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int row = (wave * (i < kLoadsX ? kLoadsX : kLoadsW) + (i < kLoadsX ? i : i - kLoadsX)) * 8 + (lane >> 3);
        const int turn = i < kLoadsX ? (row >> 1) & 7 : ((row >> 1) & 1) | ((row >> 3) & 3) << 1;
        const int piece = ((lane & 7) ^ turn) << 4;
        offset[i] = (unsigned)row * (i < kLoadsX ? a.x_pitch : a.w_pitch) + piece;
        if ((all_steps - 1) * 128 + piece >= a.row_bytes) behind |= 1u << i;
    }
    const unsigned lds0 = (unsigned)(uintptr_t)(SC_LDS char*)lds;
    int4v from_x, from_w;
    int bytes_x = 0, bytes_w = 0;
    unsigned xdst = lds0, wdst = lds0 + S * kX, tile = blockIdx.x, beyond = 0;
    int next_m = 0, next_n = 0, next_part = 0, step = 0, end = 0, set = 0;      // what is loaded: a step of a tile, whose biases go to `set`
    unsigned at = 0;                                                            // where it begins in its rows
    auto enter = [&]() {
        int tm, tn;
        tile_of(tile, tiles, down * a.parts, across, tm, tn);      // (the parts of a tile as further tiles below it)
        next_part = tm / down;
        next_m = (tm - next_part * down) * TM;
        next_n = tn * TN;
        step = next_part * steps;
        end = step + steps;
        from_x = descriptor_of(static_cast<const char*>(a.x) + (size_t)next_m * a.x_pitch, (long long)min(TM, a.M - next_m) * a.x_pitch);
        from_w = descriptor_of(static_cast<const char*>(a.w) + (size_t)next_n * a.w_pitch, (long long)min(TN, a.N - next_n) * a.w_pitch);
        bytes_x = from_x[2];
        bytes_w = from_w[2];
        if (wave * 64 < TN) {
            if (a.bias)
                load_word_to_lds(descriptor_of(a.bias + next_n, min(TN, a.N - next_n) * 4ll), threadIdx.x * 4,
                                 (unsigned)(uintptr_t)(SC_LDS float*)channel_bias[set] + wave * 256);
            else channel_bias[set][threadIdx.x] = 0.f;
        }
    };
    // (Each of these scalars is set in one place: with a branch for each reason to fetch nothing the compiler lost the descriptors' zeros.)
    auto advance = [&]() {
        if (++step == end) {
            tile += stride;
            if (kWalksOver<MB, NB> && tile < tiles) {
                set ^= 1;
                enter();
            }
        }
        const bool there = step < min(end, all_steps);      // else zeros: past the last tile, or past the rows (in the last part)
        from_x[2] = there ? bytes_x : 0;
        from_w[2] = there ? bytes_w : 0;
        at = there ? step * 128 : 0;
        beyond = step == all_steps - 1 ? behind : 0;
    };
    auto load = [&](int i) {
        if (i < kLoadsX) load_to_lds(from_x, past(offset[i], beyond, i), at, xdst + (wave * kLoadsX + i) * 1024);
        else load_to_lds(from_w, past(offset[i], beyond, i), at, wdst + (wave * kLoadsW + i - kLoadsX) * 1024);
    };
    enter();
    at = step * 128;
    beyond = step == all_steps - 1 ? behind : 0;
    int m0 = next_m, n0 = next_n, part = next_part, done = set;
    each<S>([&](auto stage) {
        if constexpr (stage > 0) advance();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load(i);
        xdst += kX;
        wdst += kW;
    });
    xdst -= S * kX;
    wdst -= S * kW;

    float4v acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};
            asm volatile("" : "+a"(acc[i][j]));
        }

    // Where a lane reads: its row of block 0 and its piece; the second 64 bytes of a step are four pieces on (an exclusive or).
    // Row r of a wavefront's block j of w stands for channel 32 (j / 2) + 8 (r / 4) + 4 (j % 2) + r % 4, so that a lane's sums of
    // two blocks are eight channels in a row.
    const int wm = wave % WM, wn = wave / WM, r = lane & 15, q = lane >> 4;
    int xa0 = (wm * 16 * MB + r) * 128 + ((q ^ (r >> 1)) << 4), xa1 = xa0 ^ 64;
    int wa0 = S * kX + (wn * 16 * NB + (r >> 2) * 8 + (r & 3)) * 128 + ((q ^ (r >> 1)) << 4), wa1 = wa0 ^ 64;
    int4v wf[2][NB], xf[2][MB];
    auto read_w = [&](int h, int j) { wf[h][j] = *reinterpret_cast<const int4v*>(lds + (h ? wa1 : wa0) + ((j >> 1) * 32 + (j & 1) * 4) * 128); };
    auto read_x = [&](int h, int i) { xf[h][i] = *reinterpret_cast<const int4v*>(lds + (h ? xa1 : xa0) + i * 2048); };
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"((S - 1) * kLoads) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int j = 0; j < NB; ++j) read_w(0, j);
#pragma unroll
    for (int i = 0; i < kHalf; ++i) read_x(0, i);
    __builtin_amdgcn_sched_barrier(0);

    // A step is two halves of MB x NB products, 64 bytes each.  In the first, all that the second needs is read, one read every few
    // products (a wavefront is alone on its SIMD and issues in order: reads or loads in a row leave the matrix unit without work).
    // Then nothing reads this buffer any more and, spread over the second half, it is loaded with the bytes of the step that is S on.
    // Halfway through, those of the next step (loaded S - 1 steps before) are waited for, and the first half's operands are read.
    int buffer = 0;
    for (unsigned current = blockIdx.x; current < tiles; current += stride) {
        for (int k = 0; k < steps; ++k) {
            advance();
            const int dx = buffer == S - 1 ? (1 - S) * kX : kX, dw = buffer == S - 1 ? (1 - S) * kW : kW;      // to the next step's buffer
            buffer = buffer == S - 1 ? 0 : buffer + 1;
            constexpr int kBlocks = MB * NB, kSlots = kBlocks * kSub<T>, kTurn = kSlots / 2;
            each<kSlots>([&](auto slot) {
                constexpr int t = slot, i = t % kBlocks / NB, j = t % NB, kOps = kHalf + NB + MB;
                multiply<T, t / kBlocks>(acc[i][j], wf[0][j], xf[0][i]);
                if constexpr (t < kBlocks) {
                    constexpr int first = (t * kOps + kBlocks - 1) / kBlocks, last = ((t + 1) * kOps + kBlocks - 1) / kBlocks;
                    each<last - first>([&](auto n) {
                        constexpr int o = first + n;
                        if constexpr (o < 2 * kHalf && o % 2 == 0) read_x(0, kHalf + o / 2);
                        else {
                            constexpr int u = o < 2 * kHalf ? o / 2 : o - kHalf;
                            if constexpr (u < NB) read_w(1, u);
                            else read_x(1, u - NB);
                        }
                    });
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            each<kSlots>([&](auto slot) {
                constexpr int t = slot, i = t % kBlocks / NB, j = t % NB;
                if constexpr (t == kTurn) {
                    constexpr int kIssued = (kTurn * kLoads + kSlots - 1) / kSlots;
                    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(kIssued + (S - 2) * kLoads) : "memory");
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    xa0 += dx;
                    xa1 += dx;
                    wa0 += dw;
                    wa1 += dw;
                    __builtin_amdgcn_sched_barrier(0);
                }
                multiply<T, t / kBlocks>(acc[i][j], wf[1][j], xf[1][i]);
                constexpr int first = (t * kLoads + kSlots - 1) / kSlots, last = ((t + 1) * kLoads + kSlots - 1) / kSlots;
                each<last - first>([&](auto n) { load(first + n); });
                if constexpr (t >= kTurn) {
                    constexpr int kReads = NB + kHalf, kRoom = kSlots - kTurn, v = t - kTurn;
                    constexpr int from = (v * kReads + kRoom - 1) / kRoom, to = ((v + 1) * kReads + kRoom - 1) / kRoom;
                    each<to - from>([&](auto n) {
                        constexpr int o = from + n;
                        if constexpr (o < NB) read_w(0, o);
                        else read_x(0, o - NB);
                    });
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            xdst += dx;
            wdst += dw;
        }

        // Bias, activation and residual, while the first steps of the next tile are on their way.  The last products are read: the matrix
        // unit's results need 18 clocks.
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
        each<NB / 2>([&](auto pair) {
            constexpr int j = 2 * pair;
            const int tile_n = wn * 16 * NB + j * 16 + q * 8, n = n0 + tile_n;
            float bias[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) bias[e] = channel_bias[done][tile_n + e];
            each<MB>([&](auto block) {
                constexpr int i = block;
                const int m = m0 + (wm * MB + i) * 16 + r;
                asm volatile("" : "+a"(acc[i][j]), "+a"(acc[i][j + 1]));
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = acc[i][j + e / 4][e % 4];
                acc[i][j] = acc[i][j + 1] = float4v{0.f, 0.f, 0.f, 0.f};
                if (m >= a.M || n >= a.N) return;
                if (a.partial) {
                    float* to = a.partial + ((size_t)part * a.M + m) * a.N + n;
                    typedef float four __attribute__((ext_vector_type(4), aligned(4)));
                    if (n + 8 <= a.N) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) reinterpret_cast<four*>(to)[c] = four{v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]};
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (n + e < a.N) to[e] = v[e];
                    }
                } else {
                    finish<T, 8>(a, v, bias, m, n, a.N - n);
                }
            });
        });
        if (!kWalksOver<MB, NB>) break;
        m0 = next_m;
        n0 = next_n;
        part = next_part;
        done = set;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (loads of zeros that nothing reads)
}

// Few rows of x: 16 MB of them by 16 NB rows of w a workgroup, whose W wavefronts go round the 128-byte units of the rows and add their
// sums up at the end.  A wavefront loads its units to a part of LDS of its own, D of them in flight, and waits for its own loads alone.
// (Loads in the order that the products take would touch 16 rows with 16 lanes in a row, at a quarter of the rate.)
template <class T, int MB, int NB, int W, int D>
__global__ __launch_bounds__(64 * W) void linear_row_kernel(ProductArgs a)
{
    constexpr int kTokens = 16 * MB, kChannels = 16 * NB, kThreads = 64 * W;
    constexpr int kLoadsX = 2 * MB, kLoads = kLoadsX + 2 * NB, kUnit = 1024 * kLoads;
    static_assert(D * kUnit >= kTokens * kChannels * 4, "the sums take the place of the units");
    __shared__ __attribute__((aligned(256))) char lds[W * D * kUnit];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, q = lane >> 4;
    const int across = (a.N + kChannels - 1) / kChannels;
    const int m0 = (int)(blockIdx.x / across) * kTokens, n0 = (int)(blockIdx.x % across) * kChannels;
    const int units = (a.row_bytes + 127) / 128;

    // Pieces of 16 bytes are permuted within the 128 bytes of a row as in the tile kernel.
    int4v from_w = descriptor_of(static_cast<const char*>(a.w) + (size_t)n0 * a.w_pitch, (long long)min(kChannels, a.N - n0) * a.w_pitch);
    int4v from_x = descriptor_of(static_cast<const char*>(a.x) + (size_t)m0 * a.x_pitch, (long long)min(kTokens, a.M - m0) * a.x_pitch);
    const int bytes_w = from_w[2], bytes_x = from_x[2];
    const unsigned lds0 = (unsigned)(uintptr_t)(SC_LDS char*)lds + wave * D * kUnit;
    unsigned row[2], piece_of[2], behind = 0;      // of the rows lane / 8 of an even and an odd load: their permutations differ
#pragma unroll
    for (int o = 0; o < 2; ++o) {
        row[o] = (unsigned)(o * 8 + (lane >> 3));
        piece_of[o] = ((lane & 7) ^ ((o * 4 + (lane >> 4)) & 7)) << 4;
        if ((units - 1) * 128 + (int)piece_of[o] >= a.row_bytes) behind |= 1u << o;
    }
    auto load = [&](int slot, int unit) {
        from_w[2] = unit < units ? bytes_w : 0;
        from_x[2] = unit < units ? bytes_x : 0;
        const unsigned beyond = unit == units - 1 ? behind : 0, at = unit < units ? unit * 128u : 0u;
        each<kLoads>([&](auto load) {
            constexpr int l = load, block = l < kLoadsX ? l / 2 : (l - kLoadsX) / 2;
            const unsigned pitch = l < kLoadsX ? a.x_pitch : a.w_pitch;
            load_to_lds(l < kLoadsX ? from_x : from_w, past((row[l & 1] + block * 16u) * pitch + piece_of[l & 1], beyond, l & 1), at,
                        lds0 + slot * kUnit + l * 1024);
        });
    };
    each<D>([&](auto d) { load(d, wave + d * W); });

    float4v acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};
    const char* mine = lds + wave * D * kUnit + r * 128;
    const int piece[2] = {(q ^ (r >> 1)) << 4, ((q + 4) ^ (r >> 1)) << 4};
    int slot = 0;
    for (int unit = wave; unit < units; unit += W) {
        asm volatile("s_waitcnt vmcnt(%0)" :: "n"((D - 1) * kLoads) : "memory");
        const char* from = mine + slot * kUnit;
        int4v wf[2][NB], xf[2][MB];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < MB; ++i) xf[h][i] = *reinterpret_cast<const int4v*>(from + i * 2048 + piece[h]);
#pragma unroll
            for (int j = 0; j < NB; ++j) wf[h][j] = *reinterpret_cast<const int4v*>(from + kLoadsX * 1024 + j * 2048 + piece[h]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        load(slot, unit + D * W);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = multiplied<T>(acc[i][j], wf[h][j], xf[h][i]);
        slot = slot + 1 == D ? 0 : slot + 1;
    }

    // Sums of each wavefront where its units were: [token][channel].
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
            *reinterpret_cast<float4v*>(lds + wave * D * kUnit + ((i * 16 + r) * kChannels + j * 16 + q * 4) * 4) = acc[i][j];
    __syncthreads();
    for (int o = threadIdx.x; o < kTokens * kChannels / 4; o += kThreads) {
        const int token = o / (kChannels / 4), channel = o % (kChannels / 4) * 4, m = m0 + token, n = n0 + channel;
        if (m >= a.M || n >= a.N) continue;
        float4v total = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < W; ++w) total += *reinterpret_cast<const float4v*>(lds + w * D * kUnit + o * 16);
        float sum[4], bias[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sum[e] = total[e];
            bias[e] = a.bias && n + e < a.N ? a.bias[n + e] : 0.f;
        }
        finish<T, 4>(a, sum, bias, m, n, a.N - n);
    }
}

// The parts of a product added up, in their order, then as in the kernels above.  Four outputs of a row a thread.
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

// ---------------------------------------------------------------- which kernel

double pieces_of(int n, int size) { return (double)((n + size - 1) / size); }

// Microseconds that a product of rows of `bytes` is estimated to take: a row kernel by what its workgroups load, a tile kernel by its
// steps.  f: clocks of the matrix unit that a piece of 16 bytes takes, over those of 16-bit types.
enum Kernel { kRow11, kRow21, kRow22, kRow41, kRow42, kTile22, kTile44, kTile88, kDeep22, kDeep42, kDeep44, kKernels };

struct RowRule {
    int MB, NB;
    double join, more, all, one, weights;      // us; MB/us of all workgroups, KB/us of one, MB/us of w
};
constexpr RowRule kRowRules[] = {{1, 1, 0.36, 1.39, 21.1, 144.0, 7.2}, {2, 1, 0.24, 1.42, 22.5, 135.0, 6.0}, {2, 2, 0.12, 0.83, 19.2, 136.0, 5.6},
                                 {4, 1, 0.33, 1.54, 24.6, 133.0, 4.75}, {4, 2, 0.91, 1.64, 19.8, 132.0, 5.05}};

double row_estimate(const RowRule& r, int M, int N, double bytes, double f)
{
    const double groups = pieces_of(M, 16 * r.MB) * pieces_of(N, 16 * r.NB), loaded = 16.0 * (r.MB + r.NB) * bytes;
    const double on_a_cu = std::ceil(groups / 256.0);
    const double load = std::max({groups * loaded / (r.all * 1e6), on_a_cu * loaded / (r.one * 1e3), (double)N * bytes / (r.weights * 1e6)});
    const double multiply = on_a_cu * r.MB * r.NB * (bytes / 64.0) * f * 16.0 / 4.0 / 2000.0;
    return 3.0 + r.join * on_a_cu + r.more * (on_a_cu - 1.0) + std::max(load, multiply);
}

struct TileRule {
    int MB, NB, share;
    double least, each, start, finish, weights;
};
constexpr TileRule kTileRules[] = {{2, 2, 4, 0.268, 0.213, 0.28, 2.35, 3.5}, {4, 4, 2, 0.063, 0.446, 0.40, 4.07, 3.2}, {8, 8, 1, 0.0, 1.16, 2.66, 9.15, 6.7},
                                   {2, 2, 2, 0.049, 0.194, 1.20, 1.90, 7.0}, {4, 2, 1, 0.0, 0.271, 1.12, 2.48, 6.6}, {4, 4, 1, 0.0, 0.396, 0.99, 3.39, 4.7}};

double tile_estimate(const TileRule& r, int M, int N, int parts, double bytes, double f)
{
    const double groups = pieces_of(M, 32 * r.MB) * pieces_of(N, 32 * r.NB) * parts, steps = std::ceil(bytes / 128.0 / parts), held = 256.0 * r.share;
    const double rounds = std::floor(groups / held), rest = groups - rounds * held, each = f > 1.0 ? std::max(r.each, 2.0 * r.MB * r.NB * f * 16.0 / 2100.0) : r.each;
    double us = r.start + rounds * (steps * each * r.share + r.finish);
    if (rest > 0.0) us += steps * std::max(r.least, each * std::ceil(rest / 256.0)) + r.finish;
    us = std::max(us, 3.0 + (double)N * bytes / (r.weights * 1e6));
    return parts > 1 ? us + 3.0 + 4.0 * M * (double)N * (parts + 1) / 4e6 : us;
}

struct Choice {
    Kernel kernel;
    int parts, steps;
};

Choice choose(int dtype, int M, int N, int row_bytes)
{
    const double f = dtype == kF32 ? 8.0 : 1.0, bytes = row_bytes;
    const int all = (row_bytes + 127) / 128;
    Choice best{kRow11, 1, all};
    double least = 0.0;
    for (int k = 0; k < kKernels; ++k) {
        if (k == kTile88 && dtype == kF32) continue;
        for (int parts = 1; parts <= (k < kTile22 ? 1 : 64); parts *= 2) {
            const int steps = (all + parts - 1) / parts;
            if (parts > 1 && steps < 8) break;
            if (k == kTile88 && steps < kStepsToWalk) break;
            const double us = k < kTile22 ? row_estimate(kRowRules[k], M, N, bytes, f) : tile_estimate(kTileRules[k - kTile22], M, N, parts, bytes, f);
            if ((k == 0 && parts == 1) || us < least) {
                best = Choice{(Kernel)k, (all + steps - 1) / steps, steps};
                least = us;
            }
        }
    }
    return best;
}

template <class T, int MB, int NB, int S>
int launch_tile(const ProductArgs& a, hipStream_t s)
{
    const long long tiles = (long long)a.parts * ((a.M + 32ll * MB - 1) / (32 * MB)) * ((a.N + 32ll * NB - 1) / (32 * NB));
    const bool walks = kWalksOver<MB, NB> && a.steps >= kStepsToWalk;
    if (tiles >= (1ll << 31) || (!walks && (unsigned long long)tiles > most_groups(256))) return kTooLarge;
    const unsigned blocks = walks ? (unsigned)std::min(tiles, 256ll) : (unsigned)tiles;
    hipLaunchKernelGGL((linear_tile_kernel<T, MB, NB, 2, 2, S>), dim3(blocks), dim3(256), 0, s, a, (unsigned)tiles, blocks);
    return (int)hipGetLastError();
}

template <class T, int MB, int NB, int W, int D>
int launch_row(const ProductArgs& a, hipStream_t s)
{
    const long long groups = ((a.M + 16ll * MB - 1) / (16 * MB)) * ((a.N + 16ll * NB - 1) / (16 * NB));
    if ((unsigned long long)groups > most_groups(64 * W)) return kTooLarge;
    hipLaunchKernelGGL((linear_row_kernel<T, MB, NB, W, D>), dim3((unsigned)groups), dim3(64 * W), 0, s, a);
    return (int)hipGetLastError();
}

template <class T>
int launch_kernel(Kernel kernel, const ProductArgs& a, hipStream_t s)
{
    switch (kernel) {
        case kRow11: return launch_row<T, 1, 1, 8, 4>(a, s);
        case kRow21: return launch_row<T, 2, 1, 8, 2>(a, s);
        case kRow22: return launch_row<T, 2, 2, 4, 2>(a, s);
        case kRow41: return launch_row<T, 4, 1, 8, 1>(a, s);
        case kRow42: return launch_row<T, 4, 2, 4, 2>(a, s);
        case kTile22: return launch_tile<T, 2, 2, 2>(a, s);
        case kTile44: return launch_tile<T, 4, 4, 2>(a, s);
        case kTile88:
            if constexpr (sizeof(T) == 2) return launch_tile<T, 8, 8, 2>(a, s);
            return kTooLarge;      // (never chosen)
        case kDeep22: return launch_tile<T, 2, 2, 4>(a, s);
        case kDeep42: return launch_tile<T, 4, 2, 4>(a, s);
        default: return launch_tile<T, 4, 4, 3>(a, s);
    }
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

long long partial_bytes(int dtype, int M, int N, int row_bytes)
{
    const Choice c = choose(dtype, M, N, row_bytes);
    return c.parts > 1 ? round_up(4ll * c.parts * M * N, 256) : 0;
}

// The product of rows that are laid out; partial: scratch memory of partial_bytes.
int product(int dtype, ProductArgs a, char* partial, hipStream_t s)
{
    const Choice c = choose(dtype, a.M, a.N, a.row_bytes);
    a.parts = c.parts;
    a.steps = c.steps;
    a.partial = c.parts > 1 ? reinterpret_cast<float*>(partial) : nullptr;
    int e = dtype == kF32 ? launch_kernel<float>(c.kernel, a, s) : dtype == kF16 ? launch_kernel<_Float16>(c.kernel, a, s) : launch_kernel<__bf16>(c.kernel, a, s);
    if (e != 0 || c.parts == 1) return e;
    return dtype == kF32 ? launch_join<float>(a, s) : dtype == kF16 ? launch_join<_Float16>(a, s) : launch_join<__bf16>(a, s);
}

// ---------------------------------------------------------------- rows laid out

// Tiles of 64 x 64 elements of [rows][cols] (ld elements from one row to the next), each of: `copy`, rows of copy_pitch elements as they
// are; `turned`, columns as rows of turned_pitch elements; both with zeros up to the pitch.  With an activation the elements are first
// multiplied by its derivative at z, in fp32, and rounded once; column_sums [tiles down][cols] receives the sums over the
// tile's rows of what was not rounded.
struct LayArgs {
    const void *from, *z;
    void *copy, *turned;
    float* column_sums;
    long long ld;
    int rows, cols, copy_pitch, turned_pitch, act;
};

template <class T>
__global__ __launch_bounds__(256) void linear_lay_kernel(LayArgs a)
{
    constexpr int kCount = 16 / sizeof(T), kPer = 64 / kCount, kTurns = 64 * kPer / 256;      // pieces a row of the tile; a thread's pieces
    typedef typename Piece<T>::type V;
    typedef T A __attribute__((ext_vector_type(16 / sizeof(T))));
    constexpr int kPitch = 64 + 16 / sizeof(T) / 2 + 1;
    __shared__ T tile[64][kPitch];
    __shared__ float sums[256 / kPer][64];
    const int across = (a.cols + 63) / 64, tr = (int)(blockIdx.x / (unsigned)across), tc = (int)(blockIdx.x % (unsigned)across);
    const int piece = threadIdx.x % kPer, first = threadIdx.x / kPer, col = tc * 64 + piece * kCount;
    float total[kCount] = {};
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        const int in = first + t * (256 / kPer), row = tr * 64 + in;
        V v;
#pragma unroll
        for (int e = 0; e < kCount; ++e) v[e] = (T)0.f;
        if (row < a.rows && col < a.cols) {
            v = load_piece<T>(static_cast<const T*>(a.from) + (size_t)row * a.ld, col, a.cols);
            float g[kCount];
#pragma unroll
            for (int e = 0; e < kCount; ++e) g[e] = (float)v[e];
            if (a.z) {
                const V z = load_piece<T>(static_cast<const T*>(a.z) + (size_t)row * a.cols, col, a.cols);
#pragma unroll
                for (int e = 0; e < kCount; ++e) {
                    g[e] = col + e < a.cols ? g[e] * slope((float)z[e], a.act) : 0.f;
                    v[e] = (T)g[e];
                }
            }
#pragma unroll
            for (int e = 0; e < kCount; ++e) total[e] += g[e];
        }
        if (a.copy && row < a.rows && col < a.copy_pitch) *reinterpret_cast<A*>(static_cast<T*>(a.copy) + (size_t)row * a.copy_pitch + col) = v;
        if (a.turned)
#pragma unroll
            for (int e = 0; e < kCount; ++e) tile[in][piece * kCount + e] = v[e];
    }
    if (a.column_sums)
#pragma unroll
        for (int e = 0; e < kCount; ++e) sums[first][piece * kCount + e] = total[e];
    __syncthreads();
    if (a.column_sums && threadIdx.x < 64 && tc * 64 + (int)threadIdx.x < a.cols) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 256 / kPer; ++i) s += sums[i][threadIdx.x];
        a.column_sums[(size_t)tr * a.cols + tc * 64 + threadIdx.x] = s;
    }
    if (!a.turned) return;
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        const int in = first + t * (256 / kPer), to = tc * 64 + in, at = tr * 64 + piece * kCount;
        if (to >= a.cols || at >= a.turned_pitch) continue;
        A v;
#pragma unroll
        for (int e = 0; e < kCount; ++e) v[e] = tile[piece * kCount + e][in];
        *reinterpret_cast<A*>(static_cast<T*>(a.turned) + (size_t)to * a.turned_pitch + at) = v;
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

int launch_lay(int dtype, const LayArgs& a, hipStream_t s)
{
    const long long groups = ((a.rows + 63ll) / 64) * ((a.cols + 63ll) / 64);
    if ((unsigned long long)groups > most_groups(256)) return kTooLarge;
    const dim3 grid((unsigned)groups), block(256);
    if (dtype == kF32) hipLaunchKernelGGL(linear_lay_kernel<float>, grid, block, 0, s, a);
    else if (dtype == kF16) hipLaunchKernelGGL(linear_lay_kernel<_Float16>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(linear_lay_kernel<__bf16>, grid, block, 0, s, a);
    return (int)hipGetLastError();
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

}  // namespace

long long linear_workspace(const LinearArgs& a, int dtype)
{
    const int b = bytes_of(dtype);
    long long bytes = 0;
    if (!laid_out(a.x, a.ldx, a.M, a.K, b)) bytes += laid_bytes(a.M, a.K, b);
    if (!laid_out(a.w, a.ldw, a.N, a.K, b)) bytes += laid_bytes(a.N, a.K, b);
    return bytes + partial_bytes(dtype, a.M, a.N, (int)pitch_of(a.K, b) * b);
}

int launch_linear(int dtype, const LinearArgs& a, char* workspace, void* stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int b = bytes_of(dtype), row_bytes = (int)pitch_of(a.K, b) * b;
    ProductArgs p{a.x, a.w, a.bias, a.residual, a.out, a.z, nullptr, a.M, a.N, row_bytes, (int)(a.M > 1 ? a.ldx * b : row_bytes), (int)(a.N > 1 ? a.ldw * b : row_bytes),
                  a.act, 0, 1, a.ldr, a.ldo};
    if (!laid_out(a.x, a.ldx, a.M, a.K, b)) {
        const int e = launch_lay(dtype, LayArgs{a.x, nullptr, workspace, nullptr, nullptr, a.ldx, a.M, a.K, row_bytes / b, 0, 0}, s);
        if (e != 0) return e;
        p.x = workspace;
        p.x_pitch = row_bytes;
        workspace += laid_bytes(a.M, a.K, b);
    }
    if (!laid_out(a.w, a.ldw, a.N, a.K, b)) {
        const int e = launch_lay(dtype, LayArgs{a.w, nullptr, workspace, nullptr, nullptr, a.ldw, a.N, a.K, row_bytes / b, 0, 0}, s);
        if (e != 0) return e;
        p.w = workspace;
        p.w_pitch = row_bytes;
        workspace += laid_bytes(a.N, a.K, b);
    }
    return product(dtype, p, workspace, s);
}

namespace {

// Where the pieces of a backward pass lie in its scratch memory.
struct GradLayout {
    bool own_dz;                                             // the gradient behind the activation is formed (else grad is it)
    long long dz, dz_turned, x_turned, w_turned, sums, partial, end;
};

GradLayout layout_of(const LinearGradArgs& a, int dtype)
{
    const int b = bytes_of(dtype);
    GradLayout l{};
    l.own_dz = a.act != kNone || !laid_out(a.grad, a.ldg, a.M, a.N, b);
    long long at = 0;
    auto take = [&](bool wanted, long long bytes) {
        const long long here = at;
        if (wanted) at += round_up(bytes, 256);
        return here;
    };
    l.dz = take(a.grad_x && l.own_dz, laid_bytes(a.M, a.N, b));
    l.dz_turned = take(a.grad_w, laid_bytes(a.N, a.M, b));
    l.x_turned = take(a.grad_w, laid_bytes(a.K, a.M, b));
    l.w_turned = take(a.grad_x, laid_bytes(a.K, a.N, b));
    l.sums = take(a.grad_bias, (a.M + 63ll) / 64 * a.N * 4);
    const long long px = a.grad_x ? partial_bytes(dtype, a.M, a.K, (int)pitch_of(a.N, b) * b) : 0;
    const long long pw = a.grad_w ? partial_bytes(dtype, a.N, a.K, (int)pitch_of(a.M, b) * b) : 0;
    l.partial = take(true, std::max(px, pw));
    l.end = at;
    return l;
}

}  // namespace

long long linear_grad_workspace(const LinearGradArgs& a, int dtype) { return layout_of(a, dtype).end; }

int launch_linear_grad(int dtype, const LinearGradArgs& a, char* workspace, void* stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int b = bytes_of(dtype);
    if (a.M == 0) {      // sums of nothing
        return launch_zeros(a.grad_w, (long long)a.N * a.K * b, a.grad_bias, a.N * 4ll, s);
    }
    const GradLayout l = layout_of(a, dtype);
    const int m_pitch = (int)pitch_of(a.M, b), n_pitch = (int)pitch_of(a.N, b);
    int e = 0;
    if ((a.grad_x && l.own_dz) || a.grad_w || a.grad_bias) {
        e = launch_lay(dtype, LayArgs{a.grad, a.act != kNone ? a.z : nullptr, a.grad_x && l.own_dz ? workspace + l.dz : nullptr, a.grad_w ? workspace + l.dz_turned : nullptr,
                                      a.grad_bias ? reinterpret_cast<float*>(workspace + l.sums) : nullptr, a.ldg, a.M, a.N, n_pitch, m_pitch, a.act}, s);
        if (e != 0) return e;
    }
    if (a.grad_bias) {
        hipLaunchKernelGGL(linear_bias_kernel, dim3((unsigned)((a.N + 15) / 16)), dim3(256), 0, s, reinterpret_cast<const float*>(workspace + l.sums), a.grad_bias,
                           (a.M + 63) / 64, a.N, (int)a.accumulate);
        if ((e = (int)hipGetLastError()) != 0) return e;
    }
    if (a.grad_x) {
        e = launch_lay(dtype, LayArgs{a.w, nullptr, nullptr, workspace + l.w_turned, nullptr, a.ldw, a.N, a.K, 0, n_pitch, 0}, s);
        if (e != 0) return e;
        const ProductArgs p{l.own_dz ? workspace + l.dz : a.grad, workspace + l.w_turned, nullptr, nullptr, a.grad_x, nullptr, nullptr, a.M, a.K, n_pitch * b,
                            l.own_dz || a.M == 1 ? n_pitch * b : (int)(a.ldg * b), n_pitch * b, kNone, 0, 1, 0, a.K};
        if ((e = product(dtype, p, workspace + l.partial, s)) != 0) return e;
    }
    if (a.grad_w) {
        e = launch_lay(dtype, LayArgs{a.x, nullptr, nullptr, workspace + l.x_turned, nullptr, a.ldx, a.M, a.K, 0, m_pitch, 0}, s);
        if (e != 0) return e;
        const ProductArgs p{workspace + l.dz_turned, workspace + l.x_turned, nullptr, a.accumulate ? a.grad_w : nullptr, a.grad_w, nullptr, nullptr, a.N, a.K, m_pitch * b,
                            m_pitch * b, m_pitch * b, kNone, 0, 1, a.K, a.K};
        if ((e = product(dtype, p, workspace + l.partial, s)) != 0) return e;
    }
    return 0;
}

}  // namespace sc

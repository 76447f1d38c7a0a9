// Products of operands that are laid out: rows along the sum at multiples of 16 bytes, or such rows the other way round ("turned").  One source
// for each type includes this.
#pragma once

#include <algorithm>

#include "linear.h"

namespace sc {

namespace {

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

template <class T>
__device__ __forceinline__ int bytes_of_rows(int terms) { return (terms * (int)sizeof(T) + 15) / 16 * 16; }

// A load of a piece that lies past the rows' end: an offset that no descriptor reaches (they describe 2^31 bytes at most).
__device__ __forceinline__ unsigned past(unsigned offset, unsigned beyond, int i) { return offset | ((beyond >> i) & 1u) << 31; }

// Large tiles: a workgroup has a CU to itself, so it walks over tiles, `stride` apart, and loads the next one's first steps before it
// finishes one.  (Three steps a tile at least: a barrier lies between what reads a tile's biases and what loads over them.)
template <int MB, int NB>
constexpr bool kWalksOver = MB * NB >= 64;

// A tile of 16 MB WM rows of x by 16 NB WN rows of w, 128 bytes of each a step; WM x WN wavefronts with MB x NB blocks of 16 x 16 sums.
// S steps are in LDS or on their way there.  kTurnX, kTurnW: that operand is given the other way round, element (i, c) at c * pitch + i, as the
// gradients need it: its step is a part of 128 / sizeof(T) such rows, which lie in LDS as they do in memory and are turned as they are read.
// The matrix cores bound it: 550 GFLOP of bfloat16, 8192 x 4096 -> 8192, take 391 us a gradient (1.41 PFLOP/s; the largest tiles, 256 x 256 of four
// wavefronts, which read 1 / 64 of a byte from L2 a product) and 450 as a layer that applies gelu and keeps z, about
// 17 more vector instructions an output, which nothing hides with one wavefront a SIMD.  (Counted: the matrix cores are busy in 70 and 59 % of the CUs' clocks, at 2.0 GHz;
// no bank conflicts.)
// (Instructions of 32 x 32 sums took as long there, where power bounds it, and made the compiler move sums.  Loads of a step all in its third quarter: slower.)
template <class T, int MB, int NB, int WM, int WN, int S, bool kTurnX, bool kTurnW>
__global__ __launch_bounds__(64 * WM * WN, MB * NB >= 64 || S > 2 ? 1 : 2) void linear_tile_kernel(ProductArgs a, unsigned tiles, unsigned stride)
{
    constexpr int TM = 16 * MB * WM, TN = 16 * NB * WN, W = WM * WN, kC = 128 / sizeof(T);
    constexpr int kLoadsX = TM / 8 / W, kLoadsW = TN / 8 / W, kLoads = kLoadsX + kLoadsW;
    constexpr int kX = TM * 128, kW = TN * 128, kHalf = MB / 2;
    static_assert(MB % 2 == 0 && NB % 2 == 0, "blocks come in pairs");
    static_assert(TN % 64 == 0 && TN <= 64 * W, "a bias a thread");
    __shared__ __attribute__((aligned(256))) char lds[S * (kX + kW)];
    constexpr int kSets = kWalksOver<MB, NB> ? 2 : 1;      // the tile that is finished, and the next one
    __shared__ __attribute__((aligned(16))) float channel_bias[kSets][TN];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row_bytes = bytes_of_rows<T>(a.terms);
    const int down = (a.M + TM - 1) / TM, across = (a.N + TN - 1) / TN, steps = a.steps, all_steps = (row_bytes + 127) / 128;
    // A row of LDS is the 128 bytes of a row's step; its eight pieces of 16 bytes are permuted by the row, so that the 16 rows that a
    // read takes one piece of lie in 16 different groups of four banks.  A lane's load fetches the piece that belongs where it lands.
    // Turned, a row of LDS is the tile's i's at one c, 32 bytes (64 of fp32) permuted by c so that the 16 (4) rows of a read lie in different banks.
    unsigned offset[kLoads], behind = 0;      // behind: bit i, load i's piece of the last step lies past the end of its row
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const bool of_x = i < kLoadsX;
        const int load = wave * (of_x ? kLoadsX : kLoadsW) + (of_x ? i : i - kLoadsX);
        if (of_x ? kTurnX : kTurnW) {
            const int pieces = (of_x ? TM : TN) * (int)sizeof(T) / 16, at = load * 64 + lane, c = at / pieces;
            offset[i] = (unsigned)c * (of_x ? a.x_pitch : a.w_pitch) + ((at % pieces ^ swizzle_of<T>(c, of_x ? TM : TN)) << 4);
        } else {
            const int row = load * 8 + (lane >> 3);
            const int turn = of_x ? (row >> 1) & 7 : ((row >> 1) & 1) | ((row >> 3) & 3) << 1;
            const int piece = ((lane & 7) ^ turn) << 4;
            offset[i] = (unsigned)row * (of_x ? a.x_pitch : a.w_pitch) + piece;
            if ((all_steps - 1) * 128 + piece >= row_bytes) behind |= 1u << i;
        }
    }
    const unsigned lds0 = (unsigned)(uintptr_t)(SC_LDS char*)lds;
    int4v from_x = {0, 0, 0, 0}, from_w = from_x;
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
        if (!kTurnX) from_x = descriptor_of(static_cast<const char*>(a.x) + (size_t)next_m * a.x_pitch, (long long)min(TM, a.M - next_m) * a.x_pitch);
        if (!kTurnW) from_w = descriptor_of(static_cast<const char*>(a.w) + (size_t)next_n * a.w_pitch, (long long)min(TN, a.N - next_n) * a.w_pitch);
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
    auto look = [&]() {
        const bool there = step < min(end, all_steps);      // else zeros: past the last tile, or past the rows (in the last part)
        const int c = there ? step * kC : 0, rows = min(kC, a.terms - c) - 1;
        if (kTurnX)
            from_x = descriptor_of(static_cast<const char*>(a.x) + (size_t)c * a.x_pitch + (size_t)next_m * sizeof(T),
                                   there ? (long long)rows * a.x_pitch + bytes_of_rows<T>(a.M - next_m) : 0ll);
        else from_x[2] = there ? bytes_x : 0;
        if (kTurnW)
            from_w = descriptor_of(static_cast<const char*>(a.w) + (size_t)c * a.w_pitch + (size_t)next_n * sizeof(T),
                                   there ? (long long)rows * a.w_pitch + bytes_of_rows<T>(a.N - next_n) : 0ll);
        else from_w[2] = there ? bytes_w : 0;
        at = there ? step * 128 : 0;
        beyond = step == all_steps - 1 ? behind : 0;
    };
    auto advance = [&]() {
        if (++step == end) {
            tile += stride;
            if (kWalksOver<MB, NB> && tile < tiles) {
                set ^= 1;
                enter();
            }
        }
        look();
    };
    auto load = [&](int i) {
        if (i < kLoadsX) load_to_lds(from_x, kTurnX ? offset[i] : past(offset[i], beyond, i), kTurnX ? 0 : at, xdst + (wave * kLoadsX + i) * 1024);
        else load_to_lds(from_w, kTurnW ? offset[i] : past(offset[i], beyond, i), kTurnW ? 0 : at, wdst + (wave * kLoadsW + i - kLoadsX) * 1024);
    };
    enter();
    look();
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
    // two blocks are eight channels in a row.  (Where w is turned, of channel 16 j + r: its reads would take twice the time.)  Turned, a lane reads
    // four c's of 16 bits at once, or one of fp32.
    const int wm = wave % WM, wn = wave / WM, r = lane & 15, q = lane >> 4;
    constexpr int kRowX = TM * (int)sizeof(T), kRowW = TN * (int)sizeof(T), kChunk = 16 * (int)sizeof(T);      // bytes of a block's i's
    int xa0 = kTurnX ? turned_address<T>(lane, wm * MB, TM) : (wm * 16 * MB + r) * 128 + ((q ^ (r >> 1)) << 4), xa1 = kTurnX ? xa0 + kC / 2 * kRowX : xa0 ^ 64;
    int wa0 = S * kX + (kTurnW ? turned_address<T>(lane, wn * NB, TN) : (wn * 16 * NB + (r >> 2) * 8 + (r & 3)) * 128 + ((q ^ (r >> 1)) << 4));
    int wa1 = kTurnW ? wa0 + kC / 2 * kRowW : wa0 ^ 64;
    int4v wf[2][NB], xf[2][MB];
    auto read_w = [&](int h, int j) {
        if constexpr (kTurnW) wf[h][j] = read_block<T>(lds + ((h ? wa1 : wa0) ^ (j * kChunk)), kRowW);
        else wf[h][j] = *reinterpret_cast<const int4v*>(lds + (h ? wa1 : wa0) + ((j >> 1) * 32 + (j & 1) * 4) * 128);
    };
    auto read_x = [&](int h, int i) {
        if constexpr (kTurnX) xf[h][i] = read_block<T>(lds + ((h ? xa1 : xa0) ^ (i * kChunk)), kRowX);
        else xf[h][i] = *reinterpret_cast<const int4v*>(lds + (h ? xa1 : xa0) + i * 2048);
    };
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"((S - 1) * kLoads) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int j = 0; j < NB; ++j) read_w(0, j);
#pragma unroll
    for (int i = 0; i < kHalf; ++i) read_x(0, i);
    __builtin_amdgcn_sched_barrier(0);

    // A step is two halves, 64 bytes each.  In the first, all that the second needs is read, one read every few
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
        constexpr int kWide = kTurnW ? 4 : 8, kPair = kWide / 4;      // a lane's channels in a row, of one block or of two
        auto epilogue = [&](auto inside, auto plain) {
            each<NB / kPair>([&](auto pair) {
                constexpr int j = pair * kPair;
                const int tile_n = wn * 16 * NB + j * 16 + q * kWide, n = n0 + tile_n;
                float bias[kWide];
#pragma unroll
                for (int e = 0; e < kWide; ++e) bias[e] = channel_bias[done][tile_n + e];
                each<MB>([&](auto block) {
                    constexpr int i = block;
                    const int m = m0 + (wm * MB + i) * 16 + r;
                    float v[kWide];
                    each<kPair>([&](auto half) {
                        float4v& c = acc[i][j + half];
                        asm volatile("" : "+a"(c));
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[half * 4 + e] = c[e];
                        c = float4v{0.f, 0.f, 0.f, 0.f};
                    });
                    if (!inside && (m >= a.M || n >= a.N)) return;
                    if (!plain && a.partial) {
                        float* to = a.partial + ((size_t)part * a.M + m) * a.N + n;
                        typedef float four __attribute__((ext_vector_type(4), aligned(4)));
                        if (inside || n + kWide <= a.N) {
#pragma unroll
                            for (int c = 0; c < kWide / 4; ++c) reinterpret_cast<four*>(to)[c] = four{v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]};
                        } else {
#pragma unroll
                            for (int e = 0; e < kWide; ++e)
                                if (n + e < a.N) to[e] = v[e];
                        }
                    } else {
                        finish<T, kWide, inside, plain>(a, v, bias, m, n, a.N - n);
                    }
                });
            });
        };
        if (m0 + TM > a.M || n0 + TN > a.N) epilogue(std::false_type{}, std::false_type{});
        else if (a.partial || a.act != kNone || a.residual || a.z) epilogue(std::true_type{}, std::false_type{});
        else epilogue(std::true_type{}, std::true_type{});
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
// (Loads in the order that the products take would touch 16 rows with 16 lanes in a row, at a quarter of the rate.)  The weights' bytes bound it, as far
// as enough of them are on their way: for 24 x 4096 -> 8192 in 16 bits two workgroups of 72 KB a CU (2 x 1 blocks, 4 wavefronts, 3 deep) take 14.5 us on three sets
// of weights in turn, which the caches hold in part, one of 128 KB (2 x 2, 8 wavefronts, 2 deep) 15.7; on 16 sets, from HBM, 17.3 and 17.0 (3.9 TB/s).
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
    const int row_bytes = bytes_of_rows<T>(a.terms), units = (row_bytes + 127) / 128;

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
        if ((units - 1) * 128 + (int)piece_of[o] >= row_bytes) behind |= 1u << o;
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

template <class T, int MB, int NB, int S, Turned turned>
int launch_tile(const ProductArgs& a, hipStream_t s)
{
    const long long tiles = (long long)a.parts * ((a.M + 32ll * MB - 1) / (32 * MB)) * ((a.N + 32ll * NB - 1) / (32 * NB));
    const bool walks = kWalksOver<MB, NB> && a.steps >= kStepsToWalk;
    if (tiles >= (1ll << 31) || (!walks && (unsigned long long)tiles > most_groups(256))) return kTooLarge;
    const unsigned blocks = walks ? (unsigned)std::min(tiles, 256ll) : (unsigned)tiles;
    hipLaunchKernelGGL((linear_tile_kernel<T, MB, NB, 2, 2, S, turned == kTurnedBoth, turned != kRows>), dim3(blocks), dim3(256), 0, s, a, (unsigned)tiles, blocks);
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

template <class T, Turned turned>
int launch_kernel(Kernel kernel, const ProductArgs& a, hipStream_t s)
{
    if constexpr (turned == kRows) switch (kernel) {
        case kRow11: return launch_row<T, 1, 1, 8, 4>(a, s);
        case kRow21: return launch_row<T, 2, 1, 4, 3>(a, s);
        case kRow22: return launch_row<T, 2, 2, 8, 2>(a, s);
        case kRow41: return launch_row<T, 4, 1, 4, 2>(a, s);
        case kRow42: return launch_row<T, 4, 2, 4, 2>(a, s);
        case kDeep42: return launch_tile<T, 4, 2, 4, turned>(a, s);
        default: break;
    }
    if constexpr (sizeof(T) == 2)
        if (kernel == kTile88) return launch_tile<T, 8, 8, 2, turned>(a, s);
    switch (kernel) {
        case kTile22: return launch_tile<T, 2, 2, 2, turned>(a, s);
        case kTile44: return launch_tile<T, 4, 4, 2, turned>(a, s);
        case kDeep22: return launch_tile<T, 2, 2, 4, turned>(a, s);
        default: return launch_tile<T, 4, 4, 3, turned>(a, s);
    }
}

template <class T>
int launch_kernel(Kernel kernel, Turned turned, const ProductArgs& a, hipStream_t s)
{
    if (turned == kRows) return launch_kernel<T, kRows>(kernel, a, s);
    return turned == kTurnedW ? launch_kernel<T, kTurnedW>(kernel, a, s) : launch_kernel<T, kTurnedBoth>(kernel, a, s);
}

}  // namespace

}  // namespace sc

// Rows of 8-bit integers with a scale each, and the fully connected layer on them (sparse_conv_int8_quantize,
// sparse_conv_int8_linear).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>
#include <utility>

#include "text_ops.h"

namespace sc {

namespace {

enum { kF32 = 0, kF16 = 1, kBF16 = 2, kI8 = 3 };   // SC_F32, SC_F16, SC_BF16, SC_I8

constexpr float kTiny = 0x1p-100f;   // a row whose largest size is below this counts as zeros (127 / a would overflow from 2^-121)

// ---------------------------------------------------------------- rows to 8-bit integers

template <class T>
struct Piece {     // what one load of 16 bytes holds, from any element on (the hardware splits what crosses a line)
    static constexpr int kCount = 16 / sizeof(T);
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};

// Elements k .. k + kCount - 1 of a row; zeros past its end.
template <class T>
__device__ __forceinline__ typename Piece<T>::type load_piece(const T* row, int k, int K)
{
    typedef typename Piece<T>::type V;
    if (k + Piece<T>::kCount <= K) return *reinterpret_cast<const V*>(row + k);
    V v;
#pragma unroll
    for (int e = 0; e < Piece<T>::kCount; ++e) v[e] = k + e < K ? row[k + e] : (T)0.f;
    return v;
}

// The largest size of a piece and of what came before, as a bit pattern: patterns order as the sizes do, and a NaN lies above all.
// 16-bit types go two by two (two patterns a word until size_of).
template <class T>
__device__ __forceinline__ unsigned largest_of(typename Piece<T>::type v, unsigned most)
{
    typedef unsigned words __attribute__((ext_vector_type(4)));
    typedef unsigned short two __attribute__((ext_vector_type(2)));
    const words w = __builtin_bit_cast(words, v);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        if constexpr (sizeof(T) == 4) most = max(most, w[c] & 0x7fffffffu);
        else most = __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(two, w[c] & 0x7fff7fffu), __builtin_bit_cast(two, most)));
    }
    return most;
}

// The fp32 pattern of the largest of largest_of.
template <class T>
__device__ __forceinline__ unsigned size_of(unsigned most)
{
    if constexpr (sizeof(T) == 4) {
        return most;
    } else {
        const unsigned short one = (unsigned short)max(most & 0xffffu, most >> 16);
        return __float_as_uint((float)__builtin_bit_cast(T, one));
    }
}

// The factor that takes a row to whole numbers, and its scale, from its largest size.
__device__ __forceinline__ float scale_of(unsigned largest, float& scale)
{
    const float a = __uint_as_float(largest);
    const bool counts = a >= kTiny && a < INFINITY;
    scale = counts ? a / 127.f : a < kTiny ? 0.f : NAN;
    return counts ? 127.f / a : 0.f;
}

// The whole numbers of a piece, four to a word.  1.5 * 2^23 added to a product of at most 127 rounds it to a whole number, ties to
// even, and leaves that number in the low bits.  A row that does not count has the factor 0 and gives zeros.
template <class T>
__device__ __forceinline__ void quantize_piece(typename Piece<T>::type v, float factor, int (&word)[Piece<T>::kCount / 4])
{
#pragma clang fp contract(off)      // (the product is rounded before it is added to)
#pragma unroll
    for (int e = 0; e < Piece<T>::kCount; e += 4) {
        unsigned y[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] = __float_as_uint((float)v[e + c] * factor + 0x1.8p23f);
        const unsigned low = __builtin_amdgcn_perm(y[1], y[0], 0x0c0c0400u), high = __builtin_amdgcn_perm(y[3], y[2], 0x04000c0cu);
        word[e / 4] = factor > 0.f ? (int)(low | high) : 0;
    }
}

__device__ __forceinline__ unsigned largest_in_wavefront(unsigned most)
{
#pragma unroll
    for (int d = 32; d > 0; d /= 2) most = max(most, (unsigned)__shfl_xor((int)most, d));
    return most;
}

// A row for kLanes threads (several rows a workgroup where that is one wavefront).  Up to kKept pieces a thread stay in registers
// between the search for the largest size and the rounding; longer rows are read again.
template <class T, int kLanes>
__global__ __launch_bounds__(kLanes < 256 ? 256 : kLanes) void quantize_kernel(const T* x, int8_t* q, float* scale, int rows, int K, int pitch, long long ldx)
{
    typedef typename Piece<T>::type V;
    constexpr int kKept = 4, kCount = Piece<T>::kCount, kRows = kLanes < 256 ? 256 / kLanes : 1, kWaves = kLanes / 64;
    const int t = threadIdx.x % kLanes;
    const long long row = (long long)blockIdx.x * kRows + threadIdx.x / kLanes;
    if (kRows > 1 && row >= rows) return;       // (a whole wavefront: no barrier follows where rows share a workgroup)
    x += row * ldx;
    q += row * pitch;
    V kept[kKept];
    unsigned most = 0;
#pragma unroll
    for (int p = 0; p < kKept; ++p) kept[p] = load_piece<T>(x, (p * kLanes + t) * kCount, K);
#pragma unroll
    for (int p = 0; p < kKept; ++p) most = largest_of<T>(kept[p], most);
    for (int k = (kKept * kLanes + t) * kCount; k < K; k += kLanes * kCount) most = largest_of<T>(load_piece<T>(x, k, K), most);
    most = largest_in_wavefront(size_of<T>(most));
    if (kWaves > 1) {
        __shared__ unsigned of_wave[kWaves];
        if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = max(most, of_wave[w]);
    }
    float s;
    const float factor = scale_of(most, s);
    if (t == 0) scale[row] = s;
    auto store = [&](V v, int k) {
        int word[kCount / 4];
        quantize_piece<T>(v, factor, word);
        if (kCount == 8) *reinterpret_cast<int2*>(q + k) = make_int2(word[0], word[kCount / 4 - 1]);
        else *reinterpret_cast<int*>(q + k) = word[0];
    };
#pragma unroll
    for (int p = 0; p < kKept; ++p) {
        const int k = (p * kLanes + t) * kCount;
        if (k < pitch) store(kept[p], k);
    }
    for (int k = (kKept * kLanes + t) * kCount; k < pitch; k += kLanes * kCount) store(load_piece<T>(x, k, K), k);
}

template <class T>
int launch_quantize(const void* x, int8_t* q, float* scale, int rows, int K, long long ldx, hipStream_t s)
{
    const int pitch = (K + 127) / 128 * 128, pieces = pitch / Piece<T>::kCount;
    const T* in = static_cast<const T*>(x);
    // one wavefront a row where a lane's pieces fit its registers; few long rows by as many threads as have a piece each
    if (pieces <= 128 || (pieces <= 256 && rows >= 1024))
        hipLaunchKernelGGL((quantize_kernel<T, 64>), dim3((rows + 3) / 4), dim3(256), 0, s, in, q, scale, rows, K, pitch, ldx);
    else if (pieces <= 512 || rows >= 512)
        hipLaunchKernelGGL((quantize_kernel<T, 256>), dim3(rows), dim3(256), 0, s, in, q, scale, rows, K, pitch, ldx);
    else
        hipLaunchKernelGGL((quantize_kernel<T, 1024>), dim3(rows), dim3(1024), 0, s, in, q, scale, rows, K, pitch, ldx);
    return (int)hipGetLastError();
}

// ---------------------------------------------------------------- product, tiles through LDS

typedef int int4v __attribute__((ext_vector_type(4)));
#define SC_LDS __attribute__((address_space(3)))

template <class F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
// f(0) .. f(N - 1), each with its number as a constant: loops that have to be unrolled whole, however long.
template <int N, class F>
__device__ __forceinline__ void each(F&& f) { each_of(f, std::make_integer_sequence<int, N>{}); }

// 16 bytes a lane from memory to LDS at `lds` + 16 * lane; bytes past the descriptor's end arrive as zeros.  Not the builtin:
// the compiler waits for every load of that kind before any later read of LDS, here the reads wait where they have to.
// A load to LDS may read m0 one wait state after a scalar instruction wrote it at the earliest; the compiler adds none inside an asm block.
// (It notes that it keeps m0 for itself, which it does not across an operation that needs it.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(int4v descriptor, unsigned offset, unsigned base, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" :: "s"(lds), "v"(offset), "s"(descriptor), "s"(base) : "m0", "memory");
}

// The same, 4 bytes a lane.
__device__ __forceinline__ void load_word_to_lds(int4v descriptor, unsigned offset, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" :: "s"(lds), "v"(offset), "s"(descriptor) : "m0", "memory");
}
#pragma clang diagnostic pop

__device__ __forceinline__ int4v descriptor_of(const void* p, long long bytes)
{
    const uint64_t b = reinterpret_cast<uint64_t>(p);
    return int4v{(int)b, (int)(b >> 32) & 0xffff, (int)bytes, 0x00020000};
}

// c += a * b over 16 x 16 outputs and 64 bytes: lane l holds bytes 16 * (l / 16) .. + 15 of row l % 16 of a and of b, and rows
// 4 * (l / 16) .. + 3 of c at column l % 16.  The sums stay in accumulation registers (as a builtin they were copied and spilled).
__device__ __forceinline__ void multiply(int4v& c, int4v a, int4v b)
{
    asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}

// An output from its sum, alike in every kernel: rounded to 32 bits before anything else (the compiler would fuse the last addition
// into a conversion to float16, which then rounds once, and not everywhere: a token's outputs would depend on the kernel).
__device__ __forceinline__ float output_of(int sum, float x_scale, float w_scale, float bias, int relu)
{
    float v = fmaf((float)sum * x_scale, w_scale, bias);
    asm("" : "+v"(v));
    return relu && v < 0.f ? 0.f : v;
}

// The tile that a workgroup takes: workgroups go round the eight XCDs, so each gets a run of tiles of its own, which goes down kGroup
// tiles before it goes across: the 32 that an XCD's CUs hold at one a CU are 4 by 8 tiles that share rows of x and of w.
__device__ __forceinline__ void tile_of(unsigned block, unsigned tiles, int down, int across, int& tm, int& tn)
{
    const unsigned xcd = block % 8, share = tiles / 8, rest = tiles % 8;
    const unsigned tile = xcd * share + (xcd < rest ? xcd : rest) + block / 8;
    constexpr int kGroup = 4;
    const unsigned per_group = kGroup * (unsigned)across, group = tile / per_group, in = tile % per_group;
    const int rows = min(kGroup, down - (int)group * kGroup);
    tm = (int)group * kGroup + (int)(in % (unsigned)rows);
    tn = (int)(in / (unsigned)rows);
}

// Large tiles: a workgroup has a CU to itself, so it walks over tiles, `stride` apart, and loads the next one's first steps before it
// finishes one.  (Three steps a tile at least: a barrier lies between what reads a set of scales and what loads over it.)
template <int MB, int NB>
constexpr bool kWalks = MB * NB >= 64;
constexpr int kWalkSteps = 3;

// A tile of 16 MB WM rows of x by 16 NB WN rows of w, 128 bytes of each a step; WM x WN wavefronts with MB x NB blocks of 16 x 16 sums.
// S steps are in LDS or on their way there.
template <class T, int MB, int NB, int WM, int WN, int S>
__global__ __launch_bounds__(64 * WM * WN, MB * NB >= 64 || S > 2 ? 1 : 2) void tile_product_kernel(Int8Args a, unsigned tiles, unsigned stride)
{
    const int8_t* x = static_cast<const int8_t*>(a.x);
    const float* x_scale = a.x_scale;
    constexpr int TM = 16 * MB * WM, TN = 16 * NB * WN, W = WM * WN;
    constexpr int kLoadsX = TM / 8 / W, kLoadsW = TN / 8 / W, kLoads = kLoadsX + kLoadsW;
    constexpr int kX = TM * 128, kW = TN * 128, kHalf = MB / 2;
    static_assert(MB % 2 == 0 && NB % 2 == 0, "blocks come in pairs");
    static_assert(TM % 64 == 0 && TN % 64 == 0 && TM <= 64 * W && TN <= 64 * W, "a scale a thread");
    __shared__ __attribute__((aligned(256))) char lds[S * (kX + kW)];
    constexpr int kSets = kWalks<MB, NB> ? 2 : 1;      // the tile that is finished, and the next one
    __shared__ __attribute__((aligned(16))) float channel_scale[kSets][TN], channel_bias[kSets][TN], token_scale[kSets][TM];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int down = (a.M + TM - 1) / TM, across = (a.N + TN - 1) / TN, steps = a.pitch / 128;
    // A row of LDS is the 128 bytes of a row's step; its eight pieces of 16 bytes are permuted by the row, so that the 16 rows that a
    // read takes one piece of lie in 16 different groups of four banks.  A lane's load fetches the piece that belongs where it lands.
    unsigned offset[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int row = (wave * (i < kLoadsX ? kLoadsX : kLoadsW) + (i < kLoadsX ? i : i - kLoadsX)) * 8 + (lane >> 3);
        const int turn = i < kLoadsX ? (row >> 1) & 7 : ((row >> 1) & 1) | ((row >> 3) & 3) << 1;
        offset[i] = (unsigned)row * a.pitch + (((lane & 7) ^ turn) << 4);
    }
    const unsigned lds0 = (unsigned)(uintptr_t)(SC_LDS char*)lds;
    int4v from_x, from_w;
    unsigned xdst = lds0, wdst = lds0 + S * kX, tile = blockIdx.x;
    int next_m = 0, next_n = 0, step = 0, set = 0;      // what is loaded: a step of a tile, whose scales go to `set`
    auto enter = [&]() {
        int tm, tn;
        tile_of(tile, tiles, down, across, tm, tn);
        next_m = tm * TM;
        next_n = tn * TN;
        from_x = descriptor_of(x + (size_t)next_m * a.pitch, (long long)min(TM, a.M - next_m) * a.pitch);
        from_w = descriptor_of(a.w + (size_t)next_n * a.pitch, (long long)min(TN, a.N - next_n) * a.pitch);
        const long long ws = min(TN, a.N - next_n) * 4ll, xs = min(TM, a.M - next_m) * 4ll;
        if (wave * 64 < TN) {
            load_word_to_lds(descriptor_of(a.w_scale + next_n, ws), threadIdx.x * 4, (unsigned)(uintptr_t)(SC_LDS float*)channel_scale[set] + wave * 256);
            if (a.bias) load_word_to_lds(descriptor_of(a.bias + next_n, ws), threadIdx.x * 4, (unsigned)(uintptr_t)(SC_LDS float*)channel_bias[set] + wave * 256);
            else channel_bias[set][threadIdx.x] = 0.f;
        }
        if (wave * 64 < TM)
            load_word_to_lds(descriptor_of(x_scale + next_m, xs), threadIdx.x * 4, (unsigned)(uintptr_t)(SC_LDS float*)token_scale[set] + wave * 256);
    };
    auto advance = [&]() {
        if (++step < steps) return;
        tile += stride;
        if (kWalks<MB, NB> && tile < tiles) {
            step = 0;
            set ^= 1;
            enter();
        } else {
            from_x[2] = from_w[2] = 0;      // past the last step: zeros, and nothing is fetched
        }
    };
    auto load = [&](int i) {
        if (i < kLoadsX) load_to_lds(from_x, offset[i], step * 128, xdst + (wave * kLoadsX + i) * 1024);
        else load_to_lds(from_w, offset[i], step * 128, wdst + (wave * kLoadsW + i - kLoadsX) * 1024);
    };
    enter();
    int m0 = next_m, n0 = next_n, done = set;
    each<S>([&](auto stage) {
        if constexpr (stage > 0) advance();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load(i);
        xdst += kX;
        wdst += kW;
    });
    xdst -= S * kX;
    wdst -= S * kW;

    int4v acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            acc[i][j] = int4v{0, 0, 0, 0};
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
            constexpr int kSlots = MB * NB, kTurn = kSlots / 2;
            each<kSlots>([&](auto slot) {
                constexpr int t = slot, i = t / NB, j = t % NB, kOps = kHalf + NB + MB;
                multiply(acc[i][j], wf[0][j], xf[0][i]);
                constexpr int first = (t * kOps + kSlots - 1) / kSlots, last = ((t + 1) * kOps + kSlots - 1) / kSlots;
                each<last - first>([&](auto n) {
                    constexpr int o = first + n;
                    if constexpr (o < 2 * kHalf && o % 2 == 0) read_x(0, kHalf + o / 2);
                    else {
                        constexpr int u = o < 2 * kHalf ? o / 2 : o - kHalf;
                        if constexpr (u < NB) read_w(1, u);
                        else read_x(1, u - NB);
                    }
                });
                __builtin_amdgcn_sched_barrier(0);
            });
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            each<kSlots>([&](auto slot) {
                constexpr int t = slot, i = t / NB, j = t % NB;
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
                multiply(acc[i][j], wf[1][j], xf[1][i]);
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

        // Scales, bias and activation, while the first steps of the next tile are on their way.  The last products are read: the matrix
        // unit's results need 18 clocks.
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
        float xs[MB];
#pragma unroll
        for (int i = 0; i < MB; ++i) xs[i] = token_scale[done][(wm * MB + i) * 16 + r];
        typedef typename Piece<T>::type V;
        constexpr int kV = Piece<T>::kCount;
        auto finish = [&](auto inside) {      // inside: the tile lies whole within the output
            each<NB / 2>([&](auto pair) {
                constexpr int j = 2 * pair;
                const int tile_n = wn * 16 * NB + j * 16 + q * 8, n = n0 + tile_n;
                float cs[8], cb[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    cs[e] = channel_scale[done][tile_n + e];
                    cb[e] = channel_bias[done][tile_n + e];
                }
                each<MB>([&](auto block) {
                    constexpr int i = block;
                    const int m = m0 + (wm * MB + i) * 16 + r;
                    asm volatile("" : "+a"(acc[i][j]), "+a"(acc[i][j + 1]));
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = output_of(acc[i][j + e / 4][e % 4], xs[i], cs[e], cb[e], a.relu);
                    acc[i][j] = acc[i][j + 1] = int4v{0, 0, 0, 0};
                    V y[8 / kV];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e / kV][e % kV] = (T)v[e];
                    T* out = static_cast<T*>(a.out) + (size_t)m * a.ldo + n;
                    if constexpr (inside) {
#pragma unroll
                        for (int c = 0; c < 8 / kV; ++c) reinterpret_cast<V*>(out)[c] = y[c];
                    } else if (m < a.M) {
                        if (n + 8 <= a.N)
#pragma unroll
                            for (int c = 0; c < 8 / kV; ++c) reinterpret_cast<V*>(out)[c] = y[c];
                        else
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (n + e < a.N) out[e] = y[e / kV][e % kV];
                    }
                });
            });
        };
        if (m0 + TM <= a.M && n0 + TN <= a.N) finish(std::true_type{});
        else finish(std::false_type{});
        if (!kWalks<MB, NB>) break;
        m0 = next_m;
        n0 = next_n;
        done = set;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (loads of zeros that nothing reads)
}

template <class T, int MB, int NB, int WM, int WN, int S>
int launch_tile_product(const Int8Args& a, hipStream_t s)
{
    const long long tiles = ((a.M + 16ll * MB * WM - 1) / (16 * MB * WM)) * ((a.N + 16ll * NB * WN - 1) / (16 * NB * WN));
    const bool walks = kWalks<MB, NB> && a.pitch >= 128 * kWalkSteps;
    if (tiles >= (1ll << 31) || (!walks && (unsigned long long)tiles > most_groups(64 * WM * WN))) return kTooLarge;
    const unsigned blocks = walks ? (unsigned)std::min(tiles, 256ll) : (unsigned)tiles;
    hipLaunchKernelGGL((tile_product_kernel<T, MB, NB, WM, WN, S>), dim3(blocks), dim3(64 * WM * WN), 0, s, a, (unsigned)tiles, blocks);
    return (int)hipGetLastError();
}

// ---------------------------------------------------------------- product, few tokens

template <class T>
struct IsByte { static constexpr bool value = false; };
template <>
struct IsByte<int8_t> { static constexpr bool value = true; };

// Rows of 8-bit integers that a workgroup can quantise for itself, in bytes.
constexpr int kOwnBytes = 16384;

// 16 MB tokens by 16 NB channels a workgroup, whose W wavefronts go round the 128-byte units of the rows and add their sums up at
// the end.  A wavefront loads its units to a part of LDS of its own, D of them in flight, and waits for its own loads alone.  (Loads
// in the order that the products take would touch 16 rows with 16 lanes in a row, at a quarter of the rate.)  X is int8_t, x then
// comes the same way as w; or the type of an input that every workgroup loads and then quantises while its first weights are on their way.
template <class T, class X, int MB, int NB, int W, int D>
__global__ __launch_bounds__(64 * W) void row_product_kernel(Int8Args a)
{
    constexpr bool kGiven = IsByte<X>::value;
    constexpr int kTokens = 16 * MB, kChannels = 16 * NB, kThreads = 64 * W;
    constexpr int kLoadsX = kGiven ? 2 * MB : 0, kLoads = kLoadsX + 2 * NB, kUnit = 1024 * kLoads;
    static_assert(kGiven || MB == 1, "rows that are quantised here are 16 at most");
    static_assert(D * kUnit >= kTokens * kChannels * 4, "the sums take the place of the units");
    __shared__ __attribute__((aligned(256))) char lds[W * D * kUnit];
    __shared__ __attribute__((aligned(16))) char rows_of_x[kGiven ? 16 : kOwnBytes];
    __shared__ __attribute__((aligned(16))) float channel_scale[64], channel_bias[64], token_scale[64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, q = lane >> 4;
    const int across = (a.N + kChannels - 1) / kChannels;
    const int m0 = (int)(blockIdx.x / across) * kTokens, n0 = (int)(blockIdx.x % across) * kChannels;
    const int units = a.pitch / 128;

    // A thread's pieces of x, of any rows, stay in registers (their number a row is a multiple of 16: 16 lanes share a row).
    typedef typename Piece<typename std::conditional<kGiven, float, X>::type>::type P;
    constexpr int kCount = kGiven ? 4 : 16 / sizeof(X), kKept = kGiven ? 1 : (kOwnBytes / kCount + kThreads - 1) / kThreads;
    P kept[kKept];
    int m_of[kKept];
    const int per_row = a.pitch / kCount, pieces = min(kTokens, a.M - m0) * per_row;
    __shared__ unsigned largest[16];
    if constexpr (!kGiven) {
        const X* x = static_cast<const X*>(a.x) + (size_t)m0 * a.ldx;
        if (threadIdx.x < 16) largest[threadIdx.x] = 0;
#pragma unroll
        for (int i = 0; i < kKept; ++i) {
            const int p = i * kThreads + threadIdx.x;
            m_of[i] = p / per_row;
            if (p < pieces) kept[i] = load_piece<X>(x + m_of[i] * a.ldx, p % per_row * kCount, a.K);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (the compiler would wait for the weights as well)
        __syncthreads();
    }

    // Pieces of 16 bytes are permuted within the 128 bytes of a row as in the tile kernel.
    int4v from_w = descriptor_of(a.w + (size_t)n0 * a.pitch, (long long)min(kChannels, a.N - n0) * a.pitch);
    int4v from_x = kGiven ? descriptor_of(static_cast<const int8_t*>(a.x) + (size_t)m0 * a.pitch, (long long)min(kTokens, a.M - m0) * a.pitch) : from_w;
    const int bytes_w = from_w[2], bytes_x = from_x[2];
    const unsigned lds0 = (unsigned)(uintptr_t)(SC_LDS char*)lds + wave * D * kUnit;
    unsigned offset[2];      // of the rows lane / 8 of an even and an odd load: their permutations differ
#pragma unroll
    for (int o = 0; o < 2; ++o) offset[o] = (unsigned)(o * 8 + (lane >> 3)) * a.pitch + (((lane & 7) ^ ((o * 4 + (lane >> 4)) & 7)) << 4);
    if (wave == 0) load_word_to_lds(descriptor_of(a.w_scale + n0, min(kChannels, a.N - n0) * 4ll), lane * 4, (unsigned)(uintptr_t)(SC_LDS float*)channel_scale);
    if (wave == 1) {
        if (a.bias) load_word_to_lds(descriptor_of(a.bias + n0, min(kChannels, a.N - n0) * 4ll), lane * 4, (unsigned)(uintptr_t)(SC_LDS float*)channel_bias);
        else channel_bias[lane] = 0.f;
    }
    if (kGiven && wave == 2)
        load_word_to_lds(descriptor_of(a.x_scale + m0, min(kTokens, a.M - m0) * 4ll), lane * 4, (unsigned)(uintptr_t)(SC_LDS float*)token_scale);
    auto load = [&](int slot, int unit) {
        from_w[2] = unit < units ? bytes_w : 0;
        from_x[2] = unit < units ? bytes_x : 0;
        each<kLoads>([&](auto load) {
            constexpr int l = load, block = l < kLoadsX ? l / 2 : (l - kLoadsX) / 2;
            load_to_lds(l < kLoadsX ? from_x : from_w, offset[l & 1] + block * 16u * a.pitch, unit * 128, lds0 + slot * kUnit + l * 1024);
        });
    };
    each<D>([&](auto d) { load(d, wave + d * W); });

    if constexpr (!kGiven) {
#pragma unroll
        for (int i = 0; i < kKept; ++i) {
            if ((int)(i * kThreads + threadIdx.x) >= pieces) continue;
            unsigned most = size_of<X>(largest_of<X>(kept[i], 0));
#pragma unroll
            for (int d = 8; d > 0; d /= 2) most = max(most, (unsigned)__shfl_xor((int)most, d));
            if (r == 0) atomicMax(&largest[m_of[i]], most);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < kKept; ++i) {
            const int p = i * kThreads + threadIdx.x;
            if (p >= pieces) continue;
            float s;
            const float factor = scale_of(largest[m_of[i]], s);
            if (p % per_row == 0) token_scale[m_of[i]] = s;
            int word[kCount / 4];
            quantize_piece<X>(kept[i], factor, word);
            int* to = reinterpret_cast<int*>(rows_of_x + p * kCount);
#pragma unroll
            for (int c = 0; c < kCount / 4; ++c) to[c] = word[c];
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }

    int4v acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = int4v{0, 0, 0, 0};
    const char* mine = lds + wave * D * kUnit + r * 128;
    const int piece[2] = {(q ^ (r >> 1)) << 4, ((q + 4) ^ (r >> 1)) << 4};
    const int my_row = min(r, a.M - m0 - 1);      // (the columns of tokens that are not there are never stored)
    int slot = 0;
    for (int unit = wave; unit < units; unit += W) {
        asm volatile("s_waitcnt vmcnt(%0)" :: "n"((D - 1) * kLoads) : "memory");
        const char* from = mine + slot * kUnit;
        int4v wf[2][NB], xf[2][MB];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                if constexpr (kGiven) xf[h][i] = *reinterpret_cast<const int4v*>(from + i * 2048 + piece[h]);
                else xf[h][i] = *reinterpret_cast<const int4v*>(rows_of_x + my_row * a.pitch + unit * 128 + h * 64 + q * 16);
            }
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
                for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[h][j], xf[h][i], acc[i][j], 0, 0, 0);
        slot = slot + 1 == D ? 0 : slot + 1;
    }

    // Sums of each wavefront where its units were: [token][channel].
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
            *reinterpret_cast<int4v*>(lds + wave * D * kUnit + ((i * 16 + r) * kChannels + j * 16 + q * 4) * 4) = acc[i][j];
    __syncthreads();
    typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    for (int o = threadIdx.x; o < kTokens * kChannels / 4; o += kThreads) {
        const int token = o / (kChannels / 4), channel = o % (kChannels / 4) * 4, m = m0 + token, n = n0 + channel;
        if (m >= a.M) continue;
        int4v sum = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < W; ++w) sum += *reinterpret_cast<const int4v*>(lds + w * D * kUnit + o * 16);
        four y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[e] = (T)output_of(sum[e], token_scale[token], channel_scale[channel + e], channel_bias[channel + e], a.relu);
        }
        T* out = static_cast<T*>(a.out) + m * a.ldo + n;
        if (n + 4 <= a.N) *reinterpret_cast<four*>(out) = y;
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < a.N) out[e] = y[e];
    }
}

template <class T, class X, int MB, int NB, int W, int D>
int launch_row_product(const Int8Args& a, hipStream_t s)
{
    const long long groups = ((a.M + 16ll * MB - 1) / (16 * MB)) * ((a.N + 16ll * NB - 1) / (16 * NB));
    if ((unsigned long long)groups > most_groups(64 * W)) return kTooLarge;
    hipLaunchKernelGGL((row_product_kernel<T, X, MB, NB, W, D>), dim3((unsigned)groups), dim3(64 * W), 0, s, a);
    return (int)hipGetLastError();
}

// ---------------------------------------------------------------- which kernel

// Microseconds that a product is estimated to take.  The constants are fitted to launches of 20 sizes of M by 16 of K and N but the two
// largest products, 318 (1 to 8192 tokens, K 128 to 16384, N 10 to 16384, weights that do not stay in a cache), each to what is near the fastest there: over
// these the kernel of the least estimate takes 1.0 % more than the fastest one, 26 % at most
// (512 x 16384 -> 512).  Depth pays where a CU has a tile or two (64 x 64 at 256 x 4096 -> 4096: 14.5 us by two steps, 10.0 by four),
// two steps where workgroups that share a CU hide each other's waits (128 x 128 at 2048 x 4096 -> 4096: 32.7 by two, 35.2 by three).

// Pieces of `size` (a power of two) that n is cut into.  (The host looks at 14 kernels a call: 0.1 us without divisions of 64 bits, 0.25 with.)
double pieces_of(int n, int size) { return (double)(((unsigned)n + (unsigned)size - 1) >> __builtin_ctz((unsigned)size)); }
double rounds_of(double groups, double held) { return (double)(long long)((groups + held - 1.0) / held); }

enum Kernel { kRow11, kRow21, kRow22, kRow41, kRow42, kTile22, kTile44, kTile88, kDeep22, kDeep42, kDeep44, kKernels };

// Row kernel: a launch, the sums of the wavefronts and the further workgroups of a CU, then the largest of what all workgroups load,
// what those of one CU load, and the weights.
struct RowRule {
    int MB, NB;                      // blocks
    double join, more;               // us
    double all, one, weights;        // MB/us of all, KB/us of one, MB/us of the weights
};
constexpr RowRule kRowRules[] = {{1, 1, 0.36, 1.39, 21.1, 144.0, 7.2}, {2, 1, 0.24, 1.42, 22.5, 135.0, 6.0}, {2, 2, 0.12, 0.83, 19.2, 136.0, 5.6},
                                 {4, 1, 0.33, 1.54, 24.6, 133.0, 4.75}, {4, 2, 0.91, 1.64, 19.8, 132.0, 5.05}};

double row_estimate(const RowRule& r, int M, int N, int pitch)
{
    const double groups = pieces_of(M, 16 * r.MB) * pieces_of(N, 16 * r.NB), bytes = 16.0 * (r.MB + r.NB) * pitch;
    const double on_a_cu = rounds_of(groups, 256.0);
    const double load = std::max({groups * bytes / (r.all * 1e6), on_a_cu * bytes / (r.one * 1e3), (double)N * pitch / (r.weights * 1e6)});
    return 3.0 + r.join * on_a_cu + r.more * (on_a_cu - 1.0) + load;
}

// Tile kernel: steps of `least` us while a workgroup has the CU to itself, `each` times the workgroups that share it beyond; the weights
// from memory at least.
struct TileRule {
    int MB, NB, share;               // blocks of a wavefront; workgroups that a CU holds
    double least, each, start, finish;
    double weights;                  // MB/us
};
constexpr TileRule kTileRules[] = {{2, 2, 4, 0.268, 0.213, 0.28, 2.35, 3.5}, {4, 4, 2, 0.063, 0.446, 0.40, 4.07, 3.2}, {8, 8, 1, 0.0, 1.16, 2.66, 9.15, 6.7},
                                   {2, 2, 2, 0.049, 0.194, 1.20, 1.90, 7.0}, {4, 2, 1, 0.0, 0.271, 1.12, 2.48, 6.6}, {4, 4, 1, 0.0, 0.396, 0.99, 3.39, 4.7}};

double tile_estimate(const TileRule& r, int M, int N, int pitch)
{
    const double groups = pieces_of(M, 32 * r.MB) * pieces_of(N, 32 * r.NB), steps = pitch / 128.0, held = 256.0 * r.share;
    const double rounds = (double)(long long)(groups / held), rest = groups - rounds * held;
    double us = r.start + rounds * (steps * r.each * r.share + r.finish);
    if (rest > 0.0) us += steps * std::max(r.least, r.each * rounds_of(rest, 256.0)) + r.finish;
    return std::max(us, 3.0 + (double)N * pitch / (r.weights * 1e6));
}

Kernel choose(int M, int N, int pitch, double& least)
{
    int best = 0;
    least = 0.0;
    for (int k = 0; k < kKernels; ++k) {
        const double us = k < kTile22 ? row_estimate(kRowRules[k], M, N, pitch) : tile_estimate(kTileRules[k - kTile22], M, N, pitch);
        if (k == 0 || us < least) {
            best = k;
            least = us;
        }
    }
    return (Kernel)best;
}

template <class T>
int launch_product(Kernel kernel, const Int8Args& a, hipStream_t s)
{
    switch (kernel) {
        case kRow11: return launch_row_product<T, int8_t, 1, 1, 8, 4>(a, s);
        case kRow21: return launch_row_product<T, int8_t, 2, 1, 8, 2>(a, s);
        case kRow22: return launch_row_product<T, int8_t, 2, 2, 4, 2>(a, s);
        case kRow41: return launch_row_product<T, int8_t, 4, 1, 8, 1>(a, s);
        case kRow42: return launch_row_product<T, int8_t, 4, 2, 4, 2>(a, s);
        case kTile22: return launch_tile_product<T, 2, 2, 2, 2, 2>(a, s);
        case kTile44: return launch_tile_product<T, 4, 4, 2, 2, 2>(a, s);
        case kTile88: return launch_tile_product<T, 8, 8, 2, 2, 2>(a, s);
        case kDeep22: return launch_tile_product<T, 2, 2, 2, 2, 4>(a, s);
        case kDeep42: return launch_tile_product<T, 4, 2, 2, 2, 4>(a, s);
        default: return launch_tile_product<T, 4, 4, 2, 2, 3>(a, s);
    }
}

// An input that is not quantised yet takes a launch of its own, 2.5 to 3.9 us more on the GPU and 2.75 on the host (kQuantise counts
// some of that), or every workgroup of a row kernel quantises its 16 rows for itself: it loads them, then asks for its first weights, and
// works the scales and whole numbers out while these are on their way.  Fitted to
// 114 sizes (1 to 593 tokens, K 128 to 4096, N 10 to 12288), the rule takes 0.5 % more than the fastest one call after another, 1.6 % in
// a graph.  1 x 2048 -> 4288 5.7 us against 8.9, 1 x 4096 -> 12288 12.5 against 15.3, 101 x 384 -> 256 5.0 against 8.9;
// 593 x 384 -> 1280 would take 11.3 against 8.7.
enum Own { kOwn16, kOwn4, kOwn4Wide, kOwns, kTwoLaunches = kOwns };

struct Choice {
    Own own;
    Kernel product;      // after another launch
};

struct OwnRule {
    int NB, resident;                                  // blocks of channels; workgroups that a CU holds
    double start, round, each, more, weights, one;     // us; us a round; us for 1000 values a round, a further workgroup on a CU; MB/us; KB/us
};
constexpr OwnRule kOwnRules[] = {{1, 1, 3.7, 3.1, 0.145, 0.0, 7.7, 53.6}, {1, 4, 2.8, 1.46, 0.312, 0.041, 5.4, 29.5}, {2, 3, 3.05, 2.44, 0.327, 0.071, 4.6, 56.5}};
constexpr double kQuantise = 4.5, kTwoAtLeast = 3.0 + kQuantise;

double own_estimate(const OwnRule& r, int M, int N, int pitch, int in_dtype)
{
    const double groups = pieces_of(M, 16) * pieces_of(N, 16 * r.NB), on_a_cu = rounds_of(groups, 256.0), rounds = rounds_of(groups, 256.0 * r.resident);
    const double values = std::min(M, 16) * (double)pitch * (in_dtype == kF32 ? 1.35e-3 : 1e-3);
    return r.start + (rounds - 1.0) * r.round + rounds * r.each * values + (on_a_cu - 1.0) * r.more * values +
           std::max((double)N * pitch / (r.weights * 1e6), on_a_cu * 16 * r.NB * pitch / (r.one * 1e3));
}

Choice choose(int M, int N, int pitch, int in_dtype)
{
    double least = 0.0, product;
    int best = kTwoLaunches;
    if (in_dtype != kI8 && (long long)std::min(M, 16) * pitch <= kOwnBytes) {
        for (int k = 0; k < kOwns; ++k) {
            const double us = own_estimate(kOwnRules[k], M, N, pitch, in_dtype);
            if (k == 0 || us < least) {
                best = k;
                least = us;
            }
        }
        if (least <= kTwoAtLeast) return {(Own)best, kKernels};      // (no product takes less than 3 us)
    }
    const Kernel kernel = choose(M, N, pitch, product);
    if (best != kTwoLaunches && least <= product + kQuantise) return {(Own)best, kKernels};
    return {kTwoLaunches, kernel};
}

template <class T, class X>
int launch_own(Own kernel, const Int8Args& a, hipStream_t s)
{
    switch (kernel) {
        case kOwn16: return launch_row_product<T, X, 1, 1, 16, 4>(a, s);
        case kOwn4: return launch_row_product<T, X, 1, 1, 4, 2>(a, s);
        default: return launch_row_product<T, X, 1, 2, 4, 2>(a, s);
    }
}

template <class T>
int launch_own(Own kernel, int in_dtype, const Int8Args& a, hipStream_t s)
{
    if (in_dtype == kF32) return launch_own<T, float>(kernel, a, s);
    if (in_dtype == kF16) return launch_own<T, _Float16>(kernel, a, s);
    return launch_own<T, __bf16>(kernel, a, s);
}

}  // namespace

int launch_int8_quantize(int dtype, const void* x, int8_t* q, float* scale, int rows, int K, long long ldx, void* stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == kF32) return launch_quantize<float>(x, q, scale, rows, K, ldx, s);
    if (dtype == kF16) return launch_quantize<_Float16>(x, q, scale, rows, K, ldx, s);
    return launch_quantize<__bf16>(x, q, scale, rows, K, ldx, s);
}

int int8_kernel(int M, int N, int K) { return choose(M, N, (K + 127) / 128 * 128, kI8).product; }

int int8_own_kernel(int M, int N, int K, int in_dtype)
{
    const Own own = choose(M, N, (K + 127) / 128 * 128, in_dtype).own;
    return own == kTwoLaunches ? -1 : own;
}

// The quantised input, then its scales.
long long int8_workspace(int M, int N, int K, int in_dtype, int)
{
    if (in_dtype == kI8 || int8_own_kernel(M, N, K, in_dtype) >= 0) return 0;
    return (long long)M * ((K + 127) / 128 * 128) + (M * 4ll + 15) / 16 * 16;
}

int launch_int8_linear(int in_dtype, int out_dtype, const Int8Args& given, char* workspace, void* stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    Int8Args a = given;
    const Choice choice = choose(a.M, a.N, a.pitch, in_dtype);
    if (choice.own != kTwoLaunches) {
        if (out_dtype == kF32) return launch_own<float>(choice.own, in_dtype, a, s);
        if (out_dtype == kF16) return launch_own<_Float16>(choice.own, in_dtype, a, s);
        return launch_own<__bf16>(choice.own, in_dtype, a, s);
    }
    if (in_dtype != kI8) {
        int8_t* q = reinterpret_cast<int8_t*>(workspace);
        float* scale = reinterpret_cast<float*>(workspace + (size_t)a.M * a.pitch);
        const int e = launch_int8_quantize(in_dtype, a.x, q, scale, a.M, a.K, a.ldx, stream);
        if (e != 0) return e;
        a.x = q;
        a.x_scale = scale;
    }
    if (out_dtype == kF32) return launch_product<float>(choice.product, a, s);
    if (out_dtype == kF16) return launch_product<_Float16>(choice.product, a, s);
    return launch_product<__bf16>(choice.product, a, s);
}

}  // namespace sc

// Word vectors and their gradient (sparse_conv_embed, sparse_conv_embed_backward).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "text_ops.h"

namespace sc {

namespace {

enum { kF32 = 0, kF16 = 1, kBF16 = 2 };   // SC_F32, SC_F16, SC_BF16

constexpr int kThreads = 256;

// VEC elements that may start at any element (the hardware splits what crosses a line).
template <class T, int VEC>
struct Piece {
    typedef T type __attribute__((ext_vector_type(VEC), aligned(sizeof(T))));
};
template <class T>
struct Piece<T, 1> {
    typedef T type __attribute__((ext_vector_type(1)));
};

__device__ __forceinline__ long long token_at(const void* tokens, bool wide, size_t i)
{
    return wide ? static_cast<const long long*>(tokens)[i] : static_cast<const int*>(tokens)[i];
}

template <class T, int VEC>
__device__ __forceinline__ typename Piece<T, VEC>::type scaled(typename Piece<T, VEC>::type v, float scale)
{
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = (T)((float)v[e] * scale);
    return v;
}

// ---------------------------------------------------------------- lookup

// Rows as they are, in pieces of VEC elements, kEach a thread; the last piece of a row ends with the row (where that does not hold
// a whole number of pieces it overlaps the one before, with the same values).
template <class T, int VEC>
__global__ __launch_bounds__(kThreads) void embed_rows_kernel(EmbedArgs a, unsigned per_row, unsigned long long pieces)
{
    typedef typename Piece<T, VEC>::type V;
    constexpr int kEach = 4;
    const unsigned long long base = (unsigned long long)blockIdx.x * (kThreads * kEach);
    const unsigned long long first = base >> 32 ? base / per_row : (unsigned)base / per_row;
    const unsigned in_row = (unsigned)(base - first * per_row);
    const T* table = static_cast<const T*>(a.table);
    T* out = static_cast<T*>(a.out);
    unsigned long long place[kEach];
    unsigned d[kEach];
    long long v[kEach];
    V piece[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const unsigned p = in_row + i * kThreads + threadIdx.x, row = p / per_row;
        place[i] = first + row;
        d[i] = min((p - row * per_row) * VEC, (unsigned)a.dim - VEC);
        v[i] = base + i * kThreads + threadIdx.x < pieces ? token_at(a.tokens, a.wide, place[i]) : -1;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        piece[i] = V{};
        if (v[i] >= 0 && v[i] < a.vocab) piece[i] = *reinterpret_cast<const V*>(table + (size_t)v[i] * a.dim + d[i]);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (base + i * kThreads + threadIdx.x < pieces) *reinterpret_cast<V*>(out + place[i] * a.dim + d[i]) = scaled<T, VEC>(piece[i], a.scale);
}

// A tile of kWords words by kDims dimensions, turned in LDS between rows of vectors and rows of words.  Pieces of 16 bytes on either
// side; the pitch is odd (in words of 4 bytes), so that neither side's columns share a bank.
template <class T>
struct Turn {
    static constexpr int kVec = 16 / sizeof(T), kWords = 64, kDims = 16 * kVec, kPitch = sizeof(T) == 4 ? kWords + 1 : kWords + 2;
    typedef typename Piece<T, kVec>::type V;
    static constexpr int kPasses = kWords * 16 / kThreads;      // 16 pieces a word's row; as many pieces the other way
};

// The piece of `count` elements from p on, zeros past them.
template <class T, int VEC>
__device__ __forceinline__ typename Piece<T, VEC>::type load_some(const T* p, int count)
{
    typedef typename Piece<T, VEC>::type V;
    if (count >= VEC) return *reinterpret_cast<const V*>(p);
    V v = V{};
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        if (e < count) v[e] = p[e];
    return v;
}

template <class T, int VEC>
__device__ __forceinline__ void store_some(T* p, typename Piece<T, VEC>::type v, int count)
{
    typedef typename Piece<T, VEC>::type V;
    if (count >= VEC) {
        *reinterpret_cast<V*>(p) = v;
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (e < count) p[e] = v[e];
    }
}

// Tile number -> sentence, first word, first dimension.
__device__ __forceinline__ void tile_at(unsigned tile, int words, int dim, int per_words, int per_dims, size_t& n, int& w0, int& d0)
{
    const unsigned across = (dim + per_dims - 1) / per_dims, along = (words + per_words - 1) / per_words;
    d0 = (int)(tile % across) * per_dims;
    w0 = (int)(tile / across % along) * per_words;
    n = tile / across / along;
}

// Vectors channels first: [sentence][dimension][word].
template <class T>
__global__ __launch_bounds__(kThreads) void embed_turned_kernel(EmbedArgs a)
{
    typedef Turn<T> U;
    typedef typename U::V V;
    __shared__ T tile[U::kDims * U::kPitch];
    size_t n;
    int w0, d0;
    tile_at(blockIdx.x, a.words, a.dim, U::kWords, U::kDims, n, w0, d0);
    const T* table = static_cast<const T*>(a.table);
    V piece[U::kPasses];
    const int p = threadIdx.x & 15, d = d0 + p * U::kVec;
#pragma unroll
    for (int i = 0; i < U::kPasses; ++i) {
        const int w = i * (kThreads / 16) + (threadIdx.x >> 4);
        const long long v = w0 + w < a.words ? token_at(a.tokens, a.wide, n * a.words + w0 + w) : -1;
        piece[i] = V{};
        if (v >= 0 && v < a.vocab) piece[i] = load_some<T, U::kVec>(table + (size_t)v * a.dim + d, a.dim - d);
    }
#pragma unroll
    for (int i = 0; i < U::kPasses; ++i) {
        const int w = i * (kThreads / 16) + (threadIdx.x >> 4);
#pragma unroll
        for (int e = 0; e < U::kVec; ++e) tile[(p * U::kVec + e) * U::kPitch + w] = (T)((float)piece[i][e] * a.scale);
    }
    __syncthreads();
    T* out = static_cast<T*>(a.out);
    constexpr int kAlong = U::kWords / U::kVec;
#pragma unroll
    for (int i = 0; i < U::kPasses; ++i) {
        const int at = i * kThreads + threadIdx.x, row = at / kAlong, w = at % kAlong * U::kVec;
        if (d0 + row >= a.dim || w0 + w >= a.words) continue;
        V v;
#pragma unroll
        for (int e = 0; e < U::kVec; ++e) v[e] = tile[row * U::kPitch + w + e];
        store_some<T, U::kVec>(out + (n * a.dim + d0 + row) * a.words + w0 + w, v, a.words - w0 - w);
    }
}

template <class T>
int launch_lookup(const EmbedArgs& a, hipStream_t s)
{
    if (a.channels_first && a.words > 1) {
        typedef Turn<T> U;
        const long long tiles = (long long)a.sentences * ((a.words + U::kWords - 1) / U::kWords) * ((a.dim + U::kDims - 1) / U::kDims);
        if (tiles >= (1ll << 31)) return (int)hipErrorInvalidValue;
        hipLaunchKernelGGL(embed_turned_kernel<T>, dim3((unsigned)tiles), dim3(kThreads), 0, s, a);
        return (int)hipGetLastError();
    }
    constexpr int kVec = 16 / sizeof(T);
    const unsigned per_row = a.dim >= kVec ? (a.dim + kVec - 1) / kVec : a.dim;
    const unsigned long long pieces = (unsigned long long)a.sentences * a.words * per_row, blocks = (pieces + 4 * kThreads - 1) / (4 * kThreads);
    if (blocks >= (1ull << 31)) return (int)hipErrorInvalidValue;
    if (a.dim >= kVec) hipLaunchKernelGGL((embed_rows_kernel<T, kVec>), dim3((unsigned)blocks), dim3(kThreads), 0, s, a, per_row, pieces);
    else hipLaunchKernelGGL((embed_rows_kernel<T, 1>), dim3((unsigned)blocks), dim3(kThreads), 0, s, a, per_row, pieces);
    return (int)hipGetLastError();
}

// ---------------------------------------------------------------- gradient: rows of the table

// A wavefront sums 512 columns of rows of grad, lane l columns 4 l .. + 3 and 256 + 4 l .. + 3 of them.
constexpr int kColumns = 512;

struct Columns {
    int first[2], count[2];      // the lane's columns: where they start, how many of the four are there
};

__device__ __forceinline__ Columns columns_of(int block, int lane, int dim)
{
    Columns c;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        c.first[s] = block * kColumns + s * 256 + lane * 4;
        c.count[s] = min(max(dim - c.first[s], 0), 4);
    }
    return c;
}

struct Sums {
    float v[2][4];
};

__device__ __forceinline__ void clear(Sums& sums)
{
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums.v[s][e] = 0.f;
}

template <class G>
struct Row {
    typename Piece<G, 4>::type v[2];
};

template <class G>
__device__ __forceinline__ Row<G> load_row(const G* row, const Columns& c)
{
    Row<G> r;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        r.v[s] = typename Piece<G, 4>::type{};
        if (c.count[s] > 0) r.v[s] = load_some<G, 4>(row + c.first[s], c.count[s]);
    }
    return r;
}

template <class G>
__device__ __forceinline__ void add(Sums& sums, const Row<G>& r)
{
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums.v[s][e] += (float)r.v[s][e];
}

// Adds rows at(0) .. at(count - 1) in that order, eight loads ahead.
template <class G, class At>
__device__ __forceinline__ void add_rows(Sums& sums, int count, const Columns& c, At at)
{
    constexpr int kAhead = 8;
    int i = 0;
#pragma unroll 1
    for (; i + kAhead <= count; i += kAhead) {
        Row<G> r[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) r[u] = load_row<G>(at(i + u), c);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) add(sums, r[u]);
    }
    if (i < count) {
        Row<G> r[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < count) r[u] = load_row<G>(at(i + u), c);
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < count) add(sums, r[u]);
    }
}

template <class W>
__device__ __forceinline__ void store_row(W* row, const Sums& sums, const Columns& c, float scale, bool accumulate)
{
    Row<W> held;
    if (accumulate) held = load_row<W>(row, c);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        if (c.count[s] <= 0) continue;
        typename Piece<W, 4>::type v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (W)(accumulate ? (float)held.v[s][e] + sums.v[s][e] * scale : sums.v[s][e] * scale);
        store_some<W, 4>(row + c.first[s], v, c.count[s]);
    }
}

// ---------------------------------------------------------------- gradient of few tokens: one launch

// Workgroup (b, c) owns rows b, b + gridDim.x, ... of the table (frequent tokens are often neighbours) and column block c.  It looks
// through all tokens, keeps those of its rows in their order, and each wavefront sums the rows of its turn; a row of many tokens is
// shared by all wavefronts, each a run of them, and joined in their order.
constexpr int kFewTokens = 8192, kFewThreads = 1024, kFewWaves = kFewThreads / 64, kShared = 32;

template <class G, class W>
__global__ __launch_bounds__(kFewThreads) void embed_grad_few_kernel(EmbedGradArgs a, const G* grad)
{
    __shared__ int row_of[kFewTokens], place_of[kFewTokens];
    __shared__ int counts[kFewWaves + 1];
    __shared__ float part[kFewWaves][kColumns];
    __shared__ int long_rows[kFewTokens / kShared + 1], long_count;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tokens = a.sentences * a.words, groups = gridDim.x;
    constexpr int kPasses = kFewTokens / kFewThreads;
    const int per_wave = (tokens + kFewThreads - 1) / kFewThreads * 64;      // tokens of a wavefront, in 64s
    // Rows are numbered within the workgroup: v = b + number * groups.
    int number[kPasses];
    unsigned long long mine[kPasses];
    int count = 0;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int t = wave * per_wave + i * 64 + lane;
        number[i] = -1;
        if (i * 64 < per_wave && t < tokens) {
            const long long v = token_at(a.tokens, a.wide, t);
            if (v >= 0 && v < a.vocab && v != a.padding && (unsigned)v % (unsigned)groups == blockIdx.x) number[i] = (int)((unsigned)v / (unsigned)groups);
        }
    }
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        mine[i] = __ballot(number[i] >= 0);
        count += __popcll(mine[i]);
    }
    if (lane == 0) counts[wave] = count;
    if (threadIdx.x == 0) long_count = 0;
    __syncthreads();
    int at = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
        at += w < wave ? counts[w] : 0;
        total += counts[w];
    }
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        if (number[i] >= 0) {
            const int to = at + __popcll(mine[i] & ((1ull << lane) - 1));
            row_of[to] = number[i];
            place_of[to] = wave * per_wave + i * 64 + lane;
        }
        at += __popcll(mine[i]);
    }
    __syncthreads();

    const Columns c = columns_of(blockIdx.y, lane, a.dim);
    W* table_grad = static_cast<W*>(a.table_grad);
    const int rows = (int)((a.vocab - blockIdx.x + groups - 1) / groups);
    for (int r = wave; r < rows; r += kFewWaves) {
        int found = 0;
        for (int j = 0; j < total; j += 64) found += __popcll(__ballot(j + lane < total && row_of[j + lane] == r));
        if (found > kShared) {
            if (lane == 0) long_rows[atomicAdd(&long_count, 1)] = r;
            continue;
        }
        if (found == 0 && a.accumulate) continue;
        Sums sums;
        clear(sums);
        for (int j = 0; found > 0; j += 64) {
            unsigned long long match = __ballot(j + lane < total && row_of[j + lane] == r);
            const int here = __popcll(match);
            add_rows<G>(sums, here, c, [&](int) {
                const int bit = __ffsll((long long)match) - 1;
                match &= match - 1;
                return grad + (size_t)__builtin_amdgcn_readfirstlane(place_of[j + bit]) * a.dim;
            });
            found -= here;
        }
        store_row<W>(table_grad + ((size_t)blockIdx.x + (size_t)r * groups) * a.dim, sums, c, a.scale, a.accumulate);
    }
    __syncthreads();
    const int shared_rows = long_count;
    for (int l = 0; l < shared_rows; ++l) {
        const int r = long_rows[l];
        int found = 0;
        for (int j = 0; j < total; j += 64) found += __popcll(__ballot(j + lane < total && row_of[j + lane] == r));
        // this wavefront's run of the row's tokens
        const int from = (int)((long long)found * wave / kFewWaves), to = (int)((long long)found * (wave + 1) / kFewWaves);
        Sums sums;
        clear(sums);
        int seen = 0;
        for (int j = 0; j < total && seen < to; j += 64) {
            unsigned long long match = __ballot(j + lane < total && row_of[j + lane] == r);
            const int here = __popcll(match), skip = max(0, from - seen), keep = min(here, to - seen) - skip;
            for (int k = 0; k < skip && match; ++k) match &= match - 1;
            if (keep > 0)
                add_rows<G>(sums, keep, c, [&](int) {
                    const int bit = __ffsll((long long)match) - 1;
                    match &= match - 1;
                    return grad + (size_t)__builtin_amdgcn_readfirstlane(place_of[j + bit]) * a.dim;
                });
            seen += here;
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[wave][s * 256 + lane * 4 + e] = sums.v[s][e];
        __syncthreads();
        if (wave == 0) {
            clear(sums);
            for (int w = 0; w < kFewWaves; ++w)
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sums.v[s][e] += part[w][s * 256 + lane * 4 + e];
            store_row<W>(table_grad + ((size_t)blockIdx.x + (size_t)r * groups) * a.dim, sums, c, a.scale, a.accumulate);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- gradient of many tokens: a sort, then rows

// A stable sort of (token, place) by the token, kDigit bits a pass from the lowest on: each workgroup counts the digits of its run
// of tokens; then each finds, from all counts, where its tokens of each digit go, and takes them there in their order.  Tokens that
// add to no row get the number `vocab` and end up last.
constexpr int kMaxDigit = 10, kSortThreads = 1024, kSortWaves = kSortThreads / 64;

struct SortPlan {
    int passes, digit, per_group, groups;     // bits a digit, tokens a workgroup
};

SortPlan sort_plan(long long vocab, long long tokens)
{
    int bits = 1;
    while (vocab >> bits) ++bits;             // of the numbers 0 .. vocab
    SortPlan p;
    p.passes = (bits + kMaxDigit - 1) / kMaxDigit;
    p.digit = (bits + p.passes - 1) / p.passes;
    long long each = kSortThreads;
    while (tokens > each * 256) each *= 2;    // (every workgroup reads the counts of all)
    p.per_group = (int)each;
    p.groups = (int)((tokens + each - 1) / each);
    return p;
}

__device__ __forceinline__ unsigned sort_key(const EmbedGradArgs& a, unsigned t)
{
    const long long v = token_at(a.tokens, a.wide, t);
    return v >= 0 && v < a.vocab && v != a.padding ? (unsigned)v : (unsigned)a.vocab;
}

// keys: null in the first pass, which reads the tokens.
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(EmbedGradArgs a, const unsigned* keys, int* counts, SortPlan plan, int shift)
{
    __shared__ int bins[1 << kMaxDigit];
    const int size = 1 << plan.digit, tokens = a.sentences * a.words;
    for (int d = threadIdx.x; d < size; d += kSortThreads) bins[d] = 0;
    __syncthreads();
    const unsigned from = blockIdx.x * (unsigned)plan.per_group, to = min((unsigned)tokens, from + (unsigned)plan.per_group);
    for (unsigned t = from + threadIdx.x; t < to; t += kSortThreads) atomicAdd(&bins[((keys ? keys[t] : sort_key(a, t)) >> shift) & (size - 1)], 1);
    __syncthreads();
    for (int d = threadIdx.x; d < size; d += kSortThreads) counts[(size_t)blockIdx.x * size + d] = bins[d];
}

__global__ __launch_bounds__(kSortThreads) void sort_move_kernel(EmbedGradArgs a, const unsigned* keys, const int* places, const int* counts,
                                                                 unsigned* keys_out, int* places_out, SortPlan plan, int shift)
{
    static_assert(kSortThreads >= 1 << kMaxDigit, "a digit a thread");
    __shared__ int of_wave[kSortWaves][1 << kMaxDigit];
    __shared__ int wave_total[kSortWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int size = 1 << plan.digit, tokens = a.sentences * a.words, digit = threadIdx.x;

    // where this workgroup's first token of `digit` goes: all smaller digits, then the same digit in the workgroups before
    int before = 0, total = 0;
    if (digit < size)
        for (int g = 0; g < plan.groups; ++g) {
            const int n = counts[(size_t)g * size + digit];
            before += g < (int)blockIdx.x ? n : 0;
            total += n;
        }
    int sum = total;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int n = __shfl_up(sum, d);
        sum += lane >= d ? n : 0;
    }
    if (lane == 63) wave_total[wave] = sum;
    __syncthreads();
    int base = sum - total + before;
    for (int w = 0; w < wave; ++w) base += wave_total[w];

    const unsigned from = blockIdx.x * (unsigned)plan.per_group, to = min((unsigned)tokens, from + (unsigned)plan.per_group);
    for (unsigned start = from; start < to; start += kSortThreads) {
        const unsigned t = start + threadIdx.x;
        const bool there = t < to;
        const unsigned key = !there ? 0u : keys ? keys[t] : sort_key(a, t);
        const int place = !there ? 0 : keys ? places[t] : (int)t;
        const int mine = (int)((key >> shift) & (unsigned)(size - 1));
        // the lanes of this wavefront with the same digit
        unsigned long long same = __ballot(there);
        for (int b = 0; b < plan.digit; ++b) {
            const unsigned long long set = __ballot(mine >> b & 1);
            same &= mine >> b & 1 ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        for (int w = 0; w < kSortWaves; ++w)
            if (digit < size) of_wave[w][digit] = 0;
        __syncthreads();
        if (there && rank == 0) of_wave[wave][mine] = __popcll(same);
        __syncthreads();
        if (digit < size)
            for (int w = 0; w < kSortWaves; ++w) {
                const int n = of_wave[w][digit];
                of_wave[w][digit] = base;
                base += n;
            }
        __syncthreads();
        if (there) {
            const int at = of_wave[wave][mine] + rank;
            keys_out[at] = key;
            places_out[at] = place;
        }
        __syncthreads();
    }
}

// Sums of kWindow sorted tokens in a row, where they are of one row of the table.
constexpr int kWindow = 32;

template <class G>
__global__ __launch_bounds__(kThreads) void window_kernel(EmbedGradArgs a, const G* grad, const unsigned* keys, const int* places, float* windows, int column_blocks)
{
    const int lane = threadIdx.x & 63;
    const long long unit = (long long)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long w = unit / column_blocks, first = w * kWindow;
    if (first + kWindow > (long long)a.sentences * a.words) return;
    const unsigned key = keys[first];
    if (key != keys[first + kWindow - 1] || key >= (unsigned)a.vocab) return;
    const Columns c = columns_of((int)(unit % column_blocks), lane, a.dim);
    Sums sums;
    clear(sums);
    add_rows<G>(sums, kWindow, c, [&](int i) { return grad + (size_t)places[first + i] * a.dim; });
    store_row<float>(windows + w * a.dim, sums, c, 1.f, false);
}

// The first of `count` sorted keys that is not below v.
__device__ __forceinline__ int lower_bound(const unsigned* keys, int count, unsigned v)
{
    int from = 0, length = count;
    while (length > 0) {
        const int half = length / 2;
        const bool below = keys[from + half] < v;
        from = below ? from + half + 1 : from;
        length = below ? length - half - 1 : half;
    }
    return from;
}

// A wavefront takes kRows rows of the table and one column block: lane l looks for the tokens of row l, then the rows go one by one.
// Its rows are `sets` apart: frequent tokens are often neighbours.
constexpr int kRows = 32;

template <class G, class W>
__global__ __launch_bounds__(kThreads) void rows_kernel(EmbedGradArgs a, const G* grad, const unsigned* keys, const int* places, const float* windows, int column_blocks,
                                                        unsigned sets)
{
    const int lane = threadIdx.x & 63, tokens = a.sentences * a.words;
    const long long unit = (long long)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned set = (unsigned)(unit / column_blocks);
    if (set >= sets) return;
    // lanes 0 .. 31: where the tokens of row l begin; lanes 32 .. 63: where they end
    const long long row = (long long)set + (long long)(lane % kRows) * sets;
    const int bound = row < a.vocab ? lower_bound(keys, tokens, (unsigned)row + lane / kRows) : 0;
    const Columns c = columns_of((int)(unit % column_blocks), lane, a.dim);
    W* table_grad = static_cast<W*>(a.table_grad);
    for (int r = 0; r < kRows; ++r) {
        const long long v = (long long)set + (long long)r * sets;
        if (v >= a.vocab) break;
        const int from = __builtin_amdgcn_readlane(bound, r), to = __builtin_amdgcn_readlane(bound, r + kRows);
        if (from == to && a.accumulate) continue;
        Sums sums;
        clear(sums);
        const int first = (from + kWindow - 1) / kWindow, last = to / kWindow;
        auto row_at = [&](int i) { return grad + (size_t)places[i] * a.dim; };
        if (first < last) {
            add_rows<G>(sums, first * kWindow - from, c, [&](int i) { return row_at(from + i); });
            add_rows<float>(sums, last - first, c, [&](int i) { return windows + (size_t)(first + i) * a.dim; });
            add_rows<G>(sums, to - last * kWindow, c, [&](int i) { return row_at(last * kWindow + i); });
        } else {
            add_rows<G>(sums, to - from, c, [&](int i) { return row_at(from + i); });
        }
        store_row<W>(table_grad + (size_t)v * a.dim, sums, c, a.scale, a.accumulate);
    }
}

// ---------------------------------------------------------------- gradient: channels first

// [sentence][dimension][word] to rows of vectors.
template <class G>
__global__ __launch_bounds__(kThreads) void turn_kernel(EmbedGradArgs a, G* rows)
{
    typedef Turn<G> U;
    typedef typename U::V V;
    __shared__ G tile[U::kDims * U::kPitch];
    size_t n;
    int w0, d0;
    tile_at(blockIdx.x, a.words, a.dim, U::kWords, U::kDims, n, w0, d0);
    const G* grad = static_cast<const G*>(a.grad);
    constexpr int kAlong = U::kWords / U::kVec;
    V piece[U::kPasses];
#pragma unroll
    for (int i = 0; i < U::kPasses; ++i) {
        const int at = i * kThreads + threadIdx.x, row = at / kAlong, w = at % kAlong * U::kVec;
        piece[i] = V{};
        if (d0 + row < a.dim && w0 + w < a.words) piece[i] = load_some<G, U::kVec>(grad + (n * a.dim + d0 + row) * a.words + w0 + w, a.words - w0 - w);
    }
#pragma unroll
    for (int i = 0; i < U::kPasses; ++i) {
        const int at = i * kThreads + threadIdx.x, row = at / kAlong, w = at % kAlong * U::kVec;
#pragma unroll
        for (int e = 0; e < U::kVec; ++e) tile[row * U::kPitch + w + e] = piece[i][e];
    }
    __syncthreads();
    const int p = threadIdx.x & 15, d = d0 + p * U::kVec;
#pragma unroll
    for (int i = 0; i < U::kPasses; ++i) {
        const int w = i * (kThreads / 16) + (threadIdx.x >> 4);
        if (w0 + w >= a.words || d >= a.dim) continue;
        V v;
#pragma unroll
        for (int e = 0; e < U::kVec; ++e) v[e] = tile[(p * U::kVec + e) * U::kPitch + w];
        store_some<G, U::kVec>(rows + (n * a.words + w0 + w) * a.dim + d, v, a.dim - d);
    }
}

int type_bytes(int dtype) { return dtype == kF32 ? 4 : 2; }
long long rounded(long long bytes) { return (bytes + 255) / 256 * 256; }

// What the workspace holds, in this order.
struct Parts {
    long long rows, keys, counts, windows, total;      // bytes; keys: of each of two pairs of (token, place)
};

Parts parts_of(const EmbedGradArgs& a, int grad_dtype)
{
    const long long tokens = (long long)a.sentences * a.words;
    Parts p{};
    if (a.channels_first && a.words > 1) p.rows = rounded(tokens * a.dim * type_bytes(grad_dtype));
    if (tokens > kFewTokens) {
        const SortPlan plan = sort_plan(a.vocab, tokens);
        p.keys = rounded(tokens * 4);
        p.counts = rounded((long long)plan.groups * (1 << plan.digit) * 4);
        p.windows = rounded(tokens / kWindow * a.dim * 4);
    }
    p.total = p.rows + 4 * p.keys + p.counts + p.windows;
    return p;
}

template <class G, class W>
int launch_grad(const EmbedGradArgs& a, const Parts& parts, hipStream_t s)
{
    const long long tokens = (long long)a.sentences * a.words;
    const G* grad = static_cast<const G*>(a.grad);
    if (parts.rows) {
        typedef Turn<G> U;
        const long long tiles = (long long)a.sentences * ((a.words + U::kWords - 1) / U::kWords) * ((a.dim + U::kDims - 1) / U::kDims);
        if (tiles >= (1ll << 31)) return (int)hipErrorInvalidValue;
        G* rows = reinterpret_cast<G*>(a.workspace);
        hipLaunchKernelGGL(turn_kernel<G>, dim3((unsigned)tiles), dim3(kThreads), 0, s, a, rows);
        grad = rows;
    }
    const long long column_blocks = ((long long)a.dim + kColumns - 1) / kColumns;
    if (tokens <= kFewTokens) {
        if (column_blocks > 65535) return (int)hipErrorInvalidValue;
        const unsigned groups = (unsigned)std::min<long long>(a.vocab, 256);
        hipLaunchKernelGGL((embed_grad_few_kernel<G, W>), dim3(groups, (unsigned)column_blocks), dim3(kFewThreads), 0, s, a, grad);
        return (int)hipGetLastError();
    }
    const SortPlan plan = sort_plan(a.vocab, tokens);
    char* at = a.workspace + parts.rows;
    unsigned* keys[2];
    int* places[2];
    for (int i = 0; i < 2; ++i) {
        keys[i] = reinterpret_cast<unsigned*>(at);
        places[i] = reinterpret_cast<int*>(at + parts.keys);
        at += 2 * parts.keys;
    }
    int* counts = reinterpret_cast<int*>(at);
    float* windows = reinterpret_cast<float*>(at + parts.counts);
    const unsigned *from = nullptr;
    const int* from_places = nullptr;
    for (int pass = 0; pass < plan.passes; ++pass) {
        hipLaunchKernelGGL(sort_count_kernel, dim3(plan.groups), dim3(kSortThreads), 0, s, a, from, counts, plan, pass * plan.digit);
        hipLaunchKernelGGL(sort_move_kernel, dim3(plan.groups), dim3(kSortThreads), 0, s, a, from, from_places, counts, keys[pass & 1], places[pass & 1], plan,
                           pass * plan.digit);
        from = keys[pass & 1];
        from_places = places[pass & 1];
    }
    constexpr int kWaves = kThreads / 64;
    const long long window_units = tokens / kWindow * column_blocks, sets = (a.vocab + kRows - 1) / kRows, row_units = sets * column_blocks;
    if ((window_units + kWaves - 1) / kWaves >= (1ll << 31) || (row_units + kWaves - 1) / kWaves >= (1ll << 31)) return (int)hipErrorInvalidValue;
    hipLaunchKernelGGL(window_kernel<G>, dim3((unsigned)((window_units + kWaves - 1) / kWaves)), dim3(kThreads), 0, s, a, grad, from, from_places, windows,
                       (int)column_blocks);
    hipLaunchKernelGGL((rows_kernel<G, W>), dim3((unsigned)((row_units + kWaves - 1) / kWaves)), dim3(kThreads), 0, s, a, grad, from, from_places, windows,
                       (int)column_blocks, (unsigned)sets);
    return (int)hipGetLastError();
}

// No tokens: all rows are zero.
template <class W>
__global__ __launch_bounds__(kThreads) void zero_kernel(W* out, unsigned long long count)
{
    for (unsigned long long i = (unsigned long long)blockIdx.x * kThreads + threadIdx.x; i < count; i += (unsigned long long)gridDim.x * kThreads) out[i] = (W)0.f;
}

}  // namespace

int launch_embed(int dtype, const EmbedArgs& a, void* stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == kF32) return launch_lookup<float>(a, s);
    if (dtype == kF16) return launch_lookup<_Float16>(a, s);
    return launch_lookup<__bf16>(a, s);
}

long long embed_grad_workspace(const EmbedGradArgs& a, int grad_dtype) { return parts_of(a, grad_dtype).total; }

int launch_embed_grad(int grad_dtype, int table_dtype, const EmbedGradArgs& a, void* stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if ((long long)a.sentences * a.words == 0) {
        const unsigned long long count = (unsigned long long)a.vocab * a.dim;
        const dim3 grid((unsigned)std::min<unsigned long long>((count + kThreads - 1) / kThreads, 16384));
        if (table_dtype == kF32) hipLaunchKernelGGL(zero_kernel<float>, grid, dim3(kThreads), 0, s, static_cast<float*>(a.table_grad), count);
        else hipLaunchKernelGGL(zero_kernel<_Float16>, grid, dim3(kThreads), 0, s, static_cast<_Float16*>(a.table_grad), count);
        return (int)hipGetLastError();
    }
    const Parts parts = parts_of(a, grad_dtype);
    if (grad_dtype == kF32) return launch_grad<float, float>(a, parts, s);
    if (grad_dtype == kF16) return table_dtype == kF32 ? launch_grad<_Float16, float>(a, parts, s) : launch_grad<_Float16, _Float16>(a, parts, s);
    return table_dtype == kF32 ? launch_grad<__bf16, float>(a, parts, s) : launch_grad<__bf16, __bf16>(a, parts, s);
}

}  // namespace sc

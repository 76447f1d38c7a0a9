// Word vectors and their gradient (sparse_conv_embed, sparse_conv_embed_backward).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "text_ops.h"

namespace sc {

namespace {

enum { kF32 = 0, kF16 = 1, kBF16 = 2 };   // SC_F32, SC_F16, SC_BF16

constexpr int kThreads = 256;
constexpr unsigned long long kCacheBytes = 256ull << 20;      // of the last-level cache

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

// A barrier for what the wavefronts of a workgroup exchange through LDS; stores to memory may still be on their way.
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
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
// PASSING: the output is larger than the caches and goes past them (64k rows of 4096 in bfloat16: 139 us instead of 149).
template <class T, int VEC, bool PASSING>
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
        if (base + i * kThreads + threadIdx.x < pieces) {
            V* to = reinterpret_cast<V*>(out + place[i] * a.dim + d[i]);
            if (PASSING) __builtin_nontemporal_store(scaled<T, VEC>(piece[i], a.scale), to);
            else *to = scaled<T, VEC>(piece[i], a.scale);
        }
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
    const unsigned across = ((unsigned)dim + per_dims - 1) / per_dims, along = ((unsigned)words + per_words - 1) / per_words;
    d0 = (int)(tile % across) * per_dims;
    w0 = (int)(tile / across % along) * per_words;
    n = tile / across / along;
}

// (Sizes go up to 2^31 - 1: what rounds them up does not do so in int.)
template <class U>
long long tiles_of(int sentences, int words, int dim)
{
    return (long long)sentences * ((words + (U::kWords - 1ll)) / U::kWords) * ((dim + (U::kDims - 1ll)) / U::kDims);
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
        const long long tiles = tiles_of<Turn<T>>(a.sentences, a.words, a.dim);
        if ((unsigned long long)tiles > most_groups(kThreads)) return kTooLarge;
        hipLaunchKernelGGL(embed_turned_kernel<T>, dim3((unsigned)tiles), dim3(kThreads), 0, s, a);
        return (int)hipGetLastError();
    }
    constexpr int kVec = 16 / sizeof(T);
    const unsigned per_row = a.dim >= kVec ? ((unsigned)a.dim + kVec - 1) / kVec : a.dim;
    const unsigned long long pieces = (unsigned long long)a.sentences * a.words * per_row, blocks = (pieces + 4 * kThreads - 1) / (4 * kThreads);
    if (blocks > most_groups(kThreads)) return kTooLarge;
    const bool passing = pieces * 16 > kCacheBytes;
    auto kernel = a.dim < kVec ? embed_rows_kernel<T, 1, false> : passing ? embed_rows_kernel<T, kVec, true> : embed_rows_kernel<T, kVec, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kThreads), 0, s, a, per_row, pieces);
    return (int)hipGetLastError();
}

// ---------------------------------------------------------------- gradient: rows of the table

// A wavefront sums 512 columns of rows of grad, lane l columns 4 l .. + 3 and 256 + 4 l .. + 3 of them.  A lane whose four are not all
// there takes the last four of the block instead: loads and stores need no branch for it, and it writes the same values as its
// neighbours.  Rows of less than four columns: a column a lane.
constexpr int kColumns = 512;

struct Columns {
    int offset[2];                // where the lane reads and writes
    bool own[2];                  // some of these columns are its own
    bool both, narrow;            // the second 256 are there; rows of less than four columns
};

__device__ __forceinline__ Columns columns_of(int block, int lane, int dim)
{
    Columns c;
    int begin = block * kColumns, end = begin + min(kColumns, dim - begin);
    c.narrow = dim < 4;
    if (end < dim && dim - end < 4) end = dim - 4;            // (a last block of less than four columns takes some of the one before)
    if (block > 0 && dim - begin < 4) begin = dim - 4;
    c.both = end - begin > 256;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int first = begin + s * 256 + lane * 4;
        c.own[s] = first < end;
        c.offset[s] = min(first, end - 4);
    }
    if (c.narrow) {
        c.own[0] = lane < dim;
        c.offset[0] = min(lane, dim - 1);
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
    typedef typename Piece<G, 4>::type V;
    Row<G> r;
    if (c.narrow) {
        r.v[0] = V{};
        r.v[0][0] = row[c.offset[0]];
    } else {
        r.v[0] = *reinterpret_cast<const V*>(row + c.offset[0]);
        if (c.both) r.v[1] = *reinterpret_cast<const V*>(row + c.offset[1]);
    }
    return r;
}

template <class G>
__device__ __forceinline__ void add(Sums& sums, const Row<G>& r, const Columns& c)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) sums.v[0][e] += (float)r.v[0][e];
    if (c.both)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums.v[1][e] += (float)r.v[1][e];
}

template <class W>
__device__ __forceinline__ void store_row(W* row, const Sums& sums, const Columns& c, float scale, bool accumulate)
{
    typedef typename Piece<W, 4>::type V;
    Row<W> held;
    if (accumulate) held = load_row<W>(row, c);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        if (s == 1 && !c.both) break;
        V v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (W)(accumulate ? (float)held.v[s][e] + sums.v[s][e] * scale : sums.v[s][e] * scale);
        if (!c.own[s]) continue;
        if (s == 0 && c.narrow) row[c.offset[0]] = v[0];
        else *reinterpret_cast<V*>(row + c.offset[s]) = v;
    }
}

constexpr int kAhead = 8;       // rows that a wavefront loads before it adds the first of them

// Adds the rows that begin at grad + place_at(0) * dim .. grad + place_at(count - 1) * dim, in that order.
template <class G, class PlaceAt>
__device__ __forceinline__ void add_rows(Sums& sums, const G* grad, int dim, int count, const Columns& c, PlaceAt place_at)
{
    const int lane = threadIdx.x & 63;
#pragma unroll 1
    for (int start = 0; start < count; start += 64) {
        const int place = start + lane < count ? place_at(start + lane) : 0, here = min(count - start, 64);
#pragma unroll 1
        for (int i = 0; i < here; i += kAhead) {
            Row<G> r[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (i + u < here) r[u] = load_row<G>(grad + (size_t)(unsigned)__builtin_amdgcn_readlane(place, i + u) * dim, c);
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (i + u < here) add(sums, r[u], c);
        }
    }
}

// One past the last of the sorted keys that equals that of `from`: 64 probes at a time, further apart until one differs, then closer.
template <class KeyAt>
__device__ __forceinline__ unsigned end_of_run(KeyAt key_at, unsigned from, unsigned count)
{
    const int lane = threadIdx.x & 63;
    const unsigned key = key_at(from);
    unsigned long long last = from, step = 1;
    auto probe = [&]() {
        const unsigned long long at = last + (unsigned long long)(lane + 1) * step;
        const int same = __popcll(__ballot(at < count && key_at((unsigned)min(at, (unsigned long long)count - 1)) == key));
        last += (unsigned long long)same * step;
        return same;
    };
    while (probe() == 64) step *= 64;
    while (step > 1) {
        step /= 64;
        probe();
    }
    return __builtin_amdgcn_readfirstlane((unsigned)last + 1);
}

// The runs of equal keys that begin among sorted tokens first .. first + kSlot - 1 (of `count`; keys from `none` on are no rows): their
// rows are loaded kAhead at a time, whatever runs they belong to.  done(key, sums) for each, but longer(its first token) for one
// of more than kLong tokens.  (us a call by slots of 4, 8 and 16: 32768 tokens to 1000 x 512 floats 31.0, 32.0, 36.0; 65536 to 32768 x 256
// 45.5, 43.0, 46.9; 16384 uniform ones to 32768 x 1024 52.0, 51.0, 53.8.  By runs of up to 16, 32 and 48: 33.1, 32.0, 34.0; 43.9, 43.0,
// 44.4; 16384 uniform ones to 300 x 1024 30.1, 30.3, 34.6.)
constexpr int kSlot = 8, kLong = 32;

template <class G, class KeyAt, class PlaceAt, class Done, class Longer>
__device__ __forceinline__ void add_slot(const G* grad, int dim, const Columns& c, unsigned first, unsigned count, unsigned none, KeyAt key_at, PlaceAt place_at, Done done,
                                         Longer longer)
{
    const int lane = threadIdx.x & 63;
    const unsigned at = first + lane;
    const bool there = at < count;
    const unsigned key = there ? key_at(at) : none;
    const int place = there ? place_at(at) : 0;
    unsigned before = (unsigned)__shfl_up((int)key, 1);
    if (lane == 0) before = first > 0 ? key_at(first - 1) : ~key;
    const unsigned long long begins = __ballot(key != before), heads = begins & __ballot(key < none) & ((1ull << kSlot) - 1);
    if (!heads) return;
    const int from = __ffsll((long long)heads) - 1, last = 63 - __clzll((long long)heads);
    const unsigned long long above = begins & ~((2ull << last) - 1);
    int to = above ? __ffsll((long long)above) - 1 : 64;
    if (!above || to - last > kLong) {
        longer(first + last);
        to = last;
    }
    Sums sums;
    clear(sums);
#pragma unroll 1
    for (int i = from; i < to; i += kAhead) {
        Row<G> r[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < to) r[u] = load_row<G>(grad + (size_t)(unsigned)__builtin_amdgcn_readlane(place, i + u) * dim, c);
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < to) {
                if (i + u > from && (begins >> (i + u) & 1)) {
                    done((unsigned)__builtin_amdgcn_readlane((int)key, i + u - 1), sums);
                    clear(sums);
                }
                add(sums, r[u], c);
            }
    }
    if (from < to) done((unsigned)__builtin_amdgcn_readlane((int)key, to - 1), sums);
}

// What the wavefronts of a workgroup leave to be joined.
__device__ __forceinline__ void leave(const Sums& sums, float (*part)[kColumns])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[wave][s * 256 + lane * 4 + e] = sums.v[s][e];
}

// Adds what `count` wavefronts in a row left, `first` the first of them, in their order.
__device__ __forceinline__ void join(Sums& sums, float (*part)[kColumns], int first, int count)
{
    const int lane = threadIdx.x & 63;
#pragma unroll 4
    for (int w = first; w < first + count; ++w)
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums.v[s][e] += part[w][s * 256 + lane * 4 + e];
}

// ---------------------------------------------------------------- gradient: channels first

// grad of the shape [sentence][dimension][word] to rows of vectors.
struct TurnArgs {
    const void* grad;
    void* rows;
    int dim, sentences, words;
    unsigned tiles;
};

// Each kThreads threads of a workgroup turn a tile: number, number + 1, ...
template <class G>
__device__ __forceinline__ void turn_tiles(const TurnArgs& a, unsigned number, G* room)
{
    typedef Turn<G> U;
    typedef typename U::V V;
    const int thread = threadIdx.x % kThreads, part = threadIdx.x / kThreads;
    G* tile = room + part * U::kDims * U::kPitch;
    const bool works = number + part < a.tiles;
    size_t n;
    int w0, d0;
    tile_at(number + part, a.words, a.dim, U::kWords, U::kDims, n, w0, d0);
    const G* grad = static_cast<const G*>(a.grad);
    constexpr int kAlong = U::kWords / U::kVec;
    if (works) {
        V piece[U::kPasses];
#pragma unroll
        for (int i = 0; i < U::kPasses; ++i) {
            const int at = i * kThreads + thread, row = at / kAlong, w = at % kAlong * U::kVec;
            piece[i] = V{};
            if (d0 + row < a.dim && w0 + w < a.words) piece[i] = load_some<G, U::kVec>(grad + (n * a.dim + d0 + row) * a.words + w0 + w, a.words - w0 - w);
        }
#pragma unroll
        for (int i = 0; i < U::kPasses; ++i) {
            const int at = i * kThreads + thread, row = at / kAlong, w = at % kAlong * U::kVec;
#pragma unroll
            for (int e = 0; e < U::kVec; ++e) tile[row * U::kPitch + w + e] = piece[i][e];
        }
    }
    lds_barrier();
    if (works) {
        const int p = thread & 15, d = d0 + p * U::kVec;
#pragma unroll
        for (int i = 0; i < U::kPasses; ++i) {
            const int w = i * (kThreads / 16) + (thread >> 4);
            if (w0 + w >= a.words || d >= a.dim) continue;
            V v;
#pragma unroll
            for (int e = 0; e < U::kVec; ++e) v[e] = tile[(p * U::kVec + e) * U::kPitch + w];
            store_some<G, U::kVec>(static_cast<G*>(a.rows) + (n * a.words + w0 + w) * a.dim + d, v, a.dim - d);
        }
    }
}

// Elements of the table's gradient to set to zero.
struct Fill {
    void* to;
    unsigned long long count;
};

// The launches of the sort turn tiles and fill in workgroups of their own beside those that sort: it takes the few CUs of a sort a
// while, and most of the table's gradient is zeros, which need nothing of it (rows with tokens are written later).
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kTiles = kSortThreads / kThreads;      // tiles a workgroup

template <class G>
constexpr int tiles_room() { return kTiles * Turn<G>::kDims * Turn<G>::kPitch * (int)sizeof(G); }

// 16 bytes a thread: zeros go out fastest (6.4 TB/s; with 16 stores a thread 6.1, with 4 5.6) as many short workgroups in order.
template <class W>
__device__ __forceinline__ void fill_part(const Fill& f, unsigned number)
{
    constexpr int kVec = 16 / sizeof(W);
    typedef typename Piece<W, kVec>::type V;
    const unsigned long long at = ((unsigned long long)number * kSortThreads + threadIdx.x) * kVec;
    if (at < f.count) store_some<W, kVec>(static_cast<W*>(f.to) + at, V{}, (int)min(f.count - at, (unsigned long long)kVec));
}

template <class G, class W>
__device__ __forceinline__ void turn_or_fill(const TurnArgs& t, const Fill& f, unsigned number, void* room)
{
    const unsigned turning = (t.tiles + kTiles - 1) / kTiles;
    if (number < turning) turn_tiles<G>(t, number * kTiles, static_cast<G*>(room));
    else fill_part<W>(f, number - turning);
}

template <class W>
unsigned long long blocks_of(unsigned tiles, const Fill& f)
{
    const unsigned long long once = (unsigned long long)kSortThreads * (16 / sizeof(W));
    return (tiles + kTiles - 1) / kTiles + (f.count + once - 1) / once;
}

// A stable sort of (token, place) by the token, `digit` bits a pass from the lowest on.  Tokens that add to no row get the number
// `vocab` and end up last.
constexpr int kMaxDigit = 10, kMoveEach = 2;      // tokens of a thread
// Every workgroup that moves tokens reads the counts of all, so that there is a most of them: work grows with the tokens, not their square.
// (2^20 tokens to 131072 x 16: 211 us a call, by twice as many 264, by half 215; 2^24 to 131072 x 4: 3.1 ms, 3.1, 3.4.)
constexpr int kMostGroups = 256;

struct SortPlan {
    int passes, digit;      // bits a digit
    int groups, rounds;     // workgroups, and how many times kMoveEach * kSortThreads tokens in a row each takes
};

SortPlan sort_plan(long long last, int most, long long tokens)      // of keys 0 .. last, by digits of at most `most` bits
{
    int bits = 1;
    while (last >> bits) ++bits;
    SortPlan p;
    p.passes = (bits + most - 1) / most;
    p.digit = (bits + p.passes - 1) / p.passes;
    const long long runs = (tokens + kMoveEach * kSortThreads - 1) / (kMoveEach * kSortThreads);
    p.rounds = (int)((runs + kMostGroups - 1) / kMostGroups);
    p.groups = (int)((runs + p.rounds - 1) / p.rounds);
    return p;
}

struct TokenArgs {
    const void* tokens;
    long long vocab, padding;
    unsigned count;
    bool wide;
};

__device__ __forceinline__ unsigned key_of(const TokenArgs& a, long long token)
{
    return token >= 0 && token < a.vocab && token != a.padding ? (unsigned)token : (unsigned)a.vocab;
}

__device__ __forceinline__ unsigned sort_key(const TokenArgs& a, unsigned t) { return key_of(a, token_at(a.tokens, a.wide, t)); }

// The tokens of a workgroup: `each` runs of 64 a wavefront, in order.
__device__ __forceinline__ unsigned own_token(int each, int i) { return ((threadIdx.x >> 6) * each + i) * 64 + (threadIdx.x & 63); }

// rank[i]: how many tokens of this wavefront with the same digit come before token i; of_wave[wavefront][digit]: how many it has.
template <int EACH, int BITS>
__device__ __forceinline__ void rank_tokens(const unsigned (&key)[EACH], const bool (&there)[EACH], int each, int shift, int bits, int (*of_wave)[1 << BITS], int (&rank)[EACH])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, size = 1 << bits;
    for (int d = lane; d < size; d += 64) of_wave[wave][d] = 0;
    volatile int* mine = of_wave[wave];       // (this wavefront's alone until the next barrier; its LDS accesses stay in order)
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (i >= each) break;
        const int digit = (int)((key[i] >> shift) & (unsigned)(size - 1));
        unsigned long long same = __ballot(there[i]);
        for (int b = 0; b < bits; ++b) {
            const unsigned long long set = __ballot(digit >> b & 1);
            same &= digit >> b & 1 ? set : ~set;
        }
        const int before = __popcll(same & ((1ull << lane) - 1)), held = mine[digit];
        rank[i] = held + before;
        if (there[i] && before == 0) mine[digit] = held + __popcll(same);
    }
}

// Sum of the values of the threads before this one.
__device__ __forceinline__ int sum_before(int value, int* of_wave)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int sum = value;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int n = __shfl_up(sum, d);
        sum += lane >= d ? n : 0;
    }
    if (lane == 63) of_wave[wave] = sum;
    lds_barrier();
    int before = sum - value;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) before += w < wave ? of_wave[w] : 0;
    return before;
}

// Turns the counts of a digit's wavefronts into where each begins, from `base` on, and returns where the last ends.
template <int BITS>
__device__ __forceinline__ int spread(int (*of_wave)[1 << BITS], int digit, int base)
{
    int n[kSortWaves];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) n[w] = of_wave[w][digit];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        of_wave[w][digit] = base;
        base += n[w];
    }
    return base;
}

struct Sorted {
    unsigned* keys;
    int* places;
};

// ---------------------------------------------------------------- gradient of few tokens: one launch, two with a turn or many zeros

// The limit is what the LDS of a workgroup holds of tokens and the registers of a thread of keys.  Few launches pay below it, many CUs
// a row above.  Skewed tokens, us a call this way and by the sort of many tokens: 20000 x 300 floats, 512 tokens 9.8 and 22.9, 2048 11.9
// and 32.0, 8192 20.0 and 38.5; 50021 x 1001 binary16 21.7 and 32.6, 25.7 and 43.2, 41.8 and 47.6.  The limit does not look at the
// width or at the tokens: 32768 x 4096 floats 100 and 102, 127 and 121, 217 and 153; and a row is summed by the one workgroup that owns
// it, so that a token that is half of them costs more (20000 x 300: 36.3 and 29.8 at 2048, 113 and 39.6 at 8192; 32768 x 4096: 1373 and
// 149).  A filler token that is declared as padding costs nothing.
constexpr int kFewTokens = 8192, kBuckets = 256, kBucketBits = 8, kBucketDigit = 9, kMarks = 1 << 15;
constexpr int kFewEach = kFewTokens / kSortThreads;
constexpr unsigned long long kOwnZeros = 64ull << 20;
constexpr unsigned kPairs = 256;
constexpr int kFewBits = 13;
constexpr int kFewAhead = 10;      // rows that a wavefront has in flight (as registers go)

__device__ __forceinline__ long long rows_of(long long vocab, unsigned bucket) { return (vocab - bucket + kBuckets - 1) >> kBucketBits; }

template <int BITS>
struct BucketRoom {
    unsigned keys[kFewTokens];                  // number of the row within the bucket
    unsigned short places[kFewTokens];
    union {
        __attribute__((aligned(16))) unsigned pairs[kPairs];
        int of_wave[kSortWaves][1 << BITS];
    };
    int counts[kSortWaves], earlier[kSortWaves];
};
static_assert(kFewTokens <= 1 << 16, "places of 16 bits");
static_assert(kFewTokens == 1 << kFewBits && kPairs % 4 == 0 && kPairs * 4 == kSortThreads, "numbers of tokens; four at a time, by four lanes");

// Leaves the tokens of a bucket in room.keys and .places, sorted, and returns their number; `marks` (if there) gets a bit for each of
// their rows; start: with EARLIER, the number of tokens of the buckets before.  between() runs when the marks are whole.
template <int BITS, bool EARLIER, class Between>
__device__ __forceinline__ unsigned sort_bucket(const TokenArgs& a, unsigned bucket, int passes, int digit_bits, BucketRoom<BITS>& room, unsigned* marks, unsigned& start,
                                                Between between)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int each = (int)((a.count + kSortThreads - 1) / kSortThreads);
    const long long rows = rows_of(a.vocab, bucket);
    unsigned key[kFewEach], place[kFewEach];
    unsigned long long mine[kFewEach];
    int count = 0, before = 0;
    // All loads before the first use.  Most groups of 64 tokens have none of this workgroup's and get one look at their low
    // bits.  Code that a size has no use for is jumped over (it would be fetched).
    auto look = [&](auto* from) {
        typename std::remove_const<typename std::remove_pointer<decltype(from)>::type>::type token[kFewEach];
#pragma unroll
        for (int i = 0; i < kFewEach; ++i) {
            if (i >= each) break;
            place[i] = own_token(each, i);
            token[i] = from[min(place[i], a.count - 1)];
        }
#pragma unroll
        for (int i = 0; i < kFewEach; ++i) {
            if (i >= each) break;
            key[i] = (unsigned)token[i];
            mine[i] = __ballot((key[i] & (kBuckets - 1)) == bucket);
            if (EARLIER) {
                const bool valid = place[i] < a.count && key_of(a, token[i]) < (unsigned)a.vocab;
                mine[i] &= __ballot(valid);
                before += __popcll(__ballot(valid && (key[i] & (kBuckets - 1)) < bucket));
            } else if (mine[i]) {
                mine[i] &= __ballot(place[i] < a.count && key_of(a, token[i]) < (unsigned)a.vocab);
            }
            count += __popcll(mine[i]);
        }
    };
    if (a.wide) look(static_cast<const long long*>(a.tokens));
    else look(static_cast<const int*>(a.tokens));
    if (lane == 0) {
        room.counts[wave] = count;
        if (EARLIER) room.earlier[wave] = before;
    }
    lds_barrier();
    int at = 0;
    unsigned total = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        at += w < wave ? room.counts[w] : 0;
        total += room.counts[w];
        if (EARLIER) start += room.earlier[w];
    }
#pragma unroll
    for (int i = 0; i < kFewEach; ++i) {
        if (i >= each) break;
        if (!mine[i]) continue;
        if (mine[i] >> lane & 1) {
            const int to = at + __popcll(mine[i] & ((1ull << lane) - 1));
            room.keys[to] = key[i] >> kBucketBits;
            room.places[to] = (unsigned short)place[i];
            if (marks) atomicOr(&marks[key[i] >> (kBucketBits + 5)], 1u << (key[i] >> kBucketBits & 31));
        }
        at += __popcll(mine[i]);
    }
    lds_barrier();
    between();

    // A stable sort by the key, in LDS: few tokens by counting those that go before each, more by digits.
    if (total <= kPairs && rows <= 1ll << (32 - kFewBits)) {
        // (key, number) as one number: all differ.  Four lanes a token.
        const unsigned t = threadIdx.x, i = t / 4, k = i < total ? room.keys[i] : 0u;
        const unsigned short own_place = i < total ? room.places[i] : 0;
        if (t < kPairs) room.pairs[t] = t < total ? room.keys[t] << kFewBits | t : ~0u;
        lds_barrier();
        if (i < total) {
            const unsigned own = k << kFewBits | i;
            unsigned before = 0;
#pragma unroll 2
            for (unsigned j = t % 4 * 4; j < total; j += 16) {
                const uint4 n = *reinterpret_cast<const uint4*>(room.pairs + j);
                before += (n.x < own) + (n.y < own) + (n.z < own) + (n.w < own);
            }
            before += (unsigned)__shfl_xor((int)before, 1);
            before += (unsigned)__shfl_xor((int)before, 2);
            if (t % 4 == 0) {
                room.keys[before] = k;
                room.places[before] = own_place;
            }
        }
        lds_barrier();
    } else {
        const int kept = (int)((total + kSortThreads - 1) / kSortThreads);
        bool there[kFewEach];
#pragma unroll
        for (int i = 0; i < kFewEach; ++i) {
            const unsigned t = own_token(kept, i);
            there[i] = i < kept && t < total;
            key[i] = there[i] ? room.keys[t] : 0u;
            place[i] = there[i] ? room.places[t] : 0u;
        }
        for (int pass = 0; pass < passes; ++pass) {
            const int shift = pass * digit_bits, digit = threadIdx.x, size = 1 << digit_bits;
            int rank[kFewEach];
            rank_tokens<kFewEach, BITS>(key, there, kept, shift, digit_bits, room.of_wave, rank);
            lds_barrier();
            int here = 0;
            if (digit < size)
#pragma unroll
                for (int w = 0; w < kSortWaves; ++w) here += room.of_wave[w][digit];
            const int base = sum_before(here, room.counts);
            if (digit < size) spread<BITS>(room.of_wave, digit, base);
            lds_barrier();
#pragma unroll
            for (int i = 0; i < kFewEach; ++i)
                if (there[i]) {
                    const int to = room.of_wave[wave][(key[i] >> shift) & (unsigned)(size - 1)] + rank[i];
                    room.keys[to] = key[i];
                    room.places[to] = (unsigned short)place[i];
                }
            lds_barrier();
            if (pass + 1 < passes)
#pragma unroll
                for (int i = 0; i < kFewEach; ++i)
                    if (there[i]) {
                        key[i] = room.keys[own_token(kept, i)];
                        place[i] = room.places[own_token(kept, i)];
                    }
        }
    }
    return total;
}

// Where a launch goes before that of the sums, it sorts the tokens: lists of all buckets, one after another, and where each begins.
struct Lists {
    unsigned start[kBuckets], count[kBuckets];
    // the rows' numbers within their bucket, then the places

    __device__ unsigned* keys() { return count + kBuckets; }
    __device__ unsigned short* places(unsigned tokens) { return reinterpret_cast<unsigned short*>(keys() + tokens); }
};
constexpr long long lists_bytes(long long tokens) { return (long long)sizeof(Lists) + tokens * 6; }

// Turns, then sorts in `groups` workgroups, one a bucket, then sets to zero: in this order, for the sort takes a while and zeros go out
// beside it (two workgroups to a CU: digits of 8 bits leave the room for it).
constexpr int kListDigit = 8;

template <class G, class W>
__global__ __launch_bounds__(kSortThreads, 8) void lists_kernel(TokenArgs a, TurnArgs turn, Fill fill, Lists* lists, int groups, short passes, short digit_bits)
{
    typedef BucketRoom<kListDigit> Room;
    __shared__ __attribute__((aligned(16))) char bytes[sizeof(Room) > tiles_room<G>() ? sizeof(Room) : tiles_room<G>()];
    const unsigned turning = (turn.tiles + kTiles - 1) / kTiles, bucket = blockIdx.x - turning;
    if (bucket >= (unsigned)groups) {
        turn_or_fill<G, W>(turn, fill, blockIdx.x < turning ? blockIdx.x : blockIdx.x - groups, bytes);
        return;
    }
    Room& room = *reinterpret_cast<Room*>(bytes);
    unsigned start = 0;
    const unsigned total = sort_bucket<kListDigit, true>(a, bucket, passes, digit_bits, room, nullptr, start, [] {});
    for (unsigned t = threadIdx.x; t < total; t += kSortThreads) {
        lists->keys()[start + t] = room.keys[t];
        lists->places(a.count)[start + t] = room.places[t];
    }
    if (threadIdx.x == 0) {
        lists->start[bucket] = start;
        lists->count[bucket] = total;
    }
}

// Workgroup (b, y) owns the rows of the table whose number ends in b (kBuckets of them: frequent tokens are often neighbours), and
// column blocks y, y + shares, ...  It takes the sorted tokens of its rows from the launch before, or looks through all tokens and sorts
// them itself, sets the rows without any to zero (`zeros`; beyond kOwnZeros bytes a launch before does that, in order: 60000 x 250 floats
// 13.9 us a call here and 14.7 there, 100000 x 250, whose rows share cache lines, 31.6 and 22.9) and deals the sorted tokens out to its
// wavefronts evenly.  Latency bounds it, and the instructions that it fetches: 9.0 us at 8192 tokens of 20000 x 300 with the fullest
// workgroup's 148 tokens sorted before (the launch before takes 10.1, 8.1 without the sort; sorting here took 3.9); 37 tokens of
// 8192 x 128 5.2 us a call, the launch included.
template <class G, class W>
__global__ __launch_bounds__(kSortThreads) void bucket_kernel(EmbedGradArgs a, const G* grad, Lists* lists, short passes, short digit_bits, int column_blocks, int shares, bool zeros)
{
    __shared__ __attribute__((aligned(16))) BucketRoom<kBucketDigit> room;
    __shared__ unsigned marks[kMarks / 32];                // rows of the bucket that have tokens
    unsigned* const keys = room.keys;
    unsigned short* const places = room.places;
    float (*const part_sums)[kColumns] = reinterpret_cast<float (*)[kColumns]>(room.of_wave);      // (the sort is over when these are written)
    static_assert(sizeof(room.of_wave) >= sizeof(float) * kSortWaves * kColumns, "a part of each wavefront fits");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const TokenArgs named{a.tokens, a.vocab, a.padding, (unsigned)a.sentences * a.words, a.wide};
    const int own_blocks = (column_blocks - (int)blockIdx.y + shares - 1) / shares;
    auto columns = [&](int block) { return columns_of((int)(blockIdx.y + block * shares), lane, a.dim); };
    W* table_grad = static_cast<W*>(a.table_grad) + (size_t)blockIdx.x * a.dim;
    const size_t apart = (size_t)kBuckets * a.dim;         // elements from one row of the bucket to the next
    Sums sums;
    unsigned total;
    if (lists) {
        const unsigned start = lists->start[blockIdx.x];
        total = lists->count[blockIdx.x];
        for (unsigned t = threadIdx.x; t < total; t += kSortThreads) {
            keys[t] = lists->keys()[start + t];
            places[t] = lists->places(named.count)[start + t];
        }
        lds_barrier();
    } else {
        if (zeros)
            for (int i = threadIdx.x; i < kMarks / 32; i += kSortThreads) marks[i] = 0;
        unsigned start;
        total = sort_bucket<kBucketDigit, false>(named, blockIdx.x, passes, digit_bits, room, zeros ? marks : nullptr, start, [&] {
            if (!zeros) return;
            // pieces of 16 bytes of all rows, one after another: a row may be a few lanes wide
            constexpr int kVec = 16 / sizeof(W);
            typedef typename Piece<W, kVec>::type V;
            const unsigned per_row = a.dim < kVec ? a.dim : (a.dim + kVec - 1) / kVec, pieces = (unsigned)rows_of(a.vocab, blockIdx.x) * per_row;
            for (unsigned f = blockIdx.y * kSortThreads + threadIdx.x; f < pieces; f += shares * kSortThreads) {
                const unsigned r = f / per_row, p = f % per_row;
                if (marks[r >> 5] >> (r & 31) & 1) continue;
                W* row = table_grad + r * apart;
                if (a.dim < kVec) row[p] = (W)0.f;
                else *reinterpret_cast<V*>(row + min((int)p * kVec, a.dim - kVec)) = V{};
            }
        });
    }

    // The sorted tokens are dealt out evenly, whatever rows they belong to: `parts` wavefronts share a column block and take `share`
    // tokens in a row each.  What a wavefront has of a run that began before its tokens it leaves in LDS; the wavefront in which the
    // run begins adds that up.
    const int parts = max(kSortWaves / own_blocks, 1), together = kSortWaves / parts;
    const unsigned share = (total + parts - 1) / parts, part = wave % parts, from = min(part * share, total), to = min(from + share, total);
    for (int first = 0; first < own_blocks; first += together) {
        const int block = first + wave / parts;
        const Columns c = columns(block);
        const bool works = wave / parts < together && block < own_blocks && from < to;
        unsigned k = 0;
        bool before = false, open = false;      // the run at hand began before; it has not ended here
        auto store = [&]() { store_row<W>(table_grad + k * apart, sums, c, a.scale, a.accumulate); };
        clear(sums);
        if (works) {
            before = from > 0 && keys[from - 1] == keys[from];
#pragma unroll 1
            for (unsigned start = from; start < to; start += 64) {
                const unsigned t = start + lane, here = min(to - start, 64u);
                const unsigned own = t < to ? keys[t] : 0u;
                const int own_place = t < to ? places[t] : 0;
                const unsigned long long ends = __ballot(t < to && (t + 1 == total || keys[min(t + 1, total - 1)] != own));
#pragma unroll 1
                for (unsigned i = 0; i < here; i += kFewAhead) {
                    Row<G> r[kFewAhead];
#pragma unroll
                    for (int u = 0; u < kFewAhead; ++u)
                        if (i + u < here) r[u] = load_row<G>(grad + (size_t)(unsigned)__builtin_amdgcn_readlane(own_place, i + u) * a.dim, c);
#pragma unroll
                    for (int u = 0; u < kFewAhead; ++u) {
                        if (i + u >= here) break;
                        add(sums, r[u], c);
                        open = !(ends >> (i + u) & 1);
                        if (open) continue;
                        k = (unsigned)__builtin_amdgcn_readlane((int)own, i + u);
                        if (before) leave(sums, part_sums);
                        else store();
                        before = false;
                        clear(sums);
                    }
                }
                k = (unsigned)__builtin_amdgcn_readlane((int)own, here - 1);
            }
            if (open && before) leave(sums, part_sums);
        }
        if (parts == 1) continue;
        lds_barrier();
        if (open && !before) {
            const unsigned t = lane * share;
            const int more = __popcll(__ballot(lane > (int)part && lane < parts && t < total && keys[min(t, total - 1)] == k));
            join(sums, part_sums, wave + 1, more);
            store();
        }
        if (first + together < own_blocks) lds_barrier();
    }
}

// ---------------------------------------------------------------- gradient of many tokens: a sort, windows, runs

// A pass of the sort is two launches.  Each workgroup counts the digits of its run of tokens ...  (from: null in the first pass, which reads
// the tokens.)
template <class G, class W>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(TokenArgs a, TurnArgs turn, Fill fill, const unsigned* from, int* counts, int groups, short rounds, short shift, short bits)
{
    __shared__ __attribute__((aligned(16))) int bins[tiles_room<G>() / 4];
    static_assert(sizeof(bins) >= sizeof(int) << kMaxDigit, "a count for each digit fits");
    if ((int)blockIdx.x >= groups) {
        turn_or_fill<G, W>(turn, fill, blockIdx.x - groups, bins);
        return;
    }
    const int size = 1 << bits;
    const int each = kMoveEach * rounds;
    const unsigned first = blockIdx.x * (unsigned)(each * kSortThreads);
    for (int d = threadIdx.x; d < size; d += kSortThreads) bins[d] = 0;
    lds_barrier();
    for (int i = 0; i < each; ++i) {
        const unsigned t = first + own_token(each, i);
        if (t < a.count) atomicAdd(&bins[((from ? from[t] : sort_key(a, t)) >> shift) & (unsigned)(size - 1)], 1);
    }
    lds_barrier();
    for (int d = threadIdx.x; d < size; d += kSortThreads) counts[(size_t)blockIdx.x * size + d] = bins[d];
}

// ... then each finds, from the counts of all, where its tokens of each digit go, and takes them there in their order.
template <class W>
__global__ __launch_bounds__(kSortThreads) void sort_move_kernel(TokenArgs a, Fill fill, Sorted from, Sorted to, const int* counts, int groups, short rounds, short shift, short bits)
{
    __shared__ int of_wave[kSortWaves][1 << kMaxDigit];
    __shared__ int wave_sums[kSortWaves];
    if ((int)blockIdx.x >= groups) {
        fill_part<W>(fill, blockIdx.x - groups);
        return;
    }
    constexpr int kEach = kMoveEach;
    const int wave = threadIdx.x >> 6, size = 1 << bits, digit = threadIdx.x;
    unsigned first = blockIdx.x * (unsigned)(kEach * kSortThreads * rounds);
    unsigned key[kEach];
    int place[kEach], rank[kEach];
    bool there[kEach];
    auto fetch = [&]() {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const unsigned t = first + own_token(kEach, i);
            there[i] = t < a.count;
            key[i] = !there[i] ? 0u : from.keys ? from.keys[t] : sort_key(a, t);
            place[i] = !there[i] ? 0 : from.keys ? from.places[t] : (int)t;
        }
    };
    fetch();
    // where this workgroup's first token of `digit` goes: all smaller digits, then the same digit in the workgroups before
    int before = 0, total = 0;
    if (digit < size) {
        int g = 0;
        for (; g + 16 <= groups; g += 16) {
            int n[16];
#pragma unroll
            for (int u = 0; u < 16; ++u) n[u] = counts[(size_t)(g + u) * size + digit];
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                before += g + u < (int)blockIdx.x ? n[u] : 0;
                total += n[u];
            }
        }
        for (; g < groups; ++g) {
            const int n = counts[(size_t)g * size + digit];
            before += g < (int)blockIdx.x ? n : 0;
            total += n;
        }
    }
    int base = 0;
    for (int round = 0; round < rounds; ++round) {
        rank_tokens<kEach, kMaxDigit>(key, there, kEach, shift, bits, of_wave, rank);
        if (round == 0) base = sum_before(total, wave_sums) + before;      // (waits for the counts of all wavefronts)
        else lds_barrier();
        if (digit < size) base = spread<kMaxDigit>(of_wave, digit, base);
        lds_barrier();
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (there[i]) {
                const int at = of_wave[wave][(key[i] >> shift) & (unsigned)(size - 1)] + rank[i];
                to.keys[at] = key[i];
                to.places[at] = place[i];
            }
        first += kEach * kSortThreads;
        if (round + 1 < rounds) fetch();
    }
}

// Sums of kWindow sorted tokens in a row, where they are of one row of the table.  (us a call by 16, 32 and 64: 32768 tokens to
// 131072 x 2048 252, 251, 255; to 1000 x 512 floats 32.2, 32.0, 35.2; to 50000 x 512, half of them one token, 89, 70, 67.)
constexpr int kWindow = 32;

template <class G>
__global__ __launch_bounds__(kThreads) void window_kernel(EmbedGradArgs a, const G* grad, Sorted sorted, float* windows, int column_blocks)
{
    const int lane = threadIdx.x & 63;
    const long long unit = (long long)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long w = unit / column_blocks, first = w * kWindow;
    if (first + kWindow > (long long)a.sentences * a.words) return;
    const unsigned key = sorted.keys[first];
    if (key != sorted.keys[first + kWindow - 1] || key >= (unsigned)a.vocab) return;
    const Columns c = columns_of((int)(unit % column_blocks), lane, a.dim);
    Sums sums;
    clear(sums);
    add_rows<G>(sums, grad, a.dim, kWindow, c, [&](int i) { return sorted.places[first + i]; });
    store_row<float>(windows + w * a.dim, sums, c, 1.f, false);
}

// The rows of the table that have tokens.  A wavefront takes a slot of sorted tokens; a run of many rows to add (tokens, and sums of
// whole windows) is shared by the wavefronts of the workgroup, each a part of either, and joined in their order.
constexpr int kRunThreads = 512, kRunWaves = kRunThreads / 64;

template <class G, class W>
__global__ __launch_bounds__(kRunThreads) void runs_kernel(EmbedGradArgs a, const G* grad, Sorted sorted, const float* windows, int column_blocks)
{
    __shared__ unsigned long_runs[kRunWaves];
    __shared__ int long_count;
    __shared__ float part[kRunWaves][kColumns];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned tokens = (unsigned)a.sentences * a.words;
    const unsigned first = (unsigned)(blockIdx.x / column_blocks) * (kRunWaves * kSlot) + wave * kSlot;
    const Columns c = columns_of((int)(blockIdx.x % column_blocks), lane, a.dim);
    W* table_grad = static_cast<W*>(a.table_grad);
    if (threadIdx.x == 0) long_count = 0;
    lds_barrier();
    auto key_at = [&](unsigned i) { return sorted.keys[i]; };
    auto done = [&](unsigned k, const Sums& of_row) { store_row<W>(table_grad + (size_t)k * a.dim, of_row, c, a.scale, a.accumulate); };
    if (first < tokens)
        add_slot<G>(grad, a.dim, c, first, tokens, (unsigned)a.vocab, key_at, [&](unsigned i) { return sorted.places[i]; }, done, [&](unsigned from) {
            if (lane == 0) long_runs[atomicAdd(&long_count, 1)] = from;
        });
    lds_barrier();
    const int shared_runs = long_count;
    for (int l = 0; l < shared_runs; ++l) {
        const unsigned from = __builtin_amdgcn_readfirstlane(long_runs[l]), to = end_of_run(key_at, from, tokens);
        // tokens before the first whole window, whole windows, tokens after the last
        unsigned w0 = (from + kWindow - 1) / kWindow, w1 = to / kWindow, lead = w0 * kWindow - from, rest = w1 * kWindow;
        if (w0 >= w1) {
            w0 = w1 = 0;
            lead = to - from;
            rest = to;
        }
        auto share = [&](unsigned n, int w) { return (unsigned)((unsigned long long)n * w / kRunWaves); };
        Sums sums;
        clear(sums);
        const unsigned l0 = share(lead, wave), l1 = share(lead, wave + 1), m0 = share(w1 - w0, wave), m1 = share(w1 - w0, wave + 1), t0 = share(to - rest, wave),
                       t1 = share(to - rest, wave + 1);
        add_rows<G>(sums, grad, a.dim, (int)(l1 - l0), c, [&](int i) { return sorted.places[from + l0 + i]; });
        add_rows<float>(sums, windows, a.dim, (int)(m1 - m0), c, [&](int i) { return (int)(w0 + m0 + i); });
        add_rows<G>(sums, grad, a.dim, (int)(t1 - t0), c, [&](int i) { return sorted.places[rest + t0 + i]; });
        leave(sums, part);
        lds_barrier();
        if (wave == 0) {
            join(sums, part, 1, kRunWaves - 1);
            done(sorted.keys[from], sums);
        }
        lds_barrier();
    }
}

int type_bytes(int dtype) { return dtype == kF32 ? 4 : 2; }
long long rounded(long long bytes) { return (bytes + 255) / 256 * 256; }

// What the workspace holds, in this order.
struct Parts {
    long long rows, keys, counts, windows, lists, total;      // bytes; keys: of each of two pairs of arrays, tokens and places
};

// Few tokens: whether the launch that sums sets the rows without tokens to zero.
bool sets_own_zeros(const EmbedGradArgs& a, int table_bytes)
{
    return (unsigned long long)a.vocab * a.dim * table_bytes <= kOwnZeros && a.vocab <= (long long)kMarks * kBuckets;
}

Parts parts_of(const EmbedGradArgs& a, int grad_dtype)
{
    const long long tokens = (long long)a.sentences * a.words;
    Parts p{};
    if (a.channels_first && a.words > 1) p.rows = rounded(tokens * a.dim * type_bytes(grad_dtype));
    if (tokens > kFewTokens) {
        const SortPlan plan = sort_plan(a.vocab, kMaxDigit, tokens);
        p.keys = rounded(tokens * 4);
        p.counts = rounded((long long)plan.groups * (1 << plan.digit) * 4);
        p.windows = rounded(tokens / kWindow * a.dim * 4);
    } else if (p.rows || (!a.accumulate && !sets_own_zeros(a, 4))) {
        p.lists = rounded(lists_bytes(tokens));
    }
    p.total = p.rows + 4 * p.keys + p.counts + p.windows + p.lists;
    return p;
}

template <class W>
__global__ __launch_bounds__(kSortThreads) void zero_kernel(Fill fill)
{
    fill_part<W>(fill, blockIdx.x);
}

// Elements that one launch sets to zero at most (16 GB).
template <class W>
constexpr unsigned long long kFillAtOnce = (1ull << 20) * kSortThreads * (16 / sizeof(W));

// Sets all but at most `left` of `count` elements to zero, in launches of their own; returns how many.
template <class W>
unsigned long long set_ahead(void* to, unsigned long long count, unsigned long long left, hipStream_t s)
{
    unsigned long long done = 0;
    while (count - done > left) {
        const Fill fill{static_cast<W*>(to) + done, std::min(count - done, kFillAtOnce<W>)};
        hipLaunchKernelGGL(zero_kernel<W>, dim3((unsigned)blocks_of<W>(0, fill)), dim3(kSortThreads), 0, s, fill);
        done += fill.count;
    }
    return done;
}

template <class G, class W>
int launch_grad(const EmbedGradArgs& a, const Parts& parts, char* workspace, hipStream_t s)
{
    const long long tokens = (long long)a.sentences * a.words, column_blocks = ((long long)a.dim + kColumns - 1) / kColumns;
    const G* grad = static_cast<const G*>(a.grad);
    G* rows = reinterpret_cast<G*>(workspace);
    long long tiles = 0;
    if (parts.rows) {
        tiles = tiles_of<Turn<G>>(a.sentences, a.words, a.dim);
        grad = rows;
    }
    const unsigned long long elements = a.accumulate ? 0 : (unsigned long long)a.vocab * a.dim;
    if (tiles >= (1ll << 23)) return kTooLarge;        // (turned, set to zero and sorted in one launch: 2^21, 2^20 and, below, at most 2^18 workgroups)
    const TurnArgs turn{a.grad, rows, a.dim, a.sentences, a.words, (unsigned)tiles};
    if (tokens <= kFewTokens) {
        const bool zeros = !a.accumulate && !tiles && sets_own_zeros(a, sizeof(W));
        const unsigned groups = (unsigned)std::min<long long>(a.vocab, kBuckets);
        const unsigned shares = (unsigned)std::min<long long>(column_blocks, kBuckets / groups);      // of the column blocks: a workgroup a CU
        Lists* lists = nullptr;
        if (tiles || (elements && !zeros)) {
            const unsigned long long filled = set_ahead<W>(a.table_grad, elements, kFillAtOnce<W>, s);
            const Fill fill{static_cast<W*>(a.table_grad) + filled, elements - filled};
            const unsigned long long blocks = groups + blocks_of<W>(turn.tiles, fill);
            const TokenArgs named{a.tokens, a.vocab, a.padding, (unsigned)tokens, a.wide};
            const SortPlan plan = sort_plan((a.vocab - 1) >> kBucketBits, kListDigit, tokens);
            lists = reinterpret_cast<Lists*>(workspace + parts.rows);
            hipLaunchKernelGGL((lists_kernel<G, W>), dim3((unsigned)blocks), dim3(kSortThreads), 0, s, named, turn, fill, lists, (int)groups, (short)plan.passes,
                               (short)plan.digit);
        }
        const SortPlan plan = sort_plan((a.vocab - 1) >> kBucketBits, kBucketDigit, tokens);
        hipLaunchKernelGGL((bucket_kernel<G, W>), dim3(groups, shares), dim3(kSortThreads), 0, s, a, grad, lists, (short)plan.passes, (short)plan.digit,
                           (int)column_blocks, (int)shares, zeros);
        return (int)hipGetLastError();
    }
    const SortPlan plan = sort_plan(a.vocab, kMaxDigit, tokens);
    const long long run_blocks = ((tokens + kRunWaves * kSlot - 1) / (kRunWaves * kSlot)) * column_blocks;
    constexpr int kWaves = kThreads / 64;
    const long long window_blocks = (tokens / kWindow * column_blocks + kWaves - 1) / kWaves;
    if ((unsigned long long)run_blocks > most_groups(kRunThreads) || (unsigned long long)window_blocks > most_groups(kThreads)) return kTooLarge;
    char* at = workspace + parts.rows;
    Sorted sorted[2];
    for (int i = 0; i < 2; ++i) {
        sorted[i].keys = reinterpret_cast<unsigned*>(at);
        sorted[i].places = reinterpret_cast<int*>(at + parts.keys);
        at += 2 * parts.keys;
    }
    int* counts = reinterpret_cast<int*>(at);
    float* windows = reinterpret_cast<float*>(at + parts.counts);
    Sorted from{nullptr, nullptr};
    const TokenArgs named{a.tokens, a.vocab, a.padding, (unsigned)tokens, a.wide};
    const int launches = 2 * plan.passes;
    const unsigned long long ahead = set_ahead<W>(a.table_grad, elements, launches * kFillAtOnce<W>, s);
    unsigned long long filled = ahead;
    for (int l = 0; l < launches; ++l) {
        const unsigned long long kVec = 16 / sizeof(W), end = l + 1 == launches ? elements : ahead + (elements - ahead) * (l + 1) / launches / kVec * kVec;
        const Fill fill{static_cast<W*>(a.table_grad) + filled, end - filled};
        filled = end;
        const short shift = (short)(l / 2 * plan.digit), bits = (short)plan.digit;
        const unsigned long long blocks = plan.groups + blocks_of<W>(l == 0 ? turn.tiles : 0, fill);
        if (l % 2 == 0) {
            TurnArgs here = turn;
            if (l > 0) here.tiles = 0;
            hipLaunchKernelGGL((sort_count_kernel<G, W>), dim3((unsigned)blocks), dim3(kSortThreads), 0, s, named, here, fill, from.keys, counts, plan.groups, (short)plan.rounds, shift, bits);
        } else {
            hipLaunchKernelGGL(sort_move_kernel<W>, dim3((unsigned)blocks), dim3(kSortThreads), 0, s, named, fill, from, sorted[l / 2 & 1], counts, plan.groups, (short)plan.rounds, shift, bits);
            from = sorted[l / 2 & 1];
        }
    }
    hipLaunchKernelGGL(window_kernel<G>, dim3((unsigned)window_blocks), dim3(kThreads), 0, s, a, grad, from, windows, (int)column_blocks);
    hipLaunchKernelGGL((runs_kernel<G, W>), dim3((unsigned)run_blocks), dim3(kRunThreads), 0, s, a, grad, from, static_cast<const float*>(windows), (int)column_blocks);
    return (int)hipGetLastError();
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

int launch_embed_grad(int grad_dtype, int table_dtype, const EmbedGradArgs& a, char* workspace, void* stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if ((long long)a.sentences * a.words == 0) {       // all rows are zero
        const unsigned long long elements = (unsigned long long)a.vocab * a.dim;
        if (table_dtype == kF32) set_ahead<float>(a.table_grad, elements, 0, s);
        else set_ahead<_Float16>(a.table_grad, elements, 0, s);      // (zeros of 16 bits)
        return (int)hipGetLastError();
    }
    const Parts parts = parts_of(a, grad_dtype);
    if (grad_dtype == kF32) return launch_grad<float, float>(a, parts, workspace, s);
    if (grad_dtype == kF16) return table_dtype == kF32 ? launch_grad<_Float16, float>(a, parts, workspace, s) : launch_grad<_Float16, _Float16>(a, parts, workspace, s);
    return table_dtype == kF32 ? launch_grad<__bf16, float>(a, parts, workspace, s) : launch_grad<__bf16, __bf16>(a, parts, workspace, s);
}

}  // namespace sc

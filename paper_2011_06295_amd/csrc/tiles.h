// What the kernels that multiply rows share: pieces of 16 bytes, loads from memory straight to LDS, the order of tiles.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>
#include <utility>

namespace sc {

namespace {

enum { kF32 = 0, kF16 = 1, kBF16 = 2, kI8 = 3 };   // SC_F32, SC_F16, SC_BF16, SC_I8

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

typedef int int4v __attribute__((ext_vector_type(4)));
#define SC_LDS __attribute__((address_space(3)))

template <class F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
// f(0) .. f(N - 1), each with its number as a constant: loops that have to be unrolled whole, however long.
template <int N, class F>
__device__ __forceinline__ void each(F&& f) { each_of(f, std::make_integer_sequence<int, N>{}); }

// 16 bytes a lane from memory to LDS at `lds` + 16 * lane; bytes past the descriptor's end arrive as zeros: those of an `offset` of the
// descriptor's bytes less `base`, or more.  (A difference that must not be negative: where nothing is to be fetched, the descriptor has no
// bytes and the base is 0.)  Not the builtin:
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

}  // namespace

}  // namespace sc

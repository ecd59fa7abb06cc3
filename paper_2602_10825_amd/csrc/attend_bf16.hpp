// What the attention kernels on bf16 operands share (attend_bf16.hip: bf16 caches; attend_kv4.hip: a clean region in 4 bits).
#pragma once

#include <utility>

#include "attend_split.hpp"

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int BQ = kWideRows;   // query rows per workgroup
constexpr int BK = 64;       // keys per tile

constexpr int NT = 64 * (BQ / 32);   // 8 wavefronts of 32 query rows, two per SIMD

// f(0), ..., f(N - 1) with the argument a compile-time constant: every choice made on it is made when
// the loop is written out
template <int N, typename F, int... I>
__device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>()), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
    static_for_impl<N>(f, std::make_integer_sequence<int, N>());
}

template <int D>
struct WideSmem {
    static constexpr int KROW = D + 8;        // padded K row (bf16): 16-byte fragment reads of 16
                                              // consecutive keys fall in distinct banks
    static constexpr int VROW = D + 32;       // padded V row: the 4 key rows of one transposing
                                              // load fall in disjoint bank quarters
    __attribute__((aligned(16))) bf16_t K[4][BK * KROW];
    __attribute__((aligned(16))) bf16_t V[2][BK * VROW];
    int seg_start[FC_MAX_ACTIVE + 2], seg_len[FC_MAX_ACTIVE + 2];
    int seg_first, off_first, n_tiles;
};

}  // namespace

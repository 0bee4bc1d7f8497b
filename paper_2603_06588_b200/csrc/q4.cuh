// Pages held in 4 bits.
//
// The slab of a page and a KV head, D elements to a head, NG groups of D / NG elements:
//   [codes of K: 16 D / 2 bytes] [codes of V] [K: 16 x NG pairs (step, lowest) of bf16] [V: 16 x NG pairs].
// A code is four bits; element = lowest + step * code.  The orders are those in which a warp's matrix instructions take their operands,
// so that a lane reads what it needs with one wide access and no two lanes meet in a bank of shared memory:
//   K  token t: 8 elements to a 32-bit word, element e in nibble e % 8 of word (e / 8 % 4) * (D / 32) + e / 32 of row t.
//   V  token t: row q4_row(t); element e in nibble e % 32 / 8 of halfword e / 32 of unit e % 8, D / 16 bytes to a unit; with D = 128 the
//      halves of rows 2, 3, 6, 7, ... are exchanged.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace hook_attn {

// Tokens of a sequence at most: far enough from 2^31 that the end of a chunk or of a few pages behind any token is an int.
constexpr int kQ4MostKeys = 0x7fffffff - 4095;

template <int HD, int NG>
struct Q4Slab {
    static constexpr int kRow = HD / 2;                       // bytes of a token's codes
    static constexpr int kCodes = kPage * kRow;               // of K, and of V
    static constexpr int kParams = kPage * NG * 4;
    static constexpr int kBytes = 2 * (kCodes + kParams);
};

__host__ __device__ constexpr int q4_slab_bytes(int head_dim, int groups) { return kPage * (head_dim + 8 * groups); }

// Where V keeps token t: even tokens, then odd ones, in each half of the page.
__device__ __forceinline__ int q4_row(int t) { return ((t >> 1) & 3) | ((t & 1) << 2) | (t & 8); }

template <int HD>
__device__ __forceinline__ int q4_unit(int row, int unit) { return HD == 128 ? unit ^ ((row & 2) << 1) : unit; }

__device__ __forceinline__ float q4_step(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float q4_lowest(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }

}  // namespace hook_attn

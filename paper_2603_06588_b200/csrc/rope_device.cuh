// Device code that the rotary appends share: where a row of the call goes, the turn of a pair, wide loads and stores.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "ops.cuh"

namespace hook_attn {

__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(float x) { return x; }

// Where a row of the call goes.
struct RowPlace {
    int64_t slot;  // element offset of its slot in the cache (block and token part)
    int pos;       // its position in the sequence
    int state;     // kGood; kBroken: zero its queries; kBehind: behind the last sequence, leave it alone
};
enum { kGood = 0, kBroken = 1, kBehind = 2 };

// A warp looks a row up: its sequence is the number of sequences that end at or before the row.  Of many, the lanes narrow them down to
// 128 first (4096 rows of as many sequences: 20.8 us, and 33.6 us counting through all).
__device__ __forceinline__ RowPlace find_row(const RopeArgs& a, int row)
{
    const int lane = threadIdx.x & 31;
    RowPlace r = {0, 0, kBehind};
    int seq = row, lo = row, n = 1;
    if (row >= a.total_q) return r;
    if (a.cu_q_lens) {
        int from = 0, to = a.num_seqs;
        while (to - from > 128) {
            const int step = (to - from + 31) / 32, s = from + (lane + 1) * step;         // where the lane's part ends
            from += step * __popc(__ballot_sync(0xffffffffu, s <= to && a.cu_q_lens[s] <= row));
            to = min(from + step, to);
        }
        seq = 0;
#pragma unroll 4
        for (int s = from + lane; s < to; s += 32) seq += a.cu_q_lens[s + 1] <= row;
        seq = from + __reduce_add_sync(0xffffffffu, seq);
        if (seq >= a.num_seqs) return r;
        lo = a.cu_q_lens[seq];
        n = a.cu_q_lens[seq + 1] - lo;
    }
    r.state = kBroken;
    const int L = a.seq_lens[seq], at = row - lo;
    if (L <= 0 || L > a.max_keys || at < 0 || at >= n || n > L) return r;
    r.pos = L - n + at;
    const int page = a.block_table[(int64_t)seq * a.max_blocks + r.pos / kPage];
    if (page < 0 || page >= a.num_blocks) return r;
    r.slot = (int64_t)page * a.bs + (int64_t)(r.pos % kPage) * a.ts;
    r.state = kGood;
    return r;
}

// Cosine and sine of one pair at one position, times the factor.
__device__ __forceinline__ float2 turn_of(const RopeArgs& a, int p, int pair)
{
    double turns = (double)p * (double)a.inv_freq[pair] * 0.15915494309189535;   // 1 / (2 pi)
    turns -= rint(turns);
    float s, c;
    sincospif(2.0f * (float)turns, &s, &c);
    return make_float2(c * a.factor, s * a.factor);
}

// V values in a row of memory: the widest accesses that V allows, then 32 bits each.
template <typename T, int V>
struct alignas(V * sizeof(T) < 16 ? V * sizeof(T) : 16) Pack {
    T x[V];
};

template <typename T, int V>
__device__ __forceinline__ void load(float (&x)[V], const T* p)
{
    const Pack<T, V> raw = *reinterpret_cast<const Pack<T, V>*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = to_f32(raw.x[i]);
}

template <int V>
__device__ __forceinline__ void store(__nv_bfloat16* p, const float (&x)[V])
{
    Pack<__nv_bfloat16, V> raw;
#pragma unroll
    for (int i = 0; i < V; ++i) raw.x[i] = __float2bfloat16(x[i]);
    *reinterpret_cast<Pack<__nv_bfloat16, V>*>(p) = raw;
}

// V pairs turn: x holds their first elements and y the second ones (halves), or x and then y the pairs one after the other.
template <int V>
__device__ __forceinline__ void turn_item(float (&x)[V], float (&y)[V], const float2* turn, bool halves)
{
    if (halves || V == 1) {
#pragma unroll
        for (int m = 0; m < V; ++m) {
            const float2 t = turn[m];
            const float u = x[m], w = y[m];
            x[m] = u * t.x - w * t.y;
            y[m] = w * t.x + u * t.y;
        }
    } else {                               // pair m: elements 2 m and 2 m + 1 of x, then of y
#pragma unroll
        for (int m = 0; m < V; ++m) {
            const float2 t = turn[m];
            float& u = m < V / 2 ? x[2 * m % V] : y[2 * m % V];
            float& w = m < V / 2 ? x[(2 * m + 1) % V] : y[(2 * m + 1) % V];
            const float u0 = u, w0 = w;
            u = u0 * t.x - w0 * t.y;
            w = w0 * t.x + u0 * t.y;
        }
    }
}

}  // namespace hook_attn

// Rotary positions with several axes, appended to the paged cache: what has to happen to the rows of a call between
// the projections and hook_attn_prefill / hook_attn_decode.  A pair (a, b) of a head's first R elements turns by
//   angle = position[axis of the pair][row] * inv_freq[pair],   (a, b) -> factor * (a cos - b sin, b cos + a sin);
// q goes to a contiguous bf16 tensor, k and v to the page slots of the rows.
//
// Angles: position * inv_freq is exact in 64 bits (31 + 24 bits) and is brought to [-1/2, 1/2] turns there; in 32 bits a
// position of a million would be off by 0.06 rad.  The rest is 32-bit, with one rounding to bf16 at the store.
#include "common.cuh"
#include "ops.cuh"

#include <cuda_fp16.h>

namespace hook_attn {

namespace {

constexpr int kRopeThreads = 256;

__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(float x) { return x; }

// Where row `row` of the call goes.
struct RowPlace {
    int seq;       // num_seqs: the row lies behind the last sequence
    int pos;       // its position in the sequence
    int64_t slot;  // element offset of its slot in the cache (token and block part)
    bool ok;
};

// The whole CTA looks one row up: the sequence is the number of sequences that end at or before the row.
__device__ __forceinline__ RowPlace find_row(const RopeArgs& a, int row)
{
    RowPlace r;
    int lo = row, n = 1;
    if (a.cu_q_lens) {
        int before = 0;
        for (int base = 0; base < a.num_seqs; base += kRopeThreads) {
            const int s = base + (int)threadIdx.x;
            before += __syncthreads_count(s < a.num_seqs && a.cu_q_lens[s + 1] <= row);
        }
        r.seq = before;
        if (before < a.num_seqs) {
            lo = a.cu_q_lens[before];
            n = a.cu_q_lens[before + 1] - lo;
        }
    } else {
        r.seq = row;
    }
    r.ok = false;
    r.pos = 0;
    r.slot = 0;
    if (r.seq >= a.num_seqs) return r;
    const int L = a.seq_lens[r.seq], at = row - lo;
    if (L <= 0 || L > a.max_keys || at < 0 || at >= n || n > L) return r;
    r.pos = L - n + at;
    const int page = a.block_table[(int64_t)r.seq * a.max_blocks + r.pos / kPage];
    if (page < 0 || page >= a.num_blocks) return r;
    r.slot = (int64_t)page * a.bs + (int64_t)(r.pos % kPage) * a.ts;
    r.ok = true;
    return r;
}

// Cosine and sine of one pair of one row, times the factor.
__device__ __forceinline__ float2 turn_of(const RopeArgs& a, int row, int pos, int pair)
{
    const int p = a.positions ? a.positions[(int64_t)a.axis_of_pair[pair] * a.axis_stride + row] : pos;
    double turns = (double)p * (double)a.inv_freq[pair] * 0.15915494309189535;   // 1 / (2 pi)
    turns -= rint(turns);
    float s, c;
    sincospif(2.0f * (float)turns, &s, &c);
    return make_float2(c * a.factor, s * a.factor);
}

// One CTA per row, one pair (or one element behind the rotated ones) per thread and step: any strides, any R.
template <typename T>
__global__ void __launch_bounds__(kRopeThreads) rope_rows_kernel(const __grid_constant__ RopeArgs a)
{
    __shared__ float2 turn[kMaxPairs];
    const int row = blockIdx.x, D = a.head_dim, half = a.pairs, items = D - half;
    const RowPlace at = find_row(a, row);
    if (at.seq >= a.num_seqs) return;                      // rows behind the last sequence stay as they are
    __nv_bfloat16* qo = a.q_out + (int64_t)row * a.Hq * D;
    if (!at.ok) {
        for (int i = threadIdx.x; i < a.Hq * D; i += kRopeThreads) qo[i] = __float2bfloat16(0.f);
        if (threadIdx.x == 0) report(a.status, HOOK_ATTN_ERR_BOUNDS);
        return;
    }
    if ((int)threadIdx.x < half) turn[threadIdx.x] = turn_of(a, row, at.pos, threadIdx.x);
    __syncthreads();
    const int step = a.halves ? half : 1, mul = a.halves ? 1 : 2;
    const int heads = a.Hq + 2 * a.Hkv;
    for (int i = threadIdx.x; i < heads * items; i += kRopeThreads) {
        int h = i / items;
        const int j = i - h * items;
        const T* src;
        __nv_bfloat16* dst;
        bool rotated = j < half;
        if (h < a.Hq) {
            src = static_cast<const T*>(a.q) + (int64_t)row * a.q_row + (int64_t)h * a.q_head;
            dst = qo + h * D;
        } else if ((h -= a.Hq) < a.Hkv) {
            src = static_cast<const T*>(a.k) + (int64_t)row * a.k_row + (int64_t)h * a.k_head;
            dst = a.k_cache + at.slot + (int64_t)h * a.hs;
        } else {
            h -= a.Hkv;
            src = static_cast<const T*>(a.v) + (int64_t)row * a.v_row + (int64_t)h * a.v_head;
            dst = a.v_cache + at.slot + (int64_t)h * a.hs;
            if (rotated) {
                const int e = j * mul;
                dst[e] = __float2bfloat16(to_f32(src[e]));
                dst[e + step] = __float2bfloat16(to_f32(src[e + step]));
                continue;
            }
        }
        if (rotated) {
            const int e = j * mul;
            const float2 t = turn[j];
            const float x = to_f32(src[e]), y = to_f32(src[e + step]);
            dst[e] = __float2bfloat16(x * t.x - y * t.y);
            dst[e + step] = __float2bfloat16(y * t.x + x * t.y);
        } else {
            const int e = j + half;
            dst[e] = __float2bfloat16(to_f32(src[e]));
        }
    }
}

}  // namespace

cudaError_t launch_rope_append(const RopeArgs& a, int dtype, cudaStream_t st)
{
    if (dtype == HOOK_DTYPE_BF16) rope_rows_kernel<__nv_bfloat16><<<a.total_q, kRopeThreads, 0, st>>>(a);
    else if (dtype == HOOK_DTYPE_F16) rope_rows_kernel<__half><<<a.total_q, kRopeThreads, 0, st>>>(a);
    else rope_rows_kernel<float><<<a.total_q, kRopeThreads, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace hook_attn

// Rotary positions with several axes, appended to the paged cache: what has to happen to the rows of a call between
// the projections and hook_attn_prefill / hook_attn_decode.  A pair (a, b) of a head's first R elements turns by
//   angle = position[axis of the pair][row] * inv_freq[pair],   (a, b) -> factor * (a cos - b sin, b cos + a sin);
// q goes to a contiguous bf16 tensor, k and v to the page slots of the rows.
//
// Angles: position * inv_freq / (2 pi) is brought to [-1/2, 1/2] turns in 64 bits.  The two products and the constant are rounded to 53
// bits each, so a turn is off by at most 3 x 2^-53 of the turns: by 1.1e-7 at 2^31 rad.  In 32 bits a position of a million would be off by
// 0.06 rad.  The rest is 32-bit, with one rounding to bf16 at the store.
#include "rope_device.cuh"

namespace hook_attn {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeRows = 8;       // rows per CTA at most: one warp looks each of them up
template <int V>
constexpr int kResident = V == 8 ? 6 : 8;      // CTAs on an SM: 40 registers with runs of eight (held to 32, 65536 rows take 443 us)

// A CTA takes a few rows.  An item is two runs of V elements of one head: V pairs that turn, or 2 V elements that are only
// moved; the thread that reads them writes them, so the queries may be rotated in place.  Bound by HBM: every element is read
// once and written once, and a row's cosines and sines (R / 2 of them) are computed once for all its heads (65536 rows of 64/8
// heads: 427 to 437 us, 6.1 to 6.3 TB/s; with the next item's loads under way during an item, 484 us: fewer CTAs fit an SM).  Small calls are
// bound by the chain of loads before the first store (one row: 3.0 us).
template <typename T, int V>
__global__ void __launch_bounds__(kRopeThreads) rope_append_kernel(const __grid_constant__ RopeArgs a)
{
    __shared__ __align__(16) float2 turn[kRopeRows][kMaxPairs];
    __shared__ RowPlace places[kRopeRows];
    const int row0 = blockIdx.x * a.rows_per_cta, warp = threadIdx.x >> 5;
    if (warp < a.rows_per_cta) {
        const RowPlace r = find_row(a, row0 + warp);
        if ((threadIdx.x & 31) == 0) {
            places[warp] = r;
            if (r.state == kBroken) report(a.status, HOOK_ATTN_ERR_BOUNDS);
        }
    }
    if (!a.positions) __syncthreads();             // the angles go by the places
    for (int i = threadIdx.x; i < a.rows_per_cta * kMaxPairs; i += kRopeThreads) {
        const int r = i / kMaxPairs, pair = i % kMaxPairs, row = row0 + r;
        if (pair < a.pairs && row < a.total_q)
            turn[r][pair] = turn_of(a, a.positions ? a.positions[a.axis_of_pair[pair] * a.axis_stride + row] : places[r].pos, pair);
    }
    __syncthreads();

    const int D = a.head_dim, heads = a.Hq + 2 * a.Hkv, per_head = D / (2 * V), turning = a.pairs / V;
    const int total = a.rows_per_cta * heads * per_head, shift = 31 - __clz(per_head);   // head_dim is a power of two
    for (int i = threadIdx.x; i < total; i += kRopeThreads) {
        const int j = i & (per_head - 1), rh = i >> shift, r = rh / heads;
        int h = rh - r * heads;
        const int state = places[r].state;
        if (state == kBehind || (state == kBroken && h >= a.Hq)) continue;
        const int64_t row = row0 + r;
        const T* src;
        __nv_bfloat16* dst;
        bool turns = j < turning;
        if (h < a.Hq) {
            src = static_cast<const T*>(a.q) + row * a.q_row + h * a.q_head;
            dst = a.q_out + (row * a.Hq + h) * D;
        } else if ((h -= a.Hq) < a.Hkv) {
            src = static_cast<const T*>(a.k) + row * a.k_row + h * a.k_head;
            dst = a.k_cache + places[r].slot + h * a.hs;
        } else {
            h -= a.Hkv;
            src = static_cast<const T*>(a.v) + row * a.v_row + h * a.v_head;
            dst = a.v_cache + places[r].slot + h * a.hs;
            turns = false;
        }
        int e0 = j * 2 * V, e1 = e0 + V;
        if (a.halves && j < turning) {             // v takes the same runs as k: which they are is of no account there
            e0 = j * V;
            e1 = a.pairs + j * V;
        }
        float x[V], y[V];
        load(x, src + e0);
        load(y, src + e1);
        if (turns) turn_item<V>(x, y, &turn[r][j * V], a.halves);
        if (state == kBroken) {
#pragma unroll
            for (int m = 0; m < V; ++m) x[m] = y[m] = 0.f;
        }
        store(dst + e0, x);
        store(dst + e1, y);
    }
}

template <typename T, int V>
cudaError_t issue(RopeArgs& a, int num_sms, cudaStream_t st)
{
    // As many rows per CTA as let all CTAs be resident at once, up to kRopeRows (1024 rows of 32/8 heads: 7.1 us, and 9.1 us with a few
    // CTAs in a second wave).
    const int resident = num_sms * kResident<V>;
    a.rows_per_cta = (a.total_q + resident - 1) / resident;
    if (a.rows_per_cta > kRopeRows) a.rows_per_cta = kRopeRows;
    rope_append_kernel<T, V><<<(a.total_q + a.rows_per_cta - 1) / a.rows_per_cta, kRopeThreads, 0, st>>>(a);
    return cudaGetLastError();
}

template <typename T>
cudaError_t launch(RopeArgs& a, int num_sms, cudaStream_t st)
{
    // The widest run that divides the rotated half and the strides and on whose multiples the tensors start (16384 rows of 32/8 heads,
    // bf16: 75, 82, 123 and 201 us with runs of 8, 4, 2 and 1: the work to find an item is the same for all).
    const int64_t strides = a.q_row | a.q_head | a.k_row | a.k_head | a.v_row | a.v_head | a.pairs;
    const uintptr_t at = (reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v)) / sizeof(T);
    const bool by16 = ((reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v)) & 15) == 0;
    if (((strides & 7) == 0) && by16) return issue<T, 8>(a, num_sms, st);
    if (((strides | at) & 3) == 0) return issue<T, 4>(a, num_sms, st);
    return ((strides | at) & 1) == 0 ? issue<T, 2>(a, num_sms, st) : issue<T, 1>(a, num_sms, st);
}

}  // namespace

cudaError_t launch_rope_append(RopeArgs& a, int dtype, int num_sms, cudaStream_t st)
{
    if (dtype == HOOK_DTYPE_BF16) return launch<__nv_bfloat16>(a, num_sms, st);
    if (dtype == HOOK_DTYPE_F16) return launch<__half>(a, num_sms, st);
    return launch<float>(a, num_sms, st);
}

}  // namespace hook_attn

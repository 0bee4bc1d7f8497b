// What fills and empties a cache held in 4 bits (its layout is in q4.cuh): the rotary append that quantises as it writes, and the read-back
// to the pages of a bf16 cache, which is what hook_attn_prefill and hook_capture_qk read.
//
// Quantising: the D / NG elements of a group, rounded to bf16, are lowest + step c with
//   lowest = min x,  step = (max x - min x) / 15 in bf16 (0 below 2^-100),  t = x - lowest in 32 bits,  c = t / step rounded to nearest,
// halves to even, 0 .. 15 -- of the quotient itself and not of a rounded one, so that a code can be told from the inputs.  An element is off
// by half a step at most (and by 15/512 of one more where the step was rounded down).
#include <type_traits>

#include "q4.cuh"
#include "rope_device.cuh"

namespace hook_attn {

namespace {

constexpr int kAppendThreads = 256;
constexpr int kAppendRows = 8;             // rows per CTA at most: one warp looks each of them up
constexpr int kAppendStage = 40 * 1024;    // bytes of the keys of its rows that a CTA holds

// The smaller of two pairs of bf16, element by element; NaN where either is.
__device__ __forceinline__ uint32_t min_pairs(uint32_t x, uint32_t y)
{
    uint32_t m;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(x), "r"(y));
    return m;
}

// The eight codes of four pairs of bf16 as a word: c with |t - c step| at most half a step, halves to even.  The quotient of t and the step's
// reciprocal, corrected once by what it leaves over, is t / step to the nearest: a half where that is one, so that adding 1.5 * 2^23 rounds as asked,
// and leaves the code in the low bits.  Only where a quotient next to a half became one can the code be a step off; that shows in what is left
// over, which is exact (t and c step lie within a step of one another).  The sum of the words so shifted holds all eight codes.
__device__ __forceinline__ uint32_t q4_codes(const uint32_t (&w)[4], float lo, float step)
{
    if (!(step > 0.f)) return 0;
    constexpr float kRound = 12582912.f;
    const float inv = 1.f / step, half = 0.5f * step;
    uint32_t codes = 0;
    bool off = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16) - lo;
        const float q = t * inv, rounded = fmaf(fmaf(-q, step, t), inv, q) + kRound;
        off |= fabsf(fmaf(kRound - rounded, step, t)) > half;
        codes += __float_as_uint(rounded) << (4 * e);
    }
    if (off) {
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {
            const uint32_t word = e < 4 ? (e < 2 ? w[0] : w[1]) : (e < 6 ? w[2] : w[3]);
            const float t = __uint_as_float(e & 1 ? word & 0xffff0000u : word << 16) - lo;
            const float q = t * inv, rounded = fmaf(fmaf(-q, step, t), inv, q) + kRound, left = fmaf(kRound - rounded, step, t);
            if (left > half) codes += 1u << (4 * e);
            if (left < -half) codes -= 1u << (4 * e);
        }
    }
    return codes - (0x4b400000u + 0xb4000000u + 0x40000000u);     // the constant's own bits: shifted three times they are gone
}

// A CTA takes a few rows.  Queries are turned and stored as in hook_rope_append; keys, turned, go to shared memory as bf16.  Then a thread takes
// eight neighbouring elements of a head of keys or values: the lanes of a group agree on its lowest and highest value, a thread's codes are
// a word of K as they are, and four lanes exchange theirs for V.
//
// 65536 rows of 64/8 heads in four groups (2.6 GB): 522 us, 4.9 TB/s, where hook_rope_append takes 437 us: the loads of one phase and the arithmetic of
// the other cover one another through the other CTAs of the SM alone (issue slots 52 %, DRAM 48 %, waits on loads first among the stalls).
// Queries in CTAs of their own took 620 us with the read-back instead of 592; four rows a CTA the same.  One row: 6 us.
template <typename T, int V, int HD, int NG>
__global__ void __launch_bounds__(kAppendThreads, 6) rope_append_q4_kernel(const __grid_constant__ RopeArgs a)
{
    using Slab = Q4Slab<HD, NG>;
    __shared__ __align__(16) float2 turn[kAppendRows][kMaxPairs];
    __shared__ RowPlace places[kAppendRows];
    extern __shared__ __align__(16) __nv_bfloat16 held[];            // [rows][Hkv][HD]
    const int row0 = blockIdx.x * a.rows_per_cta, warp = threadIdx.x >> 5;
    if (warp < a.rows_per_cta) {
        const RowPlace r = find_row(a, row0 + warp);
        if ((threadIdx.x & 31) == 0) {
            places[warp] = r;
            if (r.state == kBroken) report(a.status, HOOK_ATTN_ERR_BOUNDS);
        }
    }
    if (!a.positions) __syncthreads();             // the angles go by the places
    for (int i = threadIdx.x; i < a.rows_per_cta * kMaxPairs; i += kAppendThreads) {
        const int r = i / kMaxPairs, pair = i % kMaxPairs, row = row0 + r;
        if (pair < a.pairs && row < a.total_q)
            turn[r][pair] = turn_of(a, a.positions ? a.positions[a.axis_of_pair[pair] * a.axis_stride + row] : places[r].pos, pair);
    }
    __syncthreads();

    // `per` threads to a head: a thread keeps its place in a head, and goes through the heads of a row, or of as many rows as the CTA has threads
    // for, in steps that are powers of two.
    auto each_head = [&](int heads, int per, auto body) {
        int lanes = kAppendThreads;
        while (lanes / 2 >= heads * per) lanes /= 2;
        for (int r = threadIdx.x / lanes; r < a.rows_per_cta; r += kAppendThreads / lanes)
            for (int h = threadIdx.x % lanes / per; h < heads; h += lanes / per) body(r, h);
    };
    constexpr int PER_HEAD = HD / (2 * V);
    const int j = threadIdx.x % PER_HEAD;
    const bool turns = j < a.pairs / V;
    int e0 = j * 2 * V, e1 = e0 + V;
    if (a.halves && turns) {
        e0 = j * V;
        e1 = a.pairs + j * V;
    }
    each_head(a.Hkv, PER_HEAD, [&](int r, int h) {
        if (places[r].state != kGood) return;
        const T* src = static_cast<const T*>(a.k) + (int64_t)(row0 + r) * a.k_row + h * a.k_head;
        float x[V], y[V];
        load(x, src + e0);
        load(y, src + e1);
        if (turns) turn_item<V>(x, y, &turn[r][j * V], a.halves);
        store(held + (r * a.Hkv + h) * HD + e0, x);
        store(held + (r * a.Hkv + h) * HD + e1, y);
    });
    each_head(a.Hq, PER_HEAD, [&](int r, int h) {
        const int state = places[r].state;
        if (state == kBehind) return;
        const int64_t row = row0 + r;
        const T* src = static_cast<const T*>(a.q) + row * a.q_row + h * a.q_head;
        __nv_bfloat16* dst = a.q_out + (row * a.Hq + h) * HD;
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
    });
    __syncthreads();

    constexpr int CHUNKS = HD / 8, LANES = CHUNKS / NG;              // threads to a head and to a group
    const int c = threadIdx.x % CHUNKS;
    const uint32_t head_lanes = ((1u << CHUNKS) - 1) << (threadIdx.x & (32 - CHUNKS) & 31);
    each_head(2 * a.Hkv, CHUNKS, [&](int r, int kv) {
        if (places[r].state != kGood) return;
        const bool value = kv >= a.Hkv;
        const int h = value ? kv - a.Hkv : kv;
        uint32_t w[4] = {};
        if (!value) {
            const uint4 raw = *reinterpret_cast<const uint4*>(held + (r * a.Hkv + h) * HD + 8 * c);
            w[0] = raw.x; w[1] = raw.y; w[2] = raw.z; w[3] = raw.w;
        } else {
            const T* src = static_cast<const T*>(a.v) + (int64_t)(row0 + r) * a.v_row + h * a.v_head + 8 * c;
            if constexpr (std::is_same<T, __nv_bfloat16>::value && V == 8) {
                const uint4 raw = *reinterpret_cast<const uint4*>(src);
                w[0] = raw.x; w[1] = raw.y; w[2] = raw.z; w[3] = raw.w;
            } else {
                float x[8];
#pragma unroll
                for (int p = 0; p < 8 / V; ++p) {
                    float y[V];
                    load(y, src + p * V);
#pragma unroll
                    for (int m = 0; m < V; ++m) x[p * V + m] = y[m];
                }
#pragma unroll
                for (int p = 0; p < 4; ++p) w[p] = pack_bf16(x[2 * p], x[2 * p + 1]);
            }
        }
        // lowest, and the lowest of the negated ones, as a pair: a NaN stays in it, and an infinity leaves no finite range
        const uint32_t low = min_pairs(min_pairs(w[0], w[1]), min_pairs(w[2], w[3]));
        const uint32_t high = min_pairs(min_pairs(w[0] ^ 0x80008000u, w[1] ^ 0x80008000u), min_pairs(w[2] ^ 0x80008000u, w[3] ^ 0x80008000u));
        uint32_t range = min_pairs(__byte_perm(low, high, 0x5410), __byte_perm(low, high, 0x7632));
#pragma unroll
        for (int d = 1; d < LANES; d <<= 1) range = min_pairs(range, __shfl_xor_sync(head_lanes, range, d));
        const float lo = q4_step(range) + 0.f, width = -q4_lowest(range) - lo;    // one zero
        const float fifteenth = width * (1.f / 15.f);                             // corrected once: width / 15 to the nearest
        float step = __bfloat162float(__float2bfloat16(fmaf(fmaf(-fifteenth, 15.f, width), 1.f / 15.f, fifteenth)));
        if (step < 7.88860905e-31f) step = 0.f;                                   // 2^-100
        if (!(step <= 3.3895314e38f)) step = __int_as_float(0x7fc00000);
        const uint32_t codes = q4_codes(w, lo, step);
        const int t = places[r].pos % kPage;
        uint8_t* slab = reinterpret_cast<uint8_t*>(a.k_cache) + places[r].slot + h * a.hs;
        if (!value) {
            *reinterpret_cast<uint32_t*>(slab + t * Slab::kRow + (c % 4 * (HD / 32) + c / 4) * 4) = codes;
        } else {
            uint32_t others[4];                    // of the four chunks of 32 elements, in their order
#pragma unroll
            for (int k = 0; k < 4; ++k) others[k] = __shfl_sync(head_lanes, codes, (threadIdx.x & 28) + k);
            const int n = c % 4, row = q4_row(t);
            uint32_t even = 0, odd = 0;            // nibbles of elements 2 n and 2 n + 1 of the four chunks
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t byte = others[k] >> (8 * n);
                even |= (byte & 15u) << (4 * k);
                odd |= ((byte >> 4) & 15u) << (4 * k);
            }
            uint8_t* at = slab + Slab::kCodes + row * Slab::kRow + c / 4 * 2;
            *reinterpret_cast<uint16_t*>(at + q4_unit<HD>(row, 2 * n) * (HD / 16)) = (uint16_t)even;
            *reinterpret_cast<uint16_t*>(at + q4_unit<HD>(row, 2 * n + 1) * (HD / 16)) = (uint16_t)odd;
        }
        if (c % LANES == 0) {
            const uint32_t pair = (__float_as_uint(step) >> 16) | (__float_as_uint(lo) & 0xffff0000u);
            *reinterpret_cast<uint32_t*>(slab + 2 * Slab::kCodes + value * Slab::kParams + (t * NG + c / LANES) * 4) = pair;
        }
    });
}

template <typename T, int V, int HD, int NG>
cudaError_t issue(RopeArgs& a, int num_sms, cudaStream_t st)
{
    // as many rows per CTA as let all CTAs be resident at once, within the shared memory that holds their keys and values
    const int row_bytes = a.Hkv * HD * 2, resident = num_sms * 6;
    int rows = (a.total_q + resident - 1) / resident;
    if (rows > kAppendRows) rows = kAppendRows;
    if (rows > kAppendStage / row_bytes) rows = kAppendStage / row_bytes > 0 ? kAppendStage / row_bytes : 1;
    a.rows_per_cta = rows;
    rope_append_q4_kernel<T, V, HD, NG><<<(a.total_q + rows - 1) / rows, kAppendThreads, rows * row_bytes, st>>>(a);
    return cudaGetLastError();
}

template <typename T, int V>
cudaError_t for_group(RopeArgs& a, int group, int num_sms, cudaStream_t st)
{
    const int ng = a.head_dim / group;
    if (a.head_dim == 64) return ng == 1 ? issue<T, V, 64, 1>(a, num_sms, st) : issue<T, V, 64, 2>(a, num_sms, st);
    if (ng == 1) return issue<T, V, 128, 1>(a, num_sms, st);
    return ng == 2 ? issue<T, V, 128, 2>(a, num_sms, st) : issue<T, V, 128, 4>(a, num_sms, st);
}

template <typename T>
cudaError_t launch(RopeArgs& a, int group, int num_sms, cudaStream_t st)
{
    // the widest run that divides the rotated half and the strides and on whose multiples the tensors start, as in hook_rope_append
    const int64_t strides = a.q_row | a.q_head | a.k_row | a.k_head | a.v_row | a.v_head | a.pairs;
    const uintptr_t from = reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v);
    if (((strides & 7) == 0) && (from & 15) == 0) return for_group<T, 8>(a, group, num_sms, st);
    if (((strides | (int64_t)(from / sizeof(T))) & 3) == 0) return for_group<T, 4>(a, group, num_sms, st);
    if (((strides | (int64_t)(from / sizeof(T))) & 1) == 0) return for_group<T, 2>(a, group, num_sms, st);
    return for_group<T, 1>(a, group, num_sms, st);
}

// ---- read-back ----------------------------------------------------------------------------------------------------------------------
constexpr int kReadThreads = 256;

// A warp takes a (page, KV head) of a sequence: the slab comes to shared memory with wide loads, then a lane writes 16 bytes of a token's
// row at a time.  73728 tokens of 8 heads in four groups (397 MB, three quarters of them written): 73 us, 5.4 TB/s.
template <int HD, int NG>
__global__ void __launch_bounds__(kReadThreads) q4_read_kernel(const __grid_constant__ Q4ReadArgs a)
{
    using Slab = Q4Slab<HD, NG>;
    constexpr int WARPS = kReadThreads / 32, CHUNKS = HD / 8;
    __shared__ __align__(16) uint8_t slabs[WARPS][Slab::kBytes];
    const int s = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int L = a.seq_lens[s];
    int from = a.first ? a.first[s] : 0;
    if (L < 0 || L > a.max_keys || from < 0) {
        if (blockIdx.x == 0 && threadIdx.x == 0) report(a.status, HOOK_ATTN_ERR_BOUNDS);
        return;
    }
    const int page0 = from / kPage;
    const int64_t units = (int64_t)max(0, (L + kPage - 1) / kPage - page0) * a.Hkv;
    uint8_t* mine = slabs[warp];
    for (int64_t u = (int64_t)blockIdx.x * WARPS + warp; u < units; u += (int64_t)gridDim.x * WARPS) {
        const int j = page0 + (int)(u / a.Hkv), h = (int)(u % a.Hkv);
        const int page = a.block_table[(int64_t)s * a.max_blocks + j], to = a.to_table[(int64_t)s * a.to_max_blocks + j];
        if (page < 0 || page >= a.num_blocks || to < 0 || to >= a.to_num_blocks) {
            if (lane == 0) report(a.status, HOOK_ATTN_ERR_BOUNDS);
            continue;
        }
        const uint4* src = reinterpret_cast<const uint4*>(a.pages + (int64_t)page * a.page_block + (int64_t)h * a.page_head);
        __syncwarp();
        for (int i = lane; i < Slab::kBytes / 16; i += 32) reinterpret_cast<uint4*>(mine)[i] = src[i];
        __syncwarp();
        const int t_from = max(0, from - j * kPage), t_to = min(kPage, L - j * kPage);
        const int64_t out = (int64_t)to * a.bs + (int64_t)h * a.hs;
        const uint32_t* params = reinterpret_cast<const uint32_t*>(mine + 2 * Slab::kCodes);
        for (int i = lane; i < kPage * CHUNKS; i += 32) {
            const int t = i / CHUNKS, c = i % CHUNKS;
            if (t < t_from || t >= t_to) continue;
            const uint32_t kp = params[t * NG + c / (CHUNKS / NG)], vp = params[(kPage + t) * NG + c / (CHUNKS / NG)];
            const uint32_t codes = *reinterpret_cast<const uint32_t*>(mine + t * Slab::kRow + (c % 4 * (HD / 32) + c / 4) * 4);
            const int row = q4_row(t);
            const uint8_t* vrow = mine + Slab::kCodes + row * Slab::kRow + c / 4 * 2;
            float k[8], v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                k[e] = fmaf(q4_step(kp), (float)((codes >> (4 * e)) & 15u), q4_lowest(kp));
                const uint32_t half = *reinterpret_cast<const uint16_t*>(vrow + q4_unit<HD>(row, e) * (HD / 16));
                v[e] = fmaf(q4_step(vp), (float)((half >> (4 * (c % 4))) & 15u), q4_lowest(vp));
            }
            store(a.k_cache + out + (int64_t)t * a.ts + 8 * c, k);
            store(a.v_cache + out + (int64_t)t * a.ts + 8 * c, v);
        }
    }
}

}  // namespace

// `a.k_cache` is the pages, `a.bs` and `a.hs` their strides in bytes, `a.ts` 0.
cudaError_t launch_rope_append_q4(RopeArgs& a, int dtype, int group, int num_sms, cudaStream_t st)
{
    if (dtype == HOOK_DTYPE_BF16) return launch<__nv_bfloat16>(a, group, num_sms, st);
    if (dtype == HOOK_DTYPE_F16) return launch<__half>(a, group, num_sms, st);
    return launch<float>(a, group, num_sms, st);
}

cudaError_t launch_q4_read(const Q4ReadArgs& a, int head_dim, int group, int num_sms, cudaStream_t st)
{
    // CTAs for the longest sequence that the table allows, and no more in all than fill the device a few times
    const int64_t most = ((int64_t)a.max_keys / kPage + 1) * a.Hkv / (kReadThreads / 32) + 1, share = (int64_t)num_sms * 32 / a.num_seqs + 1;
    const dim3 grid((unsigned)(most < share ? most : share), a.num_seqs);
    const int ng = head_dim / group;
    if (head_dim == 64) {
        if (ng == 1) q4_read_kernel<64, 1><<<grid, kReadThreads, 0, st>>>(a);
        else q4_read_kernel<64, 2><<<grid, kReadThreads, 0, st>>>(a);
    } else if (ng == 1) q4_read_kernel<128, 1><<<grid, kReadThreads, 0, st>>>(a);
    else if (ng == 2) q4_read_kernel<128, 2><<<grid, kReadThreads, 0, st>>>(a);
    else q4_read_kernel<128, 4><<<grid, kReadThreads, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace hook_attn

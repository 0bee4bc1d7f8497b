// Edits of the logits before a token is chosen: penalties for tokens that have come already, sparse biases, grammar
// masks.  For token v of a row, with c the number of times it was generated and `seen` whether it is in the prompt or
// generated:
//   x <- x > 0 ? x / repetition : x * repetition  if seen;   x <- x - frequency * c - presence * (c > 0);
//   x <- x + bias[v];   x <- -inf  if the row's grammar forbids v.
#include "common.cuh"
#include "ops.cuh"

#include <cuda_fp16.h>

namespace hook_attn {

namespace {

// A token's word: the lowest bits count how often it was generated, the next hold 1 + the place of its bias in the row's list,
// the top bit says that it is in the prompt.  0: nothing but the grammar concerns it.
constexpr int kCountBits = 20, kPlaceBits = 11;
constexpr uint32_t kSeen = 0x80000000u, kCountMask = (1u << kCountBits) - 1, kPlaceMask = ((1u << kPlaceBits) - 1) << kCountBits;
static_assert(kMaxHistory == (int)kCountMask && kMaxRowBias == (int)(kPlaceMask >> kCountBits), "limits of the words");

__device__ __forceinline__ float load_f32(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float load_f32(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ float load_f32(const float* p) { return *p; }
__device__ __forceinline__ void store_f32(__nv_bfloat16* p, float x) { *p = __float2bfloat16(x); }
__device__ __forceinline__ void store_f32(__half* p, float x) { *p = __float2half(x); }
__device__ __forceinline__ void store_f32(float* p, float x) { *p = x; }

// A stretch of one row: the values [lo, hi).  Its words lie so that the eight of a vector are aligned: word 8 belongs to `base`,
// the stretch's first value whose address is a multiple of 16 bytes; the values of a row before its first such one take the words
// before it, in the row's first stretch.
struct Stretch {
    float rep, inv_rep, pres, freq;
    const float* bias;             // the row's bias values
    const uint32_t* grammar;       // its mask, or null
    int row, total, prompt, b0, b1;
    int lo, hi, base, first;       // first: the value that word 0 would belong to
    bool valid, any;               // any: the history or the biases may concern it
};

// Values of a row before the first one whose address is a multiple of 16 bytes.
template <typename TI>
__device__ __forceinline__ int values_before_aligned(const LogitsArgs& a, int row)
{
    constexpr uintptr_t kPer16 = 16 / sizeof(TI);
    const TI* in = static_cast<const TI*>(a.logits) + (int64_t)row * a.in_row;
    return (int)((kPer16 - reinterpret_cast<uintptr_t>(in) / sizeof(TI) % kPer16) % kPer16);
}

template <typename TI>
__device__ __forceinline__ Stretch place_stretch(const LogitsArgs& a, int row, int slice, int length)
{
    Stretch s;
    s.row = row;
    s.base = values_before_aligned<TI>(a, row) + slice * length;
    s.lo = slice == 0 ? 0 : min(s.base, a.vocab);             // a row with a head may need one stretch less
    s.hi = min(s.base + length, a.vocab);
    s.first = s.base - 8;
    return s;
}

// A row's numbers as they come from memory; the values are fetched between them and their use.
struct Numbers {
    int total, prompt, b0, b1, mask;
    float rep, pres, freq;
};

__device__ __forceinline__ Numbers fetch_numbers(const LogitsArgs& a, int row)
{
    Numbers n;
    n.total = a.tokens ? a.total_lens[row] : 0;
    n.prompt = a.tokens ? a.prompt_lens[row] : 0;
    n.b0 = a.bias_offsets ? a.bias_offsets[row] : 0;
    n.b1 = a.bias_offsets ? a.bias_offsets[row + 1] : 0;
    n.mask = !a.mask ? -1 : a.mask_rows ? a.mask_rows[row] : row;
    n.rep = a.repetition ? a.repetition[row] : 1.f;
    n.pres = a.presence ? a.presence[row] : 0.f;
    n.freq = a.frequency ? a.frequency[row] : 0.f;
    return n;
}

__device__ __forceinline__ void open_stretch(const LogitsArgs& a, const Numbers& n, Stretch& s)
{
    s.total = n.total;
    s.prompt = n.prompt;
    s.b0 = n.b0;
    s.b1 = n.b1;
    s.rep = n.rep;
    s.inv_rep = __frcp_rn(n.rep);
    s.pres = n.pres;
    s.freq = n.freq;
    s.valid = n.total >= 0 && n.total <= a.max_tokens && n.prompt >= 0 && n.prompt <= n.total && n.b0 >= 0 && n.b1 >= n.b0 &&
              n.b1 <= a.num_bias && n.b1 - n.b0 <= kMaxRowBias && n.mask < a.num_masks;
    s.any = s.valid && (n.total > 0 || n.b1 > n.b0);
    s.bias = a.bias_values + (s.valid ? n.b0 : 0);
    s.grammar = s.valid && n.mask >= 0 ? a.mask + (int64_t)n.mask * a.mask_row : nullptr;
}

// 1 / repetition may leave the range of the normal numbers where a quotient by it does not.  Such a row is divided value by value: chosen in
// the vectors' edits, 256 rows of 160000 values would take 75 us instead of 72.5.
__device__ __forceinline__ bool far(float rep) { return !(rep >= 0x1p-126f && rep <= 0x1p126f); }

// A value with a word that is not zero.  Multiplied by 1 / repetition, a positive value is rounded twice; FAR: divided.
template <bool FAR>
__device__ __forceinline__ float edit(float x, uint32_t word, const Stretch& r)
{
    const uint32_t made = word & kCountMask;
    const bool seen = word & (kSeen | kCountMask);
    if (FAR && seen && x > 0.f) {
        x /= r.rep;
    } else {
        x *= seen ? (x > 0.f ? r.inv_rep : r.rep) : 1.f;
    }
    x -= made ? r.freq * (float)made + r.pres : 0.f;            // an infinite penalty is none for what was not generated
    if (word & kPlaceMask) x += r.bias[((word & kPlaceMask) >> kCountBits) - 1];
    return x;
}

template <typename T>
struct alignas(16) Vec {            // eight values: one or two accesses of 16 bytes
    T x[8];
};

// The row's history as THREADS threads look through it for tokens of a stretch, four at a time.  The first eight tokens of each
// thread are fetched when it is made, so that they are there when the words are ready to count in.  Integers: the order of the
// atomics is of no account.
template <int THREADS>
struct History {
    const int32_t* tokens;
    int tid, head, quads;
    int4 held[2];

    __device__ __forceinline__ History(const LogitsArgs& a, const Stretch& s, int thread)
        : tokens(a.tokens + (int64_t)s.row * a.token_row), tid(thread),
          head(min(s.total, (int)((4 - reinterpret_cast<uintptr_t>(tokens) / 4 % 4) % 4))), quads((s.total - head) / 4)
    {
        fetch(tid);
    }
    __device__ __forceinline__ void fetch(int i0)
    {
#pragma unroll
        for (int u = 0; u < 2; ++u)
            held[u] = i0 + u * THREADS < quads ? reinterpret_cast<const int4*>(tokens + head)[i0 + u * THREADS] : make_int4(-1, -1, -1, -1);
    }
    // Most tokens belong to other stretches: a token costs its test and one predicated reduction in shared memory, no branch.
    __device__ __forceinline__ void count(const Stretch& s, uint32_t* word)
    {
        const uint32_t span = s.hi - s.lo, at = smem_u32(word) + 4 * (s.lo - s.first);
        auto see = [&](int t) {
            asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.u32 p, %0, %1;\n\t@p red.shared.or.b32 [%2], %3;\n\t}"
                         ::"r"((uint32_t)t - (uint32_t)s.lo), "r"(span), "r"(at + 4 * ((uint32_t)t - (uint32_t)s.lo)), "r"(kSeen) : "memory");
        };
        auto make = [&](int t) {
            asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.u32 p, %0, %1;\n\t@p red.shared.add.u32 [%2], %3;\n\t}"
                         ::"r"((uint32_t)t - (uint32_t)s.lo), "r"(span), "r"(at + 4 * ((uint32_t)t - (uint32_t)s.lo)), "r"(1u) : "memory");
        };
        auto take = [&](int t, int i) { i < s.prompt ? see(t) : make(t); };
        const int seen = s.prompt <= head ? 0 : (s.prompt - head) / 4;    // quads that lie in the prompt; the next may do so in part
        for (int i0 = tid; i0 < quads; i0 += 2 * THREADS) {
            const int4 now[2] = {held[0], held[1]};
            fetch(i0 + 2 * THREADS);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int quad = i0 + u * THREADS, i = head + 4 * quad;
                const int4 t = now[u];
                if (quad < seen) {
                    see(t.x); see(t.y); see(t.z); see(t.w);
                } else if (i >= s.prompt) {
                    make(t.x); make(t.y); make(t.z); make(t.w);
                } else {
                    take(t.x, i); take(t.y, i + 1); take(t.z, i + 2); take(t.w, i + 3);
                }
            }
        }
        const int i = tid < head ? tid : 4 * quads + tid;                 // what no quad covers, six tokens at most
        if (i < s.total && tid < s.total - 4 * quads) take(tokens[i], i);
    }
};

// Puts one of the row's biases into its word: of a token that is named twice the last entry counts.
__device__ __forceinline__ void place_bias(const LogitsArgs& a, const Stretch& s, uint32_t* word, int i)
{
    const int t = a.bias_tokens[i];
    if (t < 0 || t >= a.vocab) {
        if (s.lo == 0) report(a.status, HOOK_ATTN_ERR_BOUNDS);
        return;
    }
    if ((unsigned)t - (unsigned)s.lo >= (unsigned)(s.hi - s.lo)) return;
    uint32_t* w = &word[t - s.first];
    uint32_t old = *w;
    const uint32_t mine = (uint32_t)(i - s.b0 + 1) << kCountBits;
    while ((old & kPlaceMask) < mine) {
        const uint32_t was = atomicCAS(w, old, (old & ~kPlaceMask) | mine);
        if (was == old) return;
        old = was;
    }
}

// Eight values that begin at v, with the words of the stretch; `low` and `high` are the mask's words of the first and the last.
template <typename TI, typename TO>
__device__ __forceinline__ Vec<TO> edit_eight(const Vec<TI>& raw, const uint4& w0, const uint4& w1, uint32_t low, uint32_t high, int v,
                                              const Stretch& s)
{
    const uint32_t w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
    const uint32_t allowed = __funnelshift_r(low, high, v & 31);          // eight bits that may lie in two words
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        x[k] = load_f32(&raw.x[k]);
        if (w[k]) x[k] = edit<false>(x[k], w[k], s);
    }
    Vec<TO> res;
#pragma unroll
    for (int k = 0; k < 8; ++k) store_f32(&res.x[k], (allowed >> k) & 1u ? x[k] : -INFINITY);
    return res;
}

template <bool FAR, typename TI, typename TO>
__device__ __forceinline__ void edit_one(const TI* in, TO* out, int v, uint32_t w, const Stretch& s)
{
    const float x = edit<FAR>(load_f32(in + v), w, s);
    store_f32(out + v, s.grammar && !((s.grammar[v >> 5] >> (v & 31)) & 1u) ? -INFINITY : x);
}

// All of a stretch of a far row.
template <typename TI, typename TO>
__device__ __forceinline__ void edit_slowly(const TI* in, TO* out, const uint32_t* word, const Stretch& s, int threads)
{
    for (int i = s.lo + threadIdx.x; i < s.hi; i += threads) edit_one<true>(in, out, i, s.any ? word[i - s.first] : 0u, s);
}

// Small calls: a CTA takes one stretch, one vector to a thread, whose load is under way while the words are filled.  Bound by the
// chain of loads (the row's numbers, its history, the words): 2.8 us for 1 x 32000 with 300 tokens.
template <typename TI, typename TO, int THREADS>
__global__ void __launch_bounds__(THREADS) adjust_logits_kernel(const __grid_constant__ LogitsArgs a)
{
    constexpr int kLength = THREADS * 8;
    __shared__ __align__(16) uint32_t word[kLength + 8];
    const int tid = threadIdx.x;
    Stretch s = place_stretch<TI>(a, blockIdx.y, blockIdx.x, kLength);
    if (s.lo >= s.hi) return;
    const Numbers numbers = fetch_numbers(a, s.row);
    const TI* in = static_cast<const TI*>(a.logits) + (int64_t)s.row * a.in_row;
    TO* out = static_cast<TO*>(a.out) + (int64_t)s.row * a.out_row;
    const bool aligned = (reinterpret_cast<uintptr_t>(out + s.base) & 15) == 0;    // in and out reach a multiple of 16 bytes together
    const int vectors = aligned ? max(s.hi - s.base, 0) / 8 : 0, v = s.base + 8 * tid;
    Vec<TI> raw;
    if (tid < vectors) raw = *reinterpret_cast<const Vec<TI>*>(in + v);
    open_stretch(a, numbers, s);
    if (!s.valid) {
        if (tid == 0 && blockIdx.x == 0) report(a.status, HOOK_ATTN_ERR_BOUNDS);
        return;
    }
    History<THREADS> history(a, s, tid);
    uint32_t low = ~0u, high = ~0u;
    if (s.grammar && tid < vectors) {
        low = s.grammar[v >> 5];
        high = s.grammar[(v + 7) >> 5];
    }
    if (s.any) {
        for (int i = tid; i < (s.hi - s.first + 3) / 4; i += THREADS) reinterpret_cast<uint4*>(word)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        history.count(s, word);
        for (int i = s.b0 + tid; i < s.b1; i += THREADS) place_bias(a, s, word, i);
        __syncthreads();
    }
    if (far(s.rep)) return edit_slowly(in, out, word, s, THREADS);
    if (tid < vectors) {
        const uint4* w = reinterpret_cast<const uint4*>(word + 8 + 8 * tid);
        const uint4 none = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<Vec<TO>*>(out + v) = edit_eight<TI, TO>(raw, s.any ? w[0] : none, s.any ? w[1] : none, low, high, v, s);
    }
    // what no vector covers: the row's head, the values behind the last vector, all of a stretch that is not aligned
    if (s.lo == 0 && tid < min(s.base, s.hi)) edit_one<false>(in, out, tid, s.any ? word[tid - s.first] : 0u, s);
    for (int i = s.base + 8 * vectors + tid; i < s.hi; i += THREADS) edit_one<false>(in, out, i, s.any ? word[i - s.first] : 0u, s);
}

// Large calls: a CTA takes a long stretch, all of whose loads are under way while its words are filled; four CTAs of 256 threads on an
// SM or one of 1024, with 64 registers each.  Without a history it is bound by HBM (256 rows of 160000 fp32 values with masks: 54 us, 6.1
// TB/s).  With one, by phases that do not cover one another, with half of the issue slots and of the bandwidth in use: each stretch of a row looks
// through the whole history, and a warp runs the edit for each of the eight values of a lane that any of its lanes has a word for (the same with
// histories of up to 4096 tokens: 72 us, 4.6 TB/s; 64 rows of 128000 bf16 to fp32 values with up to 32768 tokens: 27 us, 2.0 TB/s, in two
// waves of CTAs: 37 rows, one wave, take 13 us).
constexpr int kTogether = 4;

template <int THREADS>
struct Large {
    static constexpr int kLength = THREADS * kTogether * 8;               // values of a stretch
    uint32_t grammar[kLength / 32 + 4];
    uint32_t word[kLength + 8];
};

template <typename TI, typename TO, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) adjust_logits_large_kernel(const __grid_constant__ LogitsArgs a)
{
    extern __shared__ __align__(16) uint8_t smem[];
    Large<THREADS>& w = *reinterpret_cast<Large<THREADS>*>(smem);
    constexpr int kLength = Large<THREADS>::kLength;
    const int tid = threadIdx.x;
    Stretch s = place_stretch<TI>(a, blockIdx.y, blockIdx.x, kLength);
    if (s.lo >= s.hi) return;
    const Numbers numbers = fetch_numbers(a, s.row);
    const TI* in = static_cast<const TI*>(a.logits) + (int64_t)s.row * a.in_row;
    TO* out = static_cast<TO*>(a.out) + (int64_t)s.row * a.out_row;
    const int vectors = (reinterpret_cast<uintptr_t>(out + s.base) & 15) == 0 ? max(s.hi - s.base, 0) / 8 : 0;
    Vec<TI> raw[kTogether];
#pragma unroll
    for (int u = 0; u < kTogether; ++u)
        if (tid + u * THREADS < vectors) raw[u] = *reinterpret_cast<const Vec<TI>*>(in + s.base + 8 * (tid + u * THREADS));
    open_stretch(a, numbers, s);
    if (!s.valid) {
        if (tid == 0 && blockIdx.x == 0) report(a.status, HOOK_ATTN_ERR_BOUNDS);
        return;
    }
    History<THREADS> history(a, s, tid);
    const int mask0 = s.lo >> 5;                                          // the stretch's part of the mask
    if (s.grammar)
        for (int i = tid; i <= ((s.hi - 1) >> 5) - mask0; i += THREADS) w.grammar[i] = s.grammar[mask0 + i];
    if (s.any)
        for (int i = tid; i < (s.hi - s.first + 3) / 4; i += THREADS) reinterpret_cast<uint4*>(w.word)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    if (s.any) {
        history.count(s, w.word);
        for (int i = s.b0 + tid; i < s.b1; i += THREADS) place_bias(a, s, w.word, i);
        __syncthreads();
    }
    if (far(s.rep)) return edit_slowly(in, out, w.word, s, THREADS);
#pragma unroll
    for (int u = 0; u < kTogether; ++u) {
        const int i = tid + u * THREADS, v = s.base + 8 * i;
        if (i >= vectors) break;
        uint4 w0 = make_uint4(0, 0, 0, 0), w1 = w0;
        if (s.any) {
            w0 = reinterpret_cast<const uint4*>(w.word + 8)[2 * i];
            w1 = reinterpret_cast<const uint4*>(w.word + 8)[2 * i + 1];
        }
        uint32_t low = ~0u, high = ~0u;
        if (s.grammar) {
            low = w.grammar[(v >> 5) - mask0];
            high = w.grammar[((v + 7) >> 5) - mask0];
        }
        *reinterpret_cast<Vec<TO>*>(out + v) = edit_eight<TI, TO>(raw[u], w0, w1, low, high, v, s);
    }
    // as in the small kernel: what no vector covers
    if (s.lo == 0 && tid < min(s.base, s.hi)) edit_one<false>(in, out, tid, s.any ? w.word[tid - s.first] : 0u, s);
    for (int i = s.base + 8 * vectors + tid; i < s.hi; i += THREADS) edit_one<false>(in, out, i, s.any ? w.word[i - s.first] : 0u, s);
}

template <typename TI, typename TO, int THREADS>
cudaError_t launch_small(const LogitsArgs& a, cudaStream_t st)
{
    adjust_logits_kernel<TI, TO, THREADS><<<dim3((a.vocab + THREADS * 8 - 1) / (THREADS * 8), a.rows), THREADS, 0, st>>>(a);
    return cudaGetLastError();
}

template <typename TI, typename TO, int THREADS>
cudaError_t launch_large(const LogitsArgs& a, cudaStream_t st)
{
    constexpr int kLength = Large<THREADS>::kLength;
    adjust_logits_large_kernel<TI, TO, THREADS>
        <<<dim3((a.vocab + kLength - 1) / kLength, a.rows), THREADS, sizeof(Large<THREADS>), st>>>(a);
    return cudaGetLastError();
}

template <typename TI, typename TO>
cudaError_t launch(const LogitsArgs& a, int num_sms, cudaStream_t st)
{
    // By the width of the token buffer, since the histories' lengths are on the device: shorter histories in a wide buffer take the times of the
    // form for wide ones.  Long stretches (8192 or 32768 values) for long rows once there are enough of them for all SMs.  Short and long ones take 4.9 and
    // 5.5 us for 8 x 128000 with 4000 tokens a row, 6.9 and 6.4 us for 12 x 128000, 13.7 and 9.3 us for 32 x 128000; 10.0 and 11.3 us
    // for 12 x 128000 with 16000 tokens, 13.6 and 12.8 us with 32768.  Of the long ones, 32768 values look through long histories less
    // often: with 8192 and 32768, 64 x 128000 takes 14.5 and 16.2 us with 4000 tokens, 20.4 and 20.5 us with 12000, 26.9 and 23.1 us
    // with 24000.
    if (a.vocab >= 16384 && (int64_t)a.rows * a.vocab >= (int64_t)num_sms * 10240)
        return a.max_tokens > 12288 ? launch_large<TI, TO, 1024>(a, st) : launch_large<TI, TO, 256>(a, st);
    // More threads look through a long history side by side: 1 x 128000 takes 7.3, 5.5, 5.3 us with 128, 256, 512 threads and 16000
    // tokens, 3.8, 3.5, 3.8 us with 4000, 3.2, 3.3, 3.7 us with 100.
    if (a.max_tokens > 8192) return launch_small<TI, TO, 512>(a, st);
    return a.max_tokens > 1024 ? launch_small<TI, TO, 256>(a, st) : launch_small<TI, TO, 128>(a, st);
}

template <typename TI, typename TO>
cudaError_t configure()
{
    const cudaError_t e = cudaFuncSetAttribute(adjust_logits_large_kernel<TI, TO, 256>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(Large<256>));
    return e != cudaSuccess ? e : cudaFuncSetAttribute(adjust_logits_large_kernel<TI, TO, 1024>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(Large<1024>));
}

}  // namespace

cudaError_t configure_logits()
{
    cudaError_t e = configure<__nv_bfloat16, __nv_bfloat16>();
    if (e == cudaSuccess) e = configure<__nv_bfloat16, float>();
    if (e == cudaSuccess) e = configure<__half, __half>();
    if (e == cudaSuccess) e = configure<__half, float>();
    if (e == cudaSuccess) e = configure<float, float>();
    return e;
}

cudaError_t launch_adjust_logits(const LogitsArgs& a, int dtype, int out_dtype, int num_sms, cudaStream_t st)
{
    if (dtype == HOOK_DTYPE_BF16) return out_dtype == dtype ? launch<__nv_bfloat16, __nv_bfloat16>(a, num_sms, st) : launch<__nv_bfloat16, float>(a, num_sms, st);
    if (dtype == HOOK_DTYPE_F16) return out_dtype == dtype ? launch<__half, __half>(a, num_sms, st) : launch<__half, float>(a, num_sms, st);
    return launch<float, float>(a, num_sms, st);
}

}  // namespace hook_attn

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

constexpr int kLogitThreads = 256;
constexpr int kSlice = 8192;                     // entries of a row per CTA: 32 KB of counters, 32 KB of bias places
constexpr uint32_t kSeen = 0x80000000u;          // top bit of a counter: the token is in the prompt

__device__ __forceinline__ float load_f32(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float load_f32(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ float load_f32(const float* p) { return *p; }
__device__ __forceinline__ void store_f32(__nv_bfloat16* p, float x) { *p = __float2bfloat16(x); }
__device__ __forceinline__ void store_f32(__half* p, float x) { *p = __float2half(x); }
__device__ __forceinline__ void store_f32(float* p, float x) { *p = x; }

// A CTA owns one slice of one row: it counts the row's tokens that fall into the slice in shared memory (integers, so
// the order of the atomics is of no account) and then passes over the slice once.
template <typename TI, typename TO>
__global__ void __launch_bounds__(kLogitThreads) adjust_logits_kernel(const __grid_constant__ LogitsArgs a)
{
    extern __shared__ uint32_t sh[];
    uint32_t* count = sh;                        // [kSlice]
    uint32_t* place = sh + kSlice;               // [kSlice], with biases: 1 + the last entry that names the token
    const int row = blockIdx.y, v0 = blockIdx.x * kSlice, n = min(kSlice, a.vocab - v0);
    const int total = a.tokens ? a.total_lens[row] : 0, prompt = a.tokens ? a.prompt_lens[row] : 0;
    const int b0 = a.bias_offsets ? a.bias_offsets[row] : 0, b1 = a.bias_offsets ? a.bias_offsets[row + 1] : 0;
    const int grammar = !a.mask ? -1 : a.mask_rows ? a.mask_rows[row] : row;
    if (total < 0 || total > a.max_tokens || prompt < 0 || prompt > total || b0 < 0 || b1 < b0 || b1 > a.num_bias || grammar >= a.num_masks) {
        if (threadIdx.x == 0 && blockIdx.x == 0) report(a.status, HOOK_ATTN_ERR_BOUNDS);
        return;
    }
    for (int i = threadIdx.x; i < n; i += kLogitThreads) {
        count[i] = 0;
        if (b1 > b0) place[i] = 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < total; i += kLogitThreads) {
        const int t = a.tokens[(int64_t)row * a.token_row + i] - v0;
        if ((unsigned)t < (unsigned)n) {
            if (i < prompt) atomicOr(&count[t], kSeen);
            else atomicAdd(&count[t], 1u);
        }
    }
    for (int i = b0 + threadIdx.x; i < b1; i += kLogitThreads) {
        const int v = a.bias_tokens[i], t = v - v0;
        if (v < 0 || v >= a.vocab) report(a.status, HOOK_ATTN_ERR_BOUNDS);
        else if ((unsigned)t < (unsigned)n) atomicMax(&place[t], (uint32_t)(i - b0) + 1u);
    }
    __syncthreads();
    const float rep = a.repetition ? a.repetition[row] : 1.f, pres = a.presence ? a.presence[row] : 0.f;
    const float freq = a.frequency ? a.frequency[row] : 0.f;
    const TI* in = static_cast<const TI*>(a.logits) + (int64_t)row * a.in_row + v0;
    TO* out = static_cast<TO*>(a.out) + (int64_t)row * a.out_row + v0;
    const uint32_t* words = grammar >= 0 ? a.mask + (int64_t)grammar * a.mask_row : nullptr;
    for (int i = threadIdx.x; i < n; i += kLogitThreads) {
        float x = load_f32(in + i);
        const uint32_t c = count[i];
        if (c) {
            x = x > 0.f ? x / rep : x * rep;
            const uint32_t made = c & ~kSeen;
            if (made) x = x - freq * (float)made - pres;
        }
        if (b1 > b0 && place[i]) x += a.bias_values[b0 + place[i] - 1];
        if (words && !((words[(v0 + i) >> 5] >> ((v0 + i) & 31)) & 1u)) x = -INFINITY;
        store_f32(out + i, x);
    }
}

template <typename TI, typename TO>
cudaError_t launch(const LogitsArgs& a, cudaStream_t st)
{
    const dim3 grid((a.vocab + kSlice - 1) / kSlice, a.rows);
    adjust_logits_kernel<TI, TO><<<grid, kLogitThreads, 2 * kSlice * 4, st>>>(a);
    return cudaGetLastError();
}

template <typename TI, typename TO>
cudaError_t configure()
{
    return cudaFuncSetAttribute(adjust_logits_kernel<TI, TO>, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * kSlice * 4);
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

cudaError_t launch_adjust_logits(const LogitsArgs& a, int dtype, int out_dtype, cudaStream_t st)
{
    if (dtype == HOOK_DTYPE_BF16) return out_dtype == dtype ? launch<__nv_bfloat16, __nv_bfloat16>(a, st) : launch<__nv_bfloat16, float>(a, st);
    if (dtype == HOOK_DTYPE_F16) return out_dtype == dtype ? launch<__half, __half>(a, st) : launch<__half, float>(a, st);
    return launch<float, float>(a, st);
}

}  // namespace hook_attn

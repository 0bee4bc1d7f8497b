// The choice of a token from a row of logits and one random number: temperature, top-k, min-p, top-p.
//
// A cluster of CTAs takes a row.  Each CTA holds a stretch of it in shared memory, so that the row is read once, and they exchange what
// little the others need through distributed shared memory.  All three filters keep the first tokens in the order of falling logits
// (equal ones by index), so what stays is a least key K and how many of the tokens at K itself: tokens are never sorted.
//
// K is found by narrowing down: a histogram of the tokens' counts (top-k) or weights (top-p) over 1024 bins, the bin in which the wanted count
// or weight is reached, a histogram of that bin, until a bin is one key: bins of equal width below the largest logit first, which spread
// what a row holds evenly, then bins of the keys' bits.
//
// Weights are exp((x - max) / T) in 64 bits, off by 2^-44 of them, and are summed as whole multiples of 2^-42: whatever the order, the
// sums are the same, and a random number that falls next to a border is on the same side in every run and for every cluster size.
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "ops.cuh"

namespace hook_attn {

namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 2 * kThreads;
constexpr int kMostCtas = 8;               // of a cluster
constexpr int kTable = 64;                 // 2^(i / 64)
constexpr double kUnit = 4398046511104.0;  // 2^42 units to a weight of 1

__device__ __forceinline__ float as_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float as_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float as_f32(float x) { return x; }

// A logit as the kernel holds it: NaN is -infinity, and there is one zero.
template <typename T>
__device__ __forceinline__ float logit(T raw)
{
    const float x = as_f32(raw) + 0.f;
    return x == x ? x : -INFINITY;
}

// Integers in the order of the floats.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key)
{
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

struct SampleShared {
    unsigned long long hist[2][kBins];     // levels take turns: a CTA may still read the one before
    double table[kTable];
    unsigned long long seg_sum[kMostCtas * kWarps];
    unsigned int seg_ties[kMostCtas * kWarps];
    float peer_max[kMostCtas], peer_sum[kMostCtas];
    unsigned int peer_count[kMostCtas], peer_first[kMostCtas];
    float warp_max[kWarps], warp_sum[kWarps];
    unsigned int warp_count[kWarps];
    unsigned long long warp_scan[kWarps];
    unsigned long long found_before;
    int found_bin, found_seg;
    double found_target;
    unsigned int found_ties;
    unsigned long long found_total;
};

// exp2(y), y <= 0, in units of 2^-42: y is brought to a multiple of 1/64, whose power is in the table, and a rest r of at most 1/128, for which
// four terms of the series of exp(r ln 2) leave out less than 4e-14.
__device__ __forceinline__ unsigned long long weight_of(double y, const double* table)
{
    if (!(y > -43.5)) return 0;
    const double shifter = 6755399441055744.0 / kTable;                    // 1.5 * 2^52 / 64: adding it rounds to a multiple of 1/64
    const double rounded = y + shifter;
    const int n = __double2loint(rounded);                                 // 64 times the multiple
    const double r = (y - (rounded - shifter)) * 0.6931471805599453;
    double p = fma(r, 1.0 / 24, 1.0 / 6);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    p *= table[n & (kTable - 1)];
    p = __hiloint2double(__double2hiint(p) + ((n >> 6) << 20), __double2loint(p));
    const double fixed = p + 6755399441055744.0 / kUnit;                   // the mantissa's low bits are the multiple of 2^-42
    return (unsigned long long)(__double_as_longlong(fixed) - __double_as_longlong(6755399441055744.0 / kUnit));
}

// Sum over the CTA's threads of those before this one; `total` over all.
__device__ __forceinline__ unsigned long long scan_cta(unsigned long long x, unsigned long long* warps, unsigned long long& total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long incl = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long y = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += y;
    }
    __syncthreads();
    if (lane == 31) warps[warp] = incl;
    __syncthreads();
    unsigned long long before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += warps[w];
        total += warps[w];
    }
    return before + incl - x;
}

template <typename T, bool HELD>
struct Row {
    const T* global;
    const float* held;
    int n;                                 // tokens of this CTA's stretch
    __device__ __forceinline__ float at(int i) const { return HELD ? held[i] : logit(global[i]); }
};

// Bins of equal width below the largest logit; what lies beyond them is in the last.
__device__ __forceinline__ int linear_bin(float x, float top, float scale)
{
    const float f = (top - x) * scale;     // 0 for x = top, also where both are infinite (scale 0 then, and NaN below compares false)
    return f < (float)(kBins - 1) ? (int)f : (f == f ? kBins - 1 : 0);
}

// The key at which the wanted number or weight of eligible tokens is reached, and how much lies above it.  WEIGHTS: `want` is the share of the
// total; otherwise it is a number of tokens.  Tokens at `tie_key` count `tie_count` times in all, in no token's own turn.  All CTAs of
// the cluster come to the same result.  `level` says which histogram is free.
struct Reached {
    uint32_t key;
    unsigned long long above, total;       // above: of the tokens with larger keys
    bool all;                              // counts: there are no more than wanted
};

template <bool WEIGHTS, typename R, typename Ok, typename Weight>
__device__ Reached reach(const R& row, SampleShared& sh, cg::cluster_group& cluster, int& level, double want, float top, float scale,
                         Ok eligible, Weight weight, uint32_t tie_key, unsigned long long tie_amount)
{
    const int ctas = (int)cluster.num_blocks();
    const bool first_cta = cluster.block_rank() == 0;
    Reached out = {0, 0, 0, false};
    int linear = -1, shift = 0;
    uint32_t key_lo = 0, key_hi = 0;
    double goal = want;
    for (int pass = 0;; ++pass) {
        unsigned long long* hist = sh.hist[level & 1];
        ++level;
        for (int i = threadIdx.x; i < kBins; i += kThreads) hist[i] = 0;
        __syncthreads();
        auto bin_of = [&](float x, uint32_t key) {
            const int l = linear_bin(x, top, scale);
            if (pass == 0) return l;
            return l == linear && key >= key_lo && key <= key_hi ? (int)((key_hi - key) >> shift) : -1;
        };
        unsigned long long rest = 0;       // of the last linear bin: most of a row, added once
        for (int i = threadIdx.x; i < row.n; i += kThreads) {
            const float x = row.at(i);
            const uint32_t key = key_of(x);
            if (!eligible(x, key)) continue;
            const int b = bin_of(x, key);
            if (b < 0) continue;
            const unsigned long long amount = WEIGHTS ? weight(x) : 1ull;
            if (pass == 0 && b == kBins - 1) rest += amount;
            else if (amount) atomicAdd(&hist[b], amount);
        }
        if (rest) atomicAdd(&hist[kBins - 1], rest);
        if (WEIGHTS && first_cta && threadIdx.x == 0 && tie_amount) {
            const int b = bin_of(value_of(tie_key), tie_key);
            if (b >= 0) atomicAdd(&hist[b], tie_amount);
        }
        cluster.sync();
        unsigned long long mine[2] = {0, 0};
        for (int c = 0; c < ctas; ++c) {
            const unsigned long long* other = cluster.map_shared_rank(hist, c);
            mine[0] += other[2 * threadIdx.x];
            mine[1] += other[2 * threadIdx.x + 1];
        }
        unsigned long long total;
        const unsigned long long before = scan_cta(mine[0] + mine[1], sh.warp_scan, total) + out.above;
        if (pass == 0) {
            out.total = total;
            if (WEIGHTS) {
                goal = want * (double)total;
            } else if ((double)total <= want) {
                out.all = true;
                return out;
            }
            if (threadIdx.x == 0) sh.found_bin = -1;
            __syncthreads();
        }
        // the first bin with which the goal is reached
        const unsigned long long after0 = before + mine[0], after1 = after0 + mine[1];
        const bool start = threadIdx.x == 0;
        if ((double)after0 >= goal && ((double)before < goal || start)) {
            sh.found_bin = 2 * threadIdx.x;
            sh.found_before = before;
        } else if ((double)after1 >= goal && (double)after0 < goal) {
            sh.found_bin = 2 * threadIdx.x + 1;
            sh.found_before = after0;
        }
        __syncthreads();
        const int b = sh.found_bin;
        out.above = sh.found_before;
        if (pass == 0) {
            linear = b;
            key_hi = key_of(top);
            key_lo = key_of(-3.402823466e38f);
            if (scale > 0.f) {             // what rounds into bin b, with a margin for the rounding of (top - x) * scale
                key_hi = min(key_hi, key_of(__double2float_ru((double)top - b * (1 - 0x1p-22) / (double)scale)));
                if (b < kBins - 1) key_lo = max(key_lo, key_of(__double2float_rd((double)top - (b + 1) * (1 + 0x1p-22) / (double)scale)));
            }
        } else {
            key_hi -= (uint32_t)b << shift;
            if (key_hi - key_lo >= 1u << shift) key_lo = key_hi - ((1u << shift) - 1);
            if (shift == 0) {
                out.key = key_hi;
                return out;
            }
        }
        shift = 0;
        while ((key_hi - key_lo) >> shift >= (uint32_t)kBins) ++shift;
    }
}

template <typename T, bool HELD>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleArgs a)
{
    __shared__ SampleShared sh;
    extern __shared__ __align__(16) float stretch[];
    cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), r = blockIdx.x / ctas;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    const float u = a.uniform[r], heat = a.temperature ? a.temperature[r] : 1.f;
    const float share = a.top_p ? a.top_p[r] : 1.f, least = a.min_p ? a.min_p[r] : 0.f;
    const int k = a.top_k ? a.top_k[r] : 0;
    const bool valid = u >= 0.f && u < 1.f && heat >= 0.f && heat < INFINITY && share >= 0.f && least >= 0.f && least <= 1.f;
    if (!valid) {                          // of the whole cluster
        if (rank == 0 && threadIdx.x == 0) {
            a.tokens[r] = -1;
            report(a.status, HOOK_ATTN_ERR_INVALID_ARG);
        }
        return;
    }

    // ---- the stretch, its largest logit, the sum and number of the finite ones ----
    const int start = rank * a.slice;
    Row<T, HELD> row;
    row.n = max(0, min(a.slice, a.vocab - start));
    row.global = static_cast<const T*>(a.logits) + (int64_t)r * a.row + start;
    float top = -INFINITY, sum = 0.f;
    unsigned int count = 0;
    auto take = [&](float x) {
        top = fmaxf(top, x);
        if (fabsf(x) < INFINITY) {
            sum += x;
            ++count;
        }
    };
    constexpr int E = 16 / sizeof(T);
    const int head = row.n > 0 ? min(row.n, (int)((16 - (reinterpret_cast<uintptr_t>(row.global) & 15)) & 15) / (int)sizeof(T)) : 0;
    float* held = stretch + ((4 - head) & 3);          // where the aligned part starts on 16 bytes
    row.held = held;
    const int vectors = (row.n - head) / E, tail = head + vectors * E;
    for (int i = threadIdx.x; i < vectors; i += kThreads) {
        const uint4 raw = reinterpret_cast<const uint4*>(row.global + head)[i];
        const T* p = reinterpret_cast<const T*>(&raw);
        float x[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            x[e] = logit(p[e]);
            take(x[e]);
        }
        if (HELD) {
#pragma unroll
            for (int e = 0; e < E; e += 4) *reinterpret_cast<float4*>(held + head + i * E + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
        }
    }
    for (int i = threadIdx.x; i < head + row.n - tail; i += kThreads) {
        const int at = i < head ? i : tail + i - head;
        const float x = logit(row.global[at]);
        take(x);
        if (HELD) held[at] = x;
    }
    for (int i = threadIdx.x; i < kTable; i += kThreads) sh.table[i] = exp2((double)i / kTable);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        sum += __shfl_xor_sync(0xffffffffu, sum, d);
        count += __shfl_xor_sync(0xffffffffu, count, d);
    }
    if (lane == 0) { sh.warp_max[warp] = top; sh.warp_sum[warp] = sum; sh.warp_count[warp] = count; }
    __syncthreads();
    if ((int)threadIdx.x < ctas) {
        float m = -INFINITY, s = 0.f;
        unsigned int c = 0;
        for (int w = 0; w < kWarps; ++w) { m = fmaxf(m, sh.warp_max[w]); s += sh.warp_sum[w]; c += sh.warp_count[w]; }
        SampleShared* other = cluster.map_shared_rank(&sh, threadIdx.x);
        other->peer_max[rank] = m;
        other->peer_sum[rank] = s;
        other->peer_count[rank] = c;
    }
    cluster.sync();
    top = -INFINITY;
    sum = 0.f;
    count = 0;
    for (int c = 0; c < ctas; ++c) { top = fmaxf(top, sh.peer_max[c]); sum += sh.peer_sum[c]; count += sh.peer_count[c]; }
    if (top == -INFINITY) {
        if (rank == 0 && threadIdx.x == 0) {
            a.tokens[r] = -1;
            report(a.status, HOOK_ATTN_ERR_INVALID_ARG);
        }
        return;
    }

    // ---- what stays: larger keys than least_key, and the first `ties` tokens at it ----
    const bool greedy = heat == 0.f;
    uint32_t least_key = greedy ? key_of(top) : 0;
    unsigned long long ties = greedy ? 1 : 0;
    const double per_logit = greedy ? 0.0 : 1.4426950408889634 / (double)heat;
    const float cutoff = least > 0.f && !greedy ? __double2float_ru((double)top + log2((double)least) / per_logit) : -INFINITY;
    // next to an infinite logit everything else weighs nothing
    auto weight = [&](float x) { return x == top ? (unsigned long long)kUnit : weight_of(((double)x - (double)top) * per_logit, sh.table); };
    int level = 0;
    auto in_play = [&](float x, uint32_t) { return x > -INFINITY && x >= cutoff; };
    const float spread = count > 0 ? top - sum / (float)count : 0.f;
    if (!greedy && k > 0 && k < a.vocab) {
        const float scale = spread > 0.f && spread < INFINITY ? (float)(kBins - 1) / spread : 0.f;
        const Reached at = reach<false>(row, sh, cluster, level, (double)k, top, isfinite(scale) ? scale : 0.f, in_play, weight, 0, 0);
        if (!at.all) {
            least_key = at.key;
            ties = k - at.above;
        }
    }
    unsigned long long tie_weight = least_key ? weight(value_of(least_key)) : 0;
    if (!greedy && share < 1.f) {
        // beyond 2^-43 of the largest weight there is nothing
        const float wide = fminf(spread, (float)(44.0 / per_logit));
        const float scale = wide > 0.f && wide < INFINITY ? (float)(kBins - 1) / wide : 0.f;
        const uint32_t bound = least_key;
        const Reached at = reach<true>(row, sh, cluster, level, (double)share, top, isfinite(scale) ? scale : 0.f,
                                       [&](float x, uint32_t key) { return key > bound && in_play(x, key); }, weight, bound, ties * tie_weight);
        const double goal = (double)share * (double)at.total;
        const unsigned long long each = at.key == least_key ? tie_weight : weight(value_of(at.key));
        unsigned long long n = 1;          // those before which less than the goal lies
        if (each > 0) {
            const double more = (goal - (double)at.above) / (double)each;
            n = more > 1.0 ? (unsigned long long)more : 1;
            while ((double)(at.above + n * each) < goal) ++n;
            while (n > 1 && (double)(at.above + (n - 1) * each) >= goal) --n;
        }
        ties = at.key == least_key ? min(ties, n) : n;
        least_key = at.key;
        tie_weight = each;
    }

    // ---- the draw: weights of stretches of the stretch, in the order of the indices ----
    const int per = ((row.n + kWarps - 1) / kWarps + 31) / 32 * 32, from = min(warp * per, row.n), to = min(from + per, row.n);
    unsigned long long mine = 0;
    unsigned int tied = 0;
    for (int i = from + lane; i < to; i += 32) {
        const float x = row.at(i);
        const uint32_t key = key_of(x);
        if (key < least_key || !in_play(x, key)) continue;
        if (least_key && key == least_key) ++tied;
        else mine += weight(x);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        mine += __shfl_xor_sync(0xffffffffu, mine, d);
        tied += __shfl_xor_sync(0xffffffffu, tied, d);
    }
    if (lane < ctas) {
        SampleShared* other = cluster.map_shared_rank(&sh, lane);
        other->seg_sum[rank * kWarps + warp] = mine;
        other->seg_ties[rank * kWarps + warp] = tied;
    }
    cluster.sync();
    if (warp == 0) {                       // a lane takes a run of stretches
        const int segs = ctas * kWarps, each = (segs + 31) / 32;
        unsigned int t = 0;
        for (int j = 0; j < each; ++j)
            if (lane * each + j < segs) t += sh.seg_ties[lane * each + j];
        unsigned int t_incl = t;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned int y = __shfl_up_sync(0xffffffffu, t_incl, d);
            if (lane >= d) t_incl += y;
        }
        auto part = [&](int s, unsigned long long t_before) {
            const unsigned long long left = ties > t_before ? ties - t_before : 0;
            return sh.seg_sum[s] + min(left, (unsigned long long)sh.seg_ties[s]) * tie_weight;
        };
        unsigned long long w = 0, tb = t_incl - t;
        for (int j = 0; j < each; ++j)
            if (lane * each + j < segs) { w += part(lane * each + j, tb); tb += sh.seg_ties[lane * each + j]; }
        unsigned long long w_incl = w;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned long long y = __shfl_up_sync(0xffffffffu, w_incl, d);
            if (lane >= d) w_incl += y;
        }
        const unsigned long long total = __shfl_sync(0xffffffffu, w_incl, 31);
        // the first weight that exceeds u of the total; rounded up to it, the last one
        const double want = fmin((double)u * (double)total, (double)total - 1.0);
        const unsigned int reached = __ballot_sync(0xffffffffu, (double)w_incl > want);
        if (lane == __ffs(reached) - 1) {
            unsigned long long before = w_incl - w;
            tb = t_incl - t;
            for (int j = 0; j < each; ++j) {
                const int s = lane * each + j;
                if (s >= segs) break;
                const unsigned long long p = part(s, tb);
                if ((double)(before + p) > want) {
                    sh.found_seg = s;
                    sh.found_before = before;
                    sh.found_ties = (unsigned int)tb;
                    sh.found_target = want;
                    break;
                }
                before += p;
                tb += sh.seg_ties[s];
            }
        }
    }
    __syncthreads();
    if (sh.found_seg != rank * kWarps + warp) return;
    unsigned long long before = sh.found_before, t_before = sh.found_ties;
    for (int i0 = from; i0 < to; i0 += 32) {
        const int i = i0 + lane;
        const float x = i < to ? row.at(i) : -INFINITY;
        const uint32_t key = key_of(x);
        const bool stays = key >= least_key && in_play(x, key), tie = stays && least_key && key == least_key;
        const unsigned int all_ties = __ballot_sync(0xffffffffu, tie);
        unsigned long long w = 0;
        if (tie) w = t_before + __popc(all_ties & ((1u << lane) - 1)) < ties ? tie_weight : 0;
        else if (stays) w = weight(x);
        unsigned long long incl = w;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned long long y = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += y;
        }
        const unsigned int reached = __ballot_sync(0xffffffffu, w > 0 && (double)(before + incl) > sh.found_target);
        if (reached) {
            if (lane == __ffs(reached) - 1) a.tokens[r] = start + i;
            return;
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
        t_before += __popc(all_ties);
    }
}

constexpr int kMostHeld = 48 * 1024;       // tokens that a CTA keeps in shared memory; longer stretches are read again

template <typename T, bool HELD>
cudaError_t issue(const SampleArgs& a, int ctas, cudaStream_t st)
{
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.rows * ctas));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = HELD ? (size_t)(a.slice + 4) * 4 : 0;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sample_kernel<T, HELD>, a);
}

template <typename T>
cudaError_t launch(SampleArgs a, int num_sms, cudaStream_t st)
{
    int ctas = 1;
    while (ctas < kMostCtas && a.vocab > ctas * 4096) ctas *= 2;
    a.slice = ((a.vocab + ctas - 1) / ctas + 7) / 8 * 8;
    return a.slice <= kMostHeld ? issue<T, true>(a, ctas, st) : issue<T, false>(a, ctas, st);
}

}  // namespace

cudaError_t configure_sample()
{
    const auto allow = [](auto* kernel) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (kMostHeld + 4) * 4); };
    cudaError_t e = allow(sample_kernel<__nv_bfloat16, true>);
    if (e == cudaSuccess) e = allow(sample_kernel<__half, true>);
    if (e == cudaSuccess) e = allow(sample_kernel<float, true>);
    return e;
}

cudaError_t launch_sample(const SampleArgs& a, int dtype, int num_sms, cudaStream_t st)
{
    if (dtype == HOOK_DTYPE_BF16) return launch<__nv_bfloat16>(a, num_sms, st);
    if (dtype == HOOK_DTYPE_F16) return launch<__half>(a, num_sms, st);
    return launch<float>(a, num_sms, st);
}

}  // namespace hook_attn

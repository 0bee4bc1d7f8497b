// The choice of a token from a row of logits and one random number: temperature, top-k, min-p, top-p.
//
// A cluster of CTAs takes a row.  Each CTA holds a stretch of it in shared memory, so that the row is read once, and they exchange what
// little the others need through distributed shared memory.  All three filters keep the first tokens in the order of falling logits
// (equal ones by index), so what stays is a least key K and how many of the tokens at K itself: tokens are never sorted.
//
// K is found by narrowing down: a histogram of the tokens' counts (top-k) or weights (top-p) over bins of equal width below the largest logit,
// then the few tokens of the bin in which the wanted count or weight is reached are listed, and each is held against all others; where they
// are many, histograms of that bin by the keys' bits, until a bin is one key.  On the way each warp lists, in order, those of its tokens that may
// stay, and what follows goes by the lists.
//
// Weights are exp((x - max) / T) in 64 bits, off by 2^-44 of them, and are summed as whole multiples of 2^-42: whatever the order, the
// sums are the same, and a random number that falls next to a border is on the same side in every run and for every cluster size.
//
// Reading the row is the least of it.  A token takes some 50 instructions where every weight is needed (12 of them in 64 bits) and 20 in a pass that only compares;
// a cluster's six exchanges, the scans and the lists cost a row about 10 us.  256 x 160000 fp32: 203 us with rows of all filters, 141 without any, 171 top-k,
// 240 top-p; 1 x 32000 bf16: 15.1, 10.3, 11.7 and 11.7 us.  Issue slots are half busy at 32 warps an SM, which barriers and loads hold up by turns.
//
// Those are steep rows.  Where a CTA has more than 64 tokens in the boundary's bin (flat rows, many ties, a border among the thousandth tokens), the passes
// by the keys' bits follow, a token at a time, and those of one key are added in shared memory one after the other: 256 x 160000 with top-p 0.9 takes 0.32 ms with
// logits of deviation 3, 0.84 with 0.05 or evenly spread ones, 1.4 with two values and 2.1 with one; top-k 50 0.19, 0.19 to 0.33, 0.6 and 1.2;
// 1 x 32000 bf16 with top-p 15, 32, 39 and 49 us.
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <utility>

#include "common.cuh"
#include "ops.cuh"

namespace hook_attn {

namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = kThreads;            // what is read from the other CTAs limits them: 64 KB took 2 us
constexpr int kMostCtas = 8;               // of a cluster
constexpr int kTable = 16;                 // 2^(i / 16): as wide as the banks of shared memory, so that lanes read any of it at once
constexpr int kList = kThreads;            // tokens of a bin that are held against one another
constexpr int kShare = kList / kMostCtas;  // of one CTA
constexpr int kMayStay = 128;              // tokens in a warp's list
constexpr double kUnit = 4398046511104.0;  // 2^42 units to a weight of 1
constexpr float kLargest = 3.402823466e38f;

__device__ __forceinline__ float as_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float as_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float as_f32(float x) { return x; }

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

struct alignas(16) SampleShared {
    alignas(16) float may_stay[kWarps][kMayStay];      // the warps' lists: logits, and where they are
    unsigned int place[kWarps][kMayStay];
    unsigned long long hist[2][kBins];     // levels take turns: a CTA may still read the one before
    double table[kTable], wide_top;
    float peer_max[kMostCtas * kWarps], peer_sum[kMostCtas * kWarps];
    unsigned int peer_count[kMostCtas * kWarps];
    unsigned long long peer_weight[kMostCtas];
    unsigned int peer_ties[kMostCtas];
    unsigned long long warp_scan[2][kWarps], draw[kWarps];
    unsigned int draw_ties[kWarps];
    double per_logit, below;               // log2(e) / T; how far below the largest logit min_p's border lies
    unsigned long long found_before;
    int found_bin, found_from, found_to;
    unsigned int listed_count, listed[kShare], all[kList], all_count[kMostCtas], keys[kList], pick;
    unsigned long long amounts[kList];
};

// 2^(i / 16)
__device__ const double kPowers[kTable] = {
    0x1.0000000000000p+0, 0x1.0b5586cf9890fp+0, 0x1.172b83c7d517bp+0, 0x1.2387a6e756238p+0,
    0x1.306fe0a31b715p+0, 0x1.3dea64c123422p+0, 0x1.4bfdad5362a27p+0, 0x1.5ab07dd485429p+0,
    0x1.6a09e667f3bcdp+0, 0x1.7a11473eb0187p+0, 0x1.8ace5422aa0dbp+0, 0x1.9c49182a3f090p+0,
    0x1.ae89f995ad3adp+0, 0x1.c199bdd85529cp+0, 0x1.d5818dcfba487p+0, 0x1.ea4afa2a490dap+0,
};

// A float as a double, by its bits: the conversion instruction takes four times as long as arithmetic.  Numbers below 2^-126 (zero among them) are off by
// as much at most, and an infinity becomes 2^128.
__device__ __forceinline__ double widened(float x)
{
    const int b = __float_as_int(x);
    return __hiloint2double(((b >> 3) & (int)0x8fffffffu) + 0x38000000, b << 29);
}

// The weights of four logits in units of 2^-42: 2^y with y = (x - top) * per_logit from -45 to 0 (of others nothing is to be made).  y is brought to a
// multiple of 1/16, whose power is in the table, and a rest r of at most 1/32, for which six terms of the series of exp(r ln 2) leave out
// less than 1e-15.  No branches: the four chains run side by side.
__device__ __forceinline__ void weights_of(unsigned long long (&w)[4], const float4& x4, const SampleShared& sh)
{
    constexpr double kShifter = 6755399441055744.0 / kTable;               // 1.5 * 2^52 / 16: adding it rounds to a multiple of 1/16
    constexpr double kFixed = 6755399441055744.0 / kUnit;                  // and this one to a multiple of 2^-42, which is what its low 51 bits are
    const float x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const double y = (widened(x[e]) - sh.wide_top) * sh.per_logit;
        const double rounded = y + kShifter;
        const int n = __double2loint(rounded);                             // 16 times the multiple
        const double r = (y - (rounded - kShifter)) * 0.6931471805599453;
        double p = fma(r, 1.0 / 720, 1.0 / 120);
        p = fma(p, r, 1.0 / 24);
        p = fma(p, r, 1.0 / 6);
        p = fma(p, r, 0.5);
        p = fma(p, r, 1.0);
        p = fma(p, r, 1.0);
        p *= sh.table[n & (kTable - 1)];
        p = __hiloint2double(__double2hiint(p) + ((n >> 4) << 20), __double2loint(p)) + kFixed;
        w[e] = (unsigned long long)(__double2hiint(p) & 0x0007ffff) << 32 | (unsigned int)__double2loint(p);
    }
}

__device__ __forceinline__ unsigned long long weight_of(float x, float top, const SampleShared& sh)
{
    unsigned long long w[4];
    weights_of(w, make_float4(x, top, top, top), sh);
    return w[0];
}

// Adds to a 64-bit sum in shared memory by its words: there the hardware adds 32 bits at a time, and the carry is known from the old value.
__device__ __forceinline__ void add_words(unsigned long long* sum, unsigned long long amount)
{
    unsigned int* words = reinterpret_cast<unsigned int*>(sum);
    const unsigned int low = (unsigned int)amount, old = atomicAdd(words, low);
    const unsigned int high = (unsigned int)(amount >> 32) + (old + low < low);
    if (high) atomicAdd(words + 1, high);
}

// Sum over a warp's lanes, below 2^63: in limbs of 22 bits, which the reduction instruction adds (five exchanges of 64 bits took 450 cycles).
__device__ __forceinline__ unsigned long long sum_warp(unsigned long long x)
{
    const unsigned int a = __reduce_add_sync(0xffffffffu, (unsigned int)x & 0x3fffffu), b = __reduce_add_sync(0xffffffffu, (unsigned int)(x >> 22) & 0x3fffffu);
    const unsigned int c = __reduce_add_sync(0xffffffffu, (unsigned int)(x >> 44));
    return ((unsigned long long)c << 44) + ((unsigned long long)b << 22) + a;
}

// Inclusive, over a warp.
template <typename N>
__device__ __forceinline__ N scan_warp(N x)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const N y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// Sum over the CTA's threads of those before this one, and over all.  `sums` is not in use by anything before the last barrier.
__device__ __forceinline__ unsigned long long scan_cta(unsigned long long x, unsigned long long& total, unsigned long long (&sums)[kWarps])
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned long long incl = scan_warp(x);
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    const unsigned long long w = lane < kWarps ? sums[lane] : 0;
    total = sum_warp(w);
    return sum_warp(lane < warp ? w : 0) + incl - x;
}

// Four logits at a time of what a warp goes through: its part of the CTA's stretch, held as floats in shared memory or read again from
// the row, or its list.
template <typename T, bool HELD>
struct Walk {
    const float4* held;
    const T* global;
    int n;                                 // of the stretch, where it is not held
    int from, to;
    bool listed;
    __device__ __forceinline__ float4 get(int v) const
    {
        if (HELD || listed) return held[v];
        float x[4] = {};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = 4 * v + e < n ? as_f32(global[4 * v + e]) + 0.f : -INFINITY;
            if (x[e] != x[e]) x[e] = -INFINITY;
        }
        return make_float4(x[0], x[1], x[2], x[3]);
    }
};

// Bins of equal width below the largest logit: (top - x) * scale to the nearest whole number, which an addition of 2^23 leaves in the low bits;
// what lies beyond them (and an infinity's difference to itself) is in the last.
__device__ __forceinline__ int linear_bin(float x, float top, float scale)
{
    return (int)min(__float_as_uint(fmaf(top - x, scale, 8388608.f)) - 0x4b000000u, (uint32_t)(kBins - 1));
}

// The key at which the wanted number or weight of the logits from `floor` on is reached, and how much lies above it.  weighted: `want` is the share
// of the total; otherwise it is a number of tokens.  Tokens at `tie_key`, below floor, count `tie_amount` in all.  All CTAs of the cluster
// come to the same result.  `level` says which histogram is free.  Warps without a list get one of what is in play, from `base` on, and not
// below the key.
struct Reached {
    uint32_t key;
    unsigned long long above, total;       // above: of the tokens with larger keys
    bool all;                              // counts: there are no more than wanted
};

template <typename R>
__device__ __forceinline__ Reached reach(const bool weighted, R& row, SampleShared& sh, int& level, double want, float top, float scale, float base,
                                      float floor, uint32_t tie_key, unsigned long long tie_amount)
{
    cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Reached out = {0, 0, 0, false};
    int linear = -1, shift = 0;
    uint32_t key_lo = 0, key_hi = 0;
    double goal = want;
#pragma unroll 1
    for (int pass = 0;; ++pass) {
        unsigned long long* hist = sh.hist[level & 1];
        ++level;
        hist[threadIdx.x] = 0;
        if (threadIdx.x == 0) sh.listed_count = 0;
        __syncthreads();
        unsigned long long rest = 0;       // of the last linear bin: most of a row, added once
        if (pass == 0) {
#pragma unroll 2
            for (int v = row.from + lane; v < row.to; v += 32) {
                const float4 x4 = row.get(v);
                if (!(fmaxf(fmaxf(x4.x, x4.y), fmaxf(x4.z, x4.w)) >= floor)) continue;
                unsigned long long w[4] = {1, 1, 1, 1};
                if (weighted) weights_of(w, x4, sh);
                const float x[4] = {x4.x, x4.y, x4.z, x4.w};
                int bin[4];
                bool in[4];
                unsigned int old[4];       // the four side by side: what they wait for is the old values
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    bin[e] = linear_bin(x[e], top, scale);
                    in[e] = x[e] >= floor && bin[e] < kBins - 1;
                    if (x[e] >= floor && bin[e] == kBins - 1) rest += w[e];
                    if (in[e]) old[e] = atomicAdd(reinterpret_cast<unsigned int*>(&hist[bin[e]]), (unsigned int)w[e]);
                }
                if (weighted)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned int high = (unsigned int)(w[e] >> 32) + (old[e] + (unsigned int)w[e] < old[e]);
                        if (in[e] && high) atomicAdd(reinterpret_cast<unsigned int*>(&hist[bin[e]]) + 1, high);
                    }
            }
        } else {
#pragma unroll 1
            for (int i = 4 * row.from + lane; i < 4 * row.to; i += 32) {
                const float4 x4 = row.get(i / 4);
                const float x = i & 2 ? (i & 1 ? x4.w : x4.z) : (i & 1 ? x4.y : x4.x);
                const uint32_t key = key_of(x);
                if (x >= floor && key >= key_lo && key <= key_hi && linear_bin(x, top, scale) == linear)
                    add_words(&hist[(key_hi - key) >> shift], weighted ? weight_of(x, top, sh) : 1);
            }
        }
        if (__any_sync(0xffffffffu, rest != 0)) {
            rest = sum_warp(rest);
            if (lane == 0) add_words(&hist[kBins - 1], rest);
        }
        if (rank == 0 && threadIdx.x == 0 && tie_amount) {
            const int l = linear_bin(value_of(tie_key), top, scale);
            if (pass == 0) add_words(&hist[l], tie_amount);
            else if (l == linear && tie_key >= key_lo && tie_key <= key_hi) add_words(&hist[(key_hi - tie_key) >> shift], tie_amount);
        }
        cluster.sync();
        unsigned long long mine = 0, theirs[kMostCtas];        // all under way at once
#pragma unroll
        for (int c = 0; c < kMostCtas; ++c) theirs[c] = c < ctas ? cluster.map_shared_rank(hist, c)[threadIdx.x] : 0;
#pragma unroll
        for (int c = 0; c < kMostCtas; ++c) mine += theirs[c];
        unsigned long long total;
        const unsigned long long before = scan_cta(mine, total, sh.warp_scan[level & 1]) + out.above;
        if (pass == 0) {
            out.total = total;
            if (weighted) {
                goal = fmax(want * (double)total, 1.0);          // a unit at least: the first token stays, and it may lie in any bin
            } else if ((double)total <= want) {
                out.all = true;
                return out;
            }
        }
        // the first bin with which the goal is reached
        if ((double)(before + mine) >= goal && (double)before < goal) {
            sh.found_bin = threadIdx.x;
            sh.found_before = before;
        }
        if (threadIdx.x == 0) sh.pick = 0xffffffffu;
        __syncthreads();
        const int b = sh.found_bin;
        out.above = sh.found_before;
        if (pass > 0) {
            key_hi -= (uint32_t)b << shift;
            if (key_hi - key_lo >= 1u << shift) key_lo = key_hi - ((1u << shift) - 1);
            if (shift == 0) {
                out.key = key_hi;
                return out;
            }
        } else {
            linear = b;
            // The tokens of bin b, for all CTAs; and for the warp's own list those up to it: none lies below `near`, with a margin for what rounds into b.
            const float near = fmaxf(base, scale > 0.f && b < kBins - 1 ? top - (b + 0.51f) / scale - fabsf(top) * 4e-7f : -kLargest);
            int n = 0;
#pragma unroll 1
            for (int v0 = row.from; v0 < row.to; v0 += 32) {
                const int v = v0 + lane;
                const float4 x4 = v < row.to ? row.get(v) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                if (!__any_sync(0xffffffffu, fmaxf(fmaxf(x4.x, x4.y), fmaxf(x4.z, x4.w)) >= near)) continue;
                const float x[4] = {x4.x, x4.y, x4.z, x4.w};
                uint32_t mine_in = 0, who[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int l = x[e] >= near ? linear_bin(x[e], top, scale) : kBins;
                    if (l == b && x[e] >= floor) {
                        const unsigned int at = atomicAdd(&sh.listed_count, 1u);
                        if (at < kShare) sh.listed[at] = key_of(x[e]);
                    }
                    mine_in |= (uint32_t)(l <= b) << e;
                    who[e] = __ballot_sync(0xffffffffu, l <= b);
                }
                if (row.listed) continue;
                const uint32_t before_me = (1u << lane) - 1;
                int at = n + __popc(who[0] & before_me) + __popc(who[1] & before_me) + __popc(who[2] & before_me) + __popc(who[3] & before_me);
                n += __popc(who[0]) + __popc(who[1]) + __popc(who[2]) + __popc(who[3]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (mine_in >> e & 1) {
                        if (at < kMayStay) {
                            sh.may_stay[warp][at] = x[e];
                            sh.place[warp][at] = 4 * v + e;
                        }
                        ++at;
                    }
            }
            if (!row.listed && n <= kMayStay) {
                if (lane < (-n & 3)) sh.may_stay[warp][n + lane] = -INFINITY;
                row.held = reinterpret_cast<const float4*>(sh.may_stay[warp]);
                row.from = 0;
                row.to = (n + 3) / 4;
                row.listed = true;
            }
            __syncthreads();
            if ((int)threadIdx.x / kShare < ctas) {        // a group of threads for every CTA
                SampleShared* other = cluster.map_shared_rank(&sh, threadIdx.x / kShare);
                const int j = threadIdx.x % kShare;
                if (j < (int)sh.listed_count) other->all[rank * kShare + j] = sh.listed[j];
                if (j == 0) other->all_count[rank] = sh.listed_count;
            }
            cluster.sync();
            bool few = true;
#pragma unroll
            for (int c = 0; c < kMostCtas; ++c) few &= c >= ctas || sh.all_count[c] <= kShare;
            if (few) {
                // each is held against all, by as many threads as there are for it
                const int from_cta = threadIdx.x / kShare, from_at = threadIdx.x % kShare;
                int n = 0, at = 0;
#pragma unroll
                for (int c = 0; c < kMostCtas; ++c) {
                    if (c == from_cta) at = n + from_at;
                    if (c < ctas) n += sh.all_count[c];
                }
                if (from_cta < ctas && from_at < (int)sh.all_count[from_cta]) {
                    sh.keys[at] = sh.all[threadIdx.x];
                    sh.amounts[at] = weighted ? weight_of(value_of(sh.all[threadIdx.x]), top, sh) : 1;
                }
                __syncthreads();
                const int split = n <= kThreads / 4 ? 4 : 1, mine_at = threadIdx.x / split;
                const bool live = mine_at < n;
                const uint32_t key = live ? sh.keys[mine_at] : 0;                  // no token in play has key 0
                unsigned long long larger = 0, whole = 0;
                if (live)
#pragma unroll 4
                    for (int j = threadIdx.x % split; j < n; j += split) {
                        const unsigned long long amount = sh.amounts[j];
                        whole += amount;
                        larger += sh.keys[j] > key ? amount : 0;
                    }
                if (split > 1)
#pragma unroll
                    for (int d = 1; d < 4; d <<= 1) {
                        whole += __shfl_xor_sync(0xffffffffu, whole, d);
                        larger += __shfl_xor_sync(0xffffffffu, larger, d);
                    }
                if (live && (double)(out.above + larger) < goal) atomicMin(&sh.pick, key);
                __syncthreads();
                const uint32_t pick = sh.pick;
                const bool none = pick == 0xffffffffu;                             // the bin holds nothing but those that have no turn
                if (none ? threadIdx.x == 0 : live && key == pick) {
                    const bool ties = tie_amount && (double)(out.above + whole) < goal;                // or the goal lies among them
                    sh.found_before = out.above + (ties ? whole : larger);
                    sh.found_bin = none || ties;
                }
                __syncthreads();
                out.key = sh.found_bin ? tie_key : pick;
                out.above = sh.found_before;
                return out;
            }
        }
        if (pass == 0) {                   // what rounds into bin b, with a margin for the rounding of top - x
            key_hi = key_of(top);
            key_lo = key_of(-kLargest);
            if (scale > 0.f) {
                const double width = 1.0 / (double)scale;
                if (b > 0) key_hi = min(key_hi, key_of(__double2float_ru((double)top - (b - 0.5) * (1 - 0x1p-22) * width)));
                if (b < kBins - 1) key_lo = max(key_lo, key_of(__double2float_rd((double)top - (b + 0.5) * (1 + 0x1p-22) * width)));
            }
        }
        shift = 0;
        while ((key_hi - key_lo) >> shift >= (uint32_t)kBins) ++shift;
    }
}

template <typename T, bool HELD>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const SampleArgs a)
{
    __shared__ SampleShared sh;
    extern __shared__ __align__(16) float4 stretch[];
    cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), r = blockIdx.x / ctas;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // the others' shared memory is there once they have all begun; by the time it is written to they have
    auto begun = cluster.barrier_arrive();

    const float u = a.uniform[r], heat = a.temperature ? a.temperature[r] : 1.f;
    const float share = a.top_p ? a.top_p[r] : 1.f, least = a.min_p ? a.min_p[r] : 0.f;
    const int k = a.top_k ? a.top_k[r] : 0;
    const bool valid = u >= 0.f && u < 1.f && heat >= 0.f && heat < INFINITY && share >= 0.f && least >= 0.f && least <= 1.f;
    const bool greedy = heat == 0.f;
    if (threadIdx.x == kThreads - 32) {    // while the others fetch
        sh.per_logit = greedy ? 0.0 : 1.4426950408889634 / (double)heat;
        sh.below = least > 0.f && !greedy ? log2((double)least) / sh.per_logit : -INFINITY;
    }
    // ---- the stretch, its largest logit, the sum and number of the finite ones ----
    const int start = rank * a.slice, n = max(0, min(a.slice, a.vocab - start));
    const T* const global = static_cast<const T*>(a.logits) + (int64_t)r * a.row + start;
    // Read in vectors of 16 bytes where they are aligned; element i is then held at place i + lead, the first vector's alignment.
    constexpr int E = 16 / sizeof(T);
    const int lead = HELD ? (int)(reinterpret_cast<uintptr_t>(global) & 15) / (int)sizeof(T) : 0;
    Walk<T, HELD> row;
    row.held = stretch;
    row.global = global;
    row.n = n;
    row.listed = false;
    {
        const int fours = (lead + n + 3) / 4, per = (fours + kWarps - 1) / kWarps;
        row.from = min(warp * per, fours);
        row.to = min(row.from + per, fours);
    }
    float top = -INFINITY, sum = 0.f;
    unsigned int count = 0;
    auto take = [&](float x) {             // NaN is -infinity, and there is one zero
        x = fmaxf(x, -INFINITY) + 0.f;
        top = fmaxf(top, x);
        return x;
    };
    auto survey = [&](const float4& x4) {  // how far the logits lie below the largest: a few of each thread tell
        const float x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool finite = fabsf(x[e]) < INFINITY;
            sum += finite ? x[e] : 0.f;
            count += finite;
        }
    };
    if constexpr (HELD) {
        const int vectors = (lead + n + E - 1) / E;
        constexpr int BATCH = 4;           // vectors of a thread under way
        for (int v0 = threadIdx.x; v0 < vectors; v0 += BATCH * kThreads) {
            uint4 raw[BATCH];
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int v = v0 + j * kThreads, i0 = v * E - lead;
                if (v < vectors && i0 >= 0 && i0 + E <= n) raw[j] = *reinterpret_cast<const uint4*>(global + i0);
            }
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int v = v0 + j * kThreads, i0 = v * E - lead;
                if (v >= vectors) break;
                T* p = reinterpret_cast<T*>(&raw[j]);
                if (i0 < 0 || i0 + E > n)
                    for (int e = 0; e < E; ++e) p[e] = i0 + e >= 0 && i0 + e < n ? global[i0 + e] : T(-INFINITY);
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const float4 x = make_float4(take(as_f32(p[e])), take(as_f32(p[e + 1])), take(as_f32(p[e + 2])), take(as_f32(p[e + 3])));
                    stretch[v * (E / 4) + e / 4] = x;
                    if (v < kThreads && e == 0) survey(x);
                }
            }
        }
    } else {
        for (int v = row.from + lane; v < row.to; v += 32) {
            const float4 x = row.get(v);
            take(x.x); take(x.y); take(x.z); take(x.w);
            if (v < row.from + 32) survey(x);
        }
    }
    if (threadIdx.x < kTable) sh.table[threadIdx.x] = kPowers[threadIdx.x];
    top = value_of(__reduce_max_sync(0xffffffffu, key_of(top)));
    count = __reduce_add_sync(0xffffffffu, count);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    cluster.barrier_wait(std::move(begun));
    if (lane < ctas) {                     // of this warp, for every CTA
        SampleShared* other = cluster.map_shared_rank(&sh, lane);
        const int at = rank * kWarps + warp;
        other->peer_max[at] = top;
        other->peer_sum[at] = sum;
        other->peer_count[at] = count;
    }
    cluster.sync();
    {                                      // a lane takes four warps; every warp comes to the same
        uint32_t most = 0;
        sum = 0.f;
        count = 0;
#pragma unroll
        for (int j = 0; j < kMostCtas * kWarps / 32; ++j) {
            const int at = 32 * j + lane;
            if (at >= ctas * kWarps) break;
            most = max(most, key_of(sh.peer_max[at]));
            sum += sh.peer_sum[at];
            count += sh.peer_count[at];
        }
        top = value_of(__reduce_max_sync(0xffffffffu, most));
        count = __reduce_add_sync(0xffffffffu, count);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    }
    if (!valid || top == -INFINITY) {      // of the whole cluster
        if (rank == 0 && threadIdx.x == 0) {
            a.tokens[r] = -1;
            report(a.status, HOOK_ATTN_ERR_INVALID_ARG);
        }
        return;
    }

    // ---- what stays: larger keys than least_key, and the first `ties` tokens at it ----
    uint32_t least_key = greedy ? key_of(top) : 0;
    unsigned long long ties = greedy ? 1 : 0;
    // what is in play: from here on
    float floor = sh.below > -INFINITY ? fmaxf(__double2float_ru((double)top + sh.below), -kLargest) : -kLargest;
    // further down weights are below 2^-44, and next to an infinite logit all others are: none of those is ever drawn
    floor = top == INFINITY ? top : fmaxf(floor, top - 31.f * heat);
    __syncthreads();
    if (threadIdx.x == 0) {
        sh.wide_top = widened(top);
        if (top == INFINITY) sh.per_logit = 1.0;               // next to an infinite logit everything else weighs nothing, whatever the temperature
    }
    __syncthreads();
    int level = 0;
    const float spread = count > 0 ? top - sum / (float)count : 0.f;
    auto scale_of = [&](float width) {
        const float scale = width > 0.f && width < INFINITY ? (float)(kBins - 1) / width : 0.f;
        return isfinite(scale) ? scale : 0.f;
    };
    unsigned long long tie_weight = (unsigned long long)kUnit;
    // Top-k, then top-p among what it left: one loop, so that the code is there once (a small call waits for its instructions more than for anything else).
#pragma unroll 1
    for (int stage = 0; stage < 2; ++stage) {
        const bool weighted = stage > 0;
        if (greedy || !(weighted ? share < 1.f : k > 0 && k < a.vocab)) continue;
        // beyond 2^-43 of the largest weight there is nothing; what follows infinity is a NaN, and nothing is from there on
        const float width = weighted ? fminf(spread, 30.5f * heat) : spread, above = weighted && least_key ? value_of(least_key + 1) : floor;
        const Reached at = reach(weighted, row, sh, level, weighted ? (double)share : (double)k, top, scale_of(width), floor, above, least_key,
                                 weighted ? ties * tie_weight : 0);
        if (at.all) continue;
        unsigned long long n = k - at.above;
        if (weighted) {                    // those before which less than the goal lies
            const double goal = (double)share * (double)at.total;
            n = 1;
            const unsigned long long each = at.key == least_key ? tie_weight : weight_of(value_of(at.key), top, sh);
            if (each > 0) {
                const double more = (goal - (double)at.above) / (double)each;
                n = more > 1.0 ? (unsigned long long)more : 1;
                while ((double)(at.above + n * each) < goal) ++n;
                while (n > 1 && (double)(at.above + (n - 1) * each) >= goal) --n;
            }
            if (at.key == least_key) n = min(ties, n);
        }
        ties = n;
        least_key = at.key;
        tie_weight = weight_of(value_of(least_key), top, sh);
    }
    if (least_key) floor = fmaxf(floor, value_of(least_key));

    // ---- the draw, in the order of the indices: weights of the warps' stretches or lists, then of their parts ----
    // What is above least_value stays, whole: without a key, the number before floor (before zero that is -2^-149, as no number lies between it and -0).
    const float least_value = least_key ? value_of(least_key) : floor == 0.f ? -1.40129846e-45f : value_of(key_of(floor) - 1);
    const unsigned int most_ties = (unsigned int)min(ties, (unsigned long long)kMaxVocab);
    auto part_of = [&](int v, unsigned long long& w, unsigned int& t) {           // weights above least_value, and how many are at it
        const float4 x4 = row.get(v);
        if (!(fmaxf(fmaxf(x4.x, x4.y), fmaxf(x4.z, x4.w)) >= least_value)) return;
        unsigned long long each[4];
        weights_of(each, x4, sh);
        const float x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            t += x[e] == least_value;
            if (x[e] > least_value) w += each[e];
        }
    };
    unsigned long long lane_weight = 0;
    unsigned int lane_ties = 0;
#pragma unroll 2
    for (int v = row.from + lane; v < row.to; v += 32) part_of(v, lane_weight, lane_ties);
    const unsigned long long warp_weight = sum_warp(lane_weight);
    const unsigned int warp_ties = __reduce_add_sync(0xffffffffu, lane_ties);
    if (lane == 0) {
        sh.draw[warp] = warp_weight;
        sh.draw_ties[warp] = warp_ties;
    }
    __syncthreads();
    // of the warps, in lanes
    const unsigned long long each_warp = lane < kWarps ? sh.draw[lane] : 0;
    const unsigned int each_ties = lane < kWarps ? sh.draw_ties[lane] : 0;
    const unsigned long long cta_weight = sum_warp(each_warp);
    const unsigned int cta_ties = __reduce_add_sync(0xffffffffu, each_ties);
    if ((int)threadIdx.x < ctas) {
        SampleShared* other = cluster.map_shared_rank(&sh, threadIdx.x);
        other->peer_weight[rank] = cta_weight;
        other->peer_ties[rank] = cta_ties;
    }
    cluster.sync();
    // the first weight that exceeds u of the total; rounded up to it, the last one
    auto of_ties = [&](unsigned int before, unsigned int n) { return min(most_ties > before ? most_ties - before : 0u, n) * tie_weight; };
    unsigned long long total = 0, before = 0;
    unsigned int seen = 0, t_before = 0;
    for (int c = 0; c < ctas; ++c) {
        if (c == rank) { before = total; t_before = seen; }
        total += sh.peer_weight[c] + of_ties(seen, sh.peer_ties[c]);
        seen += sh.peer_ties[c];
    }
    const double want = fmin((double)u * (double)total, (double)total - 1.0);
    if ((double)before > want || (double)(before + cta_weight + of_ties(t_before, cta_ties)) <= want) return;
    // the warp: all know which
    const unsigned long long warps_weight = scan_warp(each_warp);
    const unsigned int warps_ties = scan_warp(each_ties);
    const unsigned int up_to = __ballot_sync(0xffffffffu, lane < kWarps && (double)(before + warps_weight + of_ties(t_before, warps_ties)) > want);
    const int chosen = __ffs(up_to) - 1;
    if (chosen > 0) {
        const unsigned long long w0 = __shfl_sync(0xffffffffu, warps_weight, chosen - 1);
        const unsigned int t0 = __shfl_sync(0xffffffffu, warps_ties, chosen - 1);
        before += w0 + of_ties(t_before, t0);
        t_before += t0;
    }
    // the element of vector i with which the wanted weight is exceeded, where it is one
    auto pick = [&](int i) {
        const float4 x4 = row.get(i);
        unsigned long long each[4];
        weights_of(each, x4, sh);
        const float x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (x[e] < least_value) continue;
            if (x[e] == least_value) before += t_before++ < most_ties ? tie_weight : 0;
            else before += each[e];
            if ((double)before > want) {
                a.tokens[r] = start - lead + (row.listed ? (int)sh.place[chosen][4 * i + e] : 4 * i + e);
                return true;
            }
        }
        return false;
    };
    if (warp == chosen && lane == 0) {     // its part of the stretch, or its list
        sh.found_from = row.from;
        sh.found_to = row.to;
        sh.found_bin = row.listed;
    }
    const bool is_short = row.to - row.from <= 32;
    if (warp == chosen && is_short) {      // a vector to a lane, whose parts are there
        const unsigned long long w_up = scan_warp(lane_weight) - lane_weight;
        const unsigned int t_up = scan_warp(lane_ties) - lane_ties;
        before += w_up + of_ties(t_before, t_up);
        t_before += t_up;
        if ((double)before <= want && (double)(before + lane_weight + of_ties(t_before, lane_ties)) > want) pick(row.from + lane);
    }
    __syncthreads();
    if (sh.found_to - sh.found_from <= 32) return;
    row.from = sh.found_from;
    row.to = sh.found_to;
    row.listed = sh.found_bin != 0;
    row.held = row.listed ? reinterpret_cast<const float4*>(sh.may_stay[chosen]) : stretch;
    const int per = (row.to - row.from + kThreads - 1) / kThreads;
    const int my_first = min(row.from + (int)threadIdx.x * per, row.to), my_end = min(my_first + per, row.to);
    unsigned long long mine = 0, all;
    unsigned int tied = 0;
#pragma unroll 1
    for (int i = my_first; i < my_end; ++i) part_of(i, mine, tied);
    // of the threads before
    const unsigned long long w_up = scan_cta(mine, all, sh.warp_scan[0]);
    const unsigned int t_up = (unsigned int)scan_cta(tied, all, sh.warp_scan[1]);
    before += w_up + of_ties(t_before, t_up);
    t_before += t_up;
    if ((double)before > want || (double)(before + mine + of_ties(t_before, tied)) <= want) return;
#pragma unroll 1
    for (int i = my_first; i < my_end; ++i)
        if (pick(i)) return;
}

constexpr int kMostHeld = 192 * 1024;      // bytes that a CTA keeps in shared memory; longer stretches are read again

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
    cfg.dynamicSmemBytes = HELD ? (size_t)a.slice * 4 + 64 : 0;                // the stretch may begin and end inside a vector
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sample_kernel<T, HELD>, a);
}

template <typename T>
cudaError_t launch(SampleArgs a, int num_sms, cudaStream_t st)
{
    // Stretches of which two fit an SM; and as long as all rows are resident at once, shorter ones, down to 4096 tokens (what a cluster does
    // besides the stretches costs as much as some ten thousand tokens: 256 rows of 32000 take 125 us in eights, 49 us in twos).
    int ctas = 1;
    while (ctas < kMostCtas && a.vocab > ctas * 20480) ctas *= 2;
    while (ctas < kMostCtas && a.vocab > ctas * 4096 && (int64_t)a.rows * ctas * 2 <= 2 * num_sms) ctas *= 2;
    a.slice = ((a.vocab + ctas - 1) / ctas + 7) / 8 * 8;
    return (int64_t)a.slice * 4 + 64 <= kMostHeld ? issue<T, true>(a, ctas, st) : issue<T, false>(a, ctas, st);
}

}  // namespace

cudaError_t configure_sample()
{
    const auto allow = [](auto* kernel) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostHeld); };
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

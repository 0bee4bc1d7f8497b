// The hooked attention of single query rows over a cache held in 4 bits: scores, softmax, span masses, P V and steering as in decode.cu,
// whose cuts, folds and merge it shares.  Only the walk over a run of pages is its own.
//
// A warp takes a page of one KV head at a time: one bulk copy brings its slab (2.1 to 2.5 KB) into one of the warp's stages.  The codes
// go into the matrix instructions as they are: a nibble of a masked word, read as a half, is the number code * 2^-24 (or 2^-20 for the nibble
// above it), exactly, and products with subnormal halves are exact too.  So no code is converted; a word of eight costs four ANDs and a
// shift, and the powers of two go into the queries and out of the sums.  With k = lowest + step c for the tokens' groups,
//   x_t = scale * sum_g (step_tg * (q_g . c_tg) + lowest_tg * sum(q_g)),    o = sum_t sum_g p_t step_tg c_tg + sum_t p_t lowest_tg:
// the steps of K multiply the partial products of a group, those of V the probabilities before their one rounding to halves, and the lowest
// values are summed in 32 bits.
//
// Halves reach from 2^-24 to 2^16: p, in the frame of decode.cu, is at most 2^8, and a group's steps go times a power of two of their own that
// keeps the largest so far in [2^6, 2^7) and comes out of the group's sums in the end.  So a product is off by 2^-11 of itself, or by 2^-31 of
// the group's largest step where that is more (from a probability of 2^-20 of the largest on), whatever the other groups hold.
//
// What bounds it is not HBM but instructions: 345 to 425 a page and KV head of 128 (two to four groups), 180 of them on the pipe that masks, shifts and
// permutes take at half rate (58 % busy; issue slots 62 %, tensor pipe 24 %, DRAM 46 %), and the waits for their fixed latencies.  256 sequences of 1024 to
// 8192 keys (683 MB): 165 to 176 us by box, 3.9 to 4.1 TB/s; 4 x 32768 keys of 8 heads in four groups, eight spans (168 MB): 56 us, 3.0 TB/s; 128 x 4096 in
// one, two and four groups 112, 121 and 145 us.  One power of two for the steps of all groups took 55 us in four groups and lost small ones.
// A page at a time with the spans tested on each took 188 and 68 us; five CTAs an SM (96 registers) 192 us, three 167; the shifts by
// multiplication on the other pipe 182 us.
#include <type_traits>

#include "decode_device.cuh"
#include "q4.cuh"

namespace hook_attn {

// decode.cu
cudaError_t launch_decode_merge(const KernelArgs& a, const HeadCfg& hc, int head_dim, bool stream, long parts, cudaStream_t st);
long stream_parts_estimate(const KernelArgs& a, int ctas, int warps);

namespace {

constexpr int kQ4Pages = 2;           // pages that a warp takes at a time
constexpr int kQ4Stages = 2;          // such pairs in flight or in use per warp
constexpr int kQ4Keys = kQ4Pages * kPage;
constexpr int kQ4CtasPerSM = 4;       // at most
// With four groups and no span sums the registers of three CTAs do without memory: 4 x 32768 keys 51 us, and 54 with four; with span sums 59 and 56.
constexpr int q4_ctas(int ng, int ns) { return ng == 4 && ns == 0 ? 3 : kQ4CtasPerSM; }
constexpr int kQ4MaxWorkers = kQ4CtasPerSM * kDecMaxSMs * kDecWarps;
constexpr float kLargestMax = 3.40282326e38f;         // the references stay within it, below kBrokenMax; the probability of an infinite score is infinite
constexpr float kTopStep = 128.f;     // steps times their frame are below this
constexpr float kFirstFrame = 1.6225928e32f;          // 2^107: steps are at least 2^-100

__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 t = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}

// N words (1, 2 or 4) from shared memory, N * 4 bytes aligned.
template <int N>
__device__ __forceinline__ void lds(uint32_t (&r)[N], uint32_t addr)
{
    if constexpr (N == 1) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r[0]) : "r"(addr));
    else if constexpr (N == 2) asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr));
    else asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// A warp that reduces runs of 4-bit pages, two at a time.  Its stages and their barriers are its own; `turn` counts the pairs it has taken, so
// stages and phases go on from one run to the next.
template <int HD, int NG>
struct Q4Walk {
    using Slab = Q4Slab<HD, NG>;
    static constexpr int kStage = kQ4Pages * Slab::kBytes;
    static constexpr int kBytes = kQ4Stages * kStage;                 // of one warp's stages
    static constexpr int kMass = kMaxSpans * 8 * 4;                   // of one warp's span sums
    // of a CTA: the stages, where its warps' sums are folded in the end, the span sums, then the barriers, which nothing else may touch
    static constexpr int kCtaBytes = kDecWarps * (kBytes + kMass + kQ4Stages * 8);
    static_assert(kDecWarps * 8 * (HD + 4) * 4 <= kDecWarps * kBytes, "the fold's buffer fits the stages");
    uint32_t base, bars, turn = 0;
    float* mass;                                                      // [span][head]

    __device__ __forceinline__ Q4Walk(uint8_t* smem, int warp)
        : base(smem_u32(smem) + warp * kBytes), bars(smem_u32(smem) + kDecWarps * (kBytes + kMass) + warp * kQ4Stages * 8),
          mass(reinterpret_cast<float*>(smem + kDecWarps * kBytes + warp * kMass))
    {
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
            for (int i = 0; i < kQ4Stages; ++i) mbar_init(bars + 8 * i, 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
    }

    template <int NS>
    __device__ __forceinline__ void segment(const KernelArgs& a, const HeadCfg& hc, int s, int kvh, int pg, int seg, int L, int* span,
                                            float& m0, float& m1, float& l0, float& l1, float (&o)[HD / 16][4], float (&sm)[NS > 0 ? NS : 1][2])
    {
        constexpr int KS = HD / 16, W = HD / 32, PER = W / NG;        // W: words of a lane's K codes; PER: words to a group
        constexpr int NSX = NS > 0 ? NS : 1;
        const int lane = threadIdx.x & 31, g = lane >> 2, tq = lane & 3, G = a.G;

        m0 = m1 = -INFINITY;
        l0 = l1 = 0.f;
#pragma unroll
        for (int i = 0; i < KS; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
#pragma unroll
        for (int j = 0; j < NSX; ++j) sm[j][0] = sm[j][1] = 0.f;
        if (seg <= 0) return;
        m0 = m1 = -kLargestMax;                                       // finite, so that keys whose scores are all -infinity weigh nothing

        const int32_t* bt = a.block_table + (int64_t)s * a.max_blocks + pg;
        const int key_base = pg * kPage, key_end = min(L, key_base + seg * kPage);
        const char* pages = reinterpret_cast<const char*>(a.k) + (int64_t)kvh * a.hs;     // strides in bytes

        // Spans cost nothing between their edges: `run` sums the probabilities since the last edge, for the spans in `inside`, and goes to their sums
        // in shared memory at the next.
        bool broken = false;
        float run0 = 0.f, run1 = 0.f;
        uint32_t inside = 0;
        int edge = 0x7fffffff;
        int my_a = 0, my_b = 0;                                       // lane j < S: span j
        auto locate = [&](int key) {                                  // which spans hold the key, and where that next changes
            inside = __ballot_sync(0xffffffffu, key >= my_a && key < my_b);
            edge = __reduce_min_sync(0xffffffffu, my_a >= my_b ? 0x7fffffff : my_a > key ? my_a : my_b > key ? my_b : 0x7fffffff);
        };
        auto add_mass = [&](int j, float x0, float x1) {              // sums over the warp, to span j
#pragma unroll
            for (int d = 4; d <= 16; d <<= 1) {
                x0 += __shfl_xor_sync(0xffffffffu, x0, d);
                x1 += __shfl_xor_sync(0xffffffffu, x1, d);
            }
            if (g == 0) {
                mass[8 * j + 2 * tq] += x0;
                mass[8 * j + 2 * tq + 1] += x1;
            }
        };
        auto flush = [&]() {
            if (inside)
#pragma unroll 1
                for (uint32_t left = inside; left; left &= left - 1) add_mass(__ffs(left) - 1, run0, run1);
            run0 = run1 = 0.f;
        };
        if constexpr (NS > 0) {
            bool probe = false;
            for (int i = 0; i < G; ++i) probe |= (hc.slot[kvh * G + i] >= 0);
            if (probe && lane < a.S) {
                my_a = a.spans[((int64_t)s * a.S + lane) * 2];
                my_b = a.spans[((int64_t)s * a.S + lane) * 2 + 1];
            }
            for (int i = lane; i < kMaxSpans * 8; i += 32) mass[i] = 0.f;
            __syncwarp();
            locate(key_base);
        }

        // block ids of 32 consecutive pages, one per lane; the next 32 are fetched a window ahead
        int btw = 0, btw_next = (lane < seg) ? bt[lane] : 0;
        auto issue = [&](int it) {                                    // pages it and it + 1 by lanes 0 and 1
            if (it >= seg) return;
            if ((it & 31) == 0) {
                btw = btw_next;
                btw_next = (it + 32 + lane < seg) ? bt[it + 32 + lane] : 0;
            }
            const int page = __shfl_sync(0xffffffffu, btw, (it + (lane & 1)) & 31);
            const bool mine = lane < 2 && it + lane < seg, ok = mine && (uint32_t)page < (uint32_t)a.num_blocks;
            const uint32_t good = __ballot_sync(0xffffffffu, ok), wanted = __ballot_sync(0xffffffffu, mine);
            const uint32_t st = (turn + it / kQ4Pages) % kQ4Stages, bar = bars + 8 * st;
            if (lane == 0) {
                mbar_expect_tx(bar, __popc(good) * Slab::kBytes);
                if (good != wanted) report(a.status, HOOK_ATTN_ERR_BOUNDS);
            }
            broken |= good != wanted;
            __syncwarp();
            if (ok) bulk_load(base + st * kStage + lane * Slab::kBytes, pages + (int64_t)page * a.bs, Slab::kBytes, bar);
        };
        issue(0);

        // The queries of head g of the group as halves, times a power of two that brings the largest to [2^14, 2^15): what is below 2^-27 of
        // that loses bits.  In a word's pairs (element n, n + 4) the odd nibbles stand for 16 times their code.
        uint32_t qb[KS][2];
        float qs0, qs1, qsum[NG][2];
        {
            float x[W][8], most = 0.f, sum[NG];
#pragma unroll
            for (int i = 0; i < W; ++i) {
                uint4 raw = make_uint4(0, 0, 0, 0);
                if (g < G) raw = *reinterpret_cast<const uint4*>(a.q + ((int64_t)s * a.Hq + kvh * G + g) * HD + 32 * i + 8 * tq);
                const uint32_t r[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[i][2 * e] = __uint_as_float(r[e] << 16);
                    x[i][2 * e + 1] = __uint_as_float(r[e] & 0xffff0000u);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[i][e]));
            }
#pragma unroll
            for (int j = 0; j < NG; ++j) {
                sum[j] = 0.f;
#pragma unroll
                for (int i = j * PER; i < (j + 1) * PER; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[j] += x[i][e];
            }
#pragma unroll
            for (int d = 1; d <= 2; d <<= 1) {
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
#pragma unroll
                for (int j = 0; j < NG; ++j) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], d);
            }
            int up = 141 - (int)(__float_as_uint(most) >> 23);        // 14 less the exponent
            up = most > 0.f ? min(max(up, -100), 100) : 0;
            const float raise = __uint_as_float((uint32_t)(127 + up) << 23), odd = raise * 0.0625f;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                qb[2 * i][0] = pack_f16(x[i][0] * raise, x[i][4] * raise);
                qb[2 * i][1] = pack_f16(x[i][1] * odd, x[i][5] * odd);
                qb[2 * i + 1][0] = pack_f16(x[i][2] * raise, x[i][6] * raise);
                qb[2 * i + 1][1] = pack_f16(x[i][3] * odd, x[i][7] * odd);
            }
            const float back = __uint_as_float((uint32_t)(127 + min(24 - up, 127)) << 23) * a.scale_log2;   // 2^24: a code as a half
            qs0 = __shfl_sync(0xffffffffu, back, 8 * tq);             // of heads 2 tq and 2 tq + 1
            qs1 = __shfl_sync(0xffffffffu, back, 8 * tq + 4);
#pragma unroll
            for (int j = 0; j < NG; ++j) {
                qsum[j][0] = __shfl_sync(0xffffffffu, sum[j], 8 * tq) * a.scale_log2;
                qsum[j][1] = __shfl_sync(0xffffffffu, sum[j], 8 * tq + 4) * a.scale_log2;
            }
        }

        // The accumulators hold p 2^(x - m), o's codes that times their group's `frame`, the power of two that brings its largest step so far to [2^6, 2^7).
        float frame[NG], zl[NG][2];
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            frame[j] = kFirstFrame;
            zl[j][0] = zl[j][1] = 0.f;
        }

        uint64_t limit_ns = 2000000000ull;
        // LAST: the run ends among these keys, and what lies behind it may be anything.
        auto pair_of_pages = [&](auto LAST, int it) {
            constexpr bool last = decltype(LAST)::value;
            issue(it + kQ4Pages);
            const uint32_t n = turn + it / kQ4Pages, st = n % kQ4Stages;
            if (!__all_sync(0xffffffffu, mbar_wait(bars + 8 * st, (n / kQ4Stages) & 1u, nullptr, limit_ns))) {
                if (lane == 0) report(a.status, HOOK_ATTN_ERR_TIMEOUT);
                broken = true;
                limit_ns = 1000000;                           // the others in flight are waited for, but not for long
            }
            const uint32_t stage = base + st * kStage;
            const int key0 = key_base + it * kPage;

            // ---- scores: keys g and g + 8 of each page for the heads 2 tq and 2 tq + 1 ----
            float x[kQ4Pages][4], top[NG];
#pragma unroll
            for (int j = 0; j < NG; ++j) top[j] = 0.f;
#pragma unroll
            for (int u = 0; u < kQ4Pages; ++u) {
                const uint32_t kt = stage + u * Slab::kBytes, kp = kt + 2 * Slab::kCodes + g * (NG * 4), vp = kp + Slab::kParams;
                uint32_t wa[W], wb[W], pa[NG], pb[NG];
                lds<W>(wa, kt + g * Slab::kRow + tq * (W * 4));
                lds<W>(wb, kt + (g + 8) * Slab::kRow + tq * (W * 4));
                lds<NG>(pa, kp);
                lds<NG>(pb, kp + 8 * (NG * 4));
                float w0 = 0.f, w1 = 0.f, w2 = 0.f, w3 = 0.f, y0 = 0.f, y1 = 0.f, y2 = 0.f, y3 = 0.f;
#pragma unroll
                for (int j = 0; j < NG; ++j) {
                    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = j * PER; i < (j + 1) * PER; ++i) {
                        mma_f16_16816(acc, wa[i] & 0x000f000fu, wb[i] & 0x000f000fu, wa[i] & 0x00f000f0u, wb[i] & 0x00f000f0u, qb[2 * i][0], qb[2 * i][1]);
                        const uint32_t ua = wa[i] >> 8, ub = wb[i] >> 8;
                        mma_f16_16816(acc, ua & 0x000f000fu, ub & 0x000f000fu, ua & 0x00f000f0u, ub & 0x00f000f0u, qb[2 * i + 1][0], qb[2 * i + 1][1]);
                    }
                    const float sa = q4_step(pa[j]), sb = q4_step(pb[j]), la = q4_lowest(pa[j]), lb = q4_lowest(pb[j]);
                    y0 += sa * acc[0]; y1 += sa * acc[1];
                    y2 += sb * acc[2]; y3 += sb * acc[3];
                    w0 += la * qsum[j][0]; w1 += la * qsum[j][1];
                    w2 += lb * qsum[j][0]; w3 += lb * qsum[j][1];
                }
                x[u][0] = y0 * qs0 + w0; x[u][1] = y1 * qs1 + w1;
                x[u][2] = y2 * qs0 + w2; x[u][3] = y3 * qs1 + w3;
                lds<NG>(pa, vp);                              // steps of V
                lds<NG>(pb, vp + 8 * (NG * 4));
                const int t0 = key0 + u * kPage + g;
                if (last && t0 >= key_end) {
                    x[u][0] = x[u][1] = -INFINITY;
#pragma unroll
                    for (int j = 0; j < NG; ++j) pa[j] = 0;
                }
                if (last && t0 + 8 >= key_end) {
                    x[u][2] = x[u][3] = -INFINITY;
#pragma unroll
                    for (int j = 0; j < NG; ++j) pb[j] = 0;
                }
#pragma unroll
                for (int j = 0; j < NG; ++j) top[j] = fmaxf(top[j], fmaxf(q4_step(pa[j]), q4_step(pb[j])));
            }
            float mx0 = x[0][0], mx1 = x[0][1];
#pragma unroll
            for (int u = 0; u < kQ4Pages; ++u) {
                mx0 = fmaxf(mx0, fmaxf(x[u][0], x[u][2]));
                mx1 = fmaxf(mx1, fmaxf(x[u][1], x[u][3]));
            }
            // ---- the references ----
            float highest = top[0] * frame[0];
#pragma unroll
            for (int j = 1; j < NG; ++j) highest = fmaxf(highest, top[j] * frame[j]);
            if (__any_sync(0xffffffffu, mx0 > m0 + kDecRaise || mx1 > m1 + kDecRaise || highest >= kTopStep)) {
#pragma unroll
                for (int d = 4; d <= 16; d <<= 1) {
                    mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, d));
                    mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, d));
                }
                const float n0 = fminf(fmaxf(m0, mx0), kLargestMax), n1 = fminf(fmaxf(m1, mx1), kLargestMax);
                const float c0 = fast_exp2(m0 - n0), c1 = fast_exp2(m1 - n1);
                m0 = n0; m1 = n1;
                l0 *= c0; l1 *= c1;
#pragma unroll
                for (int j = 0; j < NG; ++j) {
                    const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(top[j]));
                    float k0 = c0, k1 = c1;
                    if (__uint_as_float(most) * frame[j] >= kTopStep) {
                        const float to = __uint_as_float((260u << 23) - (most & 0x7f800000u));        // 2^6 over the step's power
                        const float shrink = to * __uint_as_float((254u << 23) - __float_as_uint(frame[j]));
                        k0 *= shrink;
                        k1 *= shrink;
                        frame[j] = to;
                    }
#pragma unroll
                    for (int i = 2 * j * PER; i < 2 * (j + 1) * PER; ++i) { o[i][0] *= k0; o[i][1] *= k1; o[i][2] *= k0; o[i][3] *= k1; }
                    zl[j][0] *= c0; zl[j][1] *= c1;
                }
                if constexpr (NS > 0) {
                    run0 *= c0;
                    run1 *= c1;
                    if (g == 0)
#pragma unroll 1
                        for (int j = 0; j < a.S; ++j) { mass[8 * j + 2 * tq] *= c0; mass[8 * j + 2 * tq + 1] *= c1; }
                }
            }
            float s0 = 0.f, s1 = 0.f;
#pragma unroll
            for (int u = 0; u < kQ4Pages; ++u) {
                x[u][0] = fast_exp2(x[u][0] - m0); x[u][1] = fast_exp2(x[u][1] - m1);
                x[u][2] = fast_exp2(x[u][2] - m0); x[u][3] = fast_exp2(x[u][3] - m1);
                s0 += x[u][0] + x[u][2];
                s1 += x[u][1] + x[u][3];
            }
            l0 += s0;
            l1 += s1;
            if constexpr (NS > 0) {
                if (edge >= key0 + kQ4Keys) {
                    run0 += s0;
                    run1 += s1;
                } else {                                      // an edge among these keys
                    flush();
#pragma unroll 1
                    for (int j = 0; j < a.S; ++j) {
                        const int sa = __shfl_sync(0xffffffffu, my_a, j), sb = __shfl_sync(0xffffffffu, my_b, j);
                        float in0 = 0.f, in1 = 0.f;
#pragma unroll
                        for (int u = 0; u < kQ4Pages; ++u) {
                            const int t0 = key0 + u * kPage + g, t1 = t0 + 8;
                            if (t0 >= sa && t0 < sb) { in0 += x[u][0]; in1 += x[u][1]; }
                            if (t1 >= sa && t1 < sb) { in0 += x[u][2]; in1 += x[u][3]; }
                        }
                        add_mass(j, in0, in1);
                    }
                    locate(key0 + kQ4Keys);
                }
            }
            // ---- P V, page by page: for each group the probabilities times the steps, as the B operand (k = key, n = head) ----
#pragma unroll
            for (int u = 0; u < kQ4Pages; ++u) {
                const uint32_t vt = stage + u * Slab::kBytes + Slab::kCodes, vp = vt + Slab::kCodes + Slab::kParams + g * (NG * 4);
                uint32_t va[NG], vb[NG], pb[NG][2];
                lds<NG>(va, vp);
                lds<NG>(vb, vp + 8 * (NG * 4));
                if (last) {
                    const int t0 = key0 + u * kPage + g;
#pragma unroll
                    for (int j = 0; j < NG; ++j) {
                        if (t0 >= key_end) va[j] = 0;
                        if (t0 + 8 >= key_end) vb[j] = 0;
                    }
                }
#pragma unroll
                for (int j = 0; j < NG; ++j) {
                    const float sa = q4_step(va[j]) * frame[j], sb = q4_step(vb[j]) * frame[j], la = q4_lowest(va[j]), lb = q4_lowest(vb[j]);
                    pb[j][0] = movmatrix_trans(pack_f16(x[u][0] * sa, x[u][1] * sa));
                    pb[j][1] = movmatrix_trans(pack_f16(x[u][2] * sb, x[u][3] * sb));
                    zl[j][0] += x[u][0] * la + x[u][2] * lb;
                    zl[j][1] += x[u][1] * la + x[u][3] * lb;
                }
                constexpr int U = HD / 64;                    // words of a unit: keys 2 tq, 2 tq + 1, 2 tq + 8, 2 tq + 9 of the page
                uint32_t v0[U], v1[U], v2[U], v3[U];
                const uint32_t unit = vt + tq * Slab::kRow + q4_unit<HD>(tq, g) * (U * 4);
                lds<U>(v0, unit);
                lds<U>(v1, unit + 4 * Slab::kRow);
                lds<U>(v2, unit + 8 * Slab::kRow);
                lds<U>(v3, unit + 12 * Slab::kRow);
#pragma unroll
                for (int j = 0; j < W; ++j) {                 // 32 elements: two blocks of 16 of the output
                    const uint32_t sel = j & 1 ? 0x7632u : 0x5410u;
                    uint32_t lo = __byte_perm(v0[j / 2], v1[j / 2], sel), hi = __byte_perm(v2[j / 2], v3[j / 2], sel);
                    const int grp = j / PER;
                    mma_f16_16816(o[2 * j], lo & 0x000f000fu, lo & 0x00f000f0u, hi & 0x000f000fu, hi & 0x00f000f0u, pb[grp][0], pb[grp][1]);
                    lo >>= 8;
                    hi >>= 8;
                    mma_f16_16816(o[2 * j + 1], lo & 0x000f000fu, lo & 0x00f000f0u, hi & 0x000f000fu, hi & 0x00f000f0u, pb[grp][0], pb[grp][1]);
                }
            }
            __syncwarp();                                     // the stage may be filled again
        };
        int it = 0;
#pragma unroll 1
        for (; key_base + it * kPage + kQ4Keys <= key_end; it += kQ4Pages) pair_of_pages(std::false_type(), it);
        if (it < seg) pair_of_pages(std::true_type(), it);
        turn += (seg + kQ4Pages - 1) / kQ4Pages;

        // per-thread partial sums -> per-warp sums (lanes with the same tq hold the same heads)
#pragma unroll
        for (int d = 4; d <= 16; d <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, d);
            l1 += __shfl_xor_sync(0xffffffffu, l1, d);
#pragma unroll
            for (int j = 0; j < NG; ++j) {
                zl[j][0] += __shfl_xor_sync(0xffffffffu, zl[j][0], d);
                zl[j][1] += __shfl_xor_sync(0xffffffffu, zl[j][1], d);
            }
        }
        if constexpr (NS > 0) {
            flush();
            __syncwarp();
#pragma unroll
            for (int j = 0; j < NS; ++j) {
                sm[j][0] = mass[8 * j + 2 * tq];
                sm[j][1] = mass[8 * j + 2 * tq + 1];
            }
            __syncwarp();
        }
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            const int j = i / 2 / PER;
            const float back = __uint_as_float((254u << 23) - __float_as_uint(frame[j]));
            o[i][0] = o[i][0] * 16777216.f * back + zl[j][0]; o[i][1] = o[i][1] * 16777216.f * back + zl[j][1];   // rows g: codes times 2^-24
            o[i][2] = o[i][2] * 1048576.f * back + zl[j][0]; o[i][3] = o[i][3] * 1048576.f * back + zl[j][1];     // rows g + 8: times 2^-20
        }
        if (broken) {                                         // a page out of range: the row becomes zeros
            m0 = m1 = kBrokenMax;
            l0 = l1 = 1.f;
#pragma unroll
            for (int i = 0; i < KS; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
#pragma unroll
            for (int j = 0; j < NSX; ++j) sm[j][0] = sm[j][1] = 0.f;
        }
    }
};

template <int HD, int NG>
constexpr int q4_smem_bytes() { return Q4Walk<HD, NG>::kCtaBytes; }

template <int HD, int NG, int NS>
__global__ void __launch_bounds__(kDecWarps * 32, q4_ctas(NG, NS)) decode_q4_stream_kernel(const KernelArgs a, const HeadCfg hc)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ DecStreamShared<kDecWarps> sh;
    decode_stream_cta<HD, NS, kDecWarps, Q4Walk<HD, NG>>(a, hc, smem, blockIdx.x, sh);
}

template <int HD, int NG, int NS>
__global__ void __launch_bounds__(kDecWarps * 32, q4_ctas(NG, NS)) decode_q4_splitk_kernel(const KernelArgs a, const HeadCfg hc)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int sh_span[kDecWarps][2 * kMaxSpans];
    __shared__ DecFold sh_fold;

    const int s = blockIdx.z, kvh = blockIdx.y, c = blockIdx.x;
    const int warp = threadIdx.x >> 5;
    asm volatile("griddepcontrol.wait;" ::: "memory");        // as in decode.cu: the merge of the call before may still be running
    const int L = a.seq_lens[s];
    if (L <= 0 || L > a.max_keys) return;                     // reported and zero-filled by the merge kernel
    const int start = c * a.chunk;
    if (start >= L) return;
    const int ntiles = (min(L, start + a.chunk) - start + kPage - 1) / kPage;
    const int per = (ntiles + kDecWarps - 1) / kDecWarps;     // the four warps take contiguous quarters of the chunk's pages
    const int first = min(warp * per, ntiles);
    Q4Walk<HD, NG> walk(smem, warp);
    float m0, m1, l0, l1, o[HD / 16][4], sm[NS > 0 ? NS : 1][2];
    walk.template segment<NS>(a, hc, s, kvh, start / kPage + first, min(per, ntiles - first), L, sh_span[warp], m0, m1, l0, l1, o, sm);
    float* part = a.ws + (((size_t)s * a.Hkv + kvh) * a.max_chunks + c) * a.G * decode_partial_stride(HD);
    decode_fold_cta<HD, NS>(part, a.G, reinterpret_cast<float*>(smem), sh_fold, 1, m0, m1, l0, l1, o, sm);
}

// How a call is cut, from host-known bounds only.  Chunks of a fixed length, the largest power of two in 256 .. 2048 keys that leaves eight CTAs
// an SM, but for few units of very long sequences, whose pages are shared out evenly: there chunks would leave long merges (4 x 32768
// keys of 8 KV heads: 41 to 54 us shared out, 43 to 59 in chunks).  Elsewhere finding the shares is what costs: 1 x 2000 keys take 8.3 us in
// chunks and 12.4 shared out, 36 of up to 4096 31 to 36 and 42 to 49.
constexpr int kQ4Long = 16384;            // keys of a sequence, at most
constexpr long kQ4Shared = 4L * kQ4CtasPerSM * kDecMaxSMs * 16;   // pages of all units, at most: four waves of CTAs of 256 keys
struct Q4Plan {
    bool stream;
    int chunk, max_chunks;
};

Q4Plan q4_plan(int num_seqs, int Hkv, int max_keys)
{
    Q4Plan p = {};
    const long pages = (long)num_seqs * Hkv * (((long)max_keys + kPage - 1) / kPage);
    p.stream = (long)num_seqs * Hkv < kDecStreamUnits && max_keys >= kQ4Long && pages > kQ4Shared;
    p.chunk = 2048;
    while (p.chunk > 256) {
        const long ctas = (long)num_seqs * Hkv * (((long)max_keys + p.chunk - 1) / p.chunk);
        if (ctas >= 8L * kDecMaxSMs) break;
        p.chunk >>= 1;
    }
    p.max_chunks = (int)(((long)max_keys + p.chunk - 1) / p.chunk);
    if (p.max_chunks < 1) p.max_chunks = 1;
    return p;
}

template <int HD, int NG, int NS>
cudaError_t launch_t(KernelArgs a, const HeadCfg& hc, int num_sms, cudaStream_t st)
{
    const Q4Plan plan = q4_plan(a.num_seqs, a.Hkv, a.max_keys);
    a.chunk = plan.chunk;
    a.max_chunks = plan.max_chunks;
    long parts;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kDecWarps * 32);
    cfg.dynamicSmemBytes = q4_smem_bytes<HD, NG>();
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = plan.stream ? 0 : 1;
    cudaError_t e;
    if (plan.stream) {
        const int ctas = q4_ctas(NG, NS) * (num_sms < kDecMaxSMs ? (num_sms > 0 ? num_sms : 1) : kDecMaxSMs);
        a.workers = ctas * kDecWarps;
        cfg.gridDim = dim3(ctas);
        e = cudaLaunchKernelEx(&cfg, decode_q4_stream_kernel<HD, NG, NS>, a, hc);
        parts = stream_parts_estimate(a, ctas, kDecWarps);
    } else {
        cfg.gridDim = dim3(plan.max_chunks, a.Hkv, a.num_seqs);
        e = cudaLaunchKernelEx(&cfg, decode_q4_splitk_kernel<HD, NG, NS>, a, hc);
        parts = plan.max_chunks;
    }
    if (e != cudaSuccess) return e;
    return launch_decode_merge(a, hc, HD, plan.stream, parts, st);
}

template <int HD, int NG>
cudaError_t launch_ng(const KernelArgs& a, const HeadCfg& hc, int num_sms, cudaStream_t st)
{
    if (!a.any_probe) return launch_t<HD, NG, 0>(a, hc, num_sms, st);
    return a.S <= 4 ? launch_t<HD, NG, 4>(a, hc, num_sms, st) : launch_t<HD, NG, 8>(a, hc, num_sms, st);
}

template <int HD, int NG>
cudaError_t configure_one()
{
    const auto allow = [](auto* kernel) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, q4_smem_bytes<HD, NG>()); };
    cudaError_t e;
#define HOOK_CFG(NS) if ((e = allow(decode_q4_splitk_kernel<HD, NG, NS>)) != cudaSuccess || (e = allow(decode_q4_stream_kernel<HD, NG, NS>)) != cudaSuccess) return e;
    HOOK_CFG(0) HOOK_CFG(4) HOOK_CFG(8)
#undef HOOK_CFG
    return cudaSuccess;
}

}  // namespace

cudaError_t configure_decode_q4()
{
    cudaError_t e = configure_one<64, 1>();
    if (e == cudaSuccess) e = configure_one<64, 2>();
    if (e == cudaSuccess) e = configure_one<128, 1>();
    if (e == cudaSuccess) e = configure_one<128, 2>();
    if (e == cudaSuccess) e = configure_one<128, 4>();
    return e;
}

// As decode_workspace_bytes: one partial per (unit, chunk), or the page-count prefix and one per (unit, warp) that meet.
size_t decode_q4_workspace_bytes(int num_seqs, int Hkv, int G, int head_dim, int max_keys)
{
    const Q4Plan plan = q4_plan(num_seqs, Hkv, max_keys);
    const size_t per_part = (size_t)G * decode_partial_stride(head_dim) * sizeof(float);
    if (plan.stream) return decode_prefix_bytes(num_seqs) + ((size_t)num_seqs * Hkv + kQ4MaxWorkers) * per_part;
    return (size_t)num_seqs * Hkv * plan.max_chunks * per_part;
}

// `a.k` is the pages, `a.bs` and `a.hs` their strides in bytes.
cudaError_t launch_decode_q4(const KernelArgs& a, const HeadCfg& hc, int head_dim, int group, int num_sms, cudaStream_t st)
{
    const int ng = head_dim / group;
    if (head_dim == 64) return ng == 1 ? launch_ng<64, 1>(a, hc, num_sms, st) : launch_ng<64, 2>(a, hc, num_sms, st);
    if (ng == 1) return launch_ng<128, 1>(a, hc, num_sms, st);
    return ng == 2 ? launch_ng<128, 2>(a, hc, num_sms, st) : launch_ng<128, 4>(a, hc, num_sms, st);
}

}  // namespace hook_attn

// The pages of the cache: sequences that share pages (fork), get room for new rows (extend), give pages back (free), and a
// pool whose pages are moved together at its low end (compact).  A page's entry in page_refs counts the sequences that hold
// it; 0 (or less) is free.  All results are integers that do not depend on the order in which threads run.
#include "common.cuh"
#include "ops.cuh"

#include <cooperative_groups.h>

namespace hook_attn {

namespace {

constexpr int kListThreads = 256;
constexpr int kPoolThreads = 1024;

__device__ __forceinline__ int pages_of(int len) { return (int)(((int64_t)len + kPage - 1) / kPage); }
__device__ __forceinline__ int64_t capacity(const PoolArgs& p) { return min((int64_t)p.max_blocks * kPage, (int64_t)INT32_MAX); }
__device__ __forceinline__ bool page_ok(const PoolArgs& p, int page) { return page >= 0 && page < p.num_blocks; }

// A CTA reads the pool's reference counts in steps of EACH neighbouring pages to a thread.
template <int EACH>
__device__ __forceinline__ void load_refs(const PoolArgs& p, int base, int (&refs)[EACH], int missing)
{
    const int first = base + (int)threadIdx.x * EACH;
    if (EACH % 4 == 0 && first + EACH <= p.num_blocks && (reinterpret_cast<uintptr_t>(p.page_refs) & 15) == 0) {
#pragma unroll
        for (int u = 0; u < EACH / 4; ++u) {
            const int4 r = reinterpret_cast<const int4*>(p.page_refs + first)[u];
            refs[4 * u] = r.x; refs[4 * u + 1] = r.y; refs[4 * u + 2] = r.z; refs[4 * u + 3] = r.w;
        }
    } else {
#pragma unroll
        for (int u = 0; u < EACH; ++u) refs[u] = first + u < p.num_blocks ? p.page_refs[first + u] : missing;
    }
}

// Bit u: the thread's page u is free.
template <int EACH>
__device__ __forceinline__ uint32_t free_pages(const PoolArgs& p, int base)
{
    int refs[EACH];
    load_refs<EACH>(p, base, refs, 1);
    uint32_t bits = 0;
#pragma unroll
    for (int u = 0; u < EACH; ++u) bits |= (uint32_t)(refs[u] <= 0) << u;
    return bits;
}

// One CTA per entry: children[i] gets the pages of parents[i].  An entry is refused (status) when a row is out of range, the
// child holds pages, the child is listed earlier, the child is a parent of the same call, or the parent's row is broken: its length or
// a page is out of range, or nobody holds a page of it.  Which counts are above 0 does not change during the call.
__global__ void __launch_bounds__(kListThreads) fork_kernel(const PoolArgs p, const int32_t* __restrict__ parents,
                                                            const int32_t* __restrict__ children, int n)
{
    const int i = blockIdx.x, parent = parents[i], child = children[i];
    bool bad = parent < 0 || parent >= p.num_seqs || child < 0 || child >= p.num_seqs;
    for (int j = threadIdx.x; j < n; j += kListThreads) bad |= parents[j] == child || (j < i && children[j] == child);
    int L = 0;
    if (!bad) {
        L = p.seq_lens[parent];
        bad = p.seq_lens[child] != 0 || L < 0 || L > capacity(p);
    }
    const int pages = bad ? 0 : pages_of(L);
    const int32_t* from = p.block_table + (int64_t)parent * p.max_blocks;
    for (int j = threadIdx.x; j < pages; j += kListThreads) bad |= !page_ok(p, from[j]) || p.page_refs[from[j]] <= 0;
    if (__syncthreads_or(bad)) {
        if (threadIdx.x == 0) report(p.status, HOOK_ATTN_ERR_BOUNDS);
        return;
    }
    int32_t* to = p.block_table + (int64_t)child * p.max_blocks;
    for (int j = threadIdx.x; j < pages; j += kListThreads) {
        const int page = from[j];
        to[j] = page;
        atomicAdd(&p.page_refs[page], 1);
    }
    if (threadIdx.x == 0) p.seq_lens[child] = L;
}

// One CTA per entry: the pages of sequence seqs[i] behind its first keep_lens[i] tokens go back.  A sequence that is listed
// again is passed over.
__global__ void __launch_bounds__(kListThreads) free_kernel(const PoolArgs p, const int32_t* __restrict__ seqs,
                                                            const int32_t* __restrict__ keep_lens)
{
    const int i = blockIdx.x, s = seqs[i], keep = keep_lens ? keep_lens[i] : 0;
    bool again = false;
    for (int j = threadIdx.x; j < i; j += kListThreads) again |= seqs[j] == s;
    if (__syncthreads_or(again)) return;
    const int L = s < 0 || s >= p.num_seqs ? -1 : p.seq_lens[s];
    if (L < 0 || L > capacity(p) || keep < 0) {
        if (threadIdx.x == 0) report(p.status, HOOK_ATTN_ERR_BOUNDS);
        return;
    }
    __syncthreads();                              // every thread has read the length
    if (keep >= L) return;
    if (threadIdx.x == 0) p.seq_lens[s] = keep;
    int32_t* row = p.block_table + (int64_t)s * p.max_blocks;
    for (int j = pages_of(keep) + threadIdx.x; j < pages_of(L); j += kListThreads) {
        const int page = row[j];
        row[j] = -1;
        bool ok = page_ok(p, page);
        if (ok && atomicSub(&p.page_refs[page], 1) <= 0) {      // held by nobody: the entry does not count
            atomicAdd(&p.page_refs[page], 1);
            ok = false;
        }
        if (!ok) report(p.status, HOOK_ATTN_ERR_BOUNDS);
    }
}

// Room for new_rows[s] more tokens of every sequence.  A sequence needs its missing pages, and one more when its last page is
// partly filled and held by others too: the rows to come would write into it, so it gets a page of its own and the pair
// (old page, new page) to copy.  Needs are summed in sequence order and the k-th free page goes to the k-th need; sequences
// that the pool cannot serve in that order stay as they are.
//
// One CTA does it, since what it hands out is little: 1, 4 or 16 pages to a thread, the fewest that cover the pool in one step
// (4096 pages, 64 sequences: 5.2 us).  A pool of more steps is counted by the other CTAs of a cluster (CLUSTER) meanwhile, so that the steps
// without a free page need not be looked through one after the other (100000 pages, the last tenth of them free: 9.3 us, and 25 us
// with one CTA; 16384 pages: 8.4 us with one CTA).
constexpr int kSplit = 1 << 30;                   // flag in a need: the last page is shared
constexpr int kClusterCtas = 8;
constexpr int kUnits = 1024;                      // counts of free pages that the cluster makes
static_assert(kUnits == kPoolThreads, "a thread clears and sums one");

template <int EACH, bool CLUSTER>
__global__ void __launch_bounds__(kPoolThreads) extend_kernel(const PoolArgs p, const int32_t* __restrict__ new_rows,
                                                              int32_t* __restrict__ pairs)
{
    extern __shared__ int32_t dyn[];
    int32_t* need = dyn;                          // [num_seqs] pages, with kSplit; -1: the sequence is left out
    int32_t* first = dyn + p.num_seqs;            // [num_seqs] place of its first page among all needs
    uint16_t* list = reinterpret_cast<uint16_t*>(dyn + 2 * p.num_seqs);   // [kPoolThreads * EACH] free pages of a step
    __shared__ int sh[33];
    __shared__ int units[CLUSTER ? kUnits : 1];
    constexpr int kStep = kPoolThreads * EACH;
    const int steps = (p.num_blocks + kStep - 1) / kStep, per_unit = (steps + kUnits - 1) / kUnits;
    if (CLUSTER) {
        const cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
        const int rank = (int)cluster.block_rank();
        if (rank == 0) units[threadIdx.x] = 0;
        cluster.sync();
        if (rank > 0) {
            int* to = cluster.map_shared_rank(units, 0);
            for (int step = rank - 1; step < steps; step += kClusterCtas - 1) {
                const int n = __reduce_add_sync(0xffffffffu, __popc(free_pages<EACH>(p, step * kStep)));
                if ((threadIdx.x & 31) == 0 && n > 0) atomicAdd(to + step / per_unit, n);
            }
            cluster.sync();
            return;
        }
    }
    int wanted = 0;
    for (int base = 0; base < p.num_seqs; base += kPoolThreads) {
        const int s = base + (int)threadIdx.x;
        int k = 0;
        if (s < p.num_seqs) {
            const int L = p.seq_lens[s], n = new_rows[s];
            bool bad = L < 0 || n < 0 || (int64_t)L + n > capacity(p);
            bool split = false;
            if (!bad && n > 0 && L % kPage) {
                const int last = p.block_table[(int64_t)s * p.max_blocks + L / kPage];
                const int refs = page_ok(p, last) ? p.page_refs[last] : 0;
                bad = refs <= 0;
                split = refs > 1;
            }
            if (bad) {
                report(p.status, HOOK_ATTN_ERR_BOUNDS);
                need[s] = -1;
            } else {
                k = n > 0 ? pages_of(L + n) - pages_of(L) + (split ? 1 : 0) : 0;
                need[s] = k | (split ? kSplit : 0);
            }
        }
        int total;
        const int before = block_scan(k, sh, total);
        if (s < p.num_seqs) first[s] = wanted + before;
        wanted += total;
    }
    __syncthreads();
    // how many free pages there are
    int have = 0, sum;
    if (CLUSTER) {
        cooperative_groups::this_cluster().sync();
        (void)block_scan(units[threadIdx.x], sh, have);
    } else {
        (void)block_scan(__popc(free_pages<EACH>(p, 0)), sh, have);
    }
    // hand them out, in the order of their ids: a step's free pages as a list, then one page to a thread
    int rank = 0;
    for (int step = 0; step < steps && rank < wanted; ++step) {
        if (CLUSTER && units[step / per_unit] == 0) continue;
        const int base = step * kStep;
        uint32_t free = free_pages<EACH>(p, base);
        int i = block_scan(__popc(free), sh, sum);
        for (; free && rank + i < wanted; ++i, free &= free - 1) list[i] = (uint16_t)(threadIdx.x * EACH + __ffs(free) - 1);
        __syncthreads();
        for (i = threadIdx.x; i < sum && rank + i < wanted; i += kPoolThreads) {
            const int page = base + list[i], k = rank + i;
            int lo = 0, hi = p.num_seqs;          // the last sequence whose first place is <= k
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (first[mid] <= k) lo = mid; else hi = mid;
            }
            const int want = need[lo] & ~kSplit, j = k - first[lo];
            if (first[lo] + want > have) continue;
            const bool split = need[lo] & kSplit;
            const int L = p.seq_lens[lo];
            int32_t* row = p.block_table + (int64_t)lo * p.max_blocks + pages_of(L) - (split ? 1 : 0) + j;
            if (split && j == 0) {
                pairs[2 * lo] = *row;
                pairs[2 * lo + 1] = page;
            }
            *row = page;
            p.page_refs[page] = 1;
        }
        rank += sum;
    }
    __syncthreads();
    for (int s = threadIdx.x; s < p.num_seqs; s += kPoolThreads) {
        const int want = need[s] < 0 ? 0 : need[s] & ~kSplit;
        const bool served = need[s] >= 0 && (want == 0 || first[s] + want <= have);
        if (need[s] >= 0 && !served) report(p.status, HOOK_ATTN_ERR_NO_PAGES);
        if (served && (need[s] & kSplit)) {
            atomicSub(&p.page_refs[pairs[2 * s]], 1);
        } else {
            pairs[2 * s] = -1;
            pairs[2 * s + 1] = -1;
        }
        if (served) p.seq_lens[s] += new_rows[s];
    }
}

// The table entry of sequence s at j after a move.  In place too: an entry depends on itself alone.
template <typename Where>
__device__ __forceinline__ void remap_entry(const PoolArgs& p, int32_t* table_out, int s, int j, Where where)
{
    const int64_t at = (int64_t)s * p.max_blocks + j;
    const int L = p.seq_lens[s];
    const bool bad = L < 0 || L > capacity(p);
    int to = -1;
    if (!bad && j < pages_of(L)) {
        const int page = p.block_table[at];
        if (page_ok(p, page)) to = where(page);
        if (to < 0) report(p.status, HOOK_ATTN_ERR_BOUNDS);
    }
    if (bad) report(p.status, HOOK_ATTN_ERR_BOUNDS);
    table_out[at] = to;
}

// With U pages in use, the k-th used page at U or above moves to the k-th free page below U.  One CTA for a pool of at most one page
// a thread and small tables (700 pages: 3.4 us, and 8.1 us in three kernels).
__global__ void __launch_bounds__(kPoolThreads) compact_kernel(const PoolArgs p, int32_t* table_out, int32_t* __restrict__ refs_out, int32_t* page_map,
                                                               int32_t* __restrict__ pairs, int32_t* __restrict__ num_pairs)
{
    __shared__ int sh[33];
    const int page = threadIdx.x;
    int refs[1], used, sum;
    load_refs<1>(p, 0, refs, 0);
    (void)block_scan(refs[0] > 0, sh, used);
    const bool hole = page < used && refs[0] <= 0, source = page >= used && refs[0] > 0;
    const int k = block_scan(hole | source << 16, sh, sum), moved = sum >> 16;
    if (hole) pairs[2 * (k & 0xffff) + 1] = page;
    if (source) pairs[2 * (k >> 16)] = page;
    if (page < p.num_blocks) {
        page_map[page] = refs[0] > 0 ? page : -1;
        refs_out[page] = page < used && refs[0] > 0 ? refs[0] : 0;
    }
    __syncthreads();
    if (page < moved) {
        const int from = pairs[2 * page], to = pairs[2 * page + 1];
        page_map[from] = to;
        refs_out[to] = p.page_refs[from];
    } else if (page < p.num_blocks / 2) {
        pairs[2 * page] = -1;
        pairs[2 * page + 1] = -1;
    }
    if (page == 0) *num_pairs = moved;
    __syncthreads();
    for (int e = threadIdx.x; e < p.num_seqs * p.max_blocks; e += kPoolThreads)
        remap_entry(p, table_out, e / p.max_blocks, e % p.max_blocks, [&](int at) { return page_map[at]; });
}

// The same for larger pools and tables, in three kernels with a CTA for every kSegment pages: how many of them are used (the counts lie in refs_out,
// which is written last); the plan; what follows from all pairs.  Between the last two page_map names a moving page's pair, and a free
// page's that is moved to, as -2 - pair.  4096 pages: 8.5 to 9.7 us, and 9.1 to 9.5 us with one CTA; 100000 pages: 9 to 10 us, and 140 to
// 173 us with one CTA.
constexpr int kSegment = 4 * kPoolThreads;

__global__ void __launch_bounds__(kPoolThreads) count_used_kernel(const PoolArgs p, int32_t* __restrict__ counts)
{
    asm volatile("griddepcontrol.launch_dependents;");
    __shared__ int sh[33];
    int refs[4], n = 0, sum;
    load_refs<4>(p, blockIdx.x * kSegment, refs, 0);
#pragma unroll
    for (int u = 0; u < 4; ++u) n += refs[u] > 0;
    (void)block_scan(n, sh, sum);
    if (threadIdx.x == 0) counts[blockIdx.x] = sum;
}

__global__ void __launch_bounds__(kPoolThreads) plan_kernel(const PoolArgs p, const int32_t* counts, int32_t* __restrict__ page_map,
                                                            int32_t* __restrict__ pairs, int32_t* __restrict__ num_pairs)
{
    asm volatile("griddepcontrol.launch_dependents;");
    __shared__ int sh[33];
    const int segments = gridDim.x, start = blockIdx.x * kSegment, first = start + (int)threadIdx.x * 4;
    int refs[4], n = 0, part = 0, used, before, low = 0;
    load_refs<4>(p, start, refs, 0);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int s = threadIdx.x; s < segments; s += kPoolThreads) {
        const int c = counts[s];
        n += c;
        part += s < (int)blockIdx.x ? c : 0;
    }
    (void)block_scan(n, sh, used);
    (void)block_scan(part, sh, before);           // used pages before this segment
    if (start + kSegment >= used) {               // used pages below `used`: they stay
        const int edge = used / kSegment;
        int there[4];
        load_refs<4>(p, edge * kSegment, there, 0);
        n = 0;
        for (int s = threadIdx.x; s < edge; s += kPoolThreads) n += counts[s];
#pragma unroll
        for (int u = 0; u < 4; ++u) n += there[u] > 0 && edge * kSegment + (int)threadIdx.x * 4 + u < used;
        (void)block_scan(n, sh, low);
        if (threadIdx.x == 0 && (int)blockIdx.x == segments - 1) *num_pairs = used - low;
    }
    int both = 0, sum;                            // free pages below `used`, and 2^16 for each used page from there on
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        both += first + u < used && refs[u] <= 0;
        both += (first + u >= used && refs[u] > 0) << 16;
    }
    both = block_scan(both, sh, sum);
    int k = start - before + (both & 0xffff), l = (start > used ? before - low : 0) + (both >> 16);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int page = first + u;
        if (page >= p.num_blocks) break;
        int to = refs[u] > 0 ? page : -1;
        if (page < used && refs[u] <= 0) {
            to = -2 - k;
            pairs[2 * k++ + 1] = page;
        }
        if (page >= used && refs[u] > 0) {
            to = -2 - l;
            pairs[2 * l++] = page;
        }
        page_map[page] = to;
    }
}

__global__ void __launch_bounds__(kListThreads) finish_kernel(const PoolArgs p, int32_t* table_out, int32_t* __restrict__ refs_out, int32_t* page_map,
                                                              int32_t* pairs, const int32_t* __restrict__ num_pairs)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t step = (int64_t)gridDim.x * kListThreads, me = (int64_t)blockIdx.x * kListThreads + threadIdx.x;
    for (int64_t page = me; page < p.num_blocks; page += step) {
        const int t = page_map[page], r = p.page_refs[page];
        int refs = max(r, 0);
        if (t <= -2) {
            const int32_t* pair = pairs + 2 * (-2 - t);
            refs = r > 0 ? 0 : p.page_refs[pair[0]];
            page_map[page] = r > 0 ? pair[1] : -1;
        }
        refs_out[page] = refs;
    }
    for (int64_t k = *num_pairs + me; k < p.num_blocks / 2; k += step) pairs[2 * k] = pairs[2 * k + 1] = -1;
    // What another thread makes of a page's entry in the meantime is what is made of it here.
    for (int64_t e = me; e < (int64_t)p.num_seqs * p.max_blocks; e += step)
        remap_entry(p, table_out, (int)(e / p.max_blocks), (int)(e % p.max_blocks), [&](int page) {
            const int t = __ldcg(page_map + page);
            return t > -2 ? t : p.page_refs[page] > 0 ? pairs[2 * (-2 - t) + 1] : -1;
        });
}

// A unit is a page of one slab (the keys or the values of a layer), and from kMany pairs on eight pages of four slabs, since the pairs of
// a unit are held against all others: they must not depend on one another, and one whose destination is the destination or the source of
// another pair, or whose source is a destination, is not carried out.  How many pairs there are is known on the device alone, so a
// fixed number of CTAs goes through the units, slab after slab (page after page, all slabs of each: 62 -> 69 us for 256 pairs in 32
// slabs).  32 CTAs for an SM: with one for each unit that there could be, 20 of 2048 pairs in 32 slabs take 36 us, with 64 10 us, with
// 32 7 us; all 2048 take 1 % longer than with 64.  Bound by HBM (983 pages of 16 layers, 2.1 GB read and written: 320 us, the copy rate).
//
// The check's time grows with the square of the list, whose length the host does not know: lists of more than kMostPairs pairs are refused.
// From kLong on there are units enough for all CTAs when each has all slabs, so that its pairs are checked once (2 KB pages: 2^18 pairs 30 ms, of which
// the copies of a layer take 0.3; 2^20 pairs 0.5 s, 2^22 pairs 7.5 s).
constexpr int kChecked = 8;                      // pairs of a unit at most
constexpr int kMany = 2048;
constexpr int kLong = 1 << 16;
constexpr int kMostPairs = 1 << 22;
constexpr int kCopyCtas = 32;

// TIGHT: a page's tokens and heads follow one another without gaps, in either order.  CHECKED: 1 for lists that cannot be long (the
// registers of eight leave room for fewer CTAs on an SM: 256 pairs of (-1, -1) in 32 slabs 7.7 us, and 14 us).
template <bool TIGHT, int CHECKED>
__global__ void __launch_bounds__(kListThreads, CHECKED == 1 ? 6 : 4) copy_pages_kernel(const __grid_constant__ CopyArgs a)
{
    __shared__ uint32_t refused;
    const int n = a.num_pairs ? min(max(*a.num_pairs, 0), a.max_pairs) : a.max_pairs, slabs = 2 * a.layers;
    if (n == 0) return;
    if (CHECKED > 1 && n > kMostPairs) {
        if (blockIdx.x == 0 && threadIdx.x == 0) report(a.status, HOOK_ATTN_ERR_BOUNDS);
        return;
    }
    const bool many = CHECKED > 1 && n > kMany;
    const uint32_t pairs = many ? CHECKED : 1, some = !many ? 1 : n > kLong ? slabs : min(slabs, 4);              // of a unit
    const uint32_t groups = ((uint32_t)n + pairs - 1) / pairs, rows = (slabs + some - 1) / some;
    const uint32_t next_group = gridDim.x % groups, next_row = gridDim.x / groups;
    const int per_row = a.head_dim / 8, pieces = kPage * a.Hkv * per_row;
    auto place = [&](int e) {
        if (TIGHT) return (int64_t)e * 8;
        const int c = e % per_row, h = e / per_row % a.Hkv, t = e / per_row / a.Hkv;
        return (int64_t)t * a.ts + (int64_t)h * a.hs + c * 8;
    };
    uint32_t group = blockIdx.x % groups;
    for (uint32_t row = blockIdx.x / groups; row < rows;) {
        const int p0 = (int)(group * pairs), count = min((int)pairs, n - p0), slab0 = (int)(row * some), slab1 = min(slab0 + (int)some, slabs);
        row += next_row;
        group += next_group;
        if (group >= groups) {
            group -= groups;
            ++row;
        }
        int src[CHECKED], dst[CHECKED];
        bool live = false;
#pragma unroll
        for (int q = 0; q < CHECKED; ++q) {
            src[q] = q < count ? a.pairs[2 * (p0 + q)] : -1;
            dst[q] = q < count ? a.pairs[2 * (p0 + q) + 1] : -1;
            if (src[q] < 0 || dst[q] < 0) src[q] = dst[q] = -1;
            live |= src[q] >= 0;
        }
        if (!live) continue;
        __syncthreads();                          // the unit before is done with it
        if (threadIdx.x == 0) refused = 0;
        __syncthreads();
        uint32_t bad = 0;
        for (int j = threadIdx.x; j < n; j += kListThreads) {
            const int s = a.pairs[2 * j], d = a.pairs[2 * j + 1];
            if (s < 0 || d < 0) continue;
#pragma unroll
            for (int q = 0; q < CHECKED; ++q)
                if (j != p0 + q && (d == dst[q] || s == dst[q] || d == src[q])) bad |= 1u << q;
        }
        if (bad) atomicOr(&refused, bad);
        __syncthreads();
#pragma unroll
        for (int q = 0; q < CHECKED; ++q) {
            const int s = src[q], d = dst[q];
            if (s == d) continue;
            if ((refused >> q & 1) || s >= a.num_blocks || d >= a.num_blocks) {
                if (threadIdx.x == 0) report(a.status, HOOK_ATTN_ERR_BOUNDS);
                continue;
            }
            for (int slab = slab0; slab < slab1; ++slab) {
                __nv_bfloat16* base = slab & 1 ? a.v[slab >> 1] : a.k[slab >> 1];
                const __nv_bfloat16* in = base + (int64_t)s * a.bs;
                __nv_bfloat16* out = base + (int64_t)d * a.bs;
                for (int e0 = threadIdx.x; e0 < pieces; e0 += 4 * kListThreads) {
                    uint4 held[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (e0 + u * kListThreads < pieces) held[u] = *reinterpret_cast<const uint4*>(in + place(e0 + u * kListThreads));
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (e0 + u * kListThreads < pieces) *reinterpret_cast<uint4*>(out + place(e0 + u * kListThreads)) = held[u];
                }
            }
        }
    }
}

}  // namespace

static size_t extend_bytes(int num_seqs, int each) { return 2 * (size_t)num_seqs * 4 + (size_t)each * kPoolThreads * 2; }

cudaError_t configure_cache_pages()
{
    const auto allow = [](auto* kernel, int each) {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)extend_bytes(kMaxPoolSeqs, each));
    };
    cudaError_t e = allow(extend_kernel<1, false>, 1);
    if (e == cudaSuccess) e = allow(extend_kernel<4, false>, 4);
    if (e == cudaSuccess) e = allow(extend_kernel<16, false>, 16);
    if (e == cudaSuccess) e = allow(extend_kernel<16, true>, 16);
    return e;
}

cudaError_t launch_fork(const PoolArgs& p, const int32_t* parents, const int32_t* children, int n, cudaStream_t st)
{
    fork_kernel<<<n, kListThreads, 0, st>>>(p, parents, children, n);
    return cudaGetLastError();
}

cudaError_t launch_free(const PoolArgs& p, const int32_t* seqs, const int32_t* keep_lens, int n, cudaStream_t st)
{
    free_kernel<<<n, kListThreads, 0, st>>>(p, seqs, keep_lens);
    return cudaGetLastError();
}

template <int EACH>
static cudaError_t extend(const PoolArgs& p, const int32_t* new_rows, int32_t* pairs, cudaStream_t st)
{
    extend_kernel<EACH, false><<<1, kPoolThreads, extend_bytes(p.num_seqs, EACH), st>>>(p, new_rows, pairs);
    return cudaGetLastError();
}

cudaError_t launch_extend(const PoolArgs& p, const int32_t* new_rows, int32_t* pairs, cudaStream_t st)
{
    if (p.num_blocks <= kPoolThreads) return extend<1>(p, new_rows, pairs, st);
    if (p.num_blocks <= 4 * kPoolThreads) return extend<4>(p, new_rows, pairs, st);
    if (p.num_blocks <= 16 * kPoolThreads) return extend<16>(p, new_rows, pairs, st);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kClusterCtas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kClusterCtas);
    cfg.blockDim = dim3(kPoolThreads);
    cfg.dynamicSmemBytes = extend_bytes(p.num_seqs, 16);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, extend_kernel<16, true>, p, new_rows, pairs);
}

// A kernel that may start while the one before it in the stream runs, and waits for it itself.
template <typename... P, typename... A>
static cudaError_t launch_after(void (*kernel)(P...), int grid, int threads, cudaStream_t st, A... args)
{
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

cudaError_t launch_compact(const PoolArgs& p, int32_t* table_out, int32_t* refs_out, int32_t* page_map, int32_t* pairs,
                           int32_t* num_pairs, cudaStream_t st)
{
    const int64_t entries = (int64_t)p.num_seqs * p.max_blocks;
    if (p.num_blocks == 0 || (p.num_blocks <= kPoolThreads && entries <= 16 * kPoolThreads)) {
        compact_kernel<<<1, kPoolThreads, 0, st>>>(p, table_out, refs_out, page_map, pairs, num_pairs);
        return cudaGetLastError();
    }
    const int segments = (p.num_blocks + kSegment - 1) / kSegment;
    const int64_t blocks = ((entries > p.num_blocks ? entries : p.num_blocks) + kListThreads - 1) / kListThreads;
    count_used_kernel<<<segments, kPoolThreads, 0, st>>>(p, refs_out);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) e = launch_after(plan_kernel, segments, kPoolThreads, st, p, refs_out, page_map, pairs, num_pairs);
    if (e == cudaSuccess)
        e = launch_after(finish_kernel, (int)(blocks < 4096 ? blocks : 4096), kListThreads, st, p, table_out, refs_out, page_map, pairs, num_pairs);
    return e;
}

cudaError_t launch_copy_pages(const CopyArgs& a, int num_sms, cudaStream_t st)
{
    const int64_t units = (int64_t)a.max_pairs * 2 * a.layers, most = (int64_t)num_sms * kCopyCtas;
    const int grid = (int)(units < most ? units : most);
    const bool tight = (a.hs == a.head_dim && a.ts == (int64_t)a.Hkv * a.head_dim) || (a.ts == a.head_dim && a.hs == (int64_t)kPage * a.head_dim);
    const bool few = a.max_pairs <= kMany;
    const auto kernel = tight ? (few ? copy_pages_kernel<true, 1> : copy_pages_kernel<true, kChecked>)
                              : (few ? copy_pages_kernel<false, 1> : copy_pages_kernel<false, kChecked>);
    kernel<<<grid, kListThreads, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace hook_attn

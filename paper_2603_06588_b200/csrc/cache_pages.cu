// The pages of the cache: sequences that share pages (fork), get room for new rows (extend), give pages back (free), and a
// pool whose pages are moved together at its low end (compact).  A page's entry in page_refs counts the sequences that hold
// it; 0 is free.  All results are integers that do not depend on the order in which threads run.
#include "common.cuh"
#include "ops.cuh"

namespace hook_attn {

namespace {

constexpr int kListThreads = 256;
constexpr int kPoolThreads = 1024;

__device__ __forceinline__ int pages_of(int len) { return (int)(((int64_t)len + kPage - 1) / kPage); }
__device__ __forceinline__ int64_t capacity(const PoolArgs& p) { return min((int64_t)p.max_blocks * kPage, (int64_t)INT32_MAX); }
__device__ __forceinline__ bool page_ok(const PoolArgs& p, int page) { return page >= 0 && page < p.num_blocks; }

// A CTA passes over the pool's reference counts in steps of EACH neighbouring pages to a thread: 1, 4 or 16, the fewest that cover the
// pool in one step (700 pages in one step of 1: a compaction takes 4 us less than with 16), else 16 (100000 pages: seven steps).
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
    for (int u = 0; u < EACH; ++u) bits |= (uint32_t)(refs[u] == 0) << u;
    return bits;
}

// One CTA per entry: children[i] gets the pages of parents[i].  An entry is refused (status) when a row is out of range, the
// child holds pages, the child is listed earlier, the child is a parent of the same call, or the parent's row is broken.
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
    for (int j = threadIdx.x; j < pages; j += kListThreads) bad |= !page_ok(p, from[j]);
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
constexpr int kSplit = 1 << 30;                   // flag in a need: the last page is shared

template <int EACH>
__global__ void __launch_bounds__(kPoolThreads) extend_kernel(const PoolArgs p, const int32_t* __restrict__ new_rows,
                                                              int32_t* __restrict__ pairs)
{
    extern __shared__ int32_t dyn[];
    int32_t* need = dyn;                          // [num_seqs] pages, with kSplit; -1: the sequence is left out
    int32_t* first = dyn + p.num_seqs;            // [num_seqs] place of its first page among all needs
    __shared__ int sh[33];
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
    // how many of the wanted pages there are
    int have = 0, sum;
    for (int base = 0; base < p.num_blocks && have < wanted; base += kPoolThreads * EACH) {
        (void)block_scan(__popc(free_pages<EACH>(p, base)), sh, sum);
        have += sum;
    }
    // hand them out, in the order of their ids
    int rank = 0;
    for (int base = 0; base < p.num_blocks && rank < wanted; base += kPoolThreads * EACH) {
        uint32_t free = free_pages<EACH>(p, base);
        int k = rank + block_scan(__popc(free), sh, sum);
        rank += sum;
        for (; free && k < wanted; ++k, free &= free - 1) {
            const int page = base + (int)threadIdx.x * EACH + __ffs(free) - 1;
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
__device__ __forceinline__ void remap_entry(const PoolArgs& p, const int32_t* page_map, int32_t* table_out, int s, int j)
{
    const int64_t at = (int64_t)s * p.max_blocks + j;
    const int L = p.seq_lens[s];
    const bool bad = L < 0 || L > capacity(p);
    int to = -1;
    if (!bad && j < pages_of(L)) {
        const int page = p.block_table[at];
        if (page_ok(p, page)) to = page_map[page];
        if (to < 0) report(p.status, HOOK_ATTN_ERR_BOUNDS);
    }
    if (bad) report(p.status, HOOK_ATTN_ERR_BOUNDS);
    table_out[at] = to;
}

// The tables of a large pool, one CTA per sequence.
__global__ void __launch_bounds__(kListThreads) remap_kernel(const PoolArgs p, const int32_t* page_map, int32_t* table_out)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");       // launched while the map is being made
    for (int j = threadIdx.x; j < p.max_blocks; j += kListThreads) remap_entry(p, page_map, table_out, blockIdx.x, j);
}

// With U pages in use, the k-th used page at U or above moves to the k-th free page below U.  table_out: null where the tables are
// left to remap_kernel.
template <int EACH>
__global__ void __launch_bounds__(kPoolThreads) compact_kernel(const PoolArgs p, int32_t* table_out, int32_t* __restrict__ refs_out, int32_t* page_map,
                                                               int32_t* __restrict__ pairs, int32_t* __restrict__ num_pairs)
{
    if (!table_out) asm volatile("griddepcontrol.launch_dependents;");
    __shared__ int sh[33];
    int used = 0, sum;
    for (int base = 0; base < p.num_blocks; base += kPoolThreads * EACH) {
        int refs[EACH], n = 0;
        load_refs<EACH>(p, base, refs, 0);
#pragma unroll
        for (int u = 0; u < EACH; ++u) n += refs[u] > 0;
        (void)block_scan(n, sh, sum);
        used += sum;
    }
    int sources = 0, holes = 0;
    for (int base = 0; base < p.num_blocks; base += kPoolThreads * EACH) {
        int refs[EACH], from = 0, to = 0;
        load_refs<EACH>(p, base, refs, 0);
        const int first = base + (int)threadIdx.x * EACH;
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            to += first + u < used && refs[u] <= 0;
            from += first + u >= used && refs[u] > 0;
        }
        int k = holes + block_scan(to, sh, sum);
        holes += sum;
        int l = sources + block_scan(from, sh, sum);
        sources += sum;
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            const int page = first + u;
            if (page >= p.num_blocks) break;
            if (page < used && refs[u] <= 0) pairs[2 * k++ + 1] = page;
            if (page >= used && refs[u] > 0) pairs[2 * l++] = page;
            page_map[page] = refs[u] > 0 ? page : -1;
            refs_out[page] = page < used && refs[u] > 0 ? refs[u] : 0;
        }
    }
    __syncthreads();
    for (int k = threadIdx.x; k < p.num_blocks / 2; k += kPoolThreads) {
        if (k < sources) {
            const int from = pairs[2 * k], to = pairs[2 * k + 1];
            page_map[from] = to;
            refs_out[to] = p.page_refs[from];
        } else {
            pairs[2 * k] = -1;
            pairs[2 * k + 1] = -1;
        }
    }
    if (threadIdx.x == 0) *num_pairs = sources;
    if (!table_out) return;
    __syncthreads();
    for (int e = threadIdx.x; e < p.num_seqs * p.max_blocks; e += kPoolThreads) remap_entry(p, page_map, table_out, e / p.max_blocks, e % p.max_blocks);
}

// A CTA copies `pairs` pages in `slabs` of the caches (keys or values of a layer).  Pairs must not depend on one another: one whose
// destination is the destination or the source of another pair, or whose source is a destination, is not carried out, and a CTA looks
// through all pairs to see that.  Bound by HBM (983 pages of 16 layers, 2.1 GB read and written: 334 us, 6.2 TB/s; equal shares for a
// grid that is resident at once: 362 us).
constexpr int kChecked = 8;                      // pairs of a CTA at most

// TIGHT: a page's tokens and heads follow one another without gaps, in either order.
template <bool TIGHT>
__global__ void __launch_bounds__(kListThreads) copy_pages_kernel(const __grid_constant__ CopyArgs a, int pairs, int slabs)
{
    __shared__ uint32_t refused;
    const int n = a.num_pairs ? min(max(*a.num_pairs, 0), a.max_pairs) : a.max_pairs;
    const int p0 = blockIdx.x * pairs, count = min(pairs, n - p0), slab0 = blockIdx.y * slabs, slab1 = min(slab0 + slabs, 2 * a.layers);
    if (count <= 0) return;
    int src[kChecked], dst[kChecked];
#pragma unroll
    for (int q = 0; q < kChecked; ++q) {
        src[q] = q < count ? a.pairs[2 * (p0 + q)] : -1;
        dst[q] = q < count ? a.pairs[2 * (p0 + q) + 1] : -1;
        if (src[q] < 0 || dst[q] < 0) src[q] = dst[q] = -1;
    }
    if (threadIdx.x == 0) refused = 0;
    __syncthreads();
    uint32_t bad = 0;
    for (int j = threadIdx.x; j < n; j += kListThreads) {
        const int s = a.pairs[2 * j], d = a.pairs[2 * j + 1];
        if (s < 0 || d < 0) continue;
#pragma unroll
        for (int q = 0; q < kChecked; ++q)
            if (j != p0 + q && (d == dst[q] || s == dst[q] || d == src[q])) bad |= 1u << q;
    }
    if (bad) atomicOr(&refused, bad);
    __syncthreads();
    const int per_row = a.head_dim / 8, pieces = kPage * a.Hkv * per_row;
    auto place = [&](int e) {
        if (TIGHT) return (int64_t)e * 8;
        const int c = e % per_row, h = e / per_row % a.Hkv, t = e / per_row / a.Hkv;
        return (int64_t)t * a.ts + (int64_t)h * a.hs + c * 8;
    };
#pragma unroll
    for (int q = 0; q < kChecked; ++q) {
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

}  // namespace

cudaError_t configure_cache_pages()
{
    cudaError_t e = cudaFuncSetAttribute(extend_kernel<1>, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * kMaxPoolSeqs * 4);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(extend_kernel<4>, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * kMaxPoolSeqs * 4);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(extend_kernel<16>, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * kMaxPoolSeqs * 4);
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

cudaError_t launch_extend(const PoolArgs& p, const int32_t* new_rows, int32_t* pairs, cudaStream_t st)
{
    if (p.num_blocks <= kPoolThreads) extend_kernel<1><<<1, kPoolThreads, 2 * p.num_seqs * 4, st>>>(p, new_rows, pairs);
    else if (p.num_blocks <= 4 * kPoolThreads) extend_kernel<4><<<1, kPoolThreads, 2 * p.num_seqs * 4, st>>>(p, new_rows, pairs);
    else extend_kernel<16><<<1, kPoolThreads, 2 * p.num_seqs * 4, st>>>(p, new_rows, pairs);
    return cudaGetLastError();
}

cudaError_t launch_compact(const PoolArgs& p, int32_t* table_out, int32_t* refs_out, int32_t* page_map, int32_t* pairs,
                           int32_t* num_pairs, cudaStream_t st)
{
    // A second kernel for the tables pays from some 16 entries a thread on (48 x 29 entries: 4 us more).
    const bool small = (int64_t)p.num_seqs * p.max_blocks <= 16 * kPoolThreads;
    int32_t* here = small ? table_out : nullptr;
    if (p.num_blocks <= kPoolThreads) compact_kernel<1><<<1, kPoolThreads, 0, st>>>(p, here, refs_out, page_map, pairs, num_pairs);
    else if (p.num_blocks <= 4 * kPoolThreads) compact_kernel<4><<<1, kPoolThreads, 0, st>>>(p, here, refs_out, page_map, pairs, num_pairs);
    else compact_kernel<16><<<1, kPoolThreads, 0, st>>>(p, here, refs_out, page_map, pairs, num_pairs);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || small) return e;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.num_seqs);
    cfg.blockDim = dim3(kListThreads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, remap_kernel, p, static_cast<const int32_t*>(page_map), table_out);
}

cudaError_t launch_copy_pages(const CopyArgs& a, cudaStream_t st)
{
    // A CTA for every slab of every pair; with many pairs, which each CTA has to look through, several of both for a CTA.
    const bool many = a.max_pairs > 2048;
    const int pairs = many ? kChecked : 1, slabs = many ? (2 * a.layers < 4 ? 2 * a.layers : 4) : 1;
    const dim3 grid((a.max_pairs + pairs - 1) / pairs, (2 * a.layers + slabs - 1) / slabs);
    const bool tight = (a.hs == a.head_dim && a.ts == (int64_t)a.Hkv * a.head_dim) || (a.ts == a.head_dim && a.hs == (int64_t)kPage * a.head_dim);
    if (tight) copy_pages_kernel<true><<<grid, kListThreads, 0, st>>>(a, pairs, slabs);
    else copy_pages_kernel<false><<<grid, kListThreads, 0, st>>>(a, pairs, slabs);
    return cudaGetLastError();
}

}  // namespace hook_attn

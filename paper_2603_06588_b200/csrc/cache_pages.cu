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
__device__ __forceinline__ int64_t capacity(const PoolArgs& p) { return (int64_t)p.max_blocks * kPage; }
__device__ __forceinline__ bool page_ok(const PoolArgs& p, int page) { return page >= 0 && page < p.num_blocks; }

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
    int have = 0;
    for (int base = 0; base < p.num_blocks && have < wanted; base += kPoolThreads) {
        const int page = base + (int)threadIdx.x;
        have += __syncthreads_count(page < p.num_blocks && p.page_refs[page] == 0);
    }
    // hand them out
    int rank = 0;
    for (int base = 0; base < p.num_blocks && rank < wanted; base += kPoolThreads) {
        const int page = base + (int)threadIdx.x;
        const bool is_free = page < p.num_blocks && p.page_refs[page] == 0;
        int total;
        const int k = rank + block_scan(is_free, sh, total);
        rank += total;
        if (!is_free || k >= wanted) continue;
        int lo = 0, hi = p.num_seqs;              // the last sequence whose first place is <= k
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

// With U pages in use, the k-th used page at U or above moves to the k-th free page below U.
__global__ void __launch_bounds__(kPoolThreads) compact_kernel(const PoolArgs p, int32_t* __restrict__ table_out,
                                                               int32_t* __restrict__ refs_out, int32_t* __restrict__ page_map,
                                                               int32_t* __restrict__ pairs, int32_t* __restrict__ num_pairs)
{
    __shared__ int sh[33];
    int used = 0;
    for (int base = 0; base < p.num_blocks; base += kPoolThreads) {
        const int page = base + (int)threadIdx.x;
        used += __syncthreads_count(page < p.num_blocks && p.page_refs[page] > 0);
    }
    int sources = 0, holes = 0;
    for (int base = 0; base < p.num_blocks; base += kPoolThreads) {
        const int page = base + (int)threadIdx.x;
        const int refs = page < p.num_blocks ? p.page_refs[page] : 0;
        const bool hole = page < used && refs <= 0, source = page >= used && refs > 0;
        int total;
        int k = block_scan(hole, sh, total);
        if (hole) pairs[2 * (holes + k) + 1] = page;
        holes += total;
        k = block_scan(source, sh, total);
        if (source) pairs[2 * (sources + k)] = page;
        sources += total;
        if (page < p.num_blocks) {
            page_map[page] = refs > 0 ? page : -1;
            refs_out[page] = page < used && refs > 0 ? refs : 0;
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
    __syncthreads();
    const int64_t entries = (int64_t)p.num_seqs * p.max_blocks;
    for (int64_t e = threadIdx.x; e < entries; e += kPoolThreads) {
        const int s = (int)(e / p.max_blocks), j = (int)(e % p.max_blocks), L = p.seq_lens[s];
        int to = -1;
        if (L < 0 || L > capacity(p)) {
            report(p.status, HOOK_ATTN_ERR_BOUNDS);
        } else if (j < pages_of(L)) {
            const int page = p.block_table[e];
            if (page_ok(p, page)) to = page_map[page];
            if (to < 0) report(p.status, HOOK_ATTN_ERR_BOUNDS);
        }
        table_out[e] = to;
    }
}

// A CTA copies one page of one layer's keys or values.  Pairs must not depend on one another: one whose destination is the
// destination or the source of another pair, or whose source is a destination, is not carried out.
__global__ void __launch_bounds__(kListThreads) copy_pages_kernel(const __grid_constant__ CopyArgs a)
{
    const int i = blockIdx.x, n = a.num_pairs ? min(max(*a.num_pairs, 0), a.max_pairs) : a.max_pairs;
    if (i >= n) return;
    const int src = a.pairs[2 * i], dst = a.pairs[2 * i + 1];
    if (src < 0 || dst < 0 || src == dst) return;
    bool bad = src >= a.num_blocks || dst >= a.num_blocks;
    for (int j = threadIdx.x; j < n; j += kListThreads) {
        const int s = a.pairs[2 * j], d = a.pairs[2 * j + 1];
        if (j != i && s >= 0 && d >= 0) bad |= d == dst || s == dst || d == src;
    }
    if (__syncthreads_or(bad)) {
        if (threadIdx.x == 0) report(a.status, HOOK_ATTN_ERR_BOUNDS);
        return;
    }
    __nv_bfloat16* base = blockIdx.y & 1 ? a.v[blockIdx.y >> 1] : a.k[blockIdx.y >> 1];
    const int per_row = a.head_dim / 8, total = kPage * a.Hkv * per_row;
    for (int e = threadIdx.x; e < total; e += kListThreads) {
        const int c = e % per_row, h = e / per_row % a.Hkv, t = e / per_row / a.Hkv;
        const int64_t at = (int64_t)t * a.ts + (int64_t)h * a.hs + c * 8;
        *reinterpret_cast<uint4*>(base + (int64_t)dst * a.bs + at) = *reinterpret_cast<const uint4*>(base + (int64_t)src * a.bs + at);
    }
}

}  // namespace

cudaError_t configure_cache_pages()
{
    return cudaFuncSetAttribute(extend_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * kMaxPoolSeqs * 4);
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
    extend_kernel<<<1, kPoolThreads, 2 * p.num_seqs * 4, st>>>(p, new_rows, pairs);
    return cudaGetLastError();
}

cudaError_t launch_compact(const PoolArgs& p, int32_t* table_out, int32_t* refs_out, int32_t* page_map, int32_t* pairs,
                           int32_t* num_pairs, cudaStream_t st)
{
    compact_kernel<<<1, kPoolThreads, 0, st>>>(p, table_out, refs_out, page_map, pairs, num_pairs);
    return cudaGetLastError();
}

cudaError_t launch_copy_pages(const CopyArgs& a, cudaStream_t st)
{
    copy_pages_kernel<<<dim3(a.max_pairs, 2 * a.layers), kListThreads, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace hook_attn

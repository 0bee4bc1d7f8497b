// Launch-parameter structs of the operators around the attention: rotary append, logit edits, cache pages.
#pragma once

#include "common.cuh"

namespace hook_attn {

constexpr int kMaxPairs = 64;          // rotated pairs per head: half of the largest head_dim
constexpr int kMaxVocab = 1 << 20;     // entries per row of logits
constexpr int kMaxHistory = (1 << 20) - 1;   // tokens of a row's history
constexpr int kMaxRowBias = 2047;      // bias entries of a row
constexpr int kMaxPoolSeqs = 16384;    // sequences of a page pool
constexpr int kCopyLayers = 64;        // layers per launch of the page copy

struct RopeArgs {
    const void *q, *k, *v;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;   // strides in elements
    __nv_bfloat16 *q_out, *k_cache, *v_cache;
    int64_t bs, ts, hs;
    const int32_t *block_table, *seq_lens, *cu_q_lens, *positions;
    const float* inv_freq;
    int64_t axis_stride;
    int32_t* status;
    int32_t num_seqs, total_q, Hq, Hkv, head_dim, pairs, num_blocks, max_blocks, max_keys;
    int32_t rows_per_cta;
    float factor;
    bool halves;
    uint8_t axis_of_pair[kMaxPairs];
};

struct LogitsArgs {
    const void* logits;
    void* out;
    int64_t in_row, out_row, token_row, mask_row;          // row strides in elements (mask: in 32-bit words)
    const int32_t *tokens, *prompt_lens, *total_lens;
    const float *repetition, *presence, *frequency;
    const int32_t *bias_offsets, *bias_tokens;
    const float* bias_values;
    const uint32_t* mask;
    const int32_t* mask_rows;
    int32_t* status;
    int32_t rows, vocab, max_tokens, num_bias, num_masks;
};

struct PoolArgs {
    int32_t *block_table, *seq_lens, *page_refs, *status;
    int32_t num_seqs, max_blocks, num_blocks;
};

struct CopyArgs {
    __nv_bfloat16* k[kCopyLayers];
    __nv_bfloat16* v[kCopyLayers];
    int64_t bs, ts, hs;
    const int32_t *pairs, *num_pairs;
    int32_t* status;
    int32_t slabs;                         // arrays whose pages are copied: k[0], v[0], k[1], ...
    int32_t tokens, num_blocks, Hkv, head_dim, max_pairs;   // a page: tokens x Hkv rows of head_dim elements
};

struct Q4ReadArgs {
    const uint8_t* pages;
    int64_t page_block, page_head;         // strides in bytes
    __nv_bfloat16 *k_cache, *v_cache;
    int64_t bs, ts, hs;                    // strides in elements
    const int32_t *block_table, *seq_lens, *first, *to_table;
    int32_t* status;
    int32_t num_seqs, Hkv, num_blocks, max_blocks, max_keys, to_num_blocks, to_max_blocks;
};

struct SampleArgs {
    const void* logits;
    int64_t row;                           // in elements
    const float *uniform, *temperature, *top_p, *min_p;
    const int32_t* top_k;
    int32_t *tokens, *status;
    int32_t rows, vocab, slice;            // slice: tokens of a row that one CTA holds
};

// Exclusive prefix sum over the CTA; `total` is the sum.  `sh` holds 33 ints.
__device__ __forceinline__ int block_scan(int x, int* sh, int& total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    __syncthreads();                              // sh may still be read from the scan before
    if (lane == 31) sh[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        int w = lane < (int)(blockDim.x >> 5) ? sh[lane] : 0, wi = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, wi, o);
            if (lane >= o) wi += y;
        }
        sh[lane] = wi - w;
        if (lane == 31) sh[32] = wi;
    }
    __syncthreads();
    total = sh[32];
    return sh[warp] + incl - x;
}

}  // namespace hook_attn

// The paged key / value cache and the rows of a step as the kernels see them (paged.hip, tree.hip, logits.hip).
#pragma once

#include "common.h"

namespace atts {

struct PagedView {
    const int32_t* table;        // [n_seqs, max_pages]
    int32_t n_pages, page_log, n_kv, hd, n_seqs, max_pages;

    __device__ int slots() const { return max_pages << page_log; }                 // tokens a sequence can hold (checked to fit 31 bits)
    __device__ int page_of(int seq, int token) const { return table[(int64_t)seq * max_pages + (token >> page_log)]; }
    // element offsets of token `token` in page `page`: its key row, and the first element of its value column (then one per page_rows)
    __device__ int64_t key_at(int page, int head, int token) const {
        return ((((int64_t)page * n_kv + head) << page_log) + (token & ((1 << page_log) - 1))) * hd;
    }
    __device__ int64_t value_at(int page, int head, int token) const {
        return (((int64_t)page * n_kv + head) * hd << page_log) + (token & ((1 << page_log) - 1));
    }
};

// The sequence that owns row r: the last one whose rows begin at or before it, -1 if r lies outside all of them.
__device__ __forceinline__ int sequence_of(const int32_t* __restrict__ row_offsets, int n_seqs, int r) {
    int lo = 0, hi = n_seqs;                        // row_offsets[lo] <= r < row_offsets[hi]
    if (n_seqs < 1 || r < row_offsets[0] || r >= row_offsets[n_seqs]) return -1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (row_offsets[mid] <= r) lo = mid; else hi = mid;
    }
    return lo;
}

// The same by a whole wavefront, 64 sequences a step: a search by halves waits for memory at every one of its steps.
__device__ __forceinline__ int sequence_of_wave(const int32_t* __restrict__ row_offsets, int n_seqs, int r, int lane) {
    if (n_seqs < 1) return -1;
    int lo = 0, hi = n_seqs + 1;                    // the answer is the last index in [lo, hi) whose offset is at most r
    bool none = false;
    while (hi - lo > 1 || lo == 0) {
        const int step = (hi - lo + 63) >> 6, at = lo + lane * step;
        const int below = __popcll(__ballot(at < hi && row_offsets[at] <= r));
        if (below == 0) { none = true; break; }
        lo += (below - 1) * step;
        hi = min(lo + step, hi);
        if (step == 1) break;
    }
    return none || lo >= n_seqs ? -1 : lo;
}

// ATTS_OK, or the error of a cache that no kernel can read; *view is filled in.
int32_t check_paged(const char* fn, const atts_paged_cache* cache, PagedView* view);

}  // namespace atts

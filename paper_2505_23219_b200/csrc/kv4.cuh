// Device view of a paged 4-bit cache, shared by its kernels.
#pragma once

#include "internal.h"
#include "kv4_layout.h"

namespace ghd {

struct Kv4View {
    const int32_t* table;
    const int32_t* kv_len;
    const int32_t* row_start;
    int n_seqs, n_pages, shift, max_pages, n_rows, heads, d_head;      // page_rows = 1 << shift; heads of K and V
    uint32_t block;                                                    // bytes of one head's rows of a page
    int *status, *input_status;                                        // waits that ran out; lengths, rows and pages out of range
};

#ifdef __CUDACC__
__device__ __forceinline__ int64_t kv4_capacity(const Kv4View& w) { return (int64_t)w.max_pages << w.shift; }
__device__ __forceinline__ Kv4Seq kv4_load_seq(const Kv4View& w, int s) {
    return kv4_seq(__ldg(w.row_start + s), __ldg(w.row_start + s + 1), w.n_rows, __ldg(w.kv_len + s), kv4_capacity(w));
}
// Page of a cache row (inside the page table), or -1 after recording an id that no pool has.
__device__ __forceinline__ int kv4_page(const Kv4View& w, int seq, int row) {
    const int p = __ldg(w.table + (size_t)seq * w.max_pages + (row >> w.shift));
    if ((unsigned)p < (unsigned)w.n_pages) return p;
    atomicCAS(w.input_status, DEV_OK, DEV_KV4_PAGE);
    return -1;
}
__device__ __forceinline__ size_t kv4_block_at(const Kv4View& w, int page, int head) { return ((size_t)page * w.heads + head) * w.block; }

#endif

Kv4View kv4_view(const ghd_ctx* c, const ghd_kv4* kv, const ghd_kv4_rows* rows);
// attn_kv4.cu
ghd_status launch_attn_kv4(ghd_ctx* c, const Kv4View& w, const ghd_kv4_rows* rows, const void* pool, const void* q, void* out);

}  // namespace ghd

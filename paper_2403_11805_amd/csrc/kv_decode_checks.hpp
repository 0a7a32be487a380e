// Checks and small helpers that the host sides of decoding share.
#pragma once

#include <hip/hip_runtime.h>

#include "kv_internal.h"

namespace kvs {

inline int hip_fail(hipError_t e, const char* what) { return fail(KV_EHIP, "%s: %s", what, hipGetErrorString(e)); }

inline int launch_status(const char* what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? KV_OK : hip_fail(e, what);
}

// Workgroups that one launch may have: a grid has less than 2^32 threads.
constexpr int64_t most_groups(int threads) { return 0xffffffffLL / threads; }

inline int check_seqs(int32_t n_seqs) {
    return n_seqs < 1 || n_seqs > 65535 ? fail(KV_EINVAL, "n_seqs %d outside [1, 65535]", n_seqs) : KV_OK;
}

// The page table of sequences of at most `pages` pages.
inline int check_page_table(const kv_pages_t* pages, int32_t n_pages) {
    if (!pages) return fail(KV_EINVAL, "pages is NULL");
    if (int rc = check_seqs(pages->n_seqs)) return rc;
    if (!pages->pool || !pages->off || !pages->bits || !pages->len) return fail(KV_EINVAL, "NULL device pointer in pages");
    if (!aligned(pages->pool, 16) || !aligned(pages->off, 8) || !aligned(pages->len, 4))
        return fail(KV_EINVAL, "pages: pool must be 16-byte aligned, off 8-byte, len 4-byte aligned");
    if (pages->stride < n_pages)
        return fail(KV_EINVAL, "pages: stride %d is less than the %d pages of a sequence", pages->stride, n_pages);
    return KV_OK;
}

// The rows of a step: their number, their list, and the elements from one to the next.
inline int check_rows(const kv_pages_t* pages, int32_t n_rows, const int32_t* row_start, int64_t stride, int64_t least) {
    if (n_rows < 0) return fail(KV_EINVAL, "n_rows %d is negative", n_rows);
    if (!row_start && n_rows != pages->n_seqs)
        return fail(KV_EINVAL, "without row_start n_rows (%d) must be n_seqs (%d)", n_rows, pages->n_seqs);
    if (!aligned(row_start, 4)) return fail(KV_EINVAL, "row_start must be 4-byte aligned");
    if (stride < least || stride % 8) return fail(KV_EINVAL, "row stride %lld is less than %lld or no multiple of 8",
                                                  static_cast<long long>(stride), static_cast<long long>(least));
    return KV_OK;
}

inline int log2_of(int v) {
    int l = 0;
    while ((1 << l) < v) ++l;
    return l;
}

}  // namespace kvs

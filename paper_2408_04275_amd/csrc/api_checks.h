// Host-side checks of arguments that the C-ABI entry points share.
#pragma once
#include "../../include/mmtrain.h"
#include <initializer_list>

namespace mmt {

static inline int check_batch(const mmtrain_batch *b) {
    if (!b) return MMTRAIN_ERR_INVALID_ARG;
    if (b->total_tokens < 0 || b->n_segments < 0) return MMTRAIN_ERR_INVALID_ARG;
    if (b->mask_mode != MMTRAIN_MASK_CAUSAL && b->mask_mode != MMTRAIN_MASK_BIDIR) return MMTRAIN_ERR_INVALID_ARG;
    if (!b->cu_seqlens_host) return MMTRAIN_ERR_INVALID_ARG;
    if ((b->seg_mask_dev == nullptr) != (b->seg_mask_host == nullptr)) return MMTRAIN_ERR_INVALID_ARG;
    const int32_t *cu = b->cu_seqlens_host;
    if (cu[0] != 0) return MMTRAIN_ERR_BAD_SEGMENTS;
    for (int s = 0; s < b->n_segments; ++s)
        if (cu[s + 1] < cu[s]) return MMTRAIN_ERR_BAD_SEGMENTS;
    if (cu[b->n_segments] != b->total_tokens) return MMTRAIN_ERR_BAD_SEGMENTS;
    if (b->seg_mask_host)
        for (int s = 0; s < b->n_segments; ++s)
            if (b->seg_mask_host[s] > 1) return MMTRAIN_ERR_INVALID_ARG;
    if (b->total_tokens > 0 && !b->cu_seqlens_dev) return MMTRAIN_ERR_INVALID_ARG;
    return MMTRAIN_OK;
}

// The kernels move 16 bytes per lane (vector loads and stores, direct-to-LDS copies): every tensor pointer must be
// 16-byte aligned.  A misaligned one (a view such as tensor[1:]) is an argument error, not a memory fault.
static inline bool misaligned(std::initializer_list<const void *> ptrs) {
    uintptr_t bits = 0;
    for (const void *p : ptrs) bits |= (uintptr_t)p;
    return (bits & 15) != 0;
}

#define HIP_TRY(expr) do { hipError_t e_ = (expr); if (e_ != hipSuccess) return MMTRAIN_ERR_HIP; } while (0)

}  // namespace mmt

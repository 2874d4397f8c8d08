// Host helpers of the C ABI's operators (operators.hip, drafting.hip): limits, and checks of what calls share.
// Part of libfsd (gfx950).
#ifndef FSD_CSRC_OPERATORS_HOST_H_
#define FSD_CSRC_OPERATORS_HOST_H_

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <limits.h>

#include "fsd.h"

#include "operators_common.h"

namespace {

constexpr int kMaxRows = 2048;    // K or N, as in the verify calls
constexpr int kMaxBatch = 65535;
constexpr long kMaxGroups = (1L << 32) / kWG - 1;   // workgroups of a launch: less than 2^32 threads

inline bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
// whether two runs of bytes share one (an absent one shares none)
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && (x < y ? y - x < na : x - y < nb);
}
inline int launched() { return hipGetLastError() == hipSuccess ? FSD_OK : FSD_ERR_LAUNCH; }

inline int check_cache(const fsd_cache* c) {
    if (!c || !c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || !c->block_table || !c->cache_len) return FSD_ERR_NULL;
    if (c->layers < 1 || c->num_blocks < 1 || c->kv_heads < 1 || c->kv_heads > 1024 || c->max_blocks < 1 ||
        c->max_blocks > INT_MAX / kBlock - 1 || (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256))
        return FSD_ERR_SHAPE;
    if (!aligned16(c->k_codes) || !aligned16(c->v_codes) || reinterpret_cast<uintptr_t>(c->k_scale) % 4 != 0 ||
        reinterpret_cast<uintptr_t>(c->v_scale) % 4 != 0)
        return FSD_ERR_LAYOUT;
    return FSD_OK;
}

}  // namespace

#endif  // FSD_CSRC_OPERATORS_HOST_H_

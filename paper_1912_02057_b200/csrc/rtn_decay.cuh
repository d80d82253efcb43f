// Shared by the kernels of linear attention with a decay per head.
#pragma once
#include "rtn_internal.cuh"

namespace rtn {

// The chunked tensor-core form: shapes and types it takes, and its launches (`taken` false: a layout that the copy engine
// cannot describe; nothing was launched).
bool decay_chunk_supported(const DecayArgs& g);
cudaError_t launch_decay_chunk(const DecayArgs& g, cudaStream_t s, bool& taken);

#ifdef __CUDACC__

// First token and length of sequence b; false (with the status bit) where the bounds do not fit.
__device__ __forceinline__ bool sequence_bounds(const DecayArgs& g, int64_t b, int64_t& first, int64_t& len, int64_t& slot)
{
    first = g.start[b];
    len = (int64_t)g.start[b + 1] - first;
    slot = g.slot != nullptr ? g.slot[b] : b;
    return first >= 0 && len >= 0 && len <= g.max_len && first + len <= g.total && slot < g.n_slots;
}

#endif

}  // namespace rtn

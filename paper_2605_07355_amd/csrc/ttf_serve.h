// Internal declarations of the entry points behind the compressed rows: norm and rotation of queries and
// keys, cache append, attention over a paged cache.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "ttf.h"

namespace ttf {

constexpr int kMaxHeadDim = 256;

void set_last_hip_error(hipError_t e);   // behind ttf_last_hip_error()

hipError_t launch_qk(const ttf_qk_params& p, const ttf_kv_cache* cache, hipStream_t s);

size_t attention_workspace_bytes(const ttf_attention_params& p);   // of this call and of every smaller one
size_t attention_workspace_used(const ttf_attention_params& p);    // of this call
hipError_t launch_attention(const ttf_attention_params& p, const ttf_kv_cache& c, void* workspace, hipStream_t s);

// Rows of sequence b, clamped to the buffers: first row and number of rows (0 where the offsets make no sense).
__device__ __forceinline__ int2 rows_of(const int32_t* row_offsets, int b, int rows)
{
    const int first = row_offsets[b], end = min(row_offsets[b + 1], rows);
    return first < 0 || end <= first ? int2{0, 0} : int2{first, end - first};
}

}  // namespace ttf

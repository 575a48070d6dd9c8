// What the model's translation unit needs of the paged one.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/jot.h"

namespace jot {

constexpr int32_t kStatusBadIndex = 6;     // status word: a slot, a page or a length outside the pages (skipped, or read as zeros)

// Puts a bad index on record, unless an expired wait is there already, which says more.
__device__ __forceinline__ void report_bad_index(int32_t* status) {
    const int32_t held = *reinterpret_cast<volatile int32_t*>(status);
    if (held <= 0) atomicCAS(status, held, kStatusBadIndex);
}

// Whether the kernels can work on these pages.
int check_kv_pages(const jot_kv_pages* pages, int layer);
// Positions, slots and lengths of a pass over positions pos0 .. pos0 + rows_per_seq - 1 of B canvases of L positions, whose pages are
// table[b * table_stride + position / page_size].
int launch_page_rows(const int32_t* table, int64_t table_stride, int B, int L, int rows_per_seq, int pos0, int page_size, int n_pages,
                     int32_t* positions, int32_t* slots, int32_t* lens, int32_t* status, cudaStream_t st);
// The most jot_paged_attention_workspace_bytes() asks for with up to max_rows rows of a key head.
size_t paged_workspace_most(int64_t max_rows, int head_dim);

}  // namespace jot

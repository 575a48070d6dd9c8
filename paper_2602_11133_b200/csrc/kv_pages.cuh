// Data movement of a paged key-value cache: rows of keys and values into their slots, and whole pages to other pages.
// Bound by HBM (each byte read once, written once); 16-byte vectors, several loads in flight per thread.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "heads.cuh"

namespace jot {

struct WriteArgs {
    const uint16_t *k, *v;                           // 16-bit elements; strides in elements
    int64_t k_row, k_head, v_row, v_head;
    int n_rows, n_heads, head_dim, rows_per_cta;
    PagesDev pages;
    const int32_t* slots;
    int32_t* status;
};

constexpr int kMoveThreads = 256;

__global__ void __launch_bounds__(kMoveThreads) kv_write_kernel(const WriteArgs a) {
    grid_launch_dependents();
    grid_dependency_wait();
    const int row0 = blockIdx.x * a.rows_per_cta, rows = min(a.rows_per_cta, a.n_rows - row0);
    const int nvec = a.head_dim / 8, per_row = a.n_heads * nvec;
    for (int i = threadIdx.x; i < rows * per_row; i += kMoveThreads) {
        const int row = row0 + i / per_row, in_row = i % per_row, h = in_row / nvec, c = in_row - h * nvec;
        const int slot = a.slots[row], page = slot / a.pages.page_size;
        if (slot < 0) continue;
        if (page >= a.pages.n_pages) {
            if (in_row == 0 && a.status) report_bad_index(a.status);
            continue;
        }
        const uint4 kv = reinterpret_cast<const uint4*>(a.k + row * a.k_row + h * a.k_head)[c];
        const uint4 vv = reinterpret_cast<const uint4*>(a.v + row * a.v_row + h * a.v_head)[c];
        const int64_t in_page = ((int64_t)h * a.pages.page_size + (slot - page * a.pages.page_size)) * a.head_dim;
        reinterpret_cast<uint4*>((uint16_t*)a.pages.k + page * a.pages.k_page + in_page)[c] = kv;
        reinterpret_cast<uint4*>((uint16_t*)a.pages.v + page * a.pages.v_page + in_page)[c] = vv;
    }
}

__global__ void page_rows_kernel(const int32_t* __restrict__ table, int64_t table_stride, int B, int L, int rows_per_seq, int pos0, int page_size, int n_pages,
                                 int32_t* __restrict__ positions, int32_t* __restrict__ slots, int32_t* __restrict__ lens, int32_t* status) {
    grid_launch_dependents();
    grid_dependency_wait();
    const int r = blockIdx.x * blockDim.x + threadIdx.x;
    if (r < B) lens[r] = L;
    if (r >= B * rows_per_seq) return;
    const int b = r / rows_per_seq, pos = pos0 + r - b * rows_per_seq, p = pos / page_size, page = table[b * table_stride + p];
    positions[r] = pos;
    const bool real = (unsigned)page < (unsigned)n_pages;
    slots[r] = real ? page * page_size + pos - p * page_size : -1;
    if (!real) report_bad_index(status);
}

// The pairs travel as kernel arguments, as the caller's lists live on the host and may change right after the call.
template <int N>
struct PagePairs {
    int32_t src[N], dst[N];
};
struct CopyArgs {
    uint16_t *k, *v;
    int64_t k_layer, v_layer, k_page, v_page;        // strides, elements
    int n, n_layers, page_vecs;                      // pairs; 16-byte vectors of a page
};
constexpr int kCopyVecsPerThread = 8;

// Units of work: (pair, layer, k or v), page_vecs vectors each, laid end to end; a CTA takes the next 2048 vectors of that line.
template <int N>
__global__ void __launch_bounds__(kMoveThreads) kv_copy_kernel(const CopyArgs a, const __grid_constant__ PagePairs<N> pairs) {
    grid_launch_dependents();
    grid_dependency_wait();
    const int64_t first = (int64_t)blockIdx.x * (kMoveThreads * kCopyVecsPerThread);
    const int unit0 = (int)(first / a.page_vecs);
    const unsigned off0 = (unsigned)(first - (int64_t)unit0 * a.page_vecs);
    const int n_units = a.n * a.n_layers * 2;
    uint4 buf[kCopyVecsPerThread];
    uint4* dst[kCopyVecsPerThread];
#pragma unroll
    for (int j = 0; j < kCopyVecsPerThread; ++j) {
        const unsigned at = off0 + j * kMoveThreads + threadIdx.x, more = at / (unsigned)a.page_vecs;
        const int unit = unit0 + (int)more;
        dst[j] = nullptr;
        if (unit < n_units) {
            const int pair = unit % a.n, t = unit / a.n, layer = t >> 1;
            const unsigned c = at - more * (unsigned)a.page_vecs;
            uint16_t* base = (t & 1) ? a.v + layer * a.v_layer : a.k + layer * a.k_layer;
            const int64_t page = (t & 1) ? a.v_page : a.k_page;
            buf[j] = reinterpret_cast<const uint4*>(base + pairs.src[pair] * page)[c];
            dst[j] = reinterpret_cast<uint4*>(base + pairs.dst[pair] * page) + c;
        }
    }
#pragma unroll
    for (int j = 0; j < kCopyVecsPerThread; ++j)
        if (dst[j]) *dst[j] = buf[j];
}

}  // namespace jot

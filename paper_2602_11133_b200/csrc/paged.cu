// Entry points of decoding over a paged key-value cache: argument checks and launches (kernels: heads.cuh, kv_pages.cuh,
// paged_attention.cuh).
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <memory>
#include <new>

#include "heads.cuh"
#include "host.cuh"
#include "kv_pages.cuh"
#include "paged_attention.cuh"
#include "paged_attention_umma.cuh"

using namespace jot;

static_assert(JOT_STATUS_BAD_INDEX == kStatusBadIndex, "status word of the kernels and of the interface");

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Rows and heads are counted in 31 bits, the grid's last CTA and a row's last stretch of heads (queries, keys and values) included.
constexpr int kMostRows = INT32_MAX - 4096, kMostHeads = INT32_MAX / 4;

// A stride counts only where there is a second element along it.
bool stride_ok(int64_t s, int64_t n) { return n <= 1 || s % 8 == 0; }

PagesDev layer_pages(const jot_kv_pages* p, int layer) {
    return PagesDev{(uint16_t*)p->k + layer * p->k_layer_stride, (uint16_t*)p->v + layer * p->v_layer_stride, p->k_page_stride,
                    p->v_page_stride, p->n_pages, p->page_size};
}

int check_heads(const jot_heads* h, int n_rows, bool has_out) {
    if (!h->in || !aligned16(h->in) || !aligned16(h->gain) || h->n_heads <= 0) return JOT_ERR_ARG;
    if (!stride_ok(h->in_row_stride, n_rows) || !stride_ok(h->in_head_stride, h->n_heads)) return JOT_ERR_ARG;
    if (!has_out) return JOT_OK;
    if (!h->out || !aligned16(h->out)) return JOT_ERR_ARG;
    return stride_ok(h->out_row_stride, n_rows) && stride_ok(h->out_head_stride, h->n_heads) ? JOT_OK : JOT_ERR_ARG;
}

HeadsDev heads_dev(const jot_heads* h) {
    return HeadsDev{h->in, h->out, h->gain, h->in_row_stride, h->in_head_stride, h->out_row_stride, h->out_head_stride, h->n_heads};
}

template <typename T, int G>
int launch_heads(const HeadArgs& a, bool interleaved, cudaStream_t st) {
    const dim3 grid((unsigned)((a.n_rows + a.rows_per_cta - 1) / a.rows_per_cta));
    const size_t smem = (size_t)a.rows_per_cta * a.half * sizeof(float2);
    if (interleaved) launch_k(head_norm_rope_kernel<T, G, true>, grid, dim3(kHeadThreads), smem, st, a);
    else launch_k(head_norm_rope_kernel<T, G, false>, grid, dim3(kHeadThreads), smem, st, a);
    return launch_check();
}

template <int N>
int launch_copy(CopyArgs a, const int32_t* src, const int32_t* dst, int n, cudaStream_t st) {
    PagePairs<N> pairs;
    std::memset(&pairs, 0, sizeof(pairs));
    std::memcpy(pairs.src, src, (size_t)n * 4);
    std::memcpy(pairs.dst, dst, (size_t)n * 4);
    a.n = n;
    const int64_t vecs = (int64_t)n * a.n_layers * 2 * a.page_vecs, per_cta = kMoveThreads * kCopyVecsPerThread;
    launch_k(kv_copy_kernel<N>, dim3((unsigned)((vecs + per_cta - 1) / per_cta)), dim3(kMoveThreads), 0, st, a, pairs);
    return launch_check();
}

// Whether no page is written twice and none is both read and written.
int check_moves(int n_pages, int n, const int32_t* src, const int32_t* dst) {
    for (int i = 0; i < n; ++i)
        if (src[i] < 0 || src[i] >= n_pages || dst[i] < 0 || dst[i] >= n_pages) return JOT_ERR_ARG;
    if (n <= 32) {
        for (int i = 0; i < n; ++i)
            for (int j = 0; j < n; ++j)
                if (src[i] == dst[j] || (i != j && dst[i] == dst[j])) return JOT_ERR_ARG;
        return JOT_OK;
    }
    std::unique_ptr<uint8_t[]> role(new (std::nothrow) uint8_t[n_pages]());
    if (!role) return JOT_ERR_LIMIT;
    for (int i = 0; i < n; ++i) {
        if (role[dst[i]]) return JOT_ERR_ARG;
        role[dst[i]] = 1;
    }
    for (int i = 0; i < n; ++i)
        if (role[src[i]]) return JOT_ERR_ARG;
    return JOT_OK;
}

// Rows an attention CTA works on: a warp's 16; a tcgen05 tile of 128 that holds them four times, twice or once; two such tiles.
int paged_row_tile(int rows) { return rows <= 16 ? 16 : (rows <= 32 ? 32 : (rows <= 64 ? 64 : (rows <= 128 ? 128 : 256))); }

struct PagedSpace {
    size_t desc, ml, partial, total;
};
PagedSpace paged_space(int row_tile, int head_dim) {
    const size_t ctas = row_tile == 16 ? kPagedMaxCtas : (row_tile == 256 ? kUmmaPagedMaxCtas : 2 * kUmmaPagedMaxCtas);      // or streams of CTAs
    PagedSpace s;
    s.desc = 0;
    s.ml = align_up(ctas * sizeof(int4), 256);
    s.partial = s.ml + align_up(ctas * 2 * row_tile * sizeof(float2), 256);
    s.total = s.partial + ctas * 2 * row_tile * head_dim * sizeof(float);
    return s;
}

// Items of a call: (sequence, key head, tile of rows).
int64_t paged_items(const PagedArgs& a, int row_tile) { return (int64_t)a.B * a.nkv * ((a.T * a.group + row_tile - 1) / row_tile); }

// The second kernel: four warps to a row where an item may be in many parts (few items on many CTAs), else a warp to a row.  One row over 20011 keys
// 23 us with four and 50 with one, 224 rows over 8192 keys 22 and 36; 32 rows of 32 heads of 16 sequences 50 and 44, canvases of 704 rows 230 and 202.
template <typename T, int HD>
int launch_join(const PagedArgs& a, int shares, int row_tile, cudaStream_t st) {
    const int rows = std::min(row_tile, a.T * a.group);
    const int64_t items = paged_items(a, row_tile);
    const int grid = a.by_item ? (int)items : shares;
    auto go = [&](auto* kernel, int per_cta) { launch_k(kernel, dim3((unsigned)grid, (unsigned)((rows + per_cta - 1) / per_cta)), dim3(kPagedThreads), 0, st, a, row_tile, shares); };
    if (shares > 8 * items) go(paged_join_kernel<T, HD, 4>, 1);
    else go(paged_join_kernel<T, HD, 1>, 4);
    return launch_check();
}

// Up to so many tiles (of what a table row has room for) an item is not cut: the second kernel and the parts' way through memory cost more.
// One row over 129 keys 23.4 -> 21.6 us a call (half of it the caller's side of two launches), 384 rows of 32 heads over 384 keys 28.7 -> 16.3 us.
constexpr int kPagedWhole = 4;
// What the table can hold bounds the line of tiles: of an item, and of them all (no more than there may be CTAs).
int64_t paged_tiles(const PagedArgs& a, int keys) { return ((int64_t)a.max_pages * a.pages.page_size + keys - 1) / keys; }
int64_t paged_most(const PagedArgs& a, int64_t items, int64_t tiles) {
    const int64_t n = std::min<int64_t>(items, kPagedMaxCtas) * std::min(a.B, kPagedMaxCtas);
    return std::max<int64_t>(1, std::min<int64_t>(kPagedMaxCtas, n) * std::min<int64_t>(tiles, kPagedMaxCtas));
}

template <typename T, int HD>
int launch_paged_t(const DeviceInfo* di, PagedArgs a, int64_t items, cudaStream_t st) {
    static thread_local int per_sm[64] = {};
    int dev = 0;
    JOT_CUDA(cudaGetDevice(&dev));
    int& occ = per_sm[dev & 63];
    auto* kernel = paged_attention_kernel<T, HD>;
    constexpr int smem = PagedSmem<HD>::DYN_BYTES;
    if (occ == 0) {
        JOT_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        int n = 0;
        JOT_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, kPagedThreads, smem));
        if (n < 1) return JOT_ERR_DEVICE;
        occ = n;
    }
    const int64_t tiles = paged_tiles(a, kPagedTile);
    a.whole = tiles <= kPagedWhole;
    const int grid = (int)std::min<int64_t>(paged_most(a, items, tiles), std::min(occ * di->sms, kPagedMaxCtas));
    a.by_item = !a.whole && paged_items(a, 16) <= grid;
    launch_k(kernel, dim3((unsigned)grid), dim3(kPagedThreads), smem, st, a);
    JOT_TRY(launch_check());
    return a.whole ? JOT_OK : launch_join<T, HD>(a, grid, 16, st);
}

// (head_dim, key of the page, head, page); a box is 64 columns of a page's keys, or of 128 of them.  Out-of-range pages read as zeros.
int make_map_pages(const DeviceInfo* di, CUtensorMap* map, const PagedArgs& a, const void* ptr, int64_t page_stride, int hd, int dtype) {
    const cuuint64_t head_bytes = (cuuint64_t)a.pages.page_size * hd * 2;
    cuuint64_t dims[4] = {(cuuint64_t)hd, (cuuint64_t)a.pages.page_size, (cuuint64_t)a.nkv, (cuuint64_t)a.pages.n_pages};
    cuuint64_t strides[3] = {(cuuint64_t)hd * 2, head_bytes, a.pages.n_pages > 1 ? (cuuint64_t)page_stride * 2 : head_bytes * a.nkv};
    cuuint32_t box[4] = {64, (cuuint32_t)std::min(a.pages.page_size, 128), 1, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    CUresult r = di->encode(map, dtype == JOT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(ptr), dims, strides,
                            box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        g_last_cuda_error = (int)cudaErrorInvalidValue;
        return JOT_ERR_CUDA;
    }
    return JOT_OK;
}

template <typename T, int HD, int ROWS, bool TMA>
int launch_paged_umma_t(const DeviceInfo* di, const PagedArgs& a, int grid, cudaStream_t st) {
    static thread_local bool attr_set[64] = {};
    int dev = 0;
    JOT_CUDA(cudaGetDevice(&dev));
    auto* kernel = paged_attention_umma_kernel<T, HD, ROWS, TMA>;
    constexpr int smem = UmmaPagedSmem<HD>::DYN_BYTES;
    if (!attr_set[dev & 63]) {
        JOT_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        attr_set[dev & 63] = true;
    }
    CUtensorMap mk, mv;
    if (TMA) {
        const int dtype = PackIsBf16<T>::value ? JOT_BF16 : JOT_FP16;
        JOT_TRY(make_map_pages(di, &mk, a, a.pages.k, a.pages.k_page, HD, dtype));
        JOT_TRY(make_map_pages(di, &mv, a, a.pages.v, a.pages.v_page, HD, dtype));
    } else {
        std::memset(&mk, 0, sizeof(mk));
        mv = mk;
    }
    launch_k(kernel, dim3((unsigned)grid), dim3(UmmaPagedRoles<ROWS, TMA>::THREADS), smem, st, a, mk, mv);
    return launch_check();
}

template <typename T, int HD, int ROWS>
int launch_paged_umma(const DeviceInfo* di, PagedArgs a, int64_t items, cudaStream_t st) {
    const bool tma = paged_tma_pages(a.pages.page_size) && a.pages.k_page >= 0 && a.pages.v_page >= 0;
    const int64_t tiles = paged_tiles(a, tma ? paged_tma_keys(a.pages.page_size) : kUmmaPagedTile);
    constexpr int streams = ROWS == 256 ? 1 : 2;
    // Two tiles of rows take twice as long over a tile of keys: worth cutting unless a third of the SMs have items of their own.  224 rows over 512
    // keys: one sequence 13.3 us cut and 15.4 whole, four 16.4 and 16.3, sixteen 23.1 and 17.8; canvases of 384 rows of 32 heads 26.5 and 15.3.  (Over
    // 256 keys whole items are ahead for few sequences, too: 12.1 and 11.1 for one, 16.6 and 12.4 for eight.)
    a.whole = tiles <= 1 || (tiles <= kPagedWhole && (ROWS < 256 || 3 * items * a.B >= di->sms));
    const int grid = (int)std::min<int64_t>(paged_most(a, items, tiles), std::min(di->sms, kUmmaPagedMaxCtas));
    a.by_item = !a.whole && paged_items(a, ROWS) <= grid * streams;
    if (tma) JOT_TRY((launch_paged_umma_t<T, HD, ROWS, true>(di, a, grid, st)));
    else JOT_TRY((launch_paged_umma_t<T, HD, ROWS, false>(di, a, grid, st)));
    return a.whole ? JOT_OK : launch_join<T, HD>(a, grid * streams, ROWS, st);
}

template <typename T, int HD>
int launch_paged(const DeviceInfo* di, const PagedArgs& a, int row_tile, cudaStream_t st) {
    const int rows = a.T * a.group;
    const int64_t items = (int64_t)a.nkv * ((rows + row_tile - 1) / row_tile);
    if (row_tile == 16) return launch_paged_t<T, HD>(di, a, items, st);
    if (row_tile == 32) return launch_paged_umma<T, HD, 32>(di, a, items, st);
    if (row_tile == 64) return launch_paged_umma<T, HD, 64>(di, a, items, st);
    return row_tile == 128 ? launch_paged_umma<T, HD, 128>(di, a, items, st) : launch_paged_umma<T, HD, 256>(di, a, items, st);
}

}  // namespace

namespace jot {

int check_kv_pages(const jot_kv_pages* p, int layer) {
    if (!p || !p->k || !p->v || !aligned16(p->k) || !aligned16(p->v)) return JOT_ERR_ARG;
    if (p->n_layers <= 0 || p->n_pages <= 0 || p->n_kv_heads <= 0 || p->page_size <= 0 || p->head_dim <= 0) return JOT_ERR_ARG;
    if (layer < 0 || layer >= p->n_layers) return JOT_ERR_ARG;
    if (p->dtype != JOT_BF16 && p->dtype != JOT_FP16) return JOT_ERR_ARG;
    if (p->head_dim % 8 || (int64_t)p->n_pages * p->page_size > INT32_MAX) return JOT_ERR_SHAPE;
    const int64_t page = (int64_t)p->n_kv_heads * p->page_size * p->head_dim;
    if (page / 8 > INT32_MAX / 2) return JOT_ERR_SHAPE;
    if (!stride_ok(p->k_layer_stride, p->n_layers) || !stride_ok(p->v_layer_stride, p->n_layers) ||
        !stride_ok(p->k_page_stride, p->n_pages) || !stride_ok(p->v_page_stride, p->n_pages))
        return JOT_ERR_ARG;
    if (p->n_pages > 1 && (std::abs(p->k_page_stride) < page || std::abs(p->v_page_stride) < page)) return JOT_ERR_ARG;
    return JOT_OK;
}

int launch_page_rows(const int32_t* table, int64_t table_stride, int B, int L, int rows_per_seq, int pos0, int page_size, int n_pages, int32_t* positions,
                     int32_t* slots, int32_t* lens, int32_t* status, cudaStream_t st) {
    launch_k(page_rows_kernel, dim3((unsigned)((std::max(B, B * rows_per_seq) + 255) / 256)), dim3(256), 0, st, table, table_stride, B, L, rows_per_seq, pos0, page_size,
             n_pages, positions, slots, lens, status);
    return launch_check();
}

size_t paged_workspace_most(int64_t max_rows, int head_dim) {
    size_t most = 0;
    for (int tile : {16, 32, 64, 128, 256}) {
        most = std::max(most, paged_space(tile, head_dim).total);
        if (tile >= max_rows) break;
    }
    return most;
}

}  // namespace jot

extern "C" {

int jot_head_norm_rope(const jot_heads* q, const jot_heads* k, const jot_rope* rope, int dtype, int n_rows, int head_dim, float eps,
                       const int32_t* d_positions, const jot_heads* v, const jot_kv_pages* pages, int layer, const int32_t* d_slots,
                       int32_t* d_status, void* stream) {
    if (!q || !rope || (n_rows > 0 && !d_positions) || n_rows < 0 || (dtype != JOT_BF16 && dtype != JOT_FP16)) return JOT_ERR_ARG;
    if (head_dim < 8 || head_dim > 256 || head_dim % 8) return JOT_ERR_SHAPE;
    if (rope->rotary_dim < 0 || rope->rotary_dim > head_dim || (rope->rotary_dim > 0 && !rope->d_inv_freq)) return JOT_ERR_ARG;
    if (rope->rotary_dim % (rope->interleaved ? 8 : 16)) return JOT_ERR_SHAPE;
    if (pages && (!k || !v || (n_rows > 0 && !d_slots))) return JOT_ERR_ARG;
    if (!pages && v) return JOT_ERR_ARG;
    if (n_rows == 0) return JOT_OK;
    JOT_TRY(check_heads(q, n_rows, true));
    if (k) JOT_TRY(check_heads(k, n_rows, !pages));
    if (n_rows > kMostRows || q->n_heads > kMostHeads || (k && k->n_heads > kMostHeads)) return JOT_ERR_SHAPE;
    HeadArgs a{};
    if (pages) {
        JOT_TRY(check_heads(v, n_rows, false));
        JOT_TRY(check_kv_pages(pages, layer));
        if (pages->dtype != dtype || pages->head_dim != head_dim || pages->n_kv_heads != k->n_heads || v->n_heads != k->n_heads) return JOT_ERR_ARG;
        a.pages = layer_pages(pages, layer);
        a.to_pages = 1;
        a.v = heads_dev(v);
    }
    DeviceInfo* di = nullptr;
    JOT_TRY(device_info(&di));
    a.q = heads_dev(q);
    if (k) a.k = heads_dev(k);
    a.positions = d_positions; a.inv_freq = rope->d_inv_freq; a.half = rope->rotary_dim / 2; a.magnitude = rope->magnitude; a.eps = eps;
    a.head_dim = head_dim; a.n_rows = n_rows; a.slots = d_slots; a.status = d_status;
    // Several rows a CTA where there are many: 11264 rows of 64 heads 64 us, 79 at one a CTA, 6024 rows of 32 heads 23 and 34; from a quarter as many
    // rows on it would cost: 512 rows of 64 heads 9.5 us, 7.0 at one.
    a.rows_per_cta = n_rows >= 16 * di->sms ? 4 : (n_rows >= 8 * di->sms ? 2 : 1);
    cudaStream_t st = (cudaStream_t)stream;
    const bool il = rope->interleaved != 0;
    const int pairs = (head_dim / 8 + 1) / 2;                           // lanes a head needs
    if (dtype == JOT_BF16) {
        if (pairs <= 4) return launch_heads<__nv_bfloat16, 4>(a, il, st);
        return pairs <= 8 ? launch_heads<__nv_bfloat16, 8>(a, il, st) : launch_heads<__nv_bfloat16, 16>(a, il, st);
    }
    if (pairs <= 4) return launch_heads<__half, 4>(a, il, st);
    return pairs <= 8 ? launch_heads<__half, 8>(a, il, st) : launch_heads<__half, 16>(a, il, st);
}

int jot_kv_write(const jot_kv_pages* pages, int layer, int n_rows, const void* d_k, int64_t k_row_stride, int64_t k_head_stride,
                 const void* d_v, int64_t v_row_stride, int64_t v_head_stride, const int32_t* d_slots, int32_t* d_status, void* stream) {
    JOT_TRY(check_kv_pages(pages, layer));
    if (n_rows == 0) return JOT_OK;
    if (!d_k || !d_v || !d_slots || n_rows < 0 || !aligned16(d_k) || !aligned16(d_v)) return JOT_ERR_ARG;
    if (!stride_ok(k_row_stride, n_rows) || !stride_ok(v_row_stride, n_rows) || !stride_ok(k_head_stride, pages->n_kv_heads) ||
        !stride_ok(v_head_stride, pages->n_kv_heads))
        return JOT_ERR_ARG;
    if (n_rows > kMostRows) return JOT_ERR_SHAPE;
    DeviceInfo* di = nullptr;
    JOT_TRY(device_info(&di));
    WriteArgs a{};
    a.k = (const uint16_t*)d_k; a.v = (const uint16_t*)d_v;
    a.k_row = k_row_stride; a.k_head = k_head_stride; a.v_row = v_row_stride; a.v_head = v_head_stride;
    a.n_rows = n_rows; a.n_heads = pages->n_kv_heads; a.head_dim = pages->head_dim;
    a.pages = layer_pages(pages, layer); a.slots = d_slots; a.status = d_status;
    // Several short rows a CTA, while every SM has eight: 40000 rows of 4 heads of 128 28 us, 43 at one a CTA; 11264 rows of 4 heads 10.9 and 13.6, of
    // 32 heads (two a CTA) 57.9 and 56.2.
    const int per_row = a.n_heads * (a.head_dim / 8);
    a.rows_per_cta = std::max(1, std::min(n_rows / (8 * di->sms), 4 * kMoveThreads / per_row));
    launch_k(kv_write_kernel, dim3((unsigned)((n_rows + a.rows_per_cta - 1) / a.rows_per_cta)), dim3(kMoveThreads), 0, (cudaStream_t)stream, a);
    return launch_check();
}

int jot_kv_copy_pages(const jot_kv_pages* pages, int n, const int32_t* src, const int32_t* dst, void* stream) {
    JOT_TRY(check_kv_pages(pages, 0));
    if (n < 0 || (n > 0 && (!src || !dst))) return JOT_ERR_ARG;
    JOT_TRY(check_moves(pages->n_pages, n, src, dst));
    CopyArgs a{};
    a.k = (uint16_t*)pages->k; a.v = (uint16_t*)pages->v;
    a.k_layer = pages->k_layer_stride; a.v_layer = pages->v_layer_stride; a.k_page = pages->k_page_stride; a.v_page = pages->v_page_stride;
    a.n_layers = pages->n_layers;
    a.page_vecs = pages->n_kv_heads * pages->page_size * (pages->head_dim / 8);
    cudaStream_t st = (cudaStream_t)stream;
    constexpr int MOST = 1024;
    const int64_t vecs_per_pair = (int64_t)a.n_layers * 2 * a.page_vecs;
    if (vecs_per_pair > (int64_t)INT32_MAX * kMoveThreads) return JOT_ERR_SHAPE;
    // the grid and the units of a launch fit 31 bits
    const int step = (int)std::max<int64_t>(1, std::min<int64_t>(MOST, std::min<int64_t>((int64_t)INT32_MAX * kMoveThreads / vecs_per_pair,
                                                                                         INT32_MAX / 4 / a.n_layers)));
    for (int i = 0; i < n; i += step) {
        const int m = std::min(step, n - i);
        // (few pairs are few bytes of arguments: five pages 8.4 us a call, 9.2 with room for 1024; on the device the same)
        if (m <= 16) JOT_TRY(launch_copy<16>(a, src + i, dst + i, m, st));
        else JOT_TRY(launch_copy<MOST>(a, src + i, dst + i, m, st));
    }
    return JOT_OK;
}

size_t jot_paged_attention_workspace_bytes(int T, int n_q_heads, int n_kv_heads, int head_dim) {
    if (T <= 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads || (head_dim != 64 && head_dim != 128)) return 0;
    const int64_t rows = (int64_t)T * (n_q_heads / n_kv_heads);
    return rows > INT32_MAX ? 0 : paged_space(paged_row_tile((int)rows), head_dim).total;
}

int jot_paged_attention(const void* d_q, int64_t q_seq_stride, int64_t q_row_stride, int64_t q_head_stride, void* d_out,
                        int64_t out_seq_stride, int64_t out_row_stride, int64_t out_head_stride, float* d_lse, int B, int T, int n_q_heads,
                        const jot_kv_pages* pages, int layer, const int32_t* d_page_table, int64_t table_stride, int max_pages,
                        const int32_t* d_lens, float scale, void* d_workspace, size_t workspace_bytes, int32_t* d_status, void* stream) {
    JOT_TRY(check_kv_pages(pages, layer));
    if (B < 0 || T < 0 || n_q_heads <= 0 || max_pages < 0 || table_stride < 0) return JOT_ERR_ARG;
    if (B == 0 || T == 0) return JOT_OK;
    if (!d_q || !d_out || !d_lens || (max_pages > 0 && !d_page_table) || !aligned16(d_q) || !aligned16(d_out)) return JOT_ERR_ARG;
    if (!stride_ok(q_seq_stride, B) || !stride_ok(q_row_stride, T) || !stride_ok(q_head_stride, n_q_heads) || !stride_ok(out_seq_stride, B) ||
        !stride_ok(out_row_stride, T) || !stride_ok(out_head_stride, n_q_heads))
        return JOT_ERR_ARG;
    if (n_q_heads % pages->n_kv_heads || (pages->head_dim != 64 && pages->head_dim != 128)) return JOT_ERR_SHAPE;
    // (a scale of zero as the smallest number there is: every score is as good as zero all the same, and a key that is not there stays at minus infinity)
    const float scale_log2 = scale == 0.f ? FLT_TRUE_MIN : scale * 1.4426950408889634f;
    if (!std::isfinite(scale_log2)) return JOT_ERR_ARG;
    const int group = n_q_heads / pages->n_kv_heads;
    const int64_t rows = (int64_t)T * group;
    if (rows > INT32_MAX / 256 || (int64_t)T * n_q_heads > INT32_MAX / 32) return JOT_ERR_SHAPE;
    const int row_tile = paged_row_tile((int)rows), hd = pages->head_dim;
    const PagedSpace sp = paged_space(row_tile, hd);
    if (!d_workspace || !aligned16(d_workspace) || workspace_bytes < sp.total) return JOT_ERR_WORKSPACE;
    const int64_t row_tiles = (rows + row_tile - 1) / row_tile, items = row_tiles * pages->n_kv_heads;
    const int64_t most_keys = (int64_t)max_pages * pages->page_size;
    if (items > INT32_MAX || most_keys > INT32_MAX - kUmmaPagedTile) return JOT_ERR_SHAPE;
    // the line of tiles, were every sequence as long as its table allows, counted in 31 bits
    if ((most_keys / 64 + 1) * items > INT32_MAX / B) return JOT_ERR_SHAPE;
    DeviceInfo* di = nullptr;
    JOT_TRY(device_info(&di));
    PagedArgs a{};
    a.q = d_q; a.out = d_out; a.lse = d_lse;
    a.q_b = q_seq_stride; a.q_t = q_row_stride; a.q_h = q_head_stride;
    a.o_b = out_seq_stride; a.o_t = out_row_stride; a.o_h = out_head_stride;
    a.B = B; a.T = T; a.nq = n_q_heads; a.nkv = pages->n_kv_heads; a.group = group;
    a.pages = layer_pages(pages, layer);
    a.table = d_page_table; a.table_stride = table_stride; a.max_pages = max_pages; a.lens = d_lens;
    a.scale_log2 = scale_log2;
    uint8_t* ws = (uint8_t*)d_workspace;
    a.desc = (int4*)(ws + sp.desc); a.partial_ml = (float2*)(ws + sp.ml); a.partial = (float*)(ws + sp.partial);
    a.status = d_status;
    cudaStream_t st = (cudaStream_t)stream;
    if (pages->dtype == JOT_BF16)
        return hd == 128 ? launch_paged<__nv_bfloat16, 128>(di, a, row_tile, st) : launch_paged<__nv_bfloat16, 64>(di, a, row_tile, st);
    return hd == 128 ? launch_paged<__half, 128>(di, a, row_tile, st) : launch_paged<__half, 64>(di, a, row_tile, st);
}

}  // extern "C"

// Attention of a few new rows per sequence over the sequence's keys and values in the pages of a cache:
//
//   out[b, t, h] = sum_j softmax_j(scale q[b, t, h] . k_j) v_j,   lse[b, t, h] = ln sum_j exp(scale q . k_j),   j < lens[b]
//
// key j of sequence b in page table[b, j / page_size] at offset j % page_size.  Bidirectional: no mask but the length.  The
// rows of one key head (every new row of each of its query heads, row r = t * group + g) share its keys and are worked on
// together: up to 16 of them here, on mma.sync, for a token of each sequence or a few; more in paged_attention_umma.cuh.
//
// Bound by HBM for few rows (the cache is read once: 2 * head_dim * 2 bytes a key, for R rows 4 R head_dim flops).  Sequences are
// of any and unequal length, known on the device only, so the work is cut there: all tiles of 64 keys of all (sequence, key
// head, row tile) items form one line, and CTA i of G takes an equal share of it, whatever items that belongs to.  An item that lies in
// one CTA's share is finished there; one that spans several leaves, per CTA, the unnormalised fp32 output with its maximum and sum,
// which a second kernel joins.  Where a table row has room for a few tiles only, items are not cut and there is no second kernel.
// Nothing is added with atomics: a call gives the same bits every time.
//
// A CTA keeps three stages of 64 keys in flight (cp.async, 16 bytes a request, a page table entry and the rows' addresses fetched
// ahead), two CTAs an SM; its four warps have 16 keys of a stage each, and a maximum, a sum and an accumulator of their own until the
// item ends.  16-byte chunk c of a row sits at position c ^ (row mod 8): eight rows of one chunk are on eight different banks for
// ldmatrix.  Scores, statistics and accumulators are fp32; probabilities are rounded to the cache's type for the second product (the
// sum is taken before the rounding: the rounding's errors average out over the keys, and fp16's smallest numbers are out of their way, kPagedLift).
//
// One row of 28 query over 4 key heads for four sequences of 40007 to 131072 keys (700 MB): 116 us in a captured graph, 6.0 TB/s, 0.92 of the copy,
// and 118 to 128 a call in a stream of calls, by the board (0.84 to 0.91); what is left is the launch, the share's beginning and the second
// kernel (8 us together).  What it had been bound by: 920 instructions a warp and tile, most of them addresses (140 us); now 16 loads of
// operands, 32 products, 32 requests.  On tcgen05, whose tile of 128 rows would be 7 / 128 full, the same time, but a short call takes 2 us
// more, and pages that TMA cannot bring 168 us.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "heads.cuh"
#include "ptx.cuh"

namespace jot {

constexpr int kPagedThreads = 128;
constexpr int kPagedTile = 64;              // keys
constexpr int kPagedStages = 3;
constexpr int kPagedMaxCtas = 448;          // three per SM

struct PagedArgs {
    const void* q;
    void* out;
    float* lse;                             // [B, T, nq], nullable
    int64_t q_b, q_t, q_h, o_b, o_t, o_h;   // strides, elements
    int B, T, nq, nkv, group;
    PagesDev pages;
    const int32_t* table;                   // [B, table_stride], max_pages entries a row
    int64_t table_stride;
    int max_pages;
    const int32_t* lens;                    // [B]; 0: zeros come out; negative: the sequence's rows stay as they were
    float scale_log2;                       // scale * log2(e)
    bool whole;                             // items are not cut: shares are whole items, and nothing is left to join
    // workspace: one descriptor per CTA, then two partial results per CTA
    int4* desc;                             // (sequence, item within it, parts, share it begins in); parts 0: not cut
    bool by_item;                           // one per item (there are at most as many as shares), else one per share: the item that begins there
    float* partial;                         // [CTA][2][MT][HD] unnormalised outputs
    float2* partial_ml;                     // [CTA][2][MT] (reference of the exponentials in base 2, sum)
    int32_t* status;
};

// fp16 has no number below 2^-24: a row's exponentials are taken against a reference this far (in base 2) below its maximum, so that keys of 2^-25
// of the leading one and less, of which a long cache has many, count in the product as they do in the sum.  (tcgen05 lets probabilities grow by 2^8
// more before the reference follows: 2^15 together, and fp16 ends at 65504.)  The stored maximum of a part is its reference.
template <typename T> constexpr float kPagedLift = PackIsBf16<T>::value ? 0.f : 7.f;

template <typename T> struct MmaOp;
template <> struct MmaOp<__nv_bfloat16> {
    static __device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};
template <> struct MmaOp<__half> {
    static __device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};
__device__ __forceinline__ void ldmatrix4(uint32_t* r, uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t* r, uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
// 16 bytes global -> shared; without `real` zeros are written and nothing is read
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// one arrival on the barrier once all requests this thread has made so far have landed
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Keys of sequence b as the kernels count them: within what its table row can name.
__device__ __forceinline__ int paged_len(const PagedArgs& a, int b) {
    const int n = a.lens[b];
    const int64_t most = (int64_t)a.max_pages * a.pages.page_size;
    return n > most ? (int)most : n;
}

// The share of a CTA on the line of tiles (fewer than 2^31, which the host makes sure of), and where it begins.
struct PagedRange {
    int begin, end, total;          // tiles of the line
    int ctas;                       // CTAs, or streams of CTAs, that have a share
    int b, n, item, kt;             // sequence of the first tile, its keys; item within the sequence; tile within the item
};

// total tiles over `ctas` CTAs, the first total % ctas of them one more: where CTA i's begin, and whose tile t is
__host__ __device__ __forceinline__ int paged_share(int total, int ctas, int i) { return total / ctas * i + (i < total % ctas ? i : total % ctas); }
__host__ __device__ __forceinline__ int paged_owner(int total, int ctas, int t) {
    const int q = total / ctas, longer = total % ctas, edge = longer * (q + 1);
    return t < edge ? t / (q + 1) : longer + (t - edge) / q;
}

struct PagedRangeSmem {
    int warp_tot[16], b[2], in_seq[2];
};

// The line of tiles of `tile` keys, per_b items a sequence, and the share of it that this thread's stream has: stream `mine` of the
// STREAMS that each CTA runs.  Sequences without a key are answered here: zeros, and the logarithm of nothing.  All THREADS threads of
// the CTA call it; lens is read after the preceding kernel's end.
template <typename T, int HD, int THREADS, int STREAMS>
__device__ __forceinline__ PagedRange paged_range(const PagedArgs& a, int tile, int per_b, int mine, PagedRangeSmem& sm) {
    constexpr int WARPS = THREADS / 32, CPR = HD / 8;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    bool empty = false;             // whether a sequence of this thread has no key
    auto tiles_of = [&](int b) -> int {
        if (b >= a.B) return 0;
        const int n = paged_len(a, b);
        empty |= n == 0;
        if (blockIdx.x == 0 && a.status && a.lens[b] > (int64_t)a.max_pages * a.pages.page_size) report_bad_index(a.status);
        return n > 0 ? (a.whole ? per_b : (n + tile - 1) / tile * per_b) : 0;
    };
    auto scan = [&](int v) {        // inclusive, over the warp
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += up;
        }
        return v;
    };
    PagedRange rg;
    int in_seq = 0;
    const int first = tiles_of(a.B <= 32 ? lane : tid);
    auto cut = [](int total, int stream, int& begin, int& end) {
        const int ctas = min((int)gridDim.x * STREAMS, total), i = stream * gridDim.x + blockIdx.x;
        begin = i < ctas ? paged_share(total, ctas, i) : 0;
        end = i < ctas ? paged_share(total, ctas, i + 1) : 0;
        return ctas;
    };
    rg.b = 0;
    if (a.B <= 32) {                // every warp for itself
        const int inc = scan(first);
        rg.total = __shfl_sync(0xffffffffu, inc, 31);
        empty = __any_sync(0xffffffffu, empty);
        rg.ctas = cut(rg.total, mine, rg.begin, rg.end);
        if (rg.end > rg.begin) {
            rg.b = __popc(__ballot_sync(0xffffffffu, inc <= rg.begin));        // sequences that end before it
            in_seq = rg.begin - __shfl_sync(0xffffffffu, inc - first, rg.b);
        }
    } else {
        int sum = first;
        for (int b = tid + THREADS; b < a.B; b += THREADS) sum += tiles_of(b);
        sum = scan(sum);
        if (lane == 31) sm.warp_tot[warp] = sum;
        empty = __syncthreads_or(empty);
        auto totals = [&](int warps) {
            int t = 0;
            for (int w = 0; w < warps; ++w) t += sm.warp_tot[w];
            return t;
        };
        rg.total = totals(WARPS);
        rg.ctas = cut(rg.total, mine, rg.begin, rg.end);
        int before = 0;
        for (int b0 = 0; b0 < a.B; b0 += THREADS) {
            const int tiles = b0 == 0 ? first : tiles_of(b0 + tid), inc = scan(tiles);
            __syncthreads();                                        // warp_tot is read by everyone before it is written again
            if (lane == 31) sm.warp_tot[warp] = inc;
            __syncthreads();
            const int start = before + totals(warp) + inc - tiles;
#pragma unroll
            for (int i = 0; i < STREAMS; ++i) {
                int begin, end;
                cut(rg.total, i, begin, end);
                if (start <= begin && begin < start + tiles && begin < end) {
                    sm.b[i] = b0 + tid;
                    sm.in_seq[i] = begin - start;
                }
            }
            before += totals(WARPS);
        }
        __syncthreads();
        if (rg.end > rg.begin) {
            rg.b = sm.b[mine];
            in_seq = sm.in_seq[mine];
        }
    }
    rg.n = rg.item = rg.kt = 0;
    if (rg.end > rg.begin) {
        rg.n = paged_len(a, rg.b);
        const int nt = (rg.n + tile - 1) / tile;
        rg.item = a.whole ? in_seq : in_seq / nt;
        rg.kt = a.whole ? 0 : in_seq - rg.item * nt;
        if (a.whole) {              // a share of items so far: how many tiles that is
            int left = rg.end - rg.begin, tiles = 0;
            for (int b = rg.b, from = rg.item; left > 0; ++b) {
                const int n = paged_len(a, b);
                if (n <= 0) continue;
                const int items = min(per_b - from, left);
                tiles += items * ((n + tile - 1) / tile);
                left -= items;
                from = 0;
            }
            rg.begin = 0;
            rg.end = tiles;
        }
    }
    for (int b = blockIdx.x; empty && b < a.B; b += gridDim.x) {
        if (paged_len(a, b) != 0) continue;
        for (int i = tid; i < a.T * a.nq * CPR; i += THREADS) {
            const int row = i / CPR, t = row / a.nq, h = row - t * a.nq;
            reinterpret_cast<uint4*>((T*)a.out + b * a.o_b + t * a.o_t + h * a.o_h)[i % CPR] = make_uint4(0, 0, 0, 0);
            if (i % CPR == 0 && a.lse) a.lse[(int64_t)b * a.T * a.nq + row] = -INFINITY;
        }
    }
    return rg;
}

// What the second kernel has to know of an item that begins in `share`, whose last `behind` tiles lie behind the share's end.
__device__ __forceinline__ void paged_describe(const PagedArgs& a, const PagedRange& rg, int share, int per_b, int b, int item, int behind) {
    const int parts = behind > 0 ? paged_owner(rg.total, rg.ctas, rg.end + behind - 1) - share + 1 : 0;
    if (a.by_item) a.desc[b * per_b + item] = make_int4(b, item, parts, share);
    else if (parts > 0) a.desc[share] = make_int4(b, item, parts, share);
}

// What a CTA of the second kernel joins, and whether there is anything: by item, a descriptor that nobody has written (its CTA gave up on a wait)
// holds whatever the workspace held, so the item follows from the CTA alone, and parts that are not all in the workspace are left alone.
struct PagedJoin {
    int b, item, parts, share;
};
__host__ __device__ __forceinline__ bool paged_join_of(int4 d, bool by_item, int cta, int per_b, int shares, PagedJoin& j) {
    j = by_item ? PagedJoin{cta / per_b, cta % per_b, d.z, d.w} : PagedJoin{d.x, d.y, d.z, d.w};
    return j.parts > 0 && j.share >= 0 && j.share < shares && j.parts <= shares - j.share;
}

template <int HD>
struct PagedSmem {
    static constexpr int TILE_BYTES = kPagedTile * HD * 2;                       // K or V of one stage
    static constexpr int STAGE_BYTES = 2 * TILE_BYTES;
    static constexpr int MERGE_BYTES = 64 * (HD / 4) * 4;                        // WK * MT = 64 rows of a quarter of the columns
    static constexpr int DYN_BYTES = kPagedStages * STAGE_BYTES + MERGE_BYTES;
};

template <typename T, int HD>
__global__ void __launch_bounds__(kPagedThreads) paged_attention_kernel(const PagedArgs a) {
    using SM = PagedSmem<HD>;
    constexpr int MT = 16, WK = 4, KW = kPagedTile / WK;                // rows; ranges of keys, a warp's each; keys of a range
    constexpr int NT = KW / 8, KS = HD / 16, DT = HD / 8;               // score tiles, steps of the first product, output tiles
    constexpr int CPR = HD / 8;                                         // 16-byte chunks of a key
    extern __shared__ __align__(128) uint8_t smem[];
    float* merge = reinterpret_cast<float*>(smem + kPagedStages * SM::STAGE_BYTES);
    __shared__ float2 ml[WK][MT];
    __shared__ uint64_t row_at[2][2 * kPagedTile];                      // addresses of a tile's key rows, then of its value rows
    __shared__ PagedRangeSmem range_smem;

    grid_launch_dependents();
    grid_dependency_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int R = a.T * a.group, RT = (R + MT - 1) / MT;
    const int per_b = a.nkv * RT;                                       // items of a sequence

    const PagedRange rg = paged_range<T, HD, kPagedThreads, 1>(a, kPagedTile, per_b, 0, range_smem);
    if (tid == 0 && !a.by_item) a.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
    if ((int)blockIdx.x >= rg.ctas) return;

    // ---- loads: a walk over the tiles of the share ----
    // Three steps a tile, each one tile behind the one before: a page table entry is requested; the addresses of a key and of a
    // value row are left in shared memory (thread i < 64: key i, thread 64 + i: value i); the tile is requested.  So no step
    // waits for the one it needs, and a request costs a thread one shared-memory read and one add.
    const uint32_t s0 = smem_u32(smem);
    int lb = rg.b, ln = rg.n, lkt = rg.kt, litem = rg.item;             // sequence, its keys, tile, item (head * RT + row tile)
    int lleft = rg.end - rg.begin;                                      // tiles whose table entry is yet to be requested
    const int64_t page_stride = tid < kPagedTile ? a.pages.k_page : a.pages.v_page;
    const T* const pages = (const T*)(tid < kPagedTile ? a.pages.k : a.pages.v);
    int page = 0, in_page = 0;                                          // of this thread's row in the tile last requested; -1: no such key
    bool exists = false;
    auto request_entry = [&]() {
        exists = false;
        if (lleft <= 0) return;
        const int key = lkt * kPagedTile + (tid & (kPagedTile - 1));
        if (key < ln) {
            const int p = key / a.pages.page_size;
            in_page = (litem / RT) * a.pages.page_size + key - p * a.pages.page_size;
            page = a.table[lb * a.table_stride + p];
            exists = true;
        }
        --lleft;
        if ((lkt + 1) * kPagedTile < ln) {
            ++lkt;
        } else {
            lkt = 0;
            if (++litem == per_b) {
                litem = 0;
                if (lleft > 0) do { ++lb; ln = paged_len(a, lb); } while (ln <= 0);
            }
        }
    };
    auto leave_address = [&](int buf) {                                 // an odd address: no such row, zeros are written
        uint64_t at = reinterpret_cast<uint64_t>(pages) | 1u;
        if (exists) {
            if ((unsigned)page < (unsigned)a.pages.n_pages)
                at = reinterpret_cast<uint64_t>(pages + page * page_stride + (int64_t)in_page * HD);
            else if (a.status)
                report_bad_index(a.status);
        }
        row_at[buf][tid] = at;
    };
    constexpr int RPP = 32 / CPR;                                       // rows per request of a warp
    const int lr = lane / CPR, lc = lane % CPR;
    uint32_t ldst[8 / RPP];                                             // where this lane's chunk goes: repeats every 8 rows
#pragma unroll
    for (int i = 0; i < 8 / RPP; ++i) ldst[i] = (uint32_t)((warp * 16 + i * RPP + lr) * (HD * 2) + ((lc ^ ((i * RPP + lr) & 7)) << 4));
    auto request_tile = [&](int stage, int buf) {
        const uint32_t sk = s0 + stage * SM::STAGE_BYTES;
#pragma unroll
        for (int i = 0; i < 16 / RPP; ++i) {
            const int r = warp * 16 + i * RPP + lr;
            const uint32_t d = sk + ldst[i % (8 / RPP)] + (i * RPP / 8) * 8 * (HD * 2);
            const uint64_t kp = row_at[buf][r], vp = row_at[buf][kPagedTile + r];
            cp_async16(d, reinterpret_cast<const uint8_t*>(kp & ~1ull) + lc * 16, !(kp & 1));
            cp_async16(d + SM::TILE_BYTES, reinterpret_cast<const uint8_t*>(vp & ~1ull) + lc * 16, !(vp & 1));
        }
    };
    const int share = rg.end - rg.begin;
    int requested = 0;                                                  // tiles
    request_entry();
    leave_address(0);
    request_entry();
#pragma unroll
    for (int s = 0; s < kPagedStages - 1; ++s) {
        __syncthreads();
        if (requested < share) request_tile(s, s & 1);
        cp_async_commit();
        ++requested;
        leave_address((s + 1) & 1);
        request_entry();
    }

    // ---- products ----
    const int g = lane >> 2, t4 = lane & 3;
    // operand addresses within a tile: a lane's row, and the swizzled position of chunk 2 i (+ 1) for i < 4; the next four lie 128 bytes on
    uint32_t kofs[4], vofs[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        kofs[i] = (uint32_t)(((lane & 7) + ((lane >> 4) << 3)) * (HD * 2) + (((2 * i + ((lane >> 3) & 1)) ^ (lane & 7)) << 4));
        vofs[i] = (uint32_t)(((lane & 7) + (((lane >> 3) & 1) << 3)) * (HD * 2) + (((2 * i + (lane >> 4)) ^ (lane & 7)) << 4));
    }
    int b = rg.b, n = rg.n, nt = (n + kPagedTile - 1) / kPagedTile, item = rg.item, kt = rg.kt;
    int stage = 0;
    for (int left = rg.end - rg.begin; left > 0;) {
        const int head = item / RT, row0 = (item - head * RT) * MT;
        const int kt_first = kt, kt_end = min(nt, kt + left);
        // queries of this warp's 16 rows as operand fragments; rows past R are zeros
        uint32_t qf[KS][4];
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            const int r = row0 + g + 8 * hh, t = r / a.group, gq = r - t * a.group;
            const T* qp = (const T*)a.q + b * a.q_b + (int64_t)t * a.q_t + (int64_t)(head * a.group + gq) * a.q_h;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                qf[ks][hh] = r < R ? *reinterpret_cast<const uint32_t*>(qp + ks * 16 + 2 * t4) : 0u;
                qf[ks][2 + hh] = r < R ? *reinterpret_cast<const uint32_t*>(qp + ks * 16 + 8 + 2 * t4) : 0u;
            }
        }
        float o[DT][4], mx[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d][0] = o[d][1] = o[d][2] = o[d][3] = 0.f;

        for (; kt < kt_end; ++kt, --left) {
            cp_async_wait<kPagedStages - 2>();
            __syncthreads();                                            // the tile is there, and the stage before it is free
            if (requested < share) request_tile(stage == 0 ? kPagedStages - 1 : stage - 1, requested & 1);
            cp_async_commit();
            ++requested;
            leave_address(requested & 1);
            request_entry();
            const uint32_t sk = s0 + stage * SM::STAGE_BYTES + warp * KW * (HD * 2), sv = sk + SM::TILE_BYTES;
            if (++stage == kPagedStages) stage = 0;
            float s[NT][4];
#pragma unroll
            for (int j = 0; j < NT; ++j) s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int j = 0; j < NT; j += 2) {
                    uint32_t kb[4];
                    ldmatrix4(kb, sk + kofs[ks % 4] + (ks / 4) * 128 + j * 8 * (HD * 2));
                    MmaOp<T>::mma(s[j], qf[ks], kb[0], kb[1]);
                    MmaOp<T>::mma(s[j + 1], qf[ks], kb[2], kb[3]);
                }
            const int limit = n - kt * kPagedTile - warp * KW;            // keys of the range that exist
            float top[2] = {mx[0], mx[1]};
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[j][e] *= a.scale_log2;
            if (limit < KW) {
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (j * 8 + 2 * t4 + (e & 1) >= limit) s[j][e] = -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) top[e >> 1] = fmaxf(top[e >> 1], s[j][e]);
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                top[hh] = fmaxf(top[hh], __shfl_xor_sync(0xffffffffu, top[hh], 1));
                top[hh] = fmaxf(top[hh], __shfl_xor_sync(0xffffffffu, top[hh], 2));
            }
            float base[2] = {top[0] == -INFINITY ? 0.f : top[0] - kPagedLift<T>, top[1] == -INFINITY ? 0.f : top[1] - kPagedLift<T>};   // no key yet: all exponentials are zero
            if (__any_sync(0xffffffffu, top[0] != mx[0] || top[1] != mx[1])) {
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const float f = ex2_approx(mx[hh] - kPagedLift<T> - base[hh]);
                    mx[hh] = top[hh];
                    sum[hh] *= f;
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        o[d][2 * hh] *= f;
                        o[d][2 * hh + 1] *= f;
                    }
                }
            }
            uint32_t p[NT / 2][4];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                float e[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) e[x] = ex2_approx(s[j][x] - base[x >> 1]);
                sum[0] += e[0] + e[1];
                sum[1] += e[2] + e[3];
                typename Pack2<T>::type lo = Pack2<T>::down(e[0], e[1]), hi = Pack2<T>::down(e[2], e[3]);
                p[j >> 1][(j & 1) * 2] = *reinterpret_cast<uint32_t*>(&lo);
                p[j >> 1][(j & 1) * 2 + 1] = *reinterpret_cast<uint32_t*>(&hi);
            }
#pragma unroll
            for (int j = 0; j < NT / 2; ++j)
#pragma unroll
                for (int d = 0; d < DT; d += 2) {
                    uint32_t vb[4];
                    ldmatrix4_trans(vb, sv + vofs[d / 2 % 4] + (d / 8) * 128 + j * 16 * (HD * 2));
                    MmaOp<T>::mma(o[d], p[j], vb[0], vb[1]);
                    MmaOp<T>::mma(o[d + 1], p[j], vb[2], vb[3]);
                }
        }

        // ---- the ranges of keys meet; the item, or this CTA's part of it, goes out ----
        const bool begins = kt_first == 0, ends = kt_end == nt;
        const int slot = (int)blockIdx.x * 2 + (begins ? 1 : 0);
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            sum[hh] += __shfl_xor_sync(0xffffffffu, sum[hh], 1);
            sum[hh] += __shfl_xor_sync(0xffffffffu, sum[hh], 2);
            mx[hh] -= kPagedLift<T>;                                    // from here on the reference
            if (t4 == 0) ml[warp][g + 8 * hh] = make_float2(mx[hh], sum[hh]);
        }
        __syncthreads();
        float mine[2];                                                  // what this warp's accumulators are multiplied by
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            float m = -INFINITY;
#pragma unroll
            for (int w = 0; w < WK; ++w) m = fmaxf(m, ml[w][g + 8 * hh].x);
            mine[hh] = m == -INFINITY ? 1.f : ex2_approx(mx[hh] - m);
        }
        auto totals = [&](int r, float& m, float& l) {
            m = -INFINITY;
            l = 0.f;
#pragma unroll
            for (int w = 0; w < WK; ++w) m = fmaxf(m, ml[w][r].x);
#pragma unroll
            for (int w = 0; w < WK; ++w) l += ml[w][r].y * (m == -INFINITY ? 1.f : ex2_approx(ml[w][r].x - m));
        };
        if (tid < MT && row0 + tid < R) {
            float m, l;
            totals(tid, m, l);
            const int r = row0 + tid, t = r / a.group, gq = r - t * a.group;
            if (begins && ends) {
                if (a.lse) a.lse[((int64_t)b * a.T + t) * a.nq + head * a.group + gq] = (m + log2f(l)) * 0.69314718055994531f;
            } else {
                a.partial_ml[(int64_t)slot * MT + tid] = make_float2(m, l);
            }
        }
        constexpr int QC = HD / 4, QD = DT / 4;                         // columns and output tiles of a quarter
#pragma unroll
        for (int quarter = 0; quarter < 4; ++quarter) {
#pragma unroll
            for (int d = 0; d < QD; ++d)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh)
                    *reinterpret_cast<float2*>(merge + ((warp * MT + g + 8 * hh) * QC + d * 8 + 2 * t4)) =
                        make_float2(o[quarter * QD + d][2 * hh] * mine[hh], o[quarter * QD + d][2 * hh + 1] * mine[hh]);
            __syncthreads();
            for (int i = tid; i < MT * (QC / 8); i += kPagedThreads) {
                const int r = i / (QC / 8), c = (i % (QC / 8)) * 8;
                if (row0 + r >= R) continue;
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = 0.f;
#pragma unroll
                for (int w = 0; w < WK; ++w)
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] += merge[(w * MT + r) * QC + c + e];
                if (begins && ends) {
                    float m, l;
                    totals(r, m, l);
                    const float inv = 1.f / l;
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] *= inv;
                    const int rr = row0 + r, t = rr / a.group, gq = rr - t * a.group;
                    *reinterpret_cast<uint4*>((T*)a.out + b * a.o_b + (int64_t)t * a.o_t + (int64_t)(head * a.group + gq) * a.o_h + quarter * QC + c) = pack8<T>(x);
                } else {
                    float4* dst = reinterpret_cast<float4*>(a.partial + ((int64_t)slot * MT + r) * HD + quarter * QC + c);
                    dst[0] = make_float4(x[0], x[1], x[2], x[3]);
                    dst[1] = make_float4(x[4], x[5], x[6], x[7]);
                }
            }
            __syncthreads();
        }
        if (begins && tid == 0) paged_describe(a, rg, blockIdx.x, per_b, b, item, nt - kt_end);
        // next item
        kt = 0;
        if (++item == per_b && left > 0) {
            item = 0;
            do { ++b; n = paged_len(a, b); } while (n <= 0);
            nt = (n + kPagedTile - 1) / kPagedTile;
        }
    }
    cp_async_wait<0>();
}

// Joins the parts of the items that several CTAs worked on.  blockIdx.x: the descriptor; WPR warps share a row, a part of the parts each, a
// lane HD / 32 columns.
template <typename T, int HD, int WPR>
__global__ void __launch_bounds__(kPagedThreads) paged_join_kernel(const PagedArgs a, int MT, int shares) {
    grid_launch_dependents();
    grid_dependency_wait();
    constexpr int E = HD / 32;
    __shared__ float so[WPR > 1 ? 4 : 1][HD];
    __shared__ float2 sml[4];
    const int R = a.T * a.group, RT = (R + MT - 1) / MT;
    if (a.by_item && paged_len(a, blockIdx.x / (a.nkv * RT)) <= 0) return;      // nobody had this item
    PagedJoin d;
    if (!paged_join_of(a.desc[blockIdx.x], a.by_item, blockIdx.x, a.nkv * RT, shares, d)) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int head = d.item / RT, row0 = (d.item - head * RT) * MT;
    const int r = blockIdx.y * (4 / WPR) + warp / WPR;
    if (r >= min(MT, R - row0)) return;                                 // (with WPR = 4 all of the CTA's warps have this row)
    float m = -INFINITY, l = 0.f, o[E] = {};
#pragma unroll 4
    for (int f = warp % WPR; f < d.parts; f += WPR) {
        const int64_t at = (f == 0 ? (int64_t)d.share * 2 + 1 : (int64_t)(d.share + f) * 2) * MT + r;
        const float2 p = a.partial_ml[at];
        float x[E];
#pragma unroll
        for (int e = 0; e < E; e += 2) *reinterpret_cast<float2*>(x + e) = *reinterpret_cast<const float2*>(a.partial + at * HD + lane * E + e);
        const float top = fmaxf(m, p.x), base = top == -INFINITY ? 0.f : top;
        const float fo = ex2_approx(m - base), fn = ex2_approx(p.x - base);
        m = top;
        l = l * fo + p.y * fn;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * fo + x[e] * fn;
    }
    if (WPR > 1) {
#pragma unroll
        for (int e = 0; e < E; ++e) so[warp][lane * E + e] = o[e];
        if (lane == 0) sml[warp] = make_float2(m, l);
        __syncthreads();
        if (warp != 0) return;
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) m = fmaxf(m, sml[w].x);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = m == -INFINITY ? 1.f : ex2_approx(sml[w].x - m);
            l += sml[w].y * f;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] += so[w][lane * E + e] * f;
        }
    }
    const float inv = 1.f / l;
    const int rr = row0 + r, t = rr / a.group, gq = rr - t * a.group;
    T* out = (T*)a.out + d.b * a.o_b + (int64_t)t * a.o_t + (int64_t)(head * a.group + gq) * a.o_h + lane * E;
#pragma unroll
    for (int e = 0; e < E; e += 2) *reinterpret_cast<typename Pack2<T>::type*>(out + e) = Pack2<T>::down(o[e] * inv, o[e + 1] * inv);
    if (lane == 0 && a.lse) a.lse[((int64_t)d.b * a.T + t) * a.nq + head * a.group + gq] = (m + log2f(l)) * 0.69314718055994531f;
}

}  // namespace jot

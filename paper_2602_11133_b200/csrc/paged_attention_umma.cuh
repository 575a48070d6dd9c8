// Attention over the pages of a cache for more rows of a key head than a warp's matrix instruction holds, on tcgen05: the same
// line of tiles, shares and joined parts as paged_attention.cuh, tiles of 128 keys.
//
//   S = Q K^T, P = exp2(S c - m) written over S in tensor memory, O += P V, with Q, K, V in shared memory as their rows are in the
//   pages: the head dimension runs along 128-byte rows (16-byte chunk c of row r at c ^ (r mod 8)), which is the first product's
//   K-major operand for Q and K, and for V the second product's MN-major one, so nothing is transposed.
//
// Two streams share the tensor pipe, each with a score buffer, an accumulator, a warpgroup (thread = row) and a warp that issues its
// products: while one stream's rows are in exponentials, or on their way out, the other's products run.
//   ROWS <= 128   each stream has a share of the line to itself, with queries and a stage of keys and values of its own, as if it were a CTA.
//                 With at most 64 or 32 rows the tile of 128 holds them twice or four times over, and each copy's threads take their
//                 share of a tile's keys (the probabilities of the others are zeros): what a thread has to do for a tile, which is what
//                 few rows wait for, is a half or a quarter.  The copies are added up at the end.
//   ROWS = 256    the streams are two tiles of 128 rows over the same keys, and take turns in their exponentials: at the same time, they
//                 would only get half of the special function units each, and then both wait for the tensor pipe (512 rows over 512 keys
//                 63.4 us in turns, 67.1 without; longer ones the same).
// Where a thread has a whole row (128 or 256 rows) a stream has two score buffers of 64 keys, and the scores of one are made while the
// probabilities of the other are: a thread's chain is its exponentials alone.
// The reference of a row's exponentials, its maximum (in fp16 less kPagedLift), follows a tile's maximum only when that exceeds the one it was taken
// from by more than 2^8 (probabilities up to 256 are as exact as those up to 1); then the row of the accumulator is rescaled in tensor memory.
//
// Pages of a multiple of 8 keys come by TMA (one box per page and 64 columns; a tile is as many whole pages as fit into 128 rows, or
// 128 keys of a larger page), others by cp.async, 16 bytes a request, which costs four warps and the rate at which an SM takes
// such requests.
//
//   warps 0-3, 4-7   softmax of stream 0 and 1
//   by TMA           warps 8, 9 keys and values of a stream each (ROWS = 256: warp 8 of both), warps 10, 11 products
//   by cp.async      warps 8-11 keys and values (ROWS <= 128: two a stream), warps 12, 13 products
// The softmax warps bring the queries themselves, when a part begins: their room is the one that the previous part has left through.
//
// 32 rows of 32 heads of 16 sequences of 384 to 704 keys (143 MB): 45 us, 3.3 TB/s; bound by the chain a short item is (queries, first
// scores, exponentials, second product, way out: 11 to 12 us for its four tiles), which two streams hide half of.  Before: 59.5 us on
// mma.sync in tiles of 32 rows, 66 as one stream of even and odd tiles, which ended its items together.
// 224 rows a key head of eight sequences of 2001 to 9001 keys (20 GFLOP): 49 us, 410 TFLOP/s; bound by the exponentials' chain (1.45k cycles for
// 64 keys of 128 rows, 0.6k of them until the stores to tensor memory are done, which share it with the other products) and by start and end
// of a part (8k cycles); 104 us on mma.sync, 51.5 with one score buffer of 128 keys.  Canvases of 704 rows over 704 keys, 32 heads
// of 16 sequences: 202 us, 640 TFLOP/s.  With keys by cp.async (pages of 100 keys) the first two take 51 and 47 us.
// Registers: 168 a thread with 384 threads, of which 128 columns with 32 and 64 rows exceed by 32 and 20 bytes of local memory; 128 with 448 threads
// (by cp.async), by 20 to 168 bytes in all forms but 64 columns with 256 rows.
//
// Every barrier is waited on phase by phase by whoever waits on it, so that a parity says which phase is meant.  All waits end: one
// that gives up makes the CTA leave, after its copies and products under way have ended.
#pragma once
#include "paged_attention.cuh"

namespace jot {

constexpr int kUmmaPagedTile = 128;        // rows of a tile of keys in shared memory
constexpr int kUmmaPagedMaxCtas = 160;     // one per SM

template <int HD>
struct UmmaPagedSmem {
    static constexpr int TILE_BYTES = 128 * HD * 2;               // 128 rows: a tile of Q, K or V
    static constexpr int STAGES = HD == 128 ? 2 : 4;              // of K and of V
    static constexpr int DYN_BYTES = (2 + 2 * STAGES) * TILE_BYTES + 1024;      // and the streams' tiles of queries
};

template <int ROWS, bool TMA>
struct UmmaPagedRoles {
    static constexpr bool TWO = ROWS == 256;
    static constexpr int PROD = 8, PROD_WARPS = TMA ? 1 : (TWO ? 4 : 2);       // of a stream (TWO: of both)
    static constexpr int MMA = TMA ? 10 : 12, THREADS = TMA ? 384 : 448;
};
// Keys of a tile that TMA brings, and whether it can: whole pages in 128 rows, or parts of 128 of a page.  Pages of 72 to 120 keys leave up to 44 % of a
// tile empty; 32 rows of 32 heads are the faster for it all the same (48.5 us at 72 keys, 42.9 at 120; by cp.async 51.5), 224 rows from 120 keys on
// (60.3 us at 72, 52.3 at 96, 46.7 at 120; by cp.async 47.4).
__host__ __device__ constexpr bool paged_tma_pages(int page_size) { return page_size % 8 == 0 && (page_size <= 128 || page_size % 128 == 0); }
__host__ __device__ constexpr int paged_tma_keys(int page_size) { return page_size <= 128 ? 128 / page_size * page_size : 128; }

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int c0, int c1, int c2, int c3) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
        : "memory");
}

// Operand descriptor of an MN-major tile in rows of 64 elements (128 bytes, 128-byte swizzle), 16 KB from one run of 64 to the next:
// groups of eight rows along K are 1024 bytes apart.
__device__ __forceinline__ uint64_t umma_desc_mn128(uint32_t smem_addr) {
    uint64_t d = 0;
    d |= static_cast<uint64_t>((smem_addr & 0x3FFFFu) >> 4);
    d |= static_cast<uint64_t>(16384 >> 4) << 16;                 // from one run of 64 elements to the next
    d |= static_cast<uint64_t>(1024 >> 4) << 32;                  // from one group of eight rows to the next
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;
    return d;
}
template <typename T>
__host__ __device__ constexpr uint32_t umma_idesc16(int M, int N, bool b_mn_major) {
    const uint32_t fmt = PackIsBf16<T>::value ? 1u : 0u;
    return (1u << 4) | (fmt << 7) | (fmt << 10) | (uint32_t(b_mn_major) << 16) | (uint32_t(N >> 3) << 17) | (uint32_t(M >> 4) << 24);
}

// The parts of items that a share consists of, in order.
struct PagedWalk {
    int b, n, nt, item, kt, cnt;          // sequence, its keys and tiles, item, first tile and number of tiles of this part
    int left;                             // tiles of the share from this part on
    __device__ __forceinline__ PagedWalk(const PagedRange& rg, int tile) {
        b = rg.b;
        n = rg.n;
        nt = (n + tile - 1) / tile;
        item = rg.item;
        kt = rg.kt;
        left = rg.end - rg.begin;
        cnt = min(nt - kt, left);
    }
    __device__ __forceinline__ bool next(const PagedArgs& a, int per_b, int tile) {
        left -= cnt;
        if (left <= 0) return false;
        kt = 0;
        if (++item == per_b) {
            item = 0;
            do { ++b; n = paged_len(a, b); } while (n <= 0);
            nt = (n + tile - 1) / tile;
        }
        cnt = min(nt, left);
        return true;
    }
};

template <typename T, int HD, int ROWS, bool TMA>
__global__ void __launch_bounds__(UmmaPagedRoles<ROWS, TMA>::THREADS, 1)
paged_attention_umma_kernel(const PagedArgs a, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV) {
    using SM = UmmaPagedSmem<HD>;
    using Role = UmmaPagedRoles<ROWS, TMA>;
    constexpr bool TWO = Role::TWO;
    constexpr int KB = HD / 64, ST = SM::STAGES, RING = TWO ? ST : ST / 2, TILE = kUmmaPagedTile, THREADS = Role::THREADS;
    constexpr int STREAMS = TWO ? 1 : 2;                          // shares of the line a CTA has
    constexpr int REP = TWO ? 1 : 128 / ROWS, KC = 128 / REP;     // copies of a row, and keys of a tile that one takes
    constexpr int HV = KC == 128 ? 2 : 1, HK = 128 / HV;          // score buffers of a stream, and keys of one
    constexpr uint32_t IDESC_S = umma_idesc16<T>(128, HK, false), IDESC_O = umma_idesc16<T>(128, HD, true);
    constexpr uint32_t O_COL = 256;              // scores of the streams at columns 0 and 128, accumulators at 256 and 384
    constexpr float kRaise = 8.f + kPagedLift<T>;

    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t sQ = smem_u32(smem), sK = sQ + 2 * SM::TILE_BYTES, sV = sK + ST * SM::TILE_BYTES;
    uint8_t* const values_at = smem + (2 + ST) * SM::TILE_BYTES;
    __shared__ uint64_t k_full[ST], k_empty[ST], v_full[ST], v_empty[ST], q_full[2], s_full[2][HV], p_full[2][HV], pv_done[2][HV], o_empty[2],
        drain[2], turn[2], tail_bar, prod_bar[2], g_bar[2];
    __shared__ uint64_t row_at[TMA ? 1 : STREAMS][2][TMA ? 1 : 2 * TILE];      // by cp.async: addresses of a tile's key rows, then of its value rows; odd: no such row
    __shared__ uint64_t row_q[2][128], row_o[2][2][128];     // addresses of the rows' queries, and of their results ([parity of the part])
    __shared__ float2 x_ml[2][REP > 1 ? 128 : 1];            // [stream][row] (reference, sum) of the copies
    __shared__ PagedRangeSmem range_smem;
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag, drain_flag;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        abort_flag = drain_flag = 0;
        for (int i = 0; i < ST; ++i) {
            mbar_init(&k_full[i], TMA ? 1 : Role::PROD_WARPS * 32);          // by cp.async: every producer thread's requests
            mbar_init(&k_empty[i], TWO ? 2 : 1);                             // every stream that uses the tile
            mbar_init(&v_full[i], TMA ? 1 : Role::PROD_WARPS * 32);
            mbar_init(&v_empty[i], TWO ? 2 : 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], 128);                                      // every softmax thread's requests
            for (int h = 0; h < HV; ++h) {
                mbar_init(&s_full[i][h], 1);
                mbar_init(&p_full[i][h], 4);
                mbar_init(&pv_done[i][h], 1);
            }
            mbar_init(&o_empty[i], 4);
            mbar_init(&drain[i], 1);
            mbar_init(&turn[i], 4);
            mbar_init(&prod_bar[i], Role::PROD_WARPS);
            mbar_init(&g_bar[i], 4);
        }
        mbar_init(&tail_bar, 2);
        fence_barrier_init();
        fence_proxy_async_smem();
        if (TMA) {
            tma_prefetch_desc(&tmK);
            tma_prefetch_desc(&tmV);
        }
    }
    const int KEYS = TMA ? paged_tma_keys(a.pages.page_size) : TILE;       // of a tile
    if (TMA && KEYS < TILE) {                    // value rows that no box covers: their probabilities are zero, so they must be numbers
        for (int t = 0; t < ST * KB; ++t)
            for (int i = tid; i < (TILE - KEYS) * 8; i += THREADS) reinterpret_cast<uint4*>(values_at + t * 16384 + KEYS * 128)[i] = make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();
    }
    if (warp == Role::MMA) {
        tmem_alloc(&tmem_base_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = tmem_base_slot;
    volatile int* abortp = &abort_flag;
    // (only now: a successor that starts early and takes tensor memory must not be able to take this CTA's)
    grid_launch_dependents();
    grid_dependency_wait();

    const int R = a.T * a.group, RT = (R + ROWS - 1) / ROWS, per_b = a.nkv * RT;
    // the stream of this warp (TWO: 0 for the producers, who serve both)
    const int s = warp < 8 ? warp >> 2 : (warp >= Role::MMA ? warp - Role::MMA : (TWO ? 0 : (warp - Role::PROD) / Role::PROD_WARPS));
    const PagedRange rg = paged_range<T, HD, THREADS, STREAMS>(a, KEYS, per_b, TWO ? 0 : s, range_smem);
    const int share = (TWO ? 0 : s) * gridDim.x + blockIdx.x;      // first one for every CTA, then a second
    if (tid < STREAMS && !a.by_item) a.desc[tid * gridDim.x + blockIdx.x] = make_int4(0, 0, 0, 0);
    __syncthreads();                             // (a descriptor is written again below)
    auto wait_all = [&](uint64_t* bar, uint32_t parity) -> bool {
        const bool w = mbar_wait(bar, parity, abortp);
        return __all_sync(0xffffffffu, w);
    };

    if (rg.end <= rg.begin) {
        // no share
    } else if (warp >= Role::PROD && warp < Role::MMA) {
        // ================================ producers ================================
        constexpr int PW = Role::PROD_WARPS, CPR = HD / 8, RPP = 32 / CPR;     // warps of the stream; chunks of a row; rows per request of a warp
        const int pw = TMA ? 0 : (warp - Role::PROD) % PW, pt = pw * 32 + lane;
        const int lr = lane / CPR, lc = lane % CPR;
        uint32_t prod_ph = 0;
        auto prod_sync = [&]() -> bool {                           // of the stream's producers
            __syncwarp();
            if (PW == 1) return true;
            if (lane == 0) mbar_arrive(&prod_bar[s]);
            const bool w = wait_all(&prod_bar[s], prod_ph);
            prod_ph ^= 1;
            return w;
        };
        PagedWalk w(rg, KEYS);
        bool ok = true, more = true;
        if (TMA && TWO && warp == Role::PROD + 1) {
            // nothing to bring
        } else if (TMA) {
            // lane = page of the tile
            const int ps = a.pages.page_size, boxes = ps <= 128 ? KEYS / ps : 1, box = min(ps, 128);
            PagedWalk ahead = w;                                   // the tile whose page entry is requested next
            int ahead_j = 0;
            bool ahead_more = true;
            int page = 0;
            auto request_entry = [&]() {
                if (!ahead_more) return;
                const int key = (ahead.kt + ahead_j) * KEYS + lane * box;
                page = 0;
                if (lane < boxes && key < ahead.n) page = a.table[ahead.b * a.table_stride + key / ps];
                if (++ahead_j == ahead.cnt) {
                    ahead_j = 0;
                    ahead_more = ahead.next(a, per_b, KEYS);
                }
            };
            request_entry();
            uint32_t keys_sent = 0, values_sent = 0;
            while (ok && more) {
                const int head = w.item / RT;
                for (int j = 0; j < w.cnt; ++j) {
                    const int first = (w.kt + j) * KEYS, key = first + lane * box;
                    const int here = min(boxes, (w.n - first + box - 1) / box);        // boxes that hold a key
                    const bool real = lane < here;
                    int pg = page;
                    if (real && (unsigned)pg >= (unsigned)a.pages.n_pages) {
                        if (a.status) report_bad_index(a.status);
                        pg = a.pages.n_pages;                      // past the map's end: zeros
                    }
                    const int off = ps <= 128 ? 0 : key % ps;
                    request_entry();
                    auto fetch = [&](uint32_t dst, const CUtensorMap* map, uint64_t* bar) {
                        if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)(here * box * HD * 2));
                        __syncwarp();
                        if (real) {
#pragma unroll
                            for (int kb = 0; kb < KB; ++kb) tma_load_4d(dst + kb * 16384 + lane * box * 128, map, bar, kb * 64, off, head, pg);
                        }
                        __syncwarp();
                    };
                    const uint32_t st = (TWO ? 0 : s * RING) + keys_sent % RING, ph = (keys_sent / RING & 1) ^ 1;
                    if (!(ok = wait_all(&k_empty[st], ph))) break;
                    fetch(sK + st * SM::TILE_BYTES, &tmK, &k_full[st]);
                    ++keys_sent;
                    if (!(ok = wait_all(&v_empty[st], ph))) break;
                    fetch(sV + st * SM::TILE_BYTES, &tmV, &v_full[st]);
                    ++values_sent;
                }
                if (ok) more = w.next(a, per_b, KEYS);
            }
            // what is on its way must land before this CTA's shared memory is another's, also where somebody else has given up on using it
#pragma unroll
            for (int i = 0; i < RING; ++i) {
                const int st = (TWO ? 0 : s * RING) + i;
                const uint32_t nk = (keys_sent + RING - 1 - i) / RING, nv = (values_sent + RING - 1 - i) / RING;
                if (nk > 0) mbar_wait(&k_full[st], (nk - 1) & 1, &drain_flag);
                if (nv > 0) mbar_wait(&v_full[st], (nv - 1) & 1, &drain_flag);
            }
        } else {
            constexpr int SHARE = 128 / PW;                        // rows of this warp
            auto copy_rows = [&](uint32_t dst, const uint64_t* rows) {
#pragma unroll 8
                for (int i = 0; i < SHARE / RPP; ++i) {
                    const int r = pw * SHARE + i * RPP + lr;
                    const uint64_t at = rows[r];
                    cp_async16(dst + (lc / 8) * 16384 + r * 128 + (((lc % 8) ^ (r & 7)) << 4), reinterpret_cast<const uint8_t*>(at & ~1ull) + lc * 16, !(at & 1));
                }
            };
            // page entries two tiles ahead, addresses one
            constexpr int MINE = 128 / (PW * 32);                  // keys of a tile a thread looks up
            int lb = rg.b, ln = rg.n, lkt = rg.kt, litem = rg.item, lleft = rg.end - rg.begin;
            int page[MINE], in_page[MINE];
            bool exists[MINE];
            auto request_entry = [&]() {
#pragma unroll
                for (int i = 0; i < MINE; ++i) {
                    const int key = lkt * TILE + pt + i * PW * 32;
                    exists[i] = lleft > 0 && key < ln;
                    if (exists[i]) {
                        const int p = key / a.pages.page_size;
                        in_page[i] = (litem / RT) * a.pages.page_size + key - p * a.pages.page_size;
                        page[i] = a.table[lb * a.table_stride + p];
                    }
                }
                if (lleft <= 0) return;
                --lleft;
                if ((lkt + 1) * TILE < ln) {
                    ++lkt;
                } else {
                    lkt = 0;
                    if (++litem == per_b) {
                        litem = 0;
                        if (lleft > 0) do { ++lb; ln = paged_len(a, lb); } while (ln <= 0);
                    }
                }
            };
            uint64_t(*const at)[2 * TILE] = reinterpret_cast<uint64_t(*)[2 * TILE]>(row_at[TMA || TWO ? 0 : s]);
            auto leave_address = [&](int buf) {
#pragma unroll
                for (int i = 0; i < MINE; ++i) {
                    uint64_t ka = reinterpret_cast<uint64_t>(a.pages.k) | 1u, va = reinterpret_cast<uint64_t>(a.pages.v) | 1u;
                    if (exists[i]) {
                        if ((unsigned)page[i] < (unsigned)a.pages.n_pages) {
                            ka = reinterpret_cast<uint64_t>((const T*)a.pages.k + page[i] * a.pages.k_page + (int64_t)in_page[i] * HD);
                            va = reinterpret_cast<uint64_t>((const T*)a.pages.v + page[i] * a.pages.v_page + (int64_t)in_page[i] * HD);
                        } else if (a.status) {
                            report_bad_index(a.status);
                        }
                    }
                    at[buf][pt + i * PW * 32] = ka;
                    at[buf][TILE + pt + i * PW * 32] = va;
                }
            };
            request_entry();
            leave_address(0);
            request_entry();
            uint32_t g = 0;                                        // tiles so far
            while (ok && more) {
                for (int j = 0; j < w.cnt; ++j, ++g) {
                    const uint32_t st = (TWO ? 0 : s * RING) + g % RING, ph = (g / RING & 1) ^ 1;
                    ok = prod_sync();                              // the tile's addresses are there, the ones before are used up
                    if (ok) ok = wait_all(&k_empty[st], ph);
                    if (!ok) break;
                    copy_rows(sK + st * SM::TILE_BYTES, at[g & 1]);
                    cp_async_arrive(&k_full[st]);
                    leave_address((g & 1) ^ 1);
                    request_entry();
                    if (!(ok = wait_all(&v_empty[st], ph))) break;
                    copy_rows(sV + st * SM::TILE_BYTES, at[g & 1] + TILE);
                    cp_async_arrive(&v_full[st]);
                }
                if (ok) more = w.next(a, per_b, KEYS);
            }
        }
    } else if (warp >= Role::MMA) {
        // ================================ products of stream s ================================
        const bool elected = elect_one();
        const uint64_t qd = umma_desc_k128(sQ + s * SM::TILE_BYTES), kd0 = umma_desc_k128(sK), vd0 = umma_desc_mn128(sV);
        const uint32_t d_s = tmem_base + s * 128, d_o = tmem_base + O_COL + s * 128;
        PagedWalk w(rg, KEYS);
        uint32_t part = 0, base = 0, tails = 0, done[HV] = {};     // parts, tiles, tails so far; second products per buffer
        bool ok = true, more = true;
        for (; ok && more; ++part) {
            const int tail = w.n - (w.nt - 1) * KEYS;              // keys of the last tile of the sequence
            const bool ends = w.kt + w.cnt == w.nt, has_tail = TMA && ends && tail < KEYS;
            const int units = w.cnt * HV - (ends && tail <= (HV - 1) * HK);       // buffers' worth of keys: the last one may hold none
            auto stage = [&](int u) -> uint32_t { return (TWO ? 0 : s * RING) + (base + u / HV) % RING; };
            auto phase = [&](int u) -> uint32_t { return (base + u / HV) / RING & 1; };
            ok = wait_all(&q_full[s], part & 1);
            if (ok) fence_proxy_async_smem();                      // the queries are written as threads write; the tensor pipe reads as copies do
            auto issue_S = [&](int u) -> bool {
                const int h = u % HV;
                const uint32_t st = stage(u);
                if (h == 0 && !wait_all(&k_full[st], phase(u))) return false;
                // the score buffer holds the probabilities of its previous keys until their second product is done
                if (done[h] > 0 && !wait_all(&pv_done[s][h], (done[h] - 1) & 1)) return false;
                if (!TMA) fence_proxy_async_smem();
                tc_fence_after();
                if (elected) {
                    const uint64_t kd = kd0 + (uint64_t)(st * (SM::TILE_BYTES >> 4) + h * (HK * 8));
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                        for (int k = 0; k < 4; ++k) umma_bf16(d_s + h * HK, qd + kb * 1024 + 2 * k, kd + kb * 1024 + 2 * k, IDESC_S, (kb | k) != 0);
                    umma_commit(&s_full[s][h]);
                    if (h == HV - 1 || u == units - 1) umma_commit(&k_empty[st]);
                }
                __syncwarp();
                return true;
            };
            auto issue_PV = [&](int u) -> bool {
                const int h = u % HV;
                const uint32_t st = stage(u);
                if (h == 0) {
                    if (!wait_all(&v_full[st], phase(u))) return false;
                    if (has_tail && u / HV == w.cnt - 1) {
                        // value rows behind the sequence's end, whatever the page holds there, and those of boxes that were not fetched
                        if (!TWO || s == 0) {
                            for (int kb = 0; kb < KB; ++kb)
                                for (int i = lane; i < (KEYS - tail) * 8; i += 32)
                                    reinterpret_cast<uint4*>(values_at + st * SM::TILE_BYTES + kb * 16384 + tail * 128)[i] = make_uint4(0, 0, 0, 0);
                            fence_proxy_async_smem();
                            __syncwarp();
                        }
                        if (TWO) {                                 // the streams' warps meet: both see the zeros, and neither is a tail ahead
                            if (lane == 0) mbar_arrive(&tail_bar);
                            if (!wait_all(&tail_bar, tails & 1)) return false;
                        }
                    }
                }
                if (!wait_all(&p_full[s][h], done[h] & 1)) return false;
                if (!TMA) fence_proxy_async_smem();
                tc_fence_after();
                if (elected) {
                    const uint64_t vd = vd0 + (uint64_t)(st * (SM::TILE_BYTES >> 4));
#pragma unroll
                    for (int k = 0; k < 8 / HV; ++k) {             // 16 keys: 8 columns of probabilities (64 keys in 32 columns from 0 and from 64 on), 16 value rows
                        const int kk = h * (8 / HV) + k;
                        umma_bf16_ts(d_o, d_s + kk / 4 * 64 + kk % 4 * 8, vd + kk * 128, IDESC_O, u > 0 || k > 0);
                    }
                    umma_commit(&pv_done[s][h]);
                    if (h == HV - 1 || u == units - 1) umma_commit(&v_empty[st]);
                }
                __syncwarp();
                ++done[h];
                return true;
            };
            for (int u = 0; ok && u < min(HV, units); ++u) ok = issue_S(u);
            // the part's first products overwrite the accumulator: the previous part's rows must have left
            if (ok && part > 0) ok = wait_all(&o_empty[s], (part - 1) & 1);
            for (int u = 0; ok && u < units; ++u) {
                ok = issue_PV(u);
                if (ok && u + HV < units) ok = issue_S(u + HV);
            }
            tails += has_tail;
            base += w.cnt;
            if (ok) more = w.next(a, per_b, KEYS);
        }
        // the last arrival the tensor pipe owes this CTA's barriers; where somebody gave up, meanwhile too, the end of the products under way
        if (ok) ok = wait_all(&v_empty[(TWO ? 0 : s * RING) + (base - 1) % RING], (base - 1) / RING & 1);
        if (!ok) {
            if (elected) umma_commit(&drain[s]);
            __syncwarp();
            mbar_wait(&drain[s], 0, &drain_flag);
        }
    } else {
        // ================================ softmax: thread = row of its stream ================================
        const int quad = warp & 3, r128 = quad * 32 + lane, base0 = TWO ? s * 128 : 0;             // row of the tile; first row of the tile in the item
        const int rep = TWO ? 0 : r128 / ROWS, wr = base0 + (TWO ? quad * 32 : quad * 32 % ROWS);  // copy of the row; first row of the warp in the item
        const uint32_t lanes = tmem_base + (uint32_t(quad * 32) << 16), sc = lanes + s * 128, acc = lanes + O_COL + s * 128;
        const float c = a.scale_log2, none = c < 0.f ? INFINITY : -INFINITY;
        float* const room = reinterpret_cast<float*>(smem + s * SM::TILE_BYTES);
        PagedWalk w(rg, KEYS);
        uint32_t done = 0, seen[HV] = {}, part = 0, g_ph = 0;      // buffers' worth of keys so far, and of each buffer; parts
        bool ok = true, more = true;
        auto group_sync = [&]() -> bool {                          // of the stream's four warps
            __syncwarp();
            if (lane == 0) mbar_arrive(&g_bar[s]);
            const bool r = wait_all(&g_bar[s], g_ph);
            g_ph ^= 1;
            return r;
        };
        for (; ok && more; ++part) {
            const int head = w.item / RT, row0 = (w.item - head * RT) * ROWS;
            const bool idle = row0 + wr >= R;                      // none of the warp's rows exists: it only keeps the barriers going
            {
                // this thread's row (of the copies of a row, each), then the stream's rows together: whole rows a request
                constexpr int CPR = HD / 8, RPP = 32 / CPR;
                const int r = row0 + base0 + (TWO ? r128 : r128 % ROWS), t = r / a.group, gq = r - t * a.group;
                uint64_t at = reinterpret_cast<uint64_t>(a.q) | 1u;        // odd: no such row, zeros are written
                if (r < R) at = reinterpret_cast<uint64_t>((const T*)a.q + w.b * a.q_b + t * a.q_t + (int64_t)(head * a.group + gq) * a.q_h);
                row_q[s][r128] = at;
                row_o[part & 1][s][r128] = reinterpret_cast<uint64_t>((T*)a.out + w.b * a.o_b + t * a.o_t + (int64_t)(head * a.group + gq) * a.o_h);
                if (!(ok = group_sync())) break;                   // (which the room of the previous part is read by, too)
                const int lr = lane / CPR, lc = lane % CPR;
#pragma unroll
                for (int i = 0; i < 32 / RPP; ++i) {
                    const int rr = quad * 32 + i * RPP + lr;
                    const uint64_t from = row_q[s][rr];
                    cp_async16(sQ + s * SM::TILE_BYTES + (lc / 8) * 16384 + rr * 128 + (((lc % 8) ^ (rr & 7)) << 4),
                               reinterpret_cast<const uint8_t*>(from & ~1ull) + lc * 16, !(from & 1));
                }
                cp_async_arrive(&q_full[s]);
            }
            float mc = -INFINITY, l = 0.f;
            const int tail = w.n - (w.nt - 1) * KEYS, units = w.cnt * HV - (w.kt + w.cnt == w.nt && tail <= (HV - 1) * HK);
            for (int u = 0; u < units; ++u, ++done) {
                const int h = u % HV;
                const uint32_t sb = sc + h * HK;                   // this buffer
                if (!(ok = wait_all(&s_full[s][h], seen[h] & 1))) break;
                ++seen[h];
                if (!idle) {
                    tc_fence_after();
                    // keys of the buffer that exist, from the first one of this copy on
                    const int limit = min(w.n - (w.kt + u / HV) * KEYS, KEYS) - h * HK - rep * KC;
                    constexpr int MINE = KC / HV;                  // keys of this thread
                    float v[MINE], bm = none;
#pragma unroll
                    for (int t = 0; t < MINE; t += 32) tmem_ld32(sb + rep * KC + t, v + t);
#pragma unroll
                    for (int t = 0; t < MINE; t += 32) tmem_ld_wait_regs(v + t);
                    if (limit < MINE) {
#pragma unroll
                        for (int t = 0; t < MINE; ++t)
                            if (t >= limit) v[t] = none;
                    }
                    if (c < 0.f) {
#pragma unroll
                        for (int t = 0; t < MINE; ++t) bm = fminf(bm, v[t]);
                    } else {
                        float b1 = none;
#pragma unroll
                        for (int t = 0; t < MINE; t += 4) {
                            bm = fmaxf(bm, fmaxf(v[t], v[t + 1]));
                            b1 = fmaxf(b1, fmaxf(v[t + 2], v[t + 3]));
                        }
                        bm = fmaxf(bm, b1);
                    }
                    const float bmc = bm * c, ref = bmc - kPagedLift<T>;
                    const bool raise = bmc - mc > kRaise;                      // (the first finite score, too: mc is minus infinity)
                    const bool shrink = raise && u > 0;
                    const float f = shrink ? ex2_approx(mc - ref) : 1.f;       // (a row without a finite score so far: its sum is zero)
                    if (raise) mc = ref;
                    const float base = mc == -INFINITY ? 0.f : mc;
                    // Scores are scaled and taken off the reference in one fma, unrounded in between, and the reference is the maximum scaled and rounded:
                    // beyond 2^20 the two would be apart by a fraction of an exponent first, by more than an exponent holds in the end.  Then scores
                    // are rounded, too.  (The question costs 1 % at most: 224 rows of eight sequences 48.9 us without it, 49.2 with.)
                    float step = c;
                    const bool large = fabsf(base) > 1048576.f;
                    if (__any_sync(0xffffffffu, large)) {                      // (row by row: a row's bits do not hang on its neighbours')
                        step = large ? 1.f : c;
                        const float first = large ? c : 1.f;
#pragma unroll
                        for (int t = 0; t < MINE; ++t) v[t] *= first;
                    }
                    if (TWO && !(ok = wait_all(&turn[s], (done & 1) ^ (s == 0)))) break;       // the other stream is through with its exponentials
                    l *= f;
                    float l0 = 0.f, l1 = 0.f;
                    // 32 scores -> 16 columns of probabilities: keys 0..63 of the tile in columns 0..31, 64..127 in columns 64..95
                    auto probabilities = [&](const float* x, uint32_t col) {
                        uint32_t packed[16];
#pragma unroll
                        for (int t = 0; t < 16; ++t) {
                            const float e0 = ex2_approx(fmaf(x[2 * t], step, -base)), e1 = ex2_approx(fmaf(x[2 * t + 1], step, -base));
                            l0 += e0;
                            l1 += e1;
                            typename Pack2<T>::type h2 = Pack2<T>::down(e0, e1);
                            packed[t] = *reinterpret_cast<uint32_t*>(&h2);
                        }
                        tmem_st16(col, packed);
                    };
                    if constexpr (KC < 128) {
                        const uint32_t zeros[16] = {};
#pragma unroll
                        for (int q = 0; q < 4; ++q)                // the other copies' keys
                            if (q / (KC / 32) != rep) tmem_st16(sc + (q >> 1) * 64 + (q & 1) * 16, zeros);
                    }
#pragma unroll
                    for (int t = 0; t < MINE; t += 32) {
                        const int q = (h * HK + rep * KC + t) / 32;            // which 32 of the tile's keys
                        probabilities(v + t, sc + (q >> 1) * 64 + (q & 1) * 16);
                    }
                    l += l0 + l1;
                    __syncwarp();
                    if (TWO && lane == 0) mbar_arrive(&turn[s ^ 1]);
                    if (__any_sync(0xffffffffu, shrink)) {
                        // the stream's previous second product has to be done (with one buffer it was before these scores were made)
                        if (HV == 2 && !(ok = wait_all(&pv_done[s][h ^ 1], (seen[h ^ 1] - 1) & 1))) break;
                        tc_fence_after();
#pragma unroll
                        for (int ch = 0; ch < HD / 32; ++ch) {
                            float o[32];
                            tmem_ld32(acc + ch * 32, o);
                            tmem_ld_wait_regs(o);
#pragma unroll
                            for (int t = 0; t < 32; ++t) o[t] *= f;
                            tmem_st32(acc + ch * 32, o);
                        }
                    }
                    tmem_st_wait();
                    tc_fence_before();
                } else if (TWO) {
                    if (!(ok = wait_all(&turn[s], (done & 1) ^ (s == 0)))) break;
                    if (lane == 0) mbar_arrive(&turn[s ^ 1]);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[s][h]);
            }
            if (!ok) break;
            // ---- the part goes out ----
            // Each thread weighs what its lane holds of a row, and the rows leave through the room of the part's queries, which are used up: whole
            // rows of 16-byte chunks (chunk e of row r at e ^ (r mod 8)), the copies of a row added up on the way.
            constexpr int ROUND = HD / 2, CH4 = ROUND / 4, OWN = TWO ? 128 : ROWS, ITEMS = OWN * CH4 / 128;    // columns of a round; chunks; rows; chunks a thread takes
            const bool begins = w.kt == 0, whole = begins && w.cnt == w.nt;
            const int64_t slot = (int64_t)share * 2 + (begins ? 1 : 0);
            float weight = 1.f, m = mc, sum = l;
            if (REP > 1) {
                x_ml[s][r128] = make_float2(mc, l);
                if (!(ok = group_sync())) break;
                // reference and sum over the copies
                const int rt = r128 % ROWS;
                m = -INFINITY;
                sum = 0.f;
#pragma unroll
                for (int q = 0; q < REP; ++q) m = fmaxf(m, x_ml[s][q * ROWS + rt].x);
                const float mb = m == -INFINITY ? 0.f : m;         // (no finite score at all: every copy's exponentials are against 0)
#pragma unroll
                for (int q = 0; q < REP; ++q) {
                    const float2 x = x_ml[s][q * ROWS + rt];
                    sum += x.y * (m == -INFINITY ? 1.f : ex2_approx(x.x - mb));
                }
                weight = m == -INFINITY ? 1.f : ex2_approx(mc - mb);
            }
            if (whole) weight *= 1.f / sum;
            {
                const int h = (units - 1) % HV;                    // (the last second product's end is all products' end)
                if (!(ok = wait_all(&pv_done[s][h], (seen[h] - 1) & 1))) break;
            }
            if (!idle) tc_fence_after();
#pragma unroll
            for (int round = 0; round < 2; ++round) {
                if (!idle) {
#pragma unroll
                    for (int c0 = 0; c0 < ROUND; c0 += 32) {
                        float o[32];
                        tmem_ld32(acc + round * ROUND + c0, o);
                        tmem_ld_wait_regs(o);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            reinterpret_cast<float4*>(room + r128 * ROUND)[(c0 / 4 + e) ^ (lane & 7)] =
                                make_float4(o[4 * e] * weight, o[4 * e + 1] * weight, o[4 * e + 2] * weight, o[4 * e + 3] * weight);
                    }
                }
                if (round == 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&o_empty[s]);
                }
                if (!(ok = group_sync())) break;                   // the stream's rows are in the room
                // a thread has chunk e of rows rt0, rt0 + 128 / CH4, ..., four of them under way together
                constexpr int BATCH = ITEMS < 4 ? ITEMS : 4;
                const int e = tid % CH4, rt0 = (tid & 127) / CH4;
#pragma unroll 1
                for (int k0 = 0; k0 < ITEMS && row0 + base0 + rt0 + k0 * (128 / CH4) < R; k0 += BATCH) {
                    float4 x[BATCH];
                    uint64_t to[BATCH];
#pragma unroll
                    for (int k = 0; k < BATCH; ++k) {
                        const int rt = rt0 + (k0 + k) * (128 / CH4);
                        x[k] = reinterpret_cast<const float4*>(room + rt * ROUND)[e ^ (rt & 7)];
                        to[k] = whole ? row_o[part & 1][s][rt] : reinterpret_cast<uint64_t>(a.partial + (slot * ROWS + base0 + rt) * HD);
#pragma unroll
                        for (int q = 1; q < REP; ++q) {
                            const float4 y = reinterpret_cast<const float4*>(room + (q * ROWS + rt) * ROUND)[e ^ (rt & 7)];
                            x[k].x += y.x; x[k].y += y.y; x[k].z += y.z; x[k].w += y.w;
                        }
                    }
#pragma unroll
                    for (int k = 0; k < BATCH; ++k) {
                        if (row0 + base0 + rt0 + (k0 + k) * (128 / CH4) >= R) continue;
                        if (whole) {
                            typename Pack2<T>::type lo = Pack2<T>::down(x[k].x, x[k].y), hi = Pack2<T>::down(x[k].z, x[k].w);
                            reinterpret_cast<uint2*>(to[k])[round * CH4 + e] = make_uint2(*reinterpret_cast<uint32_t*>(&lo), *reinterpret_cast<uint32_t*>(&hi));
                        } else {
                            reinterpret_cast<float4*>(to[k])[round * CH4 + e] = x[k];
                        }
                    }
                }
                if (round == 0 && !(ok = group_sync())) break;     // the room is read
            }
            if (!ok) break;
            if (r128 < OWN && row0 + base0 + r128 < R) {           // (of the copies of a row, the first)
                const int r = row0 + base0 + r128, t = r / a.group, gq = r - t * a.group;
                if (!whole) a.partial_ml[slot * ROWS + base0 + r128] = make_float2(m, sum);
                else if (a.lse) a.lse[((int64_t)w.b * a.T + t) * a.nq + head * a.group + gq] = (m + log2f(sum)) * 0.69314718055994531f;
            }
            if (begins && (tid & 127) == 0 && (!TWO || s == 0)) paged_describe(a, rg, share, per_b, w.b, w.item, w.nt - w.cnt);
            more = w.next(a, per_b, KEYS);
        }
    }
    cp_async_wait<0>();
    tc_fence_before();
    __syncthreads();
    if (warp == Role::MMA) {
        tc_fence_after();
        tmem_dealloc(tmem_base, 512);
    }
    if (tid == 0 && abort_flag && a.status) atomicExch(a.status, 2);
}

}  // namespace jot

// Attention over the pages of a cache for more rows of a key head than a warp's matrix instruction holds, on tcgen05: the same
// line of tiles, shares and joined parts as paged_attention.cuh, tiles of 128 keys.
//
//   S = Q K^T, P = exp2(S c - m) written over S in tensor memory, O += P V, with Q, K, V in shared memory as their rows are in the
//   pages: the head dimension runs along 128-byte rows (16-byte chunk c of row r at c ^ (r mod 8)), which is the first product's
//   K-major operand for Q and K, and for V the second product's MN-major one, so nothing is transposed.
//
// Two streams of work share the tensor pipe, each with a score buffer, an accumulator and a warpgroup of its own (thread = row):
// while one stream's rows are in exponentials, the other's products run.
//   TWO    more than 128 rows: the streams are two tiles of 128 rows over the same keys
//   !TWO   at most 128 rows: the streams are the even and the odd tiles of keys over the same rows, and meet at the end
// The reference maximum of a row follows a tile's maximum only when that exceeds it by more than 2^8 (probabilities up to 256
// are as exact as those up to 1); then the row of the accumulator is rescaled in tensor memory.
//
// The keys come by cp.async, 16 bytes a request, since pages may be of any size; four producer warps look up page entries two tiles
// ahead, leave row addresses one tile ahead, and never wait for a request: each arrives on its stage's barrier when it has landed.
//
//   warps 0-3, 4-7  softmax of stream 0 and 1      warps 8-11  producers      warp 12  MMA issuer
#pragma once
#include "paged_attention.cuh"

namespace jot {

constexpr int kUmmaPagedThreads = 416;
constexpr int kUmmaPagedTile = 128;
constexpr int kUmmaPagedMaxCtas = 160;      // one per SM

enum { PAGED_SMALL = 0, PAGED_ONE = 1, PAGED_TWO = 2 };      // at most 32 rows of a key head, at most 128, more

template <int HD, int MODE>
struct UmmaPagedSmem {
    static constexpr int TILE_BYTES = 128 * HD * 2;               // 128 rows: a tile of Q, K or V
    // Two tiles of queries (the streams', or this part's and the next one's), then the stages of keys and values.  Up to 32 rows the
    // queries take the room of 32 (the products read on into what follows: rows that nobody looks at), which leaves a third stage.
    static constexpr int Q_ROWS = MODE == PAGED_SMALL ? 32 : 128;
    static constexpr int Q_BYTES = Q_ROWS * HD * 2;
    static constexpr int STAGES = MODE == PAGED_SMALL ? 3 : 2;
    static constexpr int DYN_BYTES = 2 * Q_BYTES + 2 * STAGES * TILE_BYTES + 1024;
};

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

// The parts of items a CTA's share consists of, in order.
struct PagedWalk {
    int b, n, nt, item, kt, cnt;          // sequence, its keys and tiles, item, first tile and number of tiles of this part
    int64_t left;                         // tiles of the share from this part on
    __device__ __forceinline__ PagedWalk(const PagedArgs& a, const PagedRange& rg, int tile) {
        b = rg.b;
        n = paged_len(a, b);
        nt = (n + tile - 1) / tile;
        item = (int)(rg.in_seq / nt);
        kt = (int)(rg.in_seq - (int64_t)item * nt);
        left = rg.end - rg.begin;
        cnt = (int)min((int64_t)(nt - kt), left);
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
        cnt = (int)min((int64_t)nt, left);
        return true;
    }
};

template <typename T, int HD, int MODE>
__global__ void __launch_bounds__(kUmmaPagedThreads, 1) paged_attention_umma_kernel(const PagedArgs a) {
    using SM = UmmaPagedSmem<HD, MODE>;
    constexpr bool TWO = MODE == PAGED_TWO;
    constexpr int KB = HD / 64, ST = SM::STAGES, TILE = kUmmaPagedTile;
    constexpr int MT = TWO ? 256 : 128;
    constexpr uint32_t IDESC_S = umma_idesc16<T>(128, 128, false), IDESC_O = umma_idesc16<T>(128, HD, true);
    constexpr uint32_t O_COL = 256;              // scores of the streams at columns 0 and 128, accumulators at 256 and 384
    constexpr float kRaise = 8.f;

    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t sQ = smem_u32(smem), sK = sQ + 2 * SM::Q_BYTES, sV = sK + ST * SM::TILE_BYTES;
    __shared__ uint64_t k_full[ST], k_empty[ST], v_full[ST], v_empty[ST], q_full[2], q_empty[2], s_full[2], p_full[2], pv_done[2], o_empty,
        prod_bar, x_bar;
    __shared__ uint64_t row_at[2][2 * TILE];     // addresses of a tile's key rows, then of its value rows; odd: no such row
    __shared__ uint64_t row_q[MT];
    __shared__ float2 x_ml[2][2][128];           // !TWO: [parity of the part][stream][row] (maximum, sum)
    __shared__ PagedRangeSmem range_smem;
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        abort_flag = 0;
        for (int i = 0; i < ST; ++i) {
            mbar_init(&k_full[i], 128);          // every producer thread's requests
            mbar_init(&k_empty[i], 1);
            mbar_init(&v_full[i], 128);
            mbar_init(&v_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], 128);
            mbar_init(&q_empty[i], 1);
            mbar_init(&s_full[i], 1);
            mbar_init(&p_full[i], 4);
            mbar_init(&pv_done[i], 1);
        }
        mbar_init(&o_empty, 8);
        mbar_init(&prod_bar, 4);
        mbar_init(&x_bar, 8);
        fence_barrier_init();
        fence_proxy_async_smem();
    }
    if (warp == 12) {
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

    const int R = a.T * a.group, RT = (R + MT - 1) / MT, per_b = a.nkv * RT;
    const PagedRange rg = paged_range<T, HD, kUmmaPagedThreads>(a, TILE, per_b, range_smem);
    if (tid == 0) a.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
    auto wait_all = [&](uint64_t* bar, uint32_t parity) -> bool {
        const bool w = mbar_wait(bar, parity, abortp);
        return __all_sync(0xffffffffu, w);
    };

    if (rg.end > rg.begin) {
        if (warp >= 8 && warp < 12) {
            // ================================ producers ================================
            const int pt = tid - 256, pw = pt >> 5;
            constexpr int CPR = HD / 8, RPP = 32 / CPR;            // chunks of a row; rows per request of a warp
            const int lr = lane / CPR, lc = lane % CPR;
            uint32_t ldst[8 / RPP];                                // where this lane's chunk goes: repeats every 8 rows
#pragma unroll
            for (int i = 0; i < 8 / RPP; ++i)
                ldst[i] = (uint32_t)((lc / 8) * 16384 + (pw * 32 + i * RPP + lr) * 128 + (((lc % 8) ^ ((i * RPP + lr) & 7)) << 4));
            auto copy_rows = [&](uint32_t dst, const uint64_t* rows) {
#pragma unroll
                for (int i = 0; i < 32 / RPP; ++i) {
                    const uint64_t at = rows[pw * 32 + i * RPP + lr];
                    cp_async16(dst + ldst[i % (8 / RPP)] + (i * RPP / 8) * 1024, reinterpret_cast<const uint8_t*>(at & ~1ull) + lc * 16, !(at & 1));
                }
            };
            auto copy_queries = [&](uint32_t dst, const uint64_t* rows) {
                constexpr int ROWS = SM::Q_ROWS / 4;               // of this warp
#pragma unroll
                for (int i = 0; i < ROWS / RPP; ++i) {
                    const int r = pw * ROWS + i * RPP + lr;
                    const uint64_t at = rows[r];
                    cp_async16(dst + (lc / 8) * (SM::Q_ROWS * 128) + r * 128 + (((lc % 8) ^ (r & 7)) << 4), reinterpret_cast<const uint8_t*>(at & ~1ull) + lc * 16,
                               !(at & 1));
                }
            };
            uint32_t prod_ph = 0;
            auto prod_sync = [&]() -> bool {
                __syncwarp();
                if (lane == 0) mbar_arrive(&prod_bar);
                const bool w = wait_all(&prod_bar, prod_ph);
                prod_ph ^= 1;
                return w;
            };
            // page entries two tiles ahead, addresses one
            int lb = rg.b, ln = paged_len(a, lb), lkt, litem;
            {
                const int nt = (ln + TILE - 1) / TILE;
                litem = (int)(rg.in_seq / nt);
                lkt = (int)(rg.in_seq - (int64_t)litem * nt);
            }
            int64_t lleft = rg.end - rg.begin;
            int page = 0, in_page = 0;
            bool exists = false;
            auto request_entry = [&]() {
                exists = false;
                if (lleft <= 0) return;
                const int key = lkt * TILE + pt;
                if (key < ln) {
                    const int p = key / a.pages.page_size;
                    in_page = (litem / RT) * a.pages.page_size + key - p * a.pages.page_size;
                    page = a.table[lb * a.table_stride + p];
                    exists = true;
                }
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
            auto leave_address = [&](int buf) {
                uint64_t ka = reinterpret_cast<uint64_t>(a.pages.k) | 1u, va = reinterpret_cast<uint64_t>(a.pages.v) | 1u;
                if (exists) {
                    if ((unsigned)page < (unsigned)a.pages.n_pages) {
                        ka = reinterpret_cast<uint64_t>((const T*)a.pages.k + page * a.pages.k_page + (int64_t)in_page * HD);
                        va = reinterpret_cast<uint64_t>((const T*)a.pages.v + page * a.pages.v_page + (int64_t)in_page * HD);
                    } else if (a.status) {
                        atomicExch(a.status, kStatusBadIndex);
                    }
                }
                row_at[buf][pt] = ka;
                row_at[buf][TILE + pt] = va;
            };
            PagedWalk w(a, rg, TILE);
            request_entry();
            leave_address(0);
            request_entry();
            uint32_t g = 0, part = 0;                              // tiles and parts so far
            bool ok = true, more = true;
            for (; ok && more; ++part) {
                // queries of the part
                const int head = w.item / RT, row0 = (w.item - head * RT) * MT;
                const int qb = TWO ? 0 : (part & 1);
                const uint32_t qph = TWO ? (part & 1) ^ 1 : ((part >> 1) & 1) ^ 1;
#pragma unroll
                for (int i = 0; i < MT / 128; ++i) {
                    const int r = row0 + i * 128 + pt, t = r / a.group, gq = r - t * a.group;
                    uint64_t at = reinterpret_cast<uint64_t>(a.q) | 1u;
                    if (r < R) at = reinterpret_cast<uint64_t>((const T*)a.q + w.b * a.q_b + t * a.q_t + (int64_t)(head * a.group + gq) * a.q_h);
                    row_q[i * 128 + pt] = at;
                }
                ok = prod_sync();
                if (ok) ok = wait_all(&q_empty[qb], qph);
                if (!ok) break;
#pragma unroll
                for (int i = 0; i < (TWO ? 2 : 1); ++i) copy_queries(sQ + (TWO ? i : qb) * SM::Q_BYTES, row_q + i * 128);
                cp_async_arrive(&q_full[qb]);
                for (int j = 0; j < w.cnt; ++j, ++g) {
                    const int st = g % ST, buf = g & 1;
                    const uint32_t ph = ((g / ST) & 1) ^ 1;
                    ok = prod_sync();                              // the tile's addresses are there, the ones before are used up
                    if (ok) ok = wait_all(&k_empty[st], ph);
                    if (!ok) break;
                    copy_rows(sK + st * SM::TILE_BYTES, row_at[buf]);
                    cp_async_arrive(&k_full[st]);
                    leave_address(buf ^ 1);
                    request_entry();
                    if (!(ok = wait_all(&v_empty[st], ph))) break;
                    copy_rows(sV + st * SM::TILE_BYTES, row_at[buf] + TILE);
                    cp_async_arrive(&v_full[st]);
                }
                if (ok) more = w.next(a, per_b, TILE);
            }
        } else if (warp == 12) {
            // ================================ MMA issuer ================================
            const bool elected = elect_one();
            const uint64_t qd0 = umma_desc_k128(sQ), kd0 = umma_desc_k128(sK), vd0 = umma_desc_mn128(sV);
            PagedWalk w(a, rg, TILE);
            uint32_t g0 = 0, part = 0, done[2] = {0, 0};           // tiles before this part; second products per stream so far
            bool ok = true, more = true;
            for (; ok && more; ++part) {
                const int units = TWO ? 2 * w.cnt : w.cnt;
                const int qb = TWO ? 0 : (part & 1);
                ok = wait_all(&q_full[qb], TWO ? (part & 1) : ((part >> 1) & 1));
                uint32_t made[2] = {0, 0};                         // second products of this part
                auto issue_S = [&](int u) -> bool {
                    const int s = u & 1, tile = TWO ? u >> 1 : u;
                    const uint32_t g = g0 + tile, st = g % ST;
                    if (!wait_all(&k_full[st], (g / ST) & 1)) return false;
                    // the score buffer holds the probabilities of the stream's previous tile until its second product is done
                    const uint32_t before = done[s];
                    if (before > 0 && !wait_all(&pv_done[s], (before - 1) & 1)) return false;
                    fence_proxy_async_smem();                      // the requests wrote as threads do; the tensor pipe reads as copies do
                    tc_fence_after();
                    if (elected) {
                        const uint64_t qd = qd0 + (uint64_t)((TWO ? s : qb) * (SM::Q_BYTES >> 4)), kd = kd0 + (uint64_t)(st * (SM::TILE_BYTES >> 4));
#pragma unroll
                        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                umma_bf16(tmem_base + s * 128, qd + kb * (SM::Q_ROWS * 8) + 2 * k, kd + kb * 1024 + 2 * k, IDESC_S, (kb | k) != 0);
                        umma_commit(&s_full[s]);
                        if (!TWO || s == 1) umma_commit(&k_empty[st]);
                        if (u == units - 1) umma_commit(&q_empty[qb]);
                    }
                    __syncwarp();
                    return true;
                };
                auto issue_PV = [&](int u) -> bool {
                    const int s = u & 1, tile = TWO ? u >> 1 : u;
                    const uint32_t g = g0 + tile, st = g % ST;
                    if (!wait_all(&v_full[st], (g / ST) & 1)) return false;
                    if (!wait_all(&p_full[s], done[s] & 1)) return false;
                    // the part's first products overwrite the accumulators: the previous part's rows must have left
                    if (u == 0 && part > 0 && !wait_all(&o_empty, (part - 1) & 1)) return false;
                    fence_proxy_async_smem();
                    tc_fence_after();
                    if (elected) {
                        const uint64_t vd = vd0 + (uint64_t)(st * (SM::TILE_BYTES >> 4));
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            umma_bf16_ts(tmem_base + O_COL + s * 128, tmem_base + s * 128 + (k < 4 ? 8 * k : 64 + 8 * (k - 4)), vd + k * 128, IDESC_O,
                                         made[s] > 0 || k > 0);
                        umma_commit(&pv_done[s]);
                        if (!TWO || s == 1) umma_commit(&v_empty[st]);
                    }
                    __syncwarp();
                    ++made[s];
                    ++done[s];
                    return true;
                };
                if (ok) ok = issue_S(0);
                if (ok && units > 1) ok = issue_S(1);
                for (int u = 0; ok && u < units; ++u) {
                    ok = issue_PV(u);
                    if (ok && u + 2 < units) ok = issue_S(u + 2);
                }
                g0 += w.cnt;
                if (ok) more = w.next(a, per_b, TILE);
            }
            // the last arrival the tensor pipe owes this CTA's barriers
            if (ok) wait_all(&v_empty[(g0 - 1) % ST], ((g0 - 1) / ST) & 1);
        } else {
            // ================================ softmax: thread = row of its stream ================================
            const int s = warp >> 2, quad = warp & 3, r128 = quad * 32 + lane;
            const uint32_t lanes = tmem_base + (uint32_t(quad * 32) << 16), sc = lanes + s * 128;
            const float c = a.scale_log2;
            PagedWalk w(a, rg, TILE);
            uint32_t done[2] = {0, 0}, part = 0;                   // tiles of each stream so far
            bool ok = true, more = true;
            for (; ok && more; ++part) {
                const int head = w.item / RT, row0 = (w.item - head * RT) * MT;
                const int wrow = row0 + (TWO ? s * 128 : 0) + quad * 32;           // first row of this warp
                const bool idle = wrow >= R;                                       // none of its rows exists: it only keeps the barriers going
                const int mine = TWO ? w.cnt : (w.cnt + 1 - s) / 2, other = TWO ? w.cnt : (w.cnt + s) / 2;
                float mc = -INFINITY, l = 0.f;
                for (int i = 0; i < mine; ++i) {
                    if (!(ok = wait_all(&s_full[s], (done[s] + i) & 1))) break;
                    if (!idle) {
                        tc_fence_after();
                        const int tile = w.kt + (TWO ? i : 2 * i + s), limit = w.n - tile * TILE;      // keys of the tile that exist
                        const float none = c < 0.f ? INFINITY : -INFINITY;
                        float v[64], bm = none;
                        // the maximum: keys 0..63, then 64..127, which stay in registers
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            tmem_ld32(sc + half * 64, v);
                            tmem_ld32(sc + half * 64 + 32, v + 32);
                            tmem_ld_wait_regs(v);
                            tmem_ld_wait_regs(v + 32);
                            if (limit < TILE) {
#pragma unroll
                                for (int t = 0; t < 64; ++t)
                                    if (half * 64 + t >= limit) v[t] = none;
                            }
                            if (c < 0.f) {
#pragma unroll
                                for (int t = 0; t < 64; ++t) bm = fminf(bm, v[t]);
                            } else {
#pragma unroll
                                for (int t = 0; t < 64; t += 2) bm = fmaxf(bm, fmaxf(v[t], v[t + 1]));
                            }
                        }
                        const float bmc = bm * c;
                        const bool raise = bmc > mc + kRaise || (mc == -INFINITY && bmc > -INFINITY);
                        const bool shrink = raise && i > 0;
                        const float f = shrink ? ex2_approx(mc - bmc) : 1.f;       // (a row without a finite score so far: its sum is zero)
                        if (raise) mc = bmc;
                        l *= f;
                        const float base = mc == -INFINITY ? 0.f : mc;
                        float l0 = 0.f, l1 = 0.f;
                        // 32 scores -> 16 columns of probabilities.  Keys 64..127 go to columns 64..95, whose scores have just been read, keys
                        // 0..63 to columns 0..31, behind the reads of theirs.
                        auto probabilities = [&](const float* x, uint32_t col) {
                            uint32_t packed[16];
#pragma unroll
                            for (int t = 0; t < 16; ++t) {
                                const float e0 = ex2_approx(fmaf(x[2 * t], c, -base)), e1 = ex2_approx(fmaf(x[2 * t + 1], c, -base));
                                l0 += e0;
                                l1 += e1;
                                typename Pack2<T>::type h2 = Pack2<T>::down(e0, e1);
                                packed[t] = *reinterpret_cast<uint32_t*>(&h2);
                            }
                            tmem_st16(sc + col, packed);
                        };
                        probabilities(v, 64);
                        tmem_ld32(sc, v);
                        probabilities(v + 32, 80);
                        tmem_ld_wait_regs(v);
                        tmem_ld32(sc + 32, v + 32);
                        if (limit < 64) {
#pragma unroll
                            for (int t = 0; t < 32; ++t)
                                if (t >= limit) v[t] = none;
                        }
                        probabilities(v, 0);
                        tmem_ld_wait_regs(v + 32);
                        if (limit < 64) {
#pragma unroll
                            for (int t = 0; t < 32; ++t)
                                if (32 + t >= limit) v[32 + t] = none;
                        }
                        probabilities(v + 32, 16);
                        l += l0 + l1;
                        if (__any_sync(0xffffffffu, shrink)) {
                            // (the previous second product of this stream was done before these scores were made)
#pragma unroll
                            for (int ch = 0; ch < HD / 32; ++ch) {
                                float o[32];
                                tmem_ld32(lanes + O_COL + s * 128 + ch * 32, o);
                                tmem_ld_wait_regs(o);
#pragma unroll
                                for (int t = 0; t < 32; ++t) o[t] *= f;
                                tmem_st32(lanes + O_COL + s * 128 + ch * 32, o);
                            }
                        }
                        tmem_st_wait();
                        tc_fence_before();
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_full[s]);
                }
                if (!ok) break;
                done[s] += mine;
                done[s ^ 1] += other;
                // ---- the part goes out ----
                const bool begins = w.kt == 0, whole = begins && w.cnt == w.nt;
                const int64_t slot = (int64_t)blockIdx.x * 2 + (begins ? 1 : 0);
                const int r = row0 + (TWO ? s * 128 : 0) + r128, rt = r - row0, t = r / a.group, gq = r - t * a.group;
                float wa = 0.f, wb = 0.f, m = mc, sum = l;         // weights of stream 0's and stream 1's accumulators
                if (TWO) {
                    wa = 1.f;
                    ok = wait_all(&pv_done[s], (done[s] - 1) & 1);
                } else {
                    x_ml[part & 1][s][r128] = make_float2(mc, l);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&x_bar);
                    ok = wait_all(&x_bar, part & 1);
                    if (ok) ok = wait_all(&pv_done[0], (done[0] - 1) & 1);
                    if (ok && w.cnt > 1) ok = wait_all(&pv_done[1], (done[1] - 1) & 1);
                    if (ok) {
                        const float2 x0 = x_ml[part & 1][0][r128], x1 = x_ml[part & 1][1][r128];
                        m = fmaxf(x0.x, x1.x);
                        const float mb = m == -INFINITY ? 0.f : m;
                        wa = ex2_approx(x0.x - mb);
                        wb = w.cnt > 1 ? ex2_approx(x1.x - mb) : 0.f;
                        sum = x0.y * wa + (w.cnt > 1 ? x1.y * wb : 0.f);
                        if (m == -INFINITY) wa = wb = 1.f;         // nothing but scores of minus infinity, or NaN
                    }
                }
                if (!ok) break;
                if (!idle) {
                    tc_fence_after();
                    const float inv = whole ? 1.f / sum : 1.f;
                    wa *= inv;
                    wb *= inv;
                    constexpr int COLS = TWO ? HD : HD / 2;        // columns of this thread: all of its own row, or half of the shared one
                    const int col0 = TWO ? 0 : s * (HD / 2);
#pragma unroll
                    for (int ch = 0; ch < COLS / 32; ++ch) {
                        float o[32];
                        const int col = col0 + ch * 32;
                        tmem_ld32(lanes + O_COL + (TWO ? s * 128 : 0) + col, o);
                        tmem_ld_wait_regs(o);
#pragma unroll
                        for (int x = 0; x < 32; ++x) o[x] *= wa;
                        if (!TWO && w.cnt > 1) {
                            float o2[32];
                            tmem_ld32(lanes + O_COL + 128 + col, o2);
                            tmem_ld_wait_regs(o2);
#pragma unroll
                            for (int x = 0; x < 32; ++x) o[x] += o2[x] * wb;
                        }
                        if (r < R) {
                            if (whole) {
                                uint4* dst = reinterpret_cast<uint4*>((T*)a.out + w.b * a.o_b + t * a.o_t + (int64_t)(head * a.group + gq) * a.o_h + col);
#pragma unroll
                                for (int x = 0; x < 4; ++x) dst[x] = pack8<T>(o + 8 * x);
                            } else {
                                float4* dst = reinterpret_cast<float4*>(a.partial + (slot * MT + rt) * HD + col);
#pragma unroll
                                for (int x = 0; x < 8; ++x) dst[x] = make_float4(o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]);
                            }
                        }
                    }
                    if (r < R && (TWO || s == 0)) {
                        if (!whole) a.partial_ml[slot * MT + rt] = make_float2(m, sum);
                        else if (a.lse) a.lse[((int64_t)w.b * a.T + t) * a.nq + head * a.group + gq] = (m + log2f(sum)) * 0.69314718055994531f;
                    }
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&o_empty);
                if (begins && !whole && tid == 0) {
                    const int64_t last = rg.end + (w.nt - w.cnt) - 1;
                    a.desc[blockIdx.x] = make_int4(w.b, w.item, paged_owner(rg.total, rg.ctas, last) - (int)blockIdx.x + 1, 0);
                }
                more = w.next(a, per_b, TILE);
            }
        }
    }
    cp_async_wait<0>();
    tc_fence_before();
    __syncthreads();
    if (warp == 12) {
        tc_fence_after();
        tmem_dealloc(tmem_base, 512);
    }
    if (tid == 0 && abort_flag && a.status) atomicExch(a.status, 2);
}

}  // namespace jot

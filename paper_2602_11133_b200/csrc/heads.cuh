// Norm of every query and key head with the position rotation in the same pass, and where the results go: to rows of
// their own, or (keys, with the values beside them) straight into the pages of a key-value cache.
//
//   y = x * rsqrt(mean(x^2) + eps) * gain                    over the head_dim elements of one head (with a gain)
//   (a, b) -> m (a cos t - b sin t, b cos t + a sin t)       t = position * inv_freq[i], pair i of the first rotary_dim
//
// Pairs are (i, i + rotary_dim / 2), or (2 i, 2 i + 1) where they are interleaved; elements from rotary_dim on pass.  fp32
// throughout, one rounding at the end.  The angle is the exception: position * inv_freq grows to 10^5 radians and more, of
// which fp32 keeps two digits behind the point, so the product and its reduction to one turn are made in fp64 (a handful of
// operations per pair and row, shared by all heads of the row through shared memory) and only the remainder goes to sincospif.
//
// Bound by HBM: every head is read once and written once.  A lane owns two 16-byte vectors of a head, chosen so that both
// elements of every pair are its own (vectors j and j + rotary_dim / 16, or any two where pairs are interleaved): no
// exchange between lanes but the norm's sum, and two loads in flight per head.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "paged.cuh"
#include "pdl.cuh"

namespace jot {

template <typename T> struct Pack2;
template <typename T> struct PackIsBf16 { static constexpr bool value = false; };
template <> struct PackIsBf16<__nv_bfloat16> { static constexpr bool value = true; };
template <> struct Pack2<__nv_bfloat16> {
    using type = __nv_bfloat162;
    static __device__ __forceinline__ float2 up(type v) { return __bfloat1622float2(v); }
    static __device__ __forceinline__ type down(float a, float b) { return __floats2bfloat162_rn(a, b); }
};
template <> struct Pack2<__half> {
    using type = __half2;
    static __device__ __forceinline__ float2 up(type v) { return __half22float2(v); }
    static __device__ __forceinline__ type down(float a, float b) { return __floats2half2_rn(a, b); }
};
template <typename T>
__device__ __forceinline__ void unpack8(const uint4& v, float* f) {
    const typename Pack2<T>::type* p = reinterpret_cast<const typename Pack2<T>::type*>(&v);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 t = Pack2<T>::up(p[j]);
        f[2 * j] = t.x;
        f[2 * j + 1] = t.y;
    }
}
template <typename T>
__device__ __forceinline__ uint4 pack8(const float* f) {
    uint4 v;
    typename Pack2<T>::type* p = reinterpret_cast<typename Pack2<T>::type*>(&v);
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = Pack2<T>::down(f[2 * j], f[2 * j + 1]);
    return v;
}

// One layer of a paged cache: element (page, head, offset, d) of k at k + page * k_page + ((head * page_size) + offset) * head_dim + d.
struct PagesDev {
    void *k, *v;
    int64_t k_page, v_page;       // elements from one page to the next
    int n_pages, page_size;
};

struct HeadsDev {
    const void* in;
    void* out;
    const void* gain;
    int64_t in_row, in_head, out_row, out_head;      // strides, elements
    int n;
};

struct HeadArgs {
    HeadsDev q, k, v;             // v: copied into the pages (n = 0 without them)
    const int32_t* positions;     // [n_rows]; negative: the row is padding and stays as it was
    const float* inv_freq;        // [half]
    int half;                     // rotary_dim / 2
    float magnitude, eps;
    int head_dim, n_rows, rows_per_cta;
    int to_pages;
    PagesDev pages;
    const int32_t* slots;         // [n_rows] page * page_size + offset; negative: nothing is written to the pages
    int32_t* status;
};

constexpr int kHeadThreads = 256;

// G lanes per head, two vectors a lane; rows_per_cta (a power of two) rows a CTA, each of which has an equal share of the CTA's groups of
// lanes: a group has one row, so what hangs on the row (cos and sin, position, slot) is fetched once for all of its heads, and the next
// head's vectors are requested before the present one's are used.  (The gains are read again for every head, from L1: 16 registers that
// four CTAs an SM do not leave; as it is, the bf16 instances keep 24 to 40 bytes a thread in local memory.  11264 rows of 64 heads: 66 us, 5.57 TB/s,
// 0.85 of the copy; five CTAs an SM 70 us.)
template <typename T, int G, bool INTERLEAVED>
__global__ void __launch_bounds__(kHeadThreads, 4) head_norm_rope_kernel(const HeadArgs a) {
    grid_launch_dependents();
    extern __shared__ float2 cs[];                 // [rows_per_cta][half] (cos, sin) times the magnitude
    constexpr int GROUPS = kHeadThreads / G;
    const int row0 = blockIdx.x * a.rows_per_cta, rows = min(a.rows_per_cta, a.n_rows - row0);
    const int sub = threadIdx.x % G, group = threadIdx.x / G, per_row = GROUPS / a.rows_per_cta, r = group / per_row;
    const int nvec = a.head_dim / 8, rot = a.half / 8;      // rot: vectors of each half (pairs far apart)
    // the two vectors of this lane, -1 where it has none
    int va, vb;
    bool turn = true, turn_b = true;                        // whether they are turned (each of four whole pairs where pairs are interleaved)
    if (INTERLEAVED) {
        va = 2 * sub < nvec ? 2 * sub : -1;
        vb = 2 * sub + 1 < nvec ? 2 * sub + 1 : -1;
        turn = va >= 0 && va * 4 < a.half;
        turn_b = vb >= 0 && vb * 4 < a.half;
    } else if (sub < rot) {
        va = sub;
        vb = sub + rot;
    } else {
        va = 2 * rot + 2 * (sub - rot);
        vb = va + 1 < nvec ? va + 1 : -1;
        va = va < nvec ? va : -1;
        turn = false;
    }
    grid_dependency_wait();
    const int heads = a.q.n + a.k.n + a.v.n, row = row0 + r;
    const bool real = r < rows;
    auto operand = [&](int& h) -> const HeadsDev& {         // of head h of a row's queries, keys and values; h becomes its index among its kind
        if (h < a.q.n) return a.q;
        h -= a.q.n;
        if (h < a.k.n) return a.k;
        h -= a.k.n;
        return a.v;
    };
    uint4 next_a = make_uint4(0, 0, 0, 0), next_b = next_a;
    auto request = [&](int h) {
        if (!real || h >= heads) return;
        const HeadsDev& x = operand(h);
        const uint4* src = reinterpret_cast<const uint4*>((const T*)x.in + row * x.in_row + h * x.in_head);
        if (va >= 0) next_a = src[va];
        if (vb >= 0) next_b = src[vb];
    };
    const int first = group - r * per_row;
    request(first);
    const int pos = real ? a.positions[row] : -1;
    int slot = a.to_pages && real ? a.slots[row] : -1;
    for (int i = threadIdx.x; i < rows * a.half; i += kHeadThreads) {
        const double turns = (double)a.positions[row0 + i / a.half] * (double)a.inv_freq[i % a.half] * 0.15915494309189533577;    // 1 / (2 pi)
        float s, c;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        cs[i] = make_float2(c * a.magnitude, s * a.magnitude);
    }
    __syncthreads();
    if (pos < 0) return;
    // cos and sin of this lane's pairs: eight, of vectors a and b together
    float2 t[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int i = INTERLEAVED ? (j < 4 ? va * 4 + j : vb * 4 + j - 4) : va * 8 + j;
        t[j] = (INTERLEAVED && j >= 4 ? turn_b : turn) ? cs[r * a.half + i] : make_float2(1.f, 0.f);
    }
    int64_t k_at = 0, v_at = 0;                             // head 0 of the row in its page
    if (a.to_pages && slot >= 0) {
        const int page = slot / a.pages.page_size, off = slot - page * a.pages.page_size;
        if (page >= a.pages.n_pages) {
            if (group == r * per_row && sub == 0 && a.status) report_bad_index(a.status);
            slot = -1;
        } else {
            k_at = page * a.pages.k_page + (int64_t)off * a.head_dim;
            v_at = page * a.pages.v_page + (int64_t)off * a.head_dim;
        }
    }
    const int64_t head_in_page = (int64_t)a.pages.page_size * a.head_dim;
    const unsigned mask = G == 32 ? 0xffffffffu : ((1u << G) - 1u) << (threadIdx.x % 32 / G * G);
    for (int item = first; item < heads; item += per_row) {
        uint4 ra = next_a, rb = next_b;
        request(item + per_row);
        int h = item;
        const HeadsDev& x = operand(h);
        const bool is_v = item >= a.q.n + a.k.n, to_page = a.to_pages && item >= a.q.n;
        if (to_page && slot < 0) break;                     // keys and values come last
        T* dst = to_page ? (is_v ? (T*)a.pages.v + v_at : (T*)a.pages.k + k_at) + h * head_in_page : (T*)x.out + row * x.out_row + h * x.out_head;
        if (!is_v) {
            float fa[8], fb[8];
            unpack8<T>(ra, fa);
            unpack8<T>(rb, fb);
            if (x.gain) {
                float ss = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) ss += fa[j] * fa[j] + fb[j] * fb[j];
#pragma unroll
                for (int o = G / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(mask, ss, o);
                const float inv = rsqrtf(ss / (float)a.head_dim + a.eps);
                uint4 ga = make_uint4(0, 0, 0, 0), gb = ga;
                if (va >= 0) ga = reinterpret_cast<const uint4*>(x.gain)[va];
                if (vb >= 0) gb = reinterpret_cast<const uint4*>(x.gain)[vb];
                float g[8];
                unpack8<T>(ga, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) fa[j] *= inv * g[j];
                unpack8<T>(gb, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) fb[j] *= inv * g[j];
            }
            if (INTERLEAVED) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float u = fa[2 * j], w = fa[2 * j + 1], y = fb[2 * j], z = fb[2 * j + 1];
                    if (turn) {
                        fa[2 * j] = u * t[j].x - w * t[j].y;
                        fa[2 * j + 1] = w * t[j].x + u * t[j].y;
                    }
                    if (turn_b) {
                        fb[2 * j] = y * t[4 + j].x - z * t[4 + j].y;
                        fb[2 * j + 1] = z * t[4 + j].x + y * t[4 + j].y;
                    }
                }
            } else if (turn) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float u = fa[j], w = fb[j];
                    fa[j] = u * t[j].x - w * t[j].y;
                    fb[j] = w * t[j].x + u * t[j].y;
                }
            }
            ra = pack8<T>(fa);
            rb = pack8<T>(fb);
        }
        if (va >= 0) reinterpret_cast<uint4*>(dst)[va] = ra;
        if (vb >= 0) reinterpret_cast<uint4*>(dst)[vb] = rb;
    }
}

}  // namespace jot

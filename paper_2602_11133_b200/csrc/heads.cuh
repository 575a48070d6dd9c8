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

#include "pdl.cuh"

namespace jot {

constexpr int32_t kStatusBadIndex = 6;     // a slot, a page or a length outside the pages: skipped or read as zeros

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

// G lanes per head, two vectors a lane; grid: rows_per_cta rows a CTA.
template <typename T, int G, bool INTERLEAVED>
__global__ void __launch_bounds__(kHeadThreads) head_norm_rope_kernel(const HeadArgs a) {
    grid_launch_dependents();
    extern __shared__ float2 cs[];                 // [rows_per_cta][half] (cos, sin) times the magnitude
    const int row0 = blockIdx.x * a.rows_per_cta;
    const int rows = min(a.rows_per_cta, a.n_rows - row0);
    const int sub = threadIdx.x % G, group = threadIdx.x / G;
    constexpr int GROUPS = kHeadThreads / G;
    const int nvec = a.head_dim / 8, rot = a.half / 8;      // rot: vectors of each half (pairs far apart)
    // the two vectors of this lane, -1 where it has none
    int va, vb;
    bool turn;
    if (INTERLEAVED) {
        va = 2 * sub < nvec ? 2 * sub : -1;
        vb = 2 * sub + 1 < nvec ? 2 * sub + 1 : -1;
        turn = true;
    } else if (sub < rot) {
        va = sub;
        vb = sub + rot;
        turn = true;
    } else {
        va = 2 * rot + 2 * (sub - rot);
        vb = va + 1 < nvec ? va + 1 : -1;
        va = va < nvec ? va : -1;
        turn = false;
    }
    grid_dependency_wait();
    for (int i = threadIdx.x; i < rows * a.half; i += kHeadThreads) {
        const int pos = a.positions[row0 + i / a.half];
        const double turns = (double)pos * (double)a.inv_freq[i % a.half] * 0.15915494309189533577;    // 1 / (2 pi)
        float s, c;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        cs[i] = make_float2(c * a.magnitude, s * a.magnitude);
    }
    __syncthreads();
    const int heads = a.q.n + a.k.n + a.v.n;
    const unsigned mask = G == 32 ? 0xffffffffu : ((1u << G) - 1u) << (threadIdx.x % 32 / G * G);
    for (int item = group; item < rows * heads; item += GROUPS) {
        const int r = item / heads, row = row0 + r;
        int h = item - r * heads;
        if (a.positions[row] < 0) continue;
        const bool is_v = h >= a.q.n + a.k.n, is_k = !is_v && h >= a.q.n;
        const HeadsDev& x = is_v ? a.v : (is_k ? a.k : a.q);
        h -= is_v ? a.q.n + a.k.n : (is_k ? a.q.n : 0);
        T* dst;
        if ((is_k || is_v) && a.to_pages) {
            const int slot = a.slots[row];
            const int page = slot / a.pages.page_size;
            if (slot < 0) continue;
            if (page >= a.pages.n_pages) {
                if (sub == 0 && a.status) atomicExch(a.status, kStatusBadIndex);
                continue;
            }
            const int64_t in_page = ((int64_t)h * a.pages.page_size + (slot - page * a.pages.page_size)) * a.head_dim;
            dst = is_v ? (T*)a.pages.v + page * a.pages.v_page + in_page : (T*)a.pages.k + page * a.pages.k_page + in_page;
        } else {
            dst = (T*)x.out + row * x.out_row + h * x.out_head;
        }
        const T* src = (const T*)x.in + row * x.in_row + h * x.in_head;
        uint4 ra = make_uint4(0, 0, 0, 0), rb = ra;
        if (va >= 0) ra = reinterpret_cast<const uint4*>(src)[va];
        if (vb >= 0) rb = reinterpret_cast<const uint4*>(src)[vb];
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
            const float2* t = cs + r * a.half;
            if (INTERLEAVED) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int ia = va * 4 + j, ib = vb * 4 + j;
                    if (va >= 0 && ia < a.half) {
                        const float2 e = t[ia];
                        const float u = fa[2 * j], w = fa[2 * j + 1];
                        fa[2 * j] = u * e.x - w * e.y;
                        fa[2 * j + 1] = w * e.x + u * e.y;
                    }
                    if (vb >= 0 && ib < a.half) {
                        const float2 e = t[ib];
                        const float u = fb[2 * j], w = fb[2 * j + 1];
                        fb[2 * j] = u * e.x - w * e.y;
                        fb[2 * j + 1] = w * e.x + u * e.y;
                    }
                }
            } else if (turn) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float2 e = t[va * 8 + j];
                    const float u = fa[j], w = fb[j];
                    fa[j] = u * e.x - w * e.y;
                    fb[j] = w * e.x + u * e.y;
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

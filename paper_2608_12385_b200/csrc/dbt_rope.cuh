// Rotary positions of queries and keys (sm_100a): the plain operator, forward and transposed, and the form that writes a
// step's keys and values into the paged cache.
//
//   (a, b) -> scale * (a cos t - b sin t, a sin t + b cos t),   t = position * frequency of the pair
//
// The angle is formed in 64 bits and reduced to a fraction of a turn there: position 500000 at frequency 1 is 80000 turns, of
// which fp32 keeps a few digits.  The fraction, below one half, goes through the fp32 sincospif: 2e-7 absolute on cos and sin.
//
// What bounds it: HBM, each element read and written once.  A thread keeps the cosines and sines of its pairs in registers
// and walks a group of heads with them, so the 64-bit work is done once for the group; two 16-byte vectors per head, four
// heads' loads in flight.
#pragma once

#include "dbt_common.cuh"

namespace dbt {

struct RopeParams {
    const void *x, *k, *v;  // k, v: append only
    void *y, *cache;
    const int32_t *positions, *page_table, *seq_lens, *node_counts;
    const double *freq;
    int *status;
    long long xs[3], ks[3], vs[3], ys[3];  // strides of batch, row, head in elements
    long long rows;                        // rows in all
    int per_batch;                         // rows per batch entry (a plain call is one batch entry)
    int hq, hkv, D, rot, heads_per_group;
    int num_pages, pps;
    float scale;
    int inverse, copy_rest;  // copy_rest 0: y is x, the elements that do not turn are in place
};

template <typename T>
struct RopeVec {
    static constexpr int N = 16 / sizeof(T);
};

template <typename T, int N>
__device__ __forceinline__ void rope_load(const T *p, float (&v)[N]);
template <>
__device__ __forceinline__ void rope_load<float, 4>(const float *p, float (&v)[4]) {
    const float4 a = *reinterpret_cast<const float4 *>(p);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
template <>
__device__ __forceinline__ void rope_load<__nv_bfloat16, 8>(const __nv_bfloat16 *p, float (&v)[8]) { load8(p, v); }
template <>
__device__ __forceinline__ void rope_load<float, 1>(const float *p, float (&v)[1]) { v[0] = *p; }
template <>
__device__ __forceinline__ void rope_load<__nv_bfloat16, 1>(const __nv_bfloat16 *p, float (&v)[1]) { v[0] = __bfloat162float(*p); }
__device__ __forceinline__ void rope_store(float *p, const float (&v)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void rope_store(__nv_bfloat16 *p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ void rope_store(T *p, const float (&v)[1]) { store1(p, v[0]); }

// A thread's unit: two vectors of N elements.  Units below `turning` hold N pairs (half layout: elements u*N.. and
// rot/2 + u*N..; interleaved: 2N neighbours), the others copy 2N elements behind rot.  N = 1 serves sizes, strides and
// addresses that 16-byte vectors do not fit.
// APPEND: heads 0..hq-1 are queries, the next hkv keys, the last hkv values (copied).
template <typename T, int N, bool INTER, bool APPEND>
__global__ void __launch_bounds__(256) rope_kernel(const RopeParams p) {
    const int turning = p.rot / (2 * N), units = turning + (p.copy_rest || APPEND ? (p.D - p.rot + 2 * N - 1) / (2 * N) : 0);
    const long long t = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    const long long row = t / units;
    if (row >= p.rows) return;
    const int u = (int)(t - row * units);
    const int b = (int)(row / p.per_batch), i = (int)(row - (long long)b * p.per_batch);
    const int heads = APPEND ? p.hq + 2 * p.hkv : p.hq;
    const int h0 = blockIdx.y * p.heads_per_group, h1 = min(heads, h0 + p.heads_per_group);
    const bool turns = u < turning;
    const int e0 = turns ? (INTER ? 2 * u * N : u * N) : p.rot + (u - turning) * 2 * N;
    const int e1 = turns && !INTER ? e0 + p.rot / 2 : e0 + N;
    const bool second = turns || e1 < p.D;  // (a rest of an odd number of vectors)

    T *page_k = nullptr;
    size_t plane = 0;
    if (APPEND) {
        if (p.node_counts && i >= p.node_counts[b]) return;
        const long long at = (long long)p.seq_lens[b] + i;
        const long long slot = at >> 4;
        int page = -1;
        if (at >= 0 && slot < p.pps) page = p.page_table[(size_t)b * p.pps + slot];
        if (page < 0 || page >= p.num_pages) {
            report(p.status, kStatusBadPage, page);
        } else {
            plane = (size_t)p.num_pages * p.hkv * 16 * p.D;
            page_k = reinterpret_cast<T *>(p.cache) + ((size_t)page * p.hkv * 16 + (at & 15)) * p.D;
        }
    }
    float cs[N], sn[N];
    if (turns) {
        const double pos = (double)p.positions[row] * 0.15915494309189533577;  // 1 / (2 pi)
#pragma unroll
        for (int k = 0; k < N; k++) {
            double part = pos * p.freq[u * N + k];
            part -= rint(part);
            sincospif(2.f * (float)part, &sn[k], &cs[k]);
            cs[k] *= p.scale;
            sn[k] *= p.inverse ? -p.scale : p.scale;
        }
    }
    auto source = [&](int h) -> const T * {
        if (!APPEND || h < p.hq) return reinterpret_cast<const T *>(p.x) + b * p.xs[0] + i * p.xs[1] + h * p.xs[2];
        if (h < p.hq + p.hkv) return reinterpret_cast<const T *>(p.k) + b * p.ks[0] + i * p.ks[1] + (h - p.hq) * p.ks[2];
        return reinterpret_cast<const T *>(p.v) + b * p.vs[0] + i * p.vs[1] + (h - p.hq - p.hkv) * p.vs[2];
    };
    auto target = [&](int h) -> T * {
        if (!APPEND || h < p.hq) return reinterpret_cast<T *>(p.y) + b * p.ys[0] + i * p.ys[1] + h * p.ys[2];
        if (!page_k) return nullptr;
        return h < p.hq + p.hkv ? page_k + (size_t)(h - p.hq) * 16 * p.D : page_k + plane + (size_t)(h - p.hq - p.hkv) * 16 * p.D;
    };
    constexpr int A = 4;  // heads in flight
    for (int h = h0; h < h1; h += A) {
        float x0[A][N], x1[A][N];
#pragma unroll
        for (int a = 0; a < A; a++)
            if (h + a < h1) {
                const T *s = source(h + a);
                rope_load<T, N>(s + e0, x0[a]);
                if (second) rope_load<T, N>(s + e1, x1[a]);
            }
#pragma unroll
        for (int a = 0; a < A; a++) {
            if (h + a >= h1) break;
            T *d = target(h + a);
            if (APPEND && !d) continue;
            if (turns && !(APPEND && h + a >= p.hq + p.hkv)) {
#pragma unroll
                for (int k = 0; k < N; k++) {
                    // the k-th pair: (x0[k], x1[k]), or neighbours in the 2N elements x0, x1
                    float *pa = INTER ? (2 * k < N ? &x0[a][(2 * k) % N] : &x1[a][(2 * k) % N]) : &x0[a][k];
                    float *pb = INTER ? (2 * k + 1 < N ? &x0[a][(2 * k + 1) % N] : &x1[a][(2 * k + 1) % N]) : &x1[a][k];
                    const float va = *pa, vb = *pb;
                    *pa = va * cs[k] - vb * sn[k];
                    *pb = va * sn[k] + vb * cs[k];
                }
            }
            rope_store(d + e0, x0[a]);
            if (second) rope_store(d + e1, x1[a]);
        }
    }
}

}  // namespace dbt

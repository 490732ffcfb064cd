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
// heads' loads in flight, held as they came.  Measured: 8192 rows of 32 heads of 128 (134 MB) 26.7 us, 5.0 TB/s, 77 % of the
// measured copy; 32768 rows of 16 heads (268 MB), half of the head turning, 46.4 us, 88 %.  With vectors that are neighbours in the
// interleaved layout and in the rest (each access half of its sectors) and floats in flight: 40.6 and 75.1 us.
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

// N elements of T as they stand in memory: a 16-byte vector, or one element.
template <typename T, int N>
struct RopeRaw {
    uint4 v;
    __device__ __forceinline__ void load(const T *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<uint4 *>(p) = v; }
    __device__ __forceinline__ void get(float (&x)[N]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if (sizeof(T) == 4) {
                x[i] = __uint_as_float(w[i]);
            } else {
                x[(2 * i) % N] = __uint_as_float(w[i] << 16);
                x[(2 * i + 1) % N] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
    __device__ __forceinline__ void put(const float (&x)[N]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if (sizeof(T) == 4) {
                w[i] = __float_as_uint(x[i]);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(x[(2 * i) % N], x[(2 * i + 1) % N]);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <typename T>
struct RopeRaw<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T *p) { v = *p; }
    __device__ __forceinline__ void store(T *p) const { *p = v; }
    __device__ __forceinline__ void get(float (&x)[1]) const { x[0] = load1(&v); }
    __device__ __forceinline__ void put(const float (&x)[1]) { store1(&v, x[0]); }
};

// A thread's unit: two vectors of N elements, half of the rotated part (or of the rest behind it) apart, so that neighbouring
// threads read and write neighbouring vectors in both layouts.  Half layout: the vectors hold the first and second elements of N
// pairs; interleaved: N / 2 pairs each.  Units behind those that turn copy the rest.  N = 1 serves sizes, strides and addresses that
// 16-byte vectors do not fit; its interleaved unit is one pair.
// APPEND: heads 0..hq-1 are queries, the next hkv keys, the last hkv values (copied).
template <typename T, int N, bool INTER, bool APPEND>
__global__ void __launch_bounds__(256, 3) rope_kernel(const RopeParams p) {
    const int turning = p.rot / (2 * N), resting = p.copy_rest || APPEND ? (p.D - p.rot + 2 * N - 1) / (2 * N) : 0, units = turning + resting;
    const long long t = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    const long long row = t / units;
    if (row >= p.rows) return;
    const int u = (int)(t - row * units);
    const int b = (int)(row / p.per_batch), i = (int)(row - (long long)b * p.per_batch);
    const int heads = APPEND ? p.hq + 2 * p.hkv : p.hq;
    const int h0 = blockIdx.y * p.heads_per_group, h1 = min(heads, h0 + p.heads_per_group);
    const bool turns = u < turning, pair = INTER && N == 1;
    const int e0 = turns ? (pair ? 2 * u : u * N) : p.rot + (u - turning) * N;
    const int e1 = turns ? (pair ? e0 + 1 : e0 + p.rot / 2) : e0 + resting * N;
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
            // the k-th of the unit's pairs
            const int at = !INTER || N == 1 ? u * N + k : k < N / 2 ? e0 / 2 + k : e1 / 2 + k - N / 2;
            double part = pos * p.freq[at];
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
        RopeRaw<T, N> r0[A], r1[A];
#pragma unroll
        for (int a = 0; a < A; a++)
            if (h + a < h1) {
                const T *s = source(h + a);
                r0[a].load(s + e0);
                if (second) r1[a].load(s + e1);
            }
#pragma unroll
        for (int a = 0; a < A; a++) {
            if (h + a >= h1) break;
            T *d = target(h + a);
            if (APPEND && !d) continue;
            if (turns && !(APPEND && h + a >= p.hq + p.hkv)) {
                float x0[N], x1[N];
                r0[a].get(x0);
                r1[a].get(x1);
                auto turn = [](float &va, float &vb, float c, float s) {
                    const float a0 = va, b0 = vb;
                    va = a0 * c - b0 * s;
                    vb = a0 * s + b0 * c;
                };
#pragma unroll
                for (int k = 0; k < N; k++) {
                    if (!INTER || N == 1) turn(x0[k], x1[k], cs[k], sn[k]);
                    else if (k < N / 2) turn(x0[(2 * k) % N], x0[(2 * k + 1) % N], cs[k], sn[k]);
                    else turn(x1[(2 * k) % N], x1[(2 * k + 1) % N], cs[k], sn[k]);
                }
                r0[a].put(x0);
                r1[a].put(x1);
            }
            r0[a].store(d + e0);
            if (second) r1[a].store(d + e1);
        }
    }
}

}  // namespace dbt

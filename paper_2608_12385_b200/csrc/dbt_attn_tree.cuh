// Attention of a tree of drafted tokens over the paged cache (sm_100a).
//
// Row (b, node i, query head h): softmax over the cached positions t < len_b and the nodes on the path from i to its root,
// times their values.  All rows of a sequence that share a KV head read the same keys, so a block takes up to kRows of them
// (node-major: row = node * G + head within the group) and streams the keys once in tiles.
//
// Work split.  The tiles of all (sequence, KV head, row block) items stand in one line, and the line is cut into equal runs,
// one per block: no block waits for the longest sequence, whatever the lengths.  An item inside one run is written out at
// once; of an item that is cut, each run leaves its unnormalised output with its maximum and sum in the workspace, and a second
// kernel joins them in the order of the keys (no atomics: results do not depend on timing).  Lengths are read on the
// device, so a captured call serves later lengths.
#pragma once

#include "dbt_ptx.cuh"

namespace dbt {

struct TreeAttnParams {
    const void *q, *cache;  // cache: this layer's K plane, the V plane behind it
    void *out;
    const int32_t *page_table, *seq_lens, *node_counts, *parents;
    float *part;    // [2 * blocks][rows][D] unnormalised outputs
    float2 *stats;  // [2 * blocks][rows] maximum (in units of log2) and sum
    int *status;
    long long qs[3];
    int B, N, G, hkv, num_pages, pps, blocks;
    float scale_log2;  // softmax scale * log2(e)
};

struct TreeSeq {
    int len, n;
};
// Cached positions and nodes of a sequence, cut to what the page table holds.
__device__ __forceinline__ TreeSeq tree_seq(const TreeAttnParams &p, int b, bool tell = false) {
    TreeSeq s;
    s.len = ld_mut(p.seq_lens + b);
    s.n = p.node_counts ? max(0, min(ld_mut(p.node_counts + b), p.N)) : p.N;
    const long long cap = (long long)p.pps * 16;
    if (s.n > 0 && (s.len < 0 || s.len + (long long)s.n > cap)) {
        if (tell) report(p.status, kStatusBadPage, -1);
        s.n = (int)min((long long)s.n, cap);
        s.len = (int)max(0ll, min((long long)s.len, cap - s.n));
    }
    return s;
}
// Tiles of one item of sequence b, its row blocks.
template <int ROWS, int KEYS>
struct TreePlan {
    static __device__ __forceinline__ int tiles(const TreeSeq &s) { return s.n > 0 ? (s.len + s.n + KEYS - 1) / KEYS : 0; }
    static __device__ __forceinline__ int row_blocks(const TreeAttnParams &p, const TreeSeq &s) { return (s.n * p.G + ROWS - 1) / ROWS; }
    static __device__ __forceinline__ long long units(const TreeAttnParams &p, int b) {
        const TreeSeq s = tree_seq(p, b);
        return (long long)tiles(s) * row_blocks(p, s) * p.hkv;
    }
    // By a whole warp: all units, and of sequence `upto` those before it.
    static __device__ __forceinline__ long long total(const TreeAttnParams &p, int lane, int upto, long long *before) {
        long long sum = 0, part = 0;
        for (int b = lane; b < p.B; b += 32) {
            const long long u = units(p, b);
            sum += u;
            if (b < upto) part += u;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, o);
            part += __shfl_xor_sync(0xffffffffu, part, o);
        }
        if (before) *before = part;
        return sum;
    }
    // By a whole warp: the sequence that unit `at` (< total) lies in, and the units before it.
    static __device__ __forceinline__ int locate(const TreeAttnParams &p, int lane, long long at, long long *before) {
        long long base = 0;
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            const long long mine = b0 + lane < p.B ? units(p, b0 + lane) : 0;
            long long run = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long x = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += x;
            }
            const unsigned past = __ballot_sync(0xffffffffu, base + run > at);
            if (past) {
                const int l = __ffs(past) - 1;
                *before = base + __shfl_sync(0xffffffffu, run - mine, l);
                return b0 + l;
            }
            base += __shfl_sync(0xffffffffu, run, 31);
        }
        return p.B;
    }
    static __device__ __forceinline__ long long per_block(const TreeAttnParams &p, long long all) { return (all + p.blocks - 1) / p.blocks; }
};
// Walks the items of a block's run of units.
template <int ROWS, int KEYS>
struct TreeWalk {
    long long at, end;  // next unit, end of the run
    int b, rb, h;       // current item
    TreeSeq s;
    int tiles, t0, t1, slot;  // the item's tiles, those of this run, the workspace slot (-1: the whole item is here)
    long long first;          // the run's first unit
    long long item0;          // the current item's first unit
    __device__ __forceinline__ bool start(const TreeAttnParams &p, int lane) {
        const long long all = TreePlan<ROWS, KEYS>::total(p, lane, 0, nullptr), per = TreePlan<ROWS, KEYS>::per_block(p, all);
        first = at = (long long)blockIdx.x * per;
        end = min(all, at + per);
        if (at >= end) return false;
        long long before;
        b = TreePlan<ROWS, KEYS>::locate(p, lane, at, &before);
        s = tree_seq(p, b, true);
        tiles = TreePlan<ROWS, KEYS>::tiles(s);
        const int item = (int)((at - before) / tiles), rbs = TreePlan<ROWS, KEYS>::row_blocks(p, s);
        h = item / rbs;
        rb = item - h * rbs;
        item0 = before + (long long)item * tiles;
        place();
        return true;
    }
    __device__ __forceinline__ void place() {
        t0 = (int)(at - item0);
        t1 = (int)min((long long)tiles, end - item0);
        // at most two items of a run are cut: the one it begins inside, the one it ends inside
        slot = t0 == 0 && t1 == tiles ? -1 : 2 * (int)blockIdx.x + (t0 == 0);
    }
    __device__ __forceinline__ bool next(const TreeAttnParams &p) {
        at = item0 + t1;
        if (at >= end) return false;
        item0 += tiles;
        if (++rb == TreePlan<ROWS, KEYS>::row_blocks(p, s)) {
            rb = 0;
            if (++h == p.hkv) {
                h = 0;
                do {
                    s = tree_seq(p, ++b, true);
                    tiles = TreePlan<ROWS, KEYS>::tiles(s);
                } while (tiles == 0);
            }
        }
        place();
        return true;
    }
};

// The ancestors of node i and itself as a bit mask; parents_s holds the sequence's n parents.
__device__ __forceinline__ unsigned long long tree_ancestors(const int *parents_s, int i) {
    unsigned long long m = 0;
    while (i >= 0) {
        m |= 1ull << i;
        i = parents_s[i];
    }
    return m;
}
__device__ __forceinline__ int tree_parent(const TreeAttnParams &p, int b, int i) {
    int up = p.parents[(size_t)b * p.N + i];
    if (up >= i || up < -1) {
        report(p.status, kStatusBadTree, up);
        up = -1;
    }
    return up;
}
__device__ __forceinline__ int tree_page(const TreeAttnParams &p, int b, int slot) {
    int page = p.page_table[(size_t)b * p.pps + slot];
    if (page < 0 || page >= p.num_pages) {
        report(p.status, kStatusBadPage, page);
        page = 0;
    }
    return page;
}

// ---- CUDA-core form: fp32 ------------------------------------------------------------------------------------
// 16 x 16 threads; thread (ty, tx) forms the scores of rows ty * RM .. and keys tx, tx + 16, .. of a tile of 64 keys, and owns
// columns 4 tx .. of the outputs of its rows.
constexpr int kTsKeys = 64;
template <int D, int RM>
struct TreeSimtCfg {
    static constexpr int kRows = 16 * RM;
    static constexpr int kLd = D + 4;  // row stride of Q and K: eight rows' 16-byte pieces fall on different banks
    static constexpr int kLdP = kTsKeys + 4;
    static constexpr int kSmemBytes = (kRows * kLd + kTsKeys * kLd + kTsKeys * D + kRows * kLdP) * 4;
    static constexpr int kBlocksPerSm = kSmemBytes <= 113 * 1024 ? 2 : 1;
};

template <typename T, int D, int RM>
__global__ void __launch_bounds__(256, TreeSimtCfg<D, RM>::kBlocksPerSm) attn_tree_simt_kernel(const TreeAttnParams p) {
    using Cfg = TreeSimtCfg<D, RM>;
    constexpr int ROWS = Cfg::kRows, LD = Cfg::kLd, LDP = Cfg::kLdP, CV = D / 64;
    extern __shared__ __align__(16) float smem_f[];
    float *qs = smem_f, *ks = qs + ROWS * LD, *vs = ks + kTsKeys * LD, *ps = vs + kTsKeys * D;
    __shared__ unsigned long long seen_s[64];
    __shared__ int parents_s[64];
    const int tid = threadIdx.x, lane = tid & 31, tx = tid & 15, ty = tid >> 4;
    TreeWalk<ROWS, kTsKeys> w;
    if (!w.start(p, lane)) return;  // (the same for every warp)
    const T *kplane = reinterpret_cast<const T *>(p.cache), *vplane = kplane + (size_t)p.num_pages * p.hkv * 16 * D;
    do {
        const int rows = min(ROWS, w.s.n * p.G - w.rb * ROWS), r0 = w.rb * ROWS, keys = w.s.len + w.s.n;
        __syncthreads();  // the item before is done with shared memory
        if (tid < w.s.n) parents_s[tid] = tree_parent(p, w.b, tid);
        for (int i = tid; i < ROWS * (D / 8); i += 256) {
            const int r = i / (D / 8), c = (i - r * (D / 8)) * 8, node = (r0 + r) / p.G, g = (r0 + r) - node * p.G;
            float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (r < rows) {
                const T *src = reinterpret_cast<const T *>(p.q) + w.b * p.qs[0] + node * p.qs[1] + (w.h * p.G + g) * p.qs[2] + c;
#pragma unroll
                for (int k = 0; k < 8; k++) x[k] = load1(src + k);
            }
#pragma unroll
            for (int k = 0; k < 8; k++) qs[r * LD + c + k] = x[k] * p.scale_log2;
        }
        __syncthreads();
        if (tid < w.s.n) seen_s[tid] = tree_ancestors(parents_s, tid);
        float o[RM][4 * CV], m_run[RM], l_run[RM];
#pragma unroll
        for (int i = 0; i < RM; i++) {
            m_run[i] = -INFINITY;
            l_run[i] = 0.f;
#pragma unroll
            for (int c = 0; c < 4 * CV; c++) o[i][c] = 0.f;
        }
        for (int t = w.t0; t < w.t1; t++) {
            const int key0 = t * kTsKeys;
            __syncthreads();  // (ancestors written; the tile before is read)
            for (int i = tid; i < kTsKeys * (D / 8); i += 256) {
                const int k = i / (D / 8), c = (i - k * (D / 8)) * 8;
                float a[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (key0 + k < keys) {
                    const int page = tree_page(p, w.b, (key0 + k) >> 4);
                    const size_t at = (((size_t)page * p.hkv + w.h) * 16 + ((key0 + k) & 15)) * D + c;
                    load8(kplane + at, a);
                    load8(vplane + at, v);
                }
                *reinterpret_cast<float4 *>(ks + k * LD + c) = make_float4(a[0], a[1], a[2], a[3]);
                *reinterpret_cast<float4 *>(ks + k * LD + c + 4) = make_float4(a[4], a[5], a[6], a[7]);
                *reinterpret_cast<float4 *>(vs + k * D + c) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4 *>(vs + k * D + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
            }
            __syncthreads();
            float s[RM][4];
#pragma unroll
            for (int i = 0; i < RM; i++) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
#pragma unroll 4
            for (int d = 0; d < D; d += 4) {
                float4 kk[4];
#pragma unroll
                for (int j = 0; j < 4; j++) kk[j] = *reinterpret_cast<const float4 *>(ks + (tx + 16 * j) * LD + d);
#pragma unroll
                for (int i = 0; i < RM; i++) {
                    const float4 qq = *reinterpret_cast<const float4 *>(qs + (ty * RM + i) * LD + d);
#pragma unroll
                    for (int j = 0; j < 4; j++) s[i][j] += qq.x * kk[j].x + qq.y * kk[j].y + qq.z * kk[j].z + qq.w * kk[j].w;
                }
            }
            const bool nodes_here = key0 + kTsKeys > w.s.len;
#pragma unroll
            for (int i = 0; i < RM; i++) {
                const int r = ty * RM + i;
                if (nodes_here) {
                    const unsigned long long seen = r < rows ? seen_s[(r0 + r) / p.G] : 0ull;
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const int node = key0 + tx + 16 * j - w.s.len;
                        if (node >= w.s.n || (node >= 0 && !((seen >> node) & 1))) s[i][j] = -INFINITY;
                    }
                }
                float mx = fmaxf(fmaxf(s[i][0], s[i][1]), fmaxf(s[i][2], s[i][3]));
#pragma unroll
                for (int x = 8; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
                const float m_new = fmaxf(m_run[i], mx), m_sub = m_new == -INFINITY ? 0.f : m_new;
                const float corr = exp2f(m_run[i] - m_sub);
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const float e = exp2f(s[i][j] - m_sub);
                    sum += e;
                    ps[r * LDP + tx + 16 * j] = e;
                }
#pragma unroll
                for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
                m_run[i] = m_new;
                l_run[i] = l_run[i] * corr + sum;
#pragma unroll
                for (int c = 0; c < 4 * CV; c++) o[i][c] *= corr;
            }
            __syncwarp();  // a row's probabilities are written and read by one half of a warp
#pragma unroll 2
            for (int k = 0; k < kTsKeys; k += 4) {
                float4 pp[RM];
#pragma unroll
                for (int i = 0; i < RM; i++) pp[i] = *reinterpret_cast<const float4 *>(ps + (ty * RM + i) * LDP + k);
#pragma unroll
                for (int kk = 0; kk < 4; kk++)
#pragma unroll
                    for (int c = 0; c < CV; c++) {
                        const float4 vv = *reinterpret_cast<const float4 *>(vs + (k + kk) * D + c * 64 + tx * 4);
#pragma unroll
                        for (int i = 0; i < RM; i++) {
                            const float e = kk == 0 ? pp[i].x : kk == 1 ? pp[i].y : kk == 2 ? pp[i].z : pp[i].w;
                            if (nodes_here && e == 0.f) continue;  // a node that this row does not see may hold NaN
                            o[i][4 * c + 0] += e * vv.x;
                            o[i][4 * c + 1] += e * vv.y;
                            o[i][4 * c + 2] += e * vv.z;
                            o[i][4 * c + 3] += e * vv.w;
                        }
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < RM; i++) {
            const int r = ty * RM + i;
            if (r >= rows) continue;
            if (w.slot >= 0) {
                float *dst = p.part + ((size_t)w.slot * ROWS + r) * D;
#pragma unroll
                for (int c = 0; c < CV; c++)
                    *reinterpret_cast<float4 *>(dst + c * 64 + tx * 4) = make_float4(o[i][4 * c], o[i][4 * c + 1], o[i][4 * c + 2], o[i][4 * c + 3]);
                if (tx == 0) p.stats[(size_t)w.slot * ROWS + r] = make_float2(m_run[i], l_run[i]);
            } else {
                const int node = (r0 + r) / p.G, g = (r0 + r) - node * p.G;
                T *dst = reinterpret_cast<T *>(p.out) + (((size_t)w.b * p.N + node) * p.hkv * p.G + w.h * p.G + g) * D;
                const float inv = l_run[i] == 0.f ? 0.f : 1.f / l_run[i];
#pragma unroll
                for (int c = 0; c < CV; c++)
#pragma unroll
                    for (int e = 0; e < 4; e++) store1(dst + c * 64 + tx * 4 + e, o[i][4 * c + e] * inv);
            }
        }
    } while (w.next(p));
}

// ---- joining the parts of items that were cut --------------------------------------------------------------------
// A warp per output row, in the order of the keys.
template <typename T, int D, int ROWS, int KEYS>
__global__ void __launch_bounds__(256) attn_tree_join_kernel(const TreeAttnParams p) {
    using Plan = TreePlan<ROWS, KEYS>;
    const int lane = threadIdx.x & 31, rows_per_seq = p.N * p.G;
    const long long id = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), per_b = (long long)p.hkv * rows_per_seq;
    const int b = (int)(id / per_b);
    if (b >= p.B) return;
    const int rest = (int)(id - b * per_b), h = rest / rows_per_seq, row = rest - h * rows_per_seq;
    pdl_wait();
    const TreeSeq s = tree_seq(p, b);
    if (row >= s.n * p.G) return;
    long long before;
    const long long per = Plan::per_block(p, Plan::total(p, lane, b, &before));
    const int tiles = Plan::tiles(s), rb = row / ROWS, r = row - rb * ROWS;
    const long long item0 = before + (long long)(h * Plan::row_blocks(p, s) + rb) * tiles;
    const int c0 = (int)(item0 / per), c1 = (int)((item0 + tiles - 1) / per);
    if (c0 == c1) return;
    auto slot = [&](int c) -> size_t { return (size_t)(2 * c + (c == c0)) * ROWS + r; };
    float m = -INFINITY;
    for (int c = c0 + lane; c <= c1; c += 32) m = fmaxf(m, __ldcg(p.stats + slot(c)).x);
    m = warp_max(m);
    const float m_sub = m == -INFINITY ? 0.f : m;
    constexpr int E = D / 32;
    float o[E], l = 0.f;
#pragma unroll
    for (int e = 0; e < E; e++) o[e] = 0.f;
#pragma unroll 4
    for (int c = c0; c <= c1; c++) {
        const float2 st = __ldcg(p.stats + slot(c));
        const float f = exp2f(st.x - m_sub);
        const float *src = p.part + slot(c) * D + lane * E;
        float x[E];
        if (E == 4) {
            const float4 a = __ldcg(reinterpret_cast<const float4 *>(src));
            x[0] = a.x; x[1] = a.y; x[E - 2] = a.z; x[E - 1] = a.w;
        } else {
            const float2 a = __ldcg(reinterpret_cast<const float2 *>(src));
            x[0] = a.x; x[1] = a.y;
        }
        l += f * st.y;
#pragma unroll
        for (int e = 0; e < E; e++) o[e] += f * x[e];
    }
    const int node = row / p.G, g = row - node * p.G;
    T *dst = reinterpret_cast<T *>(p.out) + (((size_t)b * p.N + node) * p.hkv * p.G + h * p.G + g) * D + lane * E;
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < E; e++) store1(dst + e, o[e] * inv);
}

}  // namespace dbt

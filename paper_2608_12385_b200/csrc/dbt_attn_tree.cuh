// Attention of a tree of drafted tokens over the paged cache (sm_100a).
//
// Row (b, node i, query head h): softmax over the cached positions t < len_b and the nodes on the path from i to its root,
// times their values.  All rows of a sequence that share a KV head read the same keys, so a block takes up to kRows of them
// (node-major: row = node * G + head within the group) and streams the keys once in tiles.
//
// Work split.  The tiles of all (sequence, KV head, row block) items stand in one line, each item headed by `lead` empty units for
// what it costs besides its tiles, and the line is cut into equal runs, one per block: no block waits for the longest
// sequence, whatever the lengths.  An item inside one run is written out at once; of an item that is cut, each run leaves its
// unnormalised output with its maximum and sum in the workspace, and a second kernel joins them in the order of the keys (no
// atomics: results do not depend on timing).  Lengths are read on the device, so a captured call serves later lengths.
//
// Measured, bf16, head dimension 128, a call with both kernels: 16 sequences of up to 2048 keys and 16 nodes, 16 heads over 8 (74 MB of
// keys and values) 35 us, 2.1 TB/s; 4 sequences of 32768 keys and 64 nodes, 32 heads over 8 (541 MB, 137 GFLOP) 175 to 184 us, 2.9 to 3.1 TB/s
// and 0.75 to 0.78 PFLOP/s, of which 156 us (3.5 TB/s, 0.88 PFLOP/s) are the first kernel's.
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
    int lead;       // empty units ahead of an item
    int q_vectors;  // queries can be read in 16-byte vectors
    int g_inverse;  // 2^16 / G rounded up: (row * g_inverse) >> 16 is row / G up to 1024 rows
    float scale_log2;  // softmax scale * log2(e)
};

struct TreeSeq {
    int len, n;
};
// Cached positions and nodes of a sequence, cut to what the page table holds.
__device__ __forceinline__ TreeSeq tree_seq(const TreeAttnParams &p, int b, bool tell = false) {
    TreeSeq s;
    s.len = p.seq_lens[b];
    s.n = p.node_counts ? max(0, min(p.node_counts[b], p.N)) : p.N;
    const long long cap = (long long)p.pps * 16;
    if (s.n > 0 && (s.len < 0 || s.len + (long long)s.n > cap)) {
        if (tell) report(p.status, kStatusBadPage, -1);
        s.n = (int)min((long long)s.n, cap);
        s.len = (int)max(0ll, min((long long)s.len, cap - s.n));
    }
    return s;
}
// The line of units.
template <int ROWS, int KEYS>
struct TreePlan {
    static __device__ __forceinline__ int tiles(const TreeSeq &s) { return s.n > 0 ? (s.len + s.n + KEYS - 1) / KEYS : 0; }
    static __device__ __forceinline__ int row_blocks(const TreeAttnParams &p, const TreeSeq &s) { return (s.n * p.G + ROWS - 1) / ROWS; }
    static __device__ __forceinline__ int units(const TreeAttnParams &p, int b) {  // (the host has checked that the line fits 31 bits)
        const TreeSeq s = tree_seq(p, b);
        return s.n > 0 ? (tiles(s) + p.lead) * row_blocks(p, s) * p.hkv : 0;
    }
    // By a whole warp: all units, and of sequence `upto` those before it.
    static __device__ __forceinline__ int total(const TreeAttnParams &p, int lane, int upto, int *before) {
        int sum = 0, part = 0;
        for (int b = lane; b < p.B; b += 32) {
            const int u = units(p, b);
            sum += u;
            if (b < upto) part += u;
        }
        if (before) *before = __reduce_add_sync(0xffffffffu, part);
        return __reduce_add_sync(0xffffffffu, sum);
    }
    // By a whole warp: the sequence that unit `at` (< total) lies in, and the units before it.
    static __device__ __forceinline__ int locate(const TreeAttnParams &p, int lane, int at, int *before) {
        int base = 0;
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            const int mine = b0 + lane < p.B ? units(p, b0 + lane) : 0;
            int run = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, run, o);
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
    static __device__ __forceinline__ int per_block(const TreeAttnParams &p, int all) { return all / p.blocks + (all % p.blocks != 0); }
};
// Walks the items of a block's run of units.
template <int ROWS, int KEYS>
struct TreeWalk {
    using Plan = TreePlan<ROWS, KEYS>;
    int end, item0;        // end of the run; the current item's first unit
    int b, rb, h;          // current item
    TreeSeq s;
    int tiles, t0, t1, slot;  // the item's tiles, those of this run, the workspace slot (-1: the whole item is here)
    // False where the run holds no tile.
    __device__ __forceinline__ bool start(const TreeAttnParams &p, int lane) {
        const int all = Plan::total(p, lane, 0, nullptr), per = Plan::per_block(p, all);
        if (all == 0 || (int)blockIdx.x > (all - 1) / per) return false;
        const int at = (int)blockIdx.x * per;
        end = at + min(per, all - at);
        int before;
        b = Plan::locate(p, lane, at, &before);
        s = tree_seq(p, b, true);
        tiles = Plan::tiles(s);
        const int units = tiles + p.lead, item = (at - before) / units, rbs = Plan::row_blocks(p, s);
        h = item / rbs;
        rb = item - h * rbs;
        item0 = before + item * units;
        return place(p, at) || next(p);
    }
    // The tiles of the current item in the run's part of it, from unit `at` on.
    __device__ __forceinline__ bool place(const TreeAttnParams &p, int at) {
        const int first = item0 + p.lead;
        t0 = max(0, at - first);
        t1 = min(tiles, end - first);
        // at most two items of a run are cut: the one it begins inside, the one it ends inside
        slot = t0 == 0 && t1 == tiles ? -1 : 2 * (int)blockIdx.x + (t0 == 0);
        return t1 > t0;
    }
    __device__ __forceinline__ bool next(const TreeAttnParams &p) {
        item0 += tiles + p.lead;
        if (item0 >= end) return false;
        if (++rb == Plan::row_blocks(p, s)) {
            rb = 0;
            if (++h == p.hkv) {
                h = 0;
                do {
                    s = tree_seq(p, ++b, true);
                    tiles = Plan::tiles(s);
                } while (tiles == 0);
            }
        }
        return place(p, item0);  // (false: the run ends in the item's empty units)
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
// columns 4 tx .. of the outputs of its rows.  RM is 1 up to 16 rows that share a KV head (two blocks per SM), else 4 (a quarter of the
// reads of keys and values from shared memory per product).
// What bounds it: the fp32 multiply-adds and the reads from shared memory that feed them: 8 sequences of 4096
// keys and 64 nodes, 32 heads of 128 over 8, 1371 us, 25 TFLOP/s; 4 of 4096 keys and 4 nodes, 4 heads of 64, 38 us, 0.9 TB/s: the
// loads of a tile are not under way while the one before is used.  Short sequences: the two launches (14 us a call with the binding).
constexpr int kTsKeys = 64;
template <int D, int RM>
struct TreeSimtCfg {
    static constexpr int kRows = 16 * RM;
    static constexpr int kLd = D + 4;  // row stride of Q and K: eight rows' 16-byte pieces fall on different banks
    static constexpr int kLdP = kTsKeys + 4;
    static constexpr int kSmemBytes = (kRows * kLd + kTsKeys * kLd + kTsKeys * D + kRows * kLdP) * 4;
    static constexpr int kBlocksPerSm = kSmemBytes <= 113 * 1024 ? 2 : 1;
};

template <int D, int RM>
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
    const float *kplane = reinterpret_cast<const float *>(p.cache), *vplane = kplane + (size_t)p.num_pages * p.hkv * 16 * D;
    do {
        const int rows = min(ROWS, w.s.n * p.G - w.rb * ROWS), r0 = w.rb * ROWS, keys = w.s.len + w.s.n;
        __syncthreads();  // the item before is done with shared memory
        if (tid < w.s.n) parents_s[tid] = tree_parent(p, w.b, tid);
        for (int i = tid; i < ROWS * (D / 8); i += 256) {
            const int r = i / (D / 8), c = (i - r * (D / 8)) * 8, node = (r0 + r) / p.G, g = (r0 + r) - node * p.G;
            float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (r < rows) {
                const float *src = reinterpret_cast<const float *>(p.q) + w.b * p.qs[0] + node * p.qs[1] + (w.h * p.G + g) * p.qs[2] + c;
#pragma unroll
                for (int k = 0; k < 8; k++) x[k] = src[k];
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
                float *dst = reinterpret_cast<float *>(p.out) + (((size_t)w.b * p.N + node) * p.hkv * p.G + w.h * p.G + g) * D;
                const float inv = l_run[i] == 0.f ? 0.f : 1.f / l_run[i];
#pragma unroll
                for (int c = 0; c < CV; c++)
#pragma unroll
                    for (int e = 0; e < 4; e++) dst[c * 64 + tx * 4 + e] = o[i][4 * c + e] * inv;
            }
        }
    } while (w.next(p));
}

// ---- tensor-core form: bf16 --------------------------------------------------------------------------------------
// Two groups of four softmax warps, a thread per row, alternate on the tensor cores: while one group turns its scores into
// probabilities the products of the other run.  PAIR (more than 128 rows share a KV head): the groups own a 128-row tile each and
// both see every tile of 128 keys.  Otherwise they share one row tile and take the key tiles in turn; the two outputs are
// joined where they stand, in tensor memory.  Per key tile: S = Q K^T into tensor memory, P = exp2 of the scaled scores less the row's
// maximum written back over S as bf16, O += P V with P from tensor memory.  O is rescaled only when a row's maximum has grown by
// more than 2^8 (P stays below 2^8: the same relative error).  P is rounded to bf16 (2^-9 on average, relative), which the
// tensor cores need; the sum adds the unrounded values.
//
// What bounds it: 256 rows over long sequences, the turns between the tensor cores and the softmax warps.  A pair of key tiles' work takes
// 4100 cycles: 2240 in which a group turns its scores into probabilities (half of that is the special-function unit, 16
// exponentials a cycle; tensor-memory and shared-memory traffic the rest) and 1640 in which it waits for its products (1200 of the
// tensor pipe, and the signals).  HBM would take 2150, and loads taken out save 4 %.  128 rows or fewer and ragged lengths: what a run
// costs besides its tiles, of 67k cycles 4k to find its place, 4k for the first queries, 12k for joining the groups and writing.
// Not better: scores of 64 keys in two buffers (240 us where this form took 156: products 64 wide take as long as 128 wide),
// 16 softmax warps with half a row a thread (176), a quarter of the exponentials as polynomials on the multiply-add pipes
// (173: registers), scores read in pieces of 32 twice (169).
//
// Values that are not finite.  A node that a row does not see has probability 0, but 0 * NaN in the product is NaN.  So the
// values of the nodes, once in shared memory, are looked through: elements that are not finite are replaced by 0 there, and
// the rows that do see the node add them at the end.  Slots behind the last node are cleared the same way.
//
// Roles: warps 0..3, 4..7 softmax, 8 TMA, 9 MMA and tensor memory, 10 and 11 queries, parents and the look through the values.
// An item's queries are loaded, and its first scores formed, while the softmax warps write the output of the item before.
// All waits are bounded.
template <int DH, bool PAIR>
struct TreeMmaCfg {
    static constexpr int kRows = PAIR ? 256 : 128;
    static constexpr int kKeys = 128;
    static constexpr int kThreads = 384;
    static constexpr int kHalves = DH / 64;
    static constexpr int kTileBytes = 128 * DH * 2;  // 128 rows of queries, keys or values
    static constexpr int kQTiles = PAIR ? 2 : 1;
    static constexpr int kStagesK = DH == 128 ? 3 : 5, kStagesV = DH == 128 ? (PAIR ? 2 : 3) : 5;
    static constexpr int kTail = 2048 + 128 + 64 + 512;  // statistics, parents, flags, barriers
    static constexpr int kSmemBytes = (kQTiles + kStagesK + kStagesV) * kTileBytes + kTail;
    static constexpr int kTmemCols = 512;
    static_assert(kSmemBytes <= 227 * 1024, "shared memory of one SM");
    static_assert(8 * (2 * kStagesK + 3 * kStagesV + 11) + 4 <= 512, "barrier area");
};
constexpr float kTreeRescaleLog2 = 8.f;

__device__ __forceinline__ uint64_t pack_f32x2(float a, float b) { return (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a); }
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }

template <int DH, bool PAIR>
__global__ void __launch_bounds__(384, 1) attn_tree_mma_kernel(const __grid_constant__ CUtensorMap tmKV, const TreeAttnParams p) {
    using Cfg = TreeMmaCfg<DH, PAIR>;
    constexpr int SK = Cfg::kStagesK, SV = Cfg::kStagesV, HALVES = Cfg::kHalves, KS = DH / 16, KEYS = Cfg::kKeys, ROWS = Cfg::kRows;
    constexpr uint32_t kHalfBytes = 128 * 128;  // queries: 128 rows of one 64-column piece
    constexpr uint32_t kGroup = HALVES * 1024;  // keys, values: 8 rows, their 64-column pieces one after the other
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t q_s = smem_u32(smem_raw), k_s = q_s + Cfg::kQTiles * Cfg::kTileBytes, v_s = k_s + SK * Cfg::kTileBytes;
    uint8_t *tail = smem_raw + (Cfg::kQTiles + SK + SV) * Cfg::kTileBytes;
    float2(*stats_s)[128] = reinterpret_cast<float2(*)[128]>(tail);                  // the groups' maxima and sums
    signed char(*parents_s)[64] = reinterpret_cast<signed char(*)[64]>(tail + 2048);     // parents, two items
    unsigned long long *bad_s = reinterpret_cast<unsigned long long *>(tail + 2176);  // nodes with values that are not finite, two items
    int *failed_s = reinterpret_cast<int *>(tail + 2192);
    const uint32_t bars = smem_u32(tail + 2240);
    auto k_full = [&](int s) { return bars + 8u * s; };
    auto k_empty = [&](int s) { return bars + 8u * (SK + s); };
    auto v_full = [&](int s) { return bars + 8u * (2 * SK + s); };
    auto v_empty = [&](int s) { return bars + 8u * (2 * SK + SV + s); };
    auto v_clean = [&](int s) { return bars + 8u * (2 * SK + 2 * SV + s); };  // looked through
    const uint32_t more = bars + 8u * (2 * SK + 3 * SV);
    auto s_full = [&](int i) { return more + 8u * i; };
    auto p_full = [&](int i) { return more + 8u * (2 + i); };
    auto o_full = [&](int i) { return more + 8u * (4 + i); };
    auto q_full = [&](int n) { return more + 8u * (6 + (n & 1)); };  // item n's queries and parents
    auto e_done = [&](int n) { return more + 8u * (8 + (n & 1)); };  // item n's output has been read by all softmax warps
    const uint32_t q_empty = more + 8u * 10;                         // all products with the queries are done
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(tail + 2240 + 8 * (2 * SK + 3 * SV + 11));

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < SK; s++) {
            mbar_init(k_full(s), 1);
            mbar_init(k_empty(s), 1);
        }
        for (int s = 0; s < SV; s++) {
            mbar_init(v_full(s), 1);
            mbar_init(v_empty(s), 1);
            mbar_init(v_clean(s), 2);
        }
        for (int i = 0; i < 2; i++) {
            mbar_init(s_full(i), 1);
            mbar_init(p_full(i), 4);
            mbar_init(o_full(i), 2);  // the tensor cores are done; the issuer passes on what it knows of the values
            mbar_init(q_full(i), 2);
            mbar_init(e_done(i), 8);
        }
        mbar_init(q_empty, 1);
        *failed_s = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)),
                     "r"((uint32_t)Cfg::kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *tmem_holder;
    auto t_s = [&](int i) { return tmem + 128u * i; };
    auto t_o = [&](int i) { return tmem + 256u + (uint32_t)DH * i; };
    pdl_launch_dependents();  // (the joining kernel waits for this one before it reads anything)

    TreeWalk<ROWS, KEYS> w;
    const bool aligned = (q_s & 1023u) == 0;  // (dynamic shared memory begins the block's: always)
    if (!aligned && tid == 0) report(p.status, kStatusWaitExpired, 940);
    const bool work = aligned && w.start(p, lane);
    bool ok = true;
    // the current item's queries by threads x of `threads`: all copies of a thread are under way at once
    auto load_q = [&](int x, int threads) {
        constexpr int CH = DH / 8;
        const __nv_bfloat16 *q = reinterpret_cast<const __nv_bfloat16 *>(p.q);
        const int row0 = w.rb * ROWS, rows = min(ROWS, w.s.n * p.G - row0), ch = x % CH;
        const __nv_bfloat16 *base = q + w.b * p.qs[0] + w.h * p.G * p.qs[2] + ch * 8;
#pragma unroll 4
        for (int row = x / CH; row < Cfg::kQTiles * 128; row += threads / CH) {
            const int node = ((row0 + row) * p.g_inverse) >> 16, g = row0 + row - node * p.G;
            const uint32_t dst = q_s + (row >> 7) * Cfg::kTileBytes + (ch >> 3) * kHalfBytes + (row & 127) * 128 + (((ch & 7) ^ (row & 7)) << 4);
            const __nv_bfloat16 *src = row < rows ? base + node * p.qs[1] + g * p.qs[2] : q;
            if (p.q_vectors) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(row < rows ? 16 : 0) : "memory");
            } else {
                uint32_t y[4] = {0, 0, 0, 0};
                if (row < rows)
#pragma unroll
                    for (int k = 0; k < 4; k++)
                        y[k] = (uint32_t)__bfloat16_as_ushort(src[2 * k]) | ((uint32_t)__bfloat16_as_ushort(src[2 * k + 1]) << 16);
                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(dst), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    };
    // waits of a whole warp, its first lane looking
    auto wait = [&](uint32_t bar, int parity) {
        bool r = true;
        if (lane == 0) r = mbar_wait(bar, parity & 1);
        return (bool)__shfl_sync(0xffffffffu, r, 0);
    };
    if (work && warp == 8) {
        // ---- TMA: lane l brings page l of the tile
        if (lane == 0) tma_prefetch_desc(&tmKV);
        const uint64_t once = l2_evict_first_policy();
        const bool reread = p.N * p.G > ROWS;  // other row blocks read the same pages soon
        const long long v_row0 = (long long)p.num_pages * p.hkv * 16;
        int c = 0, nk = 0, nv = 0;  // tiles begun; tiles of keys, of values requested
        do {
            const int pages_total = (w.s.len + w.s.n + 15) >> 4;
            const bool loads = lane < 8;
            int page = loads && w.t0 * 8 + lane < pages_total ? tree_page(p, w.b, w.t0 * 8 + lane) : 0;
            for (int t = w.t0; t < w.t1 && ok; t++, c++) {
                const int sk = c % SK, sv = c % SV, np = min(8, pages_total - t * 8);
                const int row = (int)(((long long)page * p.hkv + w.h) * 2);  // in groups of 8 rows
                auto load = [&](uint32_t dst, uint32_t bar, long long row0) {
                    if (!(loads && lane < np)) return;
                    const int at = (int)(row0 / 8) + row;
                    if (reread) tma_load_4d(dst + lane * 2 * kGroup, &tmKV, bar, 0, 0, 0, at);
                    else tma_load_4d_hint(dst + lane * 2 * kGroup, &tmKV, bar, 0, 0, 0, at, once);
                };
                const int nx = (t + 1) * 8 + lane;
                const int next_page = loads && t + 1 < w.t1 && nx < pages_total ? tree_page(p, w.b, nx) : 0;
                if (lane == 0) {
                    if (c >= SK) ok = mbar_wait(k_empty(sk), ((c / SK) - 1) & 1);
                    if (ok) mbar_expect_tx(k_full(sk), (uint32_t)np * HALVES * 2048);
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (ok) load(k_s + sk * Cfg::kTileBytes, k_full(sk), 0);
                nk += ok;
                if (lane == 0 && ok) {
                    if (c >= SV) ok = mbar_wait(v_empty(sv), ((c / SV) - 1) & 1);
                    if (ok) mbar_expect_tx(v_full(sv), (uint32_t)np * HALVES * 2048);
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (ok) load(v_s + sv * Cfg::kTileBytes, v_full(sv), v_row0);
                nv += ok;
                page = next_page;
            }
        } while (ok && w.next(p));
        if (!ok && lane == 0) report(p.status, kStatusWaitExpired, 900);
        // the last loads have landed before the block leaves, also where a wait ran out
        if (lane == 0) {
            for (int j = max(0, nk - SK); j < nk; j++) mbar_wait(k_full(j % SK), (j / SK) & 1, kWaitCycles / SK);
            for (int j = max(0, nv - SV); j < nv; j++) mbar_wait(v_full(j % SV), (j / SV) & 1, kWaitCycles / SV);
        }
    } else if (work && warp == 9) {
        // ---- MMA issuer (lane 0)
        constexpr uint32_t idesc_qk = umma_idesc(KEYS);
        constexpr uint32_t idesc_pv = umma_idesc(DH) | (1u << 16);  // B is MN-major
        auto arrive_after = [&](uint32_t bar, int parity) {
            const bool r = wait(bar, parity);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            return r;
        };
        auto qk = [&](int i, int c) {
            if (lane != 0) return;
#pragma unroll
            for (int k = 0; k < KS; k++) {
                const int h = k >> 2;
                umma_f16(t_s(i), umma_smem_desc(q_s + (PAIR ? i : 0) * Cfg::kTileBytes + h * kHalfBytes) + 2 * (k & 3),
                         umma_smem_desc_groups(k_s + (c % SK) * Cfg::kTileBytes + h * 1024, kGroup, 0) + 2 * (k & 3), idesc_qk, k != 0);
            }
            umma_commit(s_full(i));
        };
        auto pv = [&](int i, int c, bool add) {
            if (lane != 0) return;
            const uint64_t vd = umma_smem_desc_groups(v_s + (c % SV) * Cfg::kTileBytes, kGroup, 1024);
#pragma unroll
            for (int k = 0; k < KEYS / 16; k++) umma_f16_ts(t_o(i), t_s(i) + 8 * k, vd + (2 * kGroup >> 4) * k, idesc_pv, add || k != 0);
        };
        auto commit = [&](uint32_t bar) {
            if (lane == 0) umma_commit(bar);
        };
        auto done = [&](int i) {
            commit(o_full(i));
            if (lane == 0) mbar_arrive(o_full(i));
        };
        int c = 0, n = 0, pn[2] = {0, 0};
        do {
            const int T = w.t1 - w.t0, rows = min(ROWS, w.s.n * p.G - w.rb * ROWS);
            const int groups = PAIR && rows > 128 ? 2 : 1;  // PAIR: groups with rows
            ok = arrive_after(q_full(n), n >> 1);
            if (PAIR) {
                ok = ok && arrive_after(k_full(c % SK), c / SK);
                if (!ok) break;
                for (int i = 0; i < groups; i++) qk(i, c);
                commit(k_empty(c % SK));
                if (T == 1) commit(q_empty);
                if (n > 0) ok = arrive_after(e_done(n - 1), (n - 1) >> 1);  // the output's place is free
                for (int t = 0; t < T && ok; t++, c++) {
                    if (t + 1 < T) ok = arrive_after(k_full((c + 1) % SK), (c + 1) / SK);
                    ok = ok && arrive_after(v_clean(c % SV), c / SV);
                    for (int i = 0; i < groups && ok; i++) {
                        ok = arrive_after(p_full(i), pn[i]++);
                        if (!ok) break;
                        pv(i, c, t > 0);
                        if (t + 1 < T) qk(i, c + 1);
                        else done(i);
                    }
                    if (!ok) break;
                    commit(v_empty(c % SV));
                    if (t + 1 < T) commit(k_empty((c + 1) % SK));
                    if (t + 2 == T) commit(q_empty);
                }
            } else {
                for (int t = 0; t < min(2, T) && ok; t++) {
                    ok = arrive_after(k_full((c + t) % SK), (c + t) / SK);
                    if (!ok) break;
                    qk(t, c + t);
                    commit(k_empty((c + t) % SK));
                }
                if (ok && T <= 2) commit(q_empty);
                if (ok && n > 0) ok = arrive_after(e_done(n - 1), (n - 1) >> 1);  // the outputs' place is free
                for (int t = 0; t < T && ok; t++, c++) {
                    const int i = t & 1;
                    ok = arrive_after(v_clean(c % SV), c / SV) && arrive_after(p_full(i), pn[i]++);
                    if (!ok) break;
                    pv(i, c, t > 1);
                    commit(v_empty(c % SV));
                    if (t + 2 < T) {
                        ok = arrive_after(k_full((c + 2) % SK), (c + 2) / SK);
                        if (!ok) break;
                        qk(i, c + 2);
                        commit(k_empty((c + 2) % SK));
                        if (t + 3 == T) commit(q_empty);
                    } else {
                        done(i);
                    }
                }
            }
            n++;
        } while (ok && w.next(p));
        if (!ok && lane == 0) report(p.status, kStatusWaitExpired, 910);
    } else if (work && warp >= 10) {
        // ---- queries, parents, values that are not finite: 64 threads
        const int x = tid - 320;
        int c = 0, n = 0;
        do {
            const int parent = x < w.s.n ? p.parents[(size_t)w.b * p.N + x] : -1;
            if (n > 1) ok = wait(e_done(n - 2), (n - 2) >> 1);  // the buffers of the item before the last are free
            if (ok && n > 0) ok = wait(q_empty, n - 1);
            if (!ok) break;
            if (n > 0) load_q(x, 64);  // (the first item's come from the softmax warps, which have nothing else to do yet)
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            // a bad parent counts as none
            if (x < w.s.n && (parent >= x || parent < -1)) report(p.status, kStatusBadTree, parent);
            parents_s[n & 1][x] = (signed char)(parent >= x || parent < -1 ? -1 : parent);
            if (x == 0) bad_s[n & 1] = 0;
            if (n == 0) asm volatile("bar.sync 3, 320;" ::: "memory");
            asm volatile("bar.sync 2, 64;" ::: "memory");  // (both warps: bad_s is cleared before either marks a node)
            if (lane == 0) mbar_arrive(q_full(n));
            for (int t = w.t0; t < w.t1 && ok; t++, c++) {
                const int sv = c % SV;
                ok = wait(v_full(sv), c / SV);
                if (!ok) break;
                const int key0 = t * KEYS, first = max(0, w.s.len - key0), keys = min(KEYS, w.s.len + w.s.n - key0);
                if (first < KEYS) {
                    auto at = [&](int chunk) {  // address of the chunk-th 16 bytes of the rows (and pieces) in order
                        const int row = chunk / (8 * HALVES), rest = chunk - row * (8 * HALVES);
                        return v_s + sv * Cfg::kTileBytes + (row >> 3) * kGroup + (rest >> 3) * 1024 + (row & 7) * 128 + (rest & 7) * 16;
                    };
                    for (int i = keys * 8 * HALVES + x; i < KEYS * 8 * HALVES; i += 64)
                        asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(at(i)), "r"(0u) : "memory");
                    uint32_t any = 0;
#pragma unroll 8
                    for (int i = first * 8 * HALVES + x; i < keys * 8 * HALVES; i += 64) {
                        uint32_t y[4];
                        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3]) : "r"(at(i)));
                        // an exponent of ones carries into the sign's place when one is added to it (the sign itself masked off)
#pragma unroll
                        for (int k = 0; k < 4; k++) any |= (y[k] & 0x7f807f80u) + 0x00800080u;
                    }
                    if (any & 0x80008000u) {  // rare
                        for (int i = first * 8 * HALVES + x; i < keys * 8 * HALVES; i += 64) {
                            uint32_t y[4];
                            bool found = false;
                            asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3]) : "r"(at(i)));
#pragma unroll
                            for (int k = 0; k < 4; k++) {
                                if ((y[k] & 0x7f80u) == 0x7f80u) y[k] &= 0xffff0000u, found = true;
                                if ((y[k] & 0x7f800000u) == 0x7f800000u) y[k] &= 0xffffu, found = true;
                            }
                            if (!found) continue;
                            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at(i)), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
                            atomicOr(&bad_s[n & 1], 1ull << (key0 + i / (8 * HALVES) - w.s.len));
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(v_clean(sv));
            }
            n++;
        } while (ok && w.next(p));
        if (!ok && lane == 0) report(p.status, kStatusWaitExpired, 930 + warp);
    } else if (work) {
        // ---- softmax: thread = row
        const int i = warp >> 2, r = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t ts = t_s(i) + lanes;
        const float sc = p.scale_log2, grow = kTreeRescaleLog2 / sc;
        const uint64_t sc2 = pack_f32x2(sc, sc);
        load_q(tid, 256);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("bar.arrive 3, 320;" ::: "memory");
        auto wait_all = [&](uint32_t bar, int parity) { return (bool)__all_sync(0xffffffffu, mbar_wait(bar, parity & 1)); };
        int n = 0, sn = 0, on = 0, other_on = 0;
        do {
            const int T = w.t1 - w.t0, tile0 = w.rb * ROWS + (PAIR ? i * 128 : 0), rows = min(128, w.s.n * p.G - tile0);
            const int jobs = PAIR ? (rows > 0 ? T : 0) : (T + 1 - i) / 2;
            const bool mine = r < rows, active = (r & ~31) < rows;
            ok = wait_all(q_full(n), n >> 1);
            unsigned long long seen = 0;  // the nodes that this row sees
            if (mine && w.t1 * KEYS > w.s.len)
                for (int up = (tile0 + r) / p.G; up >= 0; up = parents_s[n & 1][up]) seen |= 1ull << up;
            float m_use = -INFINITY, l_run = 0.f;
            for (int j = 0; j < jobs && ok; j++) {
                const int key0 = (w.t0 + (PAIR ? j : 2 * j + i)) * KEYS;
                ok = wait_all(s_full(i), sn++);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (active) {
                    uint32_t v[128];
#pragma unroll
                    for (int c = 0; c < 4; c++) tmem_ld32_issue(ts + 32 * c, v + 32 * c);
                    tmem_ld_wait();
                    if (key0 + KEYS > w.s.len) {
                        const int at = w.s.len - key0;  // column of node 0
                        unsigned long long lo, hi;
                        if (at >= 64) {
                            lo = ~0ull;
                            hi = (at > 64 ? ~0ull >> (128 - at) : 0ull) | (seen << (at - 64));
                        } else if (at >= 0) {
                            lo = (at > 0 ? ~0ull >> (64 - at) : 0ull) | (seen << at);
                            hi = at > 0 ? seen >> (64 - at) : 0ull;
                        } else {
                            lo = at > -64 ? seen >> -at : 0ull;
                            hi = 0ull;
                        }
                        const uint32_t word[4] = {(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
#pragma unroll
                        for (int c = 0; c < 128; c++)
                            if (!((word[c >> 5] >> (c & 31)) & 1)) v[c] = 0xff800000u;
                    }
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < 128; c += 2) mx[(c >> 1) & 3] = max3(mx[(c >> 1) & 3], __uint_as_float(v[c]), __uint_as_float(v[c + 1]));
                    const float m_tile = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                    if (j == 0) {
                        m_use = m_tile;
                    } else if (__any_sync(0xffffffffu, m_tile > m_use + grow)) {
                        // s_full was signalled after the products of the tile before: O is at rest
                        const float m_new = fmaxf(m_use, m_tile), corr = m_new == m_use ? 1.f : ex2_approx((m_use - m_new) * sc);
                        m_use = m_new;
                        l_run *= corr;
#pragma unroll 1
                        for (int c = 0; c < DH; c += 16) {  // (sixteen at a time: the scores stay in registers)
                            uint32_t o[16];
                            tmem_ld16_issue(t_o(i) + lanes + c, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int k = 0; k < 16; k++) o[k] = __float_as_uint(__uint_as_float(o[k]) * corr);
                            tmem_st16(t_o(i) + lanes + c, o);
                        }
                    }
                    const float off = m_use == -INFINITY ? 0.f : -m_use * sc;  // (nothing seen so far: exp2 of -inf)
                    const uint64_t off2 = pack_f32x2(off, off);
                    uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
                    for (int h = 0; h < 4; h++) {
                        uint32_t pk[16];
#pragma unroll
                        for (int c = 0; c < 16; c++) {
                            const uint64_t y = fma_f32x2((uint64_t)v[h * 32 + 2 * c + 1] << 32 | v[h * 32 + 2 * c], sc2, off2);
                            const float a = ex2_approx(__uint_as_float((uint32_t)y)), e = ex2_approx(__uint_as_float((uint32_t)(y >> 32)));
                            sum[c & 1] = add_f32x2(sum[c & 1], pack_f32x2(a, e));
                            pk[c] = pack_bf16(a, e);
                        }
                        tmem_st16(ts + 16 * h, pk);
                    }
                    const uint64_t both = add_f32x2(sum[0], sum[1]);
                    l_run += __uint_as_float((uint32_t)both) + __uint_as_float((uint32_t)(both >> 32));
                    tmem_st_wait();
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full(i));
            }
            // ---- the item's output, or this run's part of it
            if (ok && jobs > 0) ok = wait_all(o_full(i), on++);
            const bool two = !PAIR && T > 1;  // both groups hold a part
            float f0 = 1.f, f1 = 0.f;         // weights of the two outputs
            if (!PAIR) {
                if (ok && (i == 1 || two)) ok = wait_all(o_full(1 - i), other_on++);  // the other group's output
                stats_s[i][r] = make_float2(m_use, l_run);
                if (!ok) *failed_s = 1;
                asm volatile("bar.sync 1, 256;" ::: "memory");
                ok = ok && !*(volatile int *)failed_s;
                const float2 a = stats_s[0][r], b = stats_s[1][r];
                const float m = two ? fmaxf(a.x, b.x) : a.x;
                f0 = a.x == m ? 1.f : ex2_approx((a.x - m) * sc);
                f1 = !two ? 0.f : b.x == m ? 1.f : ex2_approx((b.x - m) * sc);
                m_use = m;
                l_run = a.y * f0 + (two ? b.y * f1 : 0.f);
            }
            if (!ok) break;
            if (active && (!PAIR || jobs > 0)) {
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const unsigned long long bad = bad_s[n & 1] & seen;
                const float inv = w.slot >= 0 ? 1.f : l_run == 0.f ? 0.f : 1.f / l_run;
                f0 *= inv;
                f1 *= inv;
                const int node = (tile0 + r) / p.G, g = (tile0 + r) - node * p.G;
                float *part = p.part + ((size_t)max(w.slot, 0) * ROWS + (PAIR ? i * 128 : 0) + r) * DH;
                __nv_bfloat16 *out = reinterpret_cast<__nv_bfloat16 *>(p.out) + (((size_t)w.b * p.N + node) * p.hkv * p.G + w.h * p.G + g) * DH;
                // PAIR: the group's own tile; else the groups write half of the columns each
                constexpr int COLS = PAIR ? DH : DH / 2;
                const int col0 = PAIR ? 0 : i * COLS;
#pragma unroll 1
                for (int c = col0; c < col0 + COLS; c += 16) {
                    uint32_t o[16], o2[16];
                    __syncwarp();
                    tmem_ld16_issue(t_o(PAIR ? i : 0) + lanes + c, o);
                    if (!PAIR) tmem_ld16_issue(t_o(two ? 1 : 0) + lanes + c, o2);
                    tmem_ld_wait();
                    if (!mine) continue;
                    float y[16];
#pragma unroll
                    for (int k = 0; k < 16; k++) {
                        y[k] = __uint_as_float(o[k]) * f0;
                        if (!PAIR && two) y[k] += __uint_as_float(o2[k]) * f1;
                    }
                    for (unsigned long long m = bad; m; m &= m - 1) {  // rare: values that are not finite
                        const int at = w.s.len + __ffsll(m) - 1;
                        const __nv_bfloat16 *v = reinterpret_cast<const __nv_bfloat16 *>(p.cache) +
                                                 ((((size_t)p.num_pages + tree_page(p, w.b, at >> 4)) * p.hkv + w.h) * 16 + (at & 15)) * DH + c;
#pragma unroll
                        for (int k = 0; k < 16; k++) {
                            const float x = __bfloat162float(v[k]);
                            if (!isfinite(x)) y[k] += x;
                        }
                    }
                    if (w.slot >= 0) {
#pragma unroll
                        for (int k = 0; k < 16; k += 4) *reinterpret_cast<float4 *>(part + c + k) = make_float4(y[k], y[k + 1], y[k + 2], y[k + 3]);
                    } else {
#pragma unroll
                        for (int k = 0; k < 16; k += 8)
                            *reinterpret_cast<uint4 *>(out + c + k) = make_uint4(pack_bf16(y[k], y[k + 1]), pack_bf16(y[k + 2], y[k + 3]),
                                                                                 pack_bf16(y[k + 4], y[k + 5]), pack_bf16(y[k + 6], y[k + 7]));
                    }
                }
                if (w.slot >= 0 && mine && (PAIR || i == 0))
                    p.stats[(size_t)w.slot * ROWS + (PAIR ? i * 128 : 0) + r] = make_float2(m_use * sc, l_run);
            }
            // the outputs have been read: the next item's products may overwrite them (stats_s is rewritten behind those)
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(e_done(n));
            n++;
        } while (w.next(p));
        if (!ok && lane == 0) report(p.status, kStatusWaitExpired, 920 + warp);
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 9)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)Cfg::kTmemCols) : "memory");
}

// ---- joining the parts of items that were cut --------------------------------------------------------------------
// A warp per output row, in the order of the keys.  Its bound is latency: 16 ragged sequences' parts take 4 us behind the first kernel, 8
// sequences-by-heads cut in 148 parts 7 us.
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
    int before;
    const int per = Plan::per_block(p, Plan::total(p, lane, b, &before));
    const int tiles = Plan::tiles(s), rb = row / ROWS, r = row - rb * ROWS;
    const int item0 = before + (h * Plan::row_blocks(p, s) + rb) * (tiles + p.lead) + p.lead;  // its first tile
    const int c0 = item0 / per, c1 = (item0 + tiles - 1) / per;
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

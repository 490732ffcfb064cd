// Acceptance of one branch of a tree of drafted tokens (sm_100a): the walk along the sampled tokens, and the accepted nodes'
// cache rows moved together.
//
// The walk is at most 64 steps of one warp over at most 64 nodes held two to a lane: a ballot per step finds the children of the
// current node that carry the sampled token.  Every block walks for itself (a microsecond), then its threads move their share of
// (layer, K|V, head, 16 bytes): the j-th accepted node has a number of at least j, so a thread that takes the rows in order, some
// of them loaded together before they are stored, never reads what it has overwritten.
// What bounds it: latency of the walk and of the rows' loads; the bytes are 4 * layers * kv heads * head_dim elements a moved row.
// 8 sequences of 64 nodes, five rows moved in 32 layers of 8 heads of 128 (10 MB): 18 us a call, as for one short sequence (the host).
#pragma once

#include "dbt_common.cuh"

namespace dbt {

struct TreeAcceptParams {
    const int32_t *tokens, *parents, *sampled, *page_table, *seq_lens, *node_counts;
    char *pool;
    int32_t *path, *counts, *next_tokens, *new_lens;
    int *status;
    int N, hkv, num_pages, pps;
    int vecs;        // 16-byte vectors of a row of one head
    int planes;      // layers * 2
};

constexpr int kTreeMaxNodes = 64;

__global__ static void __launch_bounds__(256) tree_accept_kernel(const TreeAcceptParams p) {
    __shared__ int path_s[kTreeMaxNodes], count_s;
    __shared__ long long from_s[kTreeMaxNodes], to_s[kTreeMaxNodes];  // row numbers inside a plane, -1: not moved
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 31;
    const int len = p.seq_lens[b];
    const int n = p.node_counts ? max(0, min(p.node_counts[b], p.N)) : p.N;
    if (tid < 32) {
        int token[2], parent[2], drawn[2];
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const int c = lane + 32 * k;
            const bool on = c < n;
            const size_t at = (size_t)b * p.N + c;
            token[k] = on ? p.tokens[at] : 0;
            parent[k] = on ? p.parents[at] : -1;
            drawn[k] = on ? p.sampled[at] : 0;
            if (on && (parent[k] >= c || parent[k] < -1)) {
                report(p.status, kStatusBadTree, parent[k]);
                parent[k] = -1;
            }
        }
        int cur = 0, count = n > 0 ? 1 : 0, follows = -1;
        if (lane == 0) path_s[0] = 0;
        while (count > 0) {
            const int w0 = __shfl_sync(0xffffffffu, drawn[0], cur & 31), w1 = __shfl_sync(0xffffffffu, drawn[1], cur & 31);
            follows = cur < 32 ? w0 : w1;
            const unsigned m0 = __ballot_sync(0xffffffffu, lane < n && parent[0] == cur && token[0] == follows);
            const unsigned m1 = __ballot_sync(0xffffffffu, lane + 32 < n && parent[1] == cur && token[1] == follows);
            if (!(m0 | m1)) break;
            cur = m0 ? __ffs(m0) - 1 : 32 + __ffs(m1) - 1;  // (above its parent: the walk ends)
            if (lane == 0) path_s[count] = cur;
            count++;
        }
        __syncwarp();
        if (lane == 0) count_s = count;
        for (int j = lane; j < p.N; j += 32) {
            const int node = j < count ? path_s[j] : -1;
            long long from = -1, to = -1;
            if (node > j) {
                auto row = [&](int i) -> long long {
                    const long long at = (long long)len + i, slot = at >> 4;
                    const int page = at >= 0 && slot < p.pps ? p.page_table[(size_t)b * p.pps + slot] : -1;
                    if (page < 0 || page >= p.num_pages) {
                        report(p.status, kStatusBadPage, page);
                        return -1;
                    }
                    return (long long)page * p.hkv * 16 + (at & 15);
                };
                from = row(node);
                to = from >= 0 ? row(j) : -1;
            }
            from_s[j] = from;
            to_s[j] = to;
            if (blockIdx.x == 0) p.path[(size_t)b * p.N + j] = node;
        }
        if (blockIdx.x == 0 && lane == 0) {
            p.counts[b] = count;
            p.next_tokens[b] = follows;
            p.new_lens[b] = len + count;
        }
    }
    __syncthreads();
    const int count = count_s;
    const long long at = (long long)blockIdx.x * blockDim.x + tid, per_plane = (long long)p.hkv * p.vecs;
    if (at >= per_plane * p.planes) return;
    const int plane = (int)(at / per_plane), rest = (int)(at - plane * per_plane), h = rest / p.vecs, v = rest - h * p.vecs;
    uint4 *base = reinterpret_cast<uint4 *>(p.pool) + ((size_t)plane * p.num_pages * p.hkv + h) * 16 * p.vecs + v;
    constexpr int A = 4;
    for (int j = 1; j < count; j += A) {
        uint4 x[A];
#pragma unroll
        for (int a = 0; a < A; a++)
            if (j + a < count && to_s[j + a] >= 0) x[a] = base[(size_t)from_s[j + a] * p.vecs];
#pragma unroll
        for (int a = 0; a < A; a++)
            if (j + a < count && to_s[j + a] >= 0) base[(size_t)to_s[j + a] * p.vecs] = x[a];
    }
}

}  // namespace dbt

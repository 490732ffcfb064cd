// Host side of the operators for sampled and drafted tokens declared in include/dbt.h: argument checks and launches.
#undef DBT_TIMELINE  // the timeline's device array belongs to dbt_api.cu

#include <cmath>
#include <cstring>

#include "dbt_attn_tree.cuh"
#include "dbt_host.h"
#include "dbt_rope.cuh"
#include "dbt_sample.cuh"
#include "dbt_tree_accept.cuh"

using namespace dbt;

namespace {

#define CHECK(cond, status, ...) \
    do {                         \
        if (!(cond)) return op_error(status, __VA_ARGS__); \
    } while (0)

dbt_status launched(cudaError_t e, const char *what) {
    return e == cudaSuccess ? DBT_OK : op_error(DBT_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

template <typename... Params, typename... Args>
cudaError_t launch(void (*kernel)(Params...), dim3 grid, int block, size_t smem, void *stream, int cluster, bool pdl, Args &&...args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = cluster;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        n++;
    }
    if (pdl) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        n++;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kernel, Params(std::forward<Args>(args))...);
}

// A kernel's dynamic shared memory limit, raised on the current device (an attribute of the function on that device: set before each
// launch, a few hundred nanoseconds on the host).  Without it static and dynamic memory together end at 48 KB.
template <typename K>
cudaError_t allow_smem(K kernel, size_t bytes) {
    return bytes > 32 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) : cudaSuccess;
}

int sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) {
        cudaGetLastError();
        return 148;
    }
    return n;
}

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
size_t elem(int dtype) { return dtype == DBT_DTYPE_F32 ? 4 : 2; }

// What the cache operators have in common.
dbt_status check_cache(int dtype, int B, int max_nodes, int n_kv_heads, int head_dim, int num_pages, int pages_per_seq, const void *cache) {
    CHECK(dtype == DBT_DTYPE_F32 || dtype == DBT_DTYPE_BF16, DBT_ERR_UNSUPPORTED, "dtype must be DBT_DTYPE_F32 or DBT_DTYPE_BF16");
    CHECK(B >= 1 && B <= 65535, DBT_ERR_UNSUPPORTED, "1 <= B <= 65535 (B=%d)", B);
    CHECK(max_nodes >= 1 && max_nodes <= kTreeMaxNodes, DBT_ERR_UNSUPPORTED, "1 <= max_nodes <= %d (max_nodes=%d)", kTreeMaxNodes, max_nodes);
    CHECK(n_kv_heads >= 1 && n_kv_heads <= 1024, DBT_ERR_UNSUPPORTED, "1 <= n_kv_heads <= 1024");
    CHECK(head_dim == 64 || head_dim == 128, DBT_ERR_UNSUPPORTED, "head_dim must be 64 or 128 (%d)", head_dim);
    CHECK(num_pages >= 1 && pages_per_seq >= 1, DBT_ERR_INVALID_ARG, "num_pages and pages_per_seq must be positive");
    CHECK((long long)num_pages * n_kv_heads <= (1ll << 26), DBT_ERR_UNSUPPORTED, "num_pages * n_kv_heads exceeds 2^26");
    CHECK(pages_per_seq <= (1 << 26), DBT_ERR_UNSUPPORTED, "pages_per_seq exceeds 2^26");
    CHECK(cache, DBT_ERR_INVALID_ARG, "NULL cache");
    CHECK(aligned(cache, 16), DBT_ERR_INVALID_ARG, "the cache must be 16-byte aligned");
    return DBT_OK;
}

// ---- rotary positions --------------------------------------------------------------------------------------------
template <typename T, int N, bool APPEND>
cudaError_t rope_launch(RopeParams &p, int interleaved, void *stream) {
    const int heads = APPEND ? p.hq + 2 * p.hkv : p.hq;
    const int units = p.rot / (2 * N) + (p.copy_rest || APPEND ? (p.D - p.rot + 2 * N - 1) / (2 * N) : 0);
    // Heads per thread: each thread forms its angles once, whatever the heads; as many as leave so many blocks per SM (three are
    // resident), four at least so that four heads' loads are in flight.  8192 rows of 32 heads: 29.6, 26.9, 26.7, 28.7 us with 2, 4, 8, 12
    // blocks; the append of 32 trees of 64 nodes, bound by its latency: 12.9, 14.5, 14.3, 14.3.
    const int waves = APPEND ? 2 : 8;
    const long long blocks = (p.rows * units + 255) / 256, wanted = (long long)waves * sm_count();
    int groups = (int)(blocks >= wanted ? 1 : (wanted + blocks - 1) / blocks);
    if (groups > (heads + 3) / 4) groups = (heads + 3) / 4;
    p.heads_per_group = (heads + groups - 1) / groups;
    groups = (heads + p.heads_per_group - 1) / p.heads_per_group;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    const dim3 grid((unsigned)blocks, groups);
    return interleaved ? launch(rope_kernel<T, N, true, APPEND>, grid, 256, 0, stream, 1, false, p)
                       : launch(rope_kernel<T, N, false, APPEND>, grid, 256, 0, stream, 1, false, p);
}
template <bool APPEND>
dbt_status rope_run(RopeParams &p, int dtype, int interleaved, bool vectors, void *stream) {
    const int n = dtype == DBT_DTYPE_F32 ? 4 : 8;
    vectors = vectors && p.rot % (2 * n) == 0 && p.D % n == 0;
    cudaError_t e;
    if (dtype == DBT_DTYPE_F32)
        e = vectors ? rope_launch<float, 4, APPEND>(p, interleaved, stream) : rope_launch<float, 1, APPEND>(p, interleaved, stream);
    else
        e = vectors ? rope_launch<__nv_bfloat16, 8, APPEND>(p, interleaved, stream) : rope_launch<__nv_bfloat16, 1, APPEND>(p, interleaved, stream);
    return launched(e, "rope");
}
bool strides_fit(const int64_t *s, int n, int dtype) {
    for (int i = 0; i < n; i++)
        if (s[i] % (16 / (int)elem(dtype))) return false;
    return true;
}

// ---- tree attention ----------------------------------------------------------------------------------------------
// An item costs about as much as five (fp32: one) of its tiles besides them: 16 ragged sequences 63 us without, 42 us with four to six
// (then), 37, 36, 39 us with three, five, eight (now); long items do not care.  Measured with head dimension 128 and up to 128 rows a key;
// 64 and 256 rows take the same number unmeasured.
constexpr int kTreeLead = 5;
struct TreeShape {
    int rows, keys, blocks, per_sm, lead;
};
// The longest line of units that these arguments allow.
long long tree_units(const dbt_attn_tree_args &a) {
    const int rows = a.max_nodes * (a.n_q_heads / a.n_kv_heads), keys = a.dtype == DBT_DTYPE_BF16 ? 128 : kTsKeys;
    return ((long long)a.pages_per_seq * 16 / keys + 1 + kTreeLead) * ((rows + 15) / 16) * a.n_kv_heads * a.B;
}
// Blocks: one for each SM, two of the fp32 form for 16 rows (the one for 64 rows of 64 elements would fit twice as well; one was not held
// against two), no more than there can be tiles.
TreeShape tree_shape(const dbt_attn_tree_args &a) {
    TreeShape s;
    const int G = a.n_q_heads / a.n_kv_heads, rows = a.max_nodes * G;
    const bool mma = a.dtype == DBT_DTYPE_BF16;
    s.rows = mma ? (rows <= 128 ? 128 : 256) : (rows <= 16 ? 16 : 64);
    s.keys = mma ? 128 : kTsKeys;
    s.per_sm = s.rows == 16 ? 2 : 1;
    s.lead = mma ? kTreeLead : 1;
    const long long tiles = ((long long)a.pages_per_seq * 16 + s.keys - 1) / s.keys, rbs = (a.max_nodes * G + s.rows - 1) / s.rows;
    const long long most = tiles * rbs * a.n_kv_heads * a.B, fit = (long long)sm_count() * s.per_sm;
    s.blocks = (int)(most < fit ? most : fit);
    return s;
}
size_t tree_stats_bytes(const TreeShape &s) { return ((size_t)2 * s.blocks * s.rows * sizeof(float2) + 255) / 256 * 256; }
size_t tree_bytes(const TreeShape &s, int D) { return tree_stats_bytes(s) + (size_t)2 * s.blocks * s.rows * D * 4; }

dbt_status check_tree(const dbt_attn_tree_args *a, bool pointers) {
    CHECK(a, DBT_ERR_INVALID_ARG, "NULL arguments");
    CHECK(a->struct_size == sizeof(dbt_attn_tree_args), DBT_ERR_INVALID_ARG, "struct_size %u, expected %zu", a->struct_size, sizeof(dbt_attn_tree_args));
    static const char here = 0;
    dbt_status st = check_cache(a->dtype, a->B, a->max_nodes, a->n_kv_heads, a->head_dim, a->num_pages, a->pages_per_seq,
                                pointers ? a->cache_layer : reinterpret_cast<const void *>(reinterpret_cast<uintptr_t>(&here) & ~(uintptr_t)15));
    if (st != DBT_OK) return st;
    CHECK(a->n_q_heads >= 1 && a->n_q_heads % a->n_kv_heads == 0, DBT_ERR_UNSUPPORTED, "n_q_heads must be a multiple of n_kv_heads");
    CHECK(a->n_q_heads / a->n_kv_heads <= 16, DBT_ERR_UNSUPPORTED, "at most 16 query heads per KV head");
    CHECK(tree_units(*a) <= 0x7fffffff, DBT_ERR_UNSUPPORTED, "B * n_kv_heads * pages_per_seq are too many tiles for one call");
    if (!pointers) return DBT_OK;
    CHECK(a->q && a->out && a->page_table && a->seq_lens && a->parents && a->workspace && a->status_dev, DBT_ERR_INVALID_ARG, "NULL pointer");
    CHECK(a->q != a->out, DBT_ERR_INVALID_ARG, "out must not be q");
    CHECK(aligned(a->q, elem(a->dtype)) && aligned(a->out, 16), DBT_ERR_INVALID_ARG, "out must be 16-byte aligned, q aligned to its elements");
    CHECK(aligned(a->workspace, 256), DBT_ERR_INVALID_ARG, "the workspace must be 256-byte aligned");
    CHECK(std::isfinite(a->softmax_scale) && a->softmax_scale >= 0.f, DBT_ERR_INVALID_ARG, "softmax_scale must be finite and not negative");
    return DBT_OK;
}

template <int D, int RM>
cudaError_t tree_simt(const TreeAttnParams &p, void *stream) {
    using Cfg = TreeSimtCfg<D, RM>;
    cudaError_t e = allow_smem(attn_tree_simt_kernel<D, RM>, Cfg::kSmemBytes);
    if (e == cudaSuccess) e = launch(attn_tree_simt_kernel<D, RM>, dim3(p.blocks), 256, Cfg::kSmemBytes, stream, 1, false, p);
    if (e != cudaSuccess) return e;
    const long long warps = (long long)p.B * p.hkv * p.N * p.G;
    return launch(attn_tree_join_kernel<float, D, Cfg::kRows, kTsKeys>, dim3((unsigned)((warps + 7) / 8)), 256, 0, stream, 1, true, p);
}

template <typename T, int NT>
cudaError_t sample_launch(const SampleParams &p, int rows, int cluster, void *stream) {
    const size_t smem = sm_scratch_bytes(NT);
    cudaError_t e = allow_smem(sample_kernel<T, NT>, smem);
    return e == cudaSuccess ? launch(sample_kernel<T, NT>, dim3(rows * cluster), NT, smem, stream, cluster, false, p) : e;
}

template <int D, bool PAIR>
cudaError_t tree_mma(const TreeAttnParams &p, void *stream) {
    using Cfg = TreeMmaCfg<D, PAIR>;
    CUtensorMap map;
    if (!make_prompt_kv_map(&map, p.cache, (uint64_t)2 * p.num_pages * p.hkv * 16, D)) return cudaErrorInvalidValue;
    cudaError_t e = allow_smem(attn_tree_mma_kernel<D, PAIR>, Cfg::kSmemBytes);
    if (e == cudaSuccess) e = launch(attn_tree_mma_kernel<D, PAIR>, dim3(p.blocks), Cfg::kThreads, Cfg::kSmemBytes, stream, 1, false, map, p);
    if (e != cudaSuccess) return e;
    const long long warps = (long long)p.B * p.hkv * p.N * p.G;
    return launch(attn_tree_join_kernel<__nv_bfloat16, D, Cfg::kRows, Cfg::kKeys>, dim3((unsigned)((warps + 7) / 8)), 256, 0, stream, 1, true, p);
}

}  // namespace

extern "C" {

dbt_status dbt_rope_frequencies(const dbt_rope_spec *s, double *freq, float *scale) {
    CHECK(s && freq && scale, DBT_ERR_INVALID_ARG, "NULL pointer");
    CHECK(s->struct_size == sizeof(dbt_rope_spec), DBT_ERR_INVALID_ARG, "struct_size %u, expected %zu", s->struct_size, sizeof(dbt_rope_spec));
    CHECK(s->kind >= DBT_ROPE_PLAIN && s->kind <= DBT_ROPE_BANDS, DBT_ERR_UNSUPPORTED, "unknown kind %d", s->kind);
    CHECK(s->rot_dim >= 2 && s->rot_dim % 2 == 0 && s->rot_dim <= 4096, DBT_ERR_INVALID_ARG, "rot_dim must be even, 2..4096 (%d)", s->rot_dim);
    CHECK(std::isfinite(s->base) && s->base > 1.0, DBT_ERR_INVALID_ARG, "base must be above 1");
    if (s->kind != DBT_ROPE_PLAIN) CHECK(std::isfinite(s->factor) && s->factor >= 1.0, DBT_ERR_INVALID_ARG, "factor must be at least 1");
    if (s->kind == DBT_ROPE_BASE) CHECK(s->rot_dim > 2, DBT_ERR_INVALID_ARG, "a scaled base needs rot_dim > 2");
    const bool ranges = s->kind == DBT_ROPE_RAMP || s->kind == DBT_ROPE_BANDS;
    if (ranges) {
        CHECK(std::isfinite(s->trained_len) && s->trained_len > 0.0, DBT_ERR_INVALID_ARG, "trained_len must be positive");
        CHECK(std::isfinite(s->high) && s->low > 0.0 && s->low < s->high, DBT_ERR_INVALID_ARG, "0 < low < high");
    }
    const int rot = s->rot_dim, pairs = rot / 2;
    const double two_pi = 6.283185307179586;
    const double base = s->kind == DBT_ROPE_BASE ? s->base * std::pow(s->factor, rot / (rot - 2.0)) : s->base;
    // RAMP: the pair that makes `turns` turns over the trained length
    auto pair_of = [&](double turns) { return rot * std::log(s->trained_len / (turns * two_pi)) / (2.0 * std::log(s->base)); };
    // The ramp's ends, the upper one at most rot - 1 (YaRN, Peng et al. 2023): it may lie behind the last pair, which then makes more than
    // `low` turns and is slowed by a part.
    double first = 0.0, last = 0.0;
    if (s->kind == DBT_ROPE_RAMP) {
        first = std::fmax(std::floor(pair_of(s->high)), 0.0);
        last = std::fmin(std::ceil(pair_of(s->low)), rot - 1.0);
    }
    for (int i = 0; i < pairs; i++) {
        const double f = std::pow(base, -2.0 * i / rot);
        double slow = 0.0;  // share of the slowed frequency
        if (s->kind == DBT_ROPE_LINEAR) slow = 1.0;
        if (s->kind == DBT_ROPE_RAMP) slow = i >= last ? 1.0 : i <= first ? 0.0 : (i - first) / (last - first);
        if (s->kind == DBT_ROPE_BANDS) slow = 1.0 - std::fmin(1.0, std::fmax(0.0, (s->trained_len * f / two_pi - s->low) / (s->high - s->low)));
        freq[i] = slow == 0.0 ? f : f / s->factor * slow + f * (1.0 - slow);
    }
    *scale = s->kind == DBT_ROPE_RAMP ? (float)(0.1 * std::log(s->factor) + 1.0) : 1.f;
    return DBT_OK;
}

dbt_status dbt_op_rope(const void *x, void *y, const int32_t *positions, const double *freq, int64_t rows, int32_t heads, int32_t head_dim,
                       int32_t rot_dim, int64_t x_row_stride, int64_t x_head_stride, int64_t y_row_stride, int64_t y_head_stride, float scale,
                       int32_t interleaved, int32_t inverse, int32_t dtype, void *cuda_stream) {
    CHECK(dtype == DBT_DTYPE_F32 || dtype == DBT_DTYPE_BF16, DBT_ERR_UNSUPPORTED, "dtype must be DBT_DTYPE_F32 or DBT_DTYPE_BF16");
    CHECK(rows >= 0 && rows <= 0x7fffffff, DBT_ERR_UNSUPPORTED, "0 <= rows < 2^31");
    CHECK(heads >= 1 && heads <= 65535, DBT_ERR_UNSUPPORTED, "1 <= heads <= 65535");
    CHECK(head_dim >= 2 && head_dim <= 4096, DBT_ERR_UNSUPPORTED, "2 <= head_dim <= 4096");
    CHECK(rot_dim >= 2 && rot_dim % 2 == 0 && rot_dim <= head_dim, DBT_ERR_INVALID_ARG, "rot_dim must be even, 2..head_dim (%d)", rot_dim);
    if (rows == 0) return DBT_OK;
    CHECK(x && y && positions && freq, DBT_ERR_INVALID_ARG, "NULL pointer");
    CHECK(aligned(x, elem(dtype)) && aligned(y, elem(dtype)), DBT_ERR_INVALID_ARG, "x and y must be aligned to their elements");
    CHECK(x != y || (x_row_stride == y_row_stride && x_head_stride == y_head_stride), DBT_ERR_INVALID_ARG, "y is x with other strides");
    RopeParams p{};
    p.x = x;
    p.y = y;
    p.positions = positions;
    p.freq = freq;
    p.xs[1] = x_row_stride;
    p.xs[2] = x_head_stride;
    p.ys[1] = y_row_stride;
    p.ys[2] = y_head_stride;
    p.rows = rows;
    p.per_batch = (int)rows;
    p.hq = heads;
    p.D = head_dim;
    p.rot = rot_dim;
    p.scale = scale;
    p.inverse = inverse != 0;
    p.copy_rest = x != y;
    const int64_t strides[4] = {x_row_stride, x_head_stride, y_row_stride, y_head_stride};
    return rope_run<false>(p, dtype, interleaved, aligned(x, 16) && aligned(y, 16) && strides_fit(strides, 4, dtype), cuda_stream);
}

dbt_status dbt_op_rope_append(const dbt_rope_append_args *a, void *cuda_stream) {
    CHECK(a, DBT_ERR_INVALID_ARG, "NULL arguments");
    CHECK(a->struct_size == sizeof(dbt_rope_append_args), DBT_ERR_INVALID_ARG, "struct_size %u, expected %zu", a->struct_size,
          sizeof(dbt_rope_append_args));
    dbt_status st = check_cache(a->dtype, a->B, a->max_nodes, a->n_kv_heads, a->head_dim, a->num_pages, a->pages_per_seq, a->cache_layer);
    if (st != DBT_OK) return st;
    CHECK(a->n_q_heads >= 1 && a->n_q_heads <= 32768, DBT_ERR_UNSUPPORTED, "1 <= n_q_heads <= 32768");
    CHECK(a->rot_dim >= 2 && a->rot_dim % 2 == 0 && a->rot_dim <= a->head_dim, DBT_ERR_INVALID_ARG, "rot_dim must be even, 2..head_dim (%d)", a->rot_dim);
    CHECK(a->q && a->k && a->v && a->q_out && a->positions && a->page_table && a->seq_lens && a->freq && a->status_dev, DBT_ERR_INVALID_ARG, "NULL pointer");
    CHECK(a->q != a->q_out, DBT_ERR_INVALID_ARG, "q_out must not be q");
    const size_t e = elem(a->dtype);
    CHECK(aligned(a->q, e) && aligned(a->k, e) && aligned(a->v, e) && aligned(a->q_out, e), DBT_ERR_INVALID_ARG, "q, k, v, q_out must be aligned to their elements");
    RopeParams p{};
    p.x = a->q;
    p.k = a->k;
    p.v = a->v;
    p.y = a->q_out;
    p.cache = a->cache_layer;
    p.positions = a->positions;
    p.page_table = a->page_table;
    p.seq_lens = a->seq_lens;
    p.node_counts = a->node_counts;
    p.freq = a->freq;
    p.status = a->status_dev;
    for (int i = 0; i < 3; i++) {
        p.xs[i] = a->q_stride[i];
        p.ks[i] = a->k_stride[i];
        p.vs[i] = a->v_stride[i];
    }
    p.ys[2] = a->head_dim;
    p.ys[1] = (long long)a->n_q_heads * a->head_dim;
    p.ys[0] = p.ys[1] * a->max_nodes;
    p.rows = (long long)a->B * a->max_nodes;
    p.per_batch = a->max_nodes;
    p.hq = a->n_q_heads;
    p.hkv = a->n_kv_heads;
    p.D = a->head_dim;
    p.rot = a->rot_dim;
    p.scale = a->scale;
    p.num_pages = a->num_pages;
    p.pps = a->pages_per_seq;
    p.copy_rest = 1;
    const bool vectors = aligned(a->q, 16) && aligned(a->k, 16) && aligned(a->v, 16) && aligned(a->q_out, 16) && strides_fit(a->q_stride, 3, a->dtype) &&
                         strides_fit(a->k_stride, 3, a->dtype) && strides_fit(a->v_stride, 3, a->dtype);
    return rope_run<true>(p, a->dtype, a->interleaved, vectors, cuda_stream);
}

dbt_status dbt_op_attn_tree_workspace(const dbt_attn_tree_args *a, size_t *bytes) {
    CHECK(bytes, DBT_ERR_INVALID_ARG, "NULL pointer");
    dbt_status st = check_tree(a, false);
    if (st != DBT_OK) return st;
    *bytes = tree_bytes(tree_shape(*a), a->head_dim);
    return DBT_OK;
}

dbt_status dbt_op_attn_tree(const dbt_attn_tree_args *a, void *cuda_stream) {
    dbt_status st = check_tree(a, true);
    if (st != DBT_OK) return st;
    const TreeShape s = tree_shape(*a);
    CHECK(a->workspace_bytes >= tree_bytes(s, a->head_dim), DBT_ERR_CAPACITY, "the workspace holds %zu bytes, %zu are needed", a->workspace_bytes,
          tree_bytes(s, a->head_dim));
    TreeAttnParams p{};
    p.q = a->q;
    p.cache = a->cache_layer;
    p.out = a->out;
    p.page_table = a->page_table;
    p.seq_lens = a->seq_lens;
    p.node_counts = a->node_counts;
    p.parents = a->parents;
    p.stats = static_cast<float2 *>(a->workspace);
    p.part = reinterpret_cast<float *>(static_cast<char *>(a->workspace) + tree_stats_bytes(s));
    p.status = a->status_dev;
    for (int i = 0; i < 3; i++) p.qs[i] = a->q_stride[i];
    p.B = a->B;
    p.N = a->max_nodes;
    p.G = a->n_q_heads / a->n_kv_heads;
    p.hkv = a->n_kv_heads;
    p.num_pages = a->num_pages;
    p.pps = a->pages_per_seq;
    p.blocks = s.blocks;
    p.lead = s.lead;
    p.g_inverse = (65536 + p.G - 1) / p.G;
    p.q_vectors = aligned(a->q, 16) && strides_fit(a->q_stride, 3, a->dtype);
    p.scale_log2 = (a->softmax_scale > 0.f ? a->softmax_scale : 1.f / std::sqrt((float)a->head_dim)) * 1.4426950408889634f;
    cudaError_t e;
    const bool few = s.rows == 16, wide = a->head_dim == 128;
    if (a->dtype == DBT_DTYPE_F32)
        e = wide ? (few ? tree_simt<128, 1>(p, cuda_stream) : tree_simt<128, 4>(p, cuda_stream))
                 : (few ? tree_simt<64, 1>(p, cuda_stream) : tree_simt<64, 4>(p, cuda_stream));
    else
        e = wide ? (s.rows == 128 ? tree_mma<128, false>(p, cuda_stream) : tree_mma<128, true>(p, cuda_stream))
                 : (s.rows == 128 ? tree_mma<64, false>(p, cuda_stream) : tree_mma<64, true>(p, cuda_stream));
    return launched(e, "attn_tree");
}

dbt_status dbt_op_sample(const void *logits, int32_t dtype, int32_t rows, int32_t vocab, int64_t row_stride, const float *uniforms,
                         const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p, int32_t *tokens, float *logprobs,
                         void *cuda_stream) {
    CHECK(dtype == DBT_DTYPE_F32 || dtype == DBT_DTYPE_BF16, DBT_ERR_UNSUPPORTED, "dtype must be DBT_DTYPE_F32 or DBT_DTYPE_BF16");
    CHECK(rows >= 0 && rows <= (1 << 24), DBT_ERR_UNSUPPORTED, "0 <= rows <= 2^24");
    CHECK(vocab >= 2 && vocab <= kSmMaxSlice * kSmMaxCluster, DBT_ERR_UNSUPPORTED, "2 <= vocab <= %d (%d)", kSmMaxSlice * kSmMaxCluster, vocab);
    CHECK(row_stride >= vocab, DBT_ERR_INVALID_ARG, "row_stride is below vocab");
    if (rows == 0) return DBT_OK;
    CHECK(logits && uniforms && tokens, DBT_ERR_INVALID_ARG, "NULL pointer");
    CHECK(aligned(logits, elem(dtype)), DBT_ERR_INVALID_ARG, "logits must be aligned to their elements");
    SampleParams p{};
    p.logits = logits;
    p.row_stride = row_stride;
    p.uniforms = uniforms;
    p.temperature = temperature;
    p.top_k = top_k;
    p.top_p = top_p;
    p.min_p = min_p;
    p.tokens = tokens;
    p.logprobs = logprobs;
    p.vocab = vocab;
    // Blocks per row: enough to fill the device (four are resident per SM), or two per SM where a block's share is short already;
    // and no more than leave a block 4096 values.  256 rows of 128256, top-k 50 with top-p and min-p: 69 us with 8 blocks a row, 56 with 4;
    // top-k 400: 109, 78; without filters 90, 88; settings of all kinds 118, 127.  256 rows of 32000, the same filters: 72, 34, 24 us with 8,
    // 4, 2 (then; 21 now); one row of 128256 without filters: 25, 42, 73 with 8, 4, 2 (then; 13 now).  Between and
    // beyond these sizes the rule is a guess.
    const long long sms = sm_count();
    int cluster = 1;
    while (vocab > cluster * kSmMaxSlice ||
           (cluster < kSmMaxCluster && vocab > cluster * 4096 && (long long)rows * cluster < 4 * sms &&
            !((long long)rows * cluster >= 2 * sms && vocab <= cluster * 16384)))
        cluster *= 2;
    p.slice = ((vocab + cluster - 1) / cluster + 7) / 8 * 8;
    // Few rows: twice the threads, one block per SM: top-k 2000 of one row of 128256 62 us with 256 threads, 52 with 512 (1024 spill: 60; then).
    // Many rows, two blocks of 512 against four of 256 per SM: settings of all kinds 123 us, 133; without filters 35, 28 (64 rows).
    const bool few = (long long)rows * cluster <= sms;
    p.rows = rows;
    // More blocks than can be resident: the rows that may take long first (256 rows of 128256 with settings of all kinds 126 us, else 133).
    p.order = top_p && (long long)rows * cluster > 4 * sms;
    cudaError_t e;
    if (dtype == DBT_DTYPE_F32)
        e = few ? sample_launch<float, 512>(p, rows, cluster, cuda_stream) : sample_launch<float, 256>(p, rows, cluster, cuda_stream);
    else
        e = few ? sample_launch<__nv_bfloat16, 512>(p, rows, cluster, cuda_stream) : sample_launch<__nv_bfloat16, 256>(p, rows, cluster, cuda_stream);
    return launched(e, "sample");
}

dbt_status dbt_op_tree_accept(const dbt_tree_accept_args *a, void *cuda_stream) {
    CHECK(a, DBT_ERR_INVALID_ARG, "NULL arguments");
    CHECK(a->struct_size == sizeof(dbt_tree_accept_args), DBT_ERR_INVALID_ARG, "struct_size %u, expected %zu", a->struct_size,
          sizeof(dbt_tree_accept_args));
    dbt_status st = check_cache(a->dtype, a->B, a->max_nodes, a->n_kv_heads, a->head_dim, a->num_pages, a->pages_per_seq, a->pool);
    if (st != DBT_OK) return st;
    CHECK(a->n_layers >= 1 && a->n_layers <= 4096, DBT_ERR_UNSUPPORTED, "1 <= n_layers <= 4096");
    CHECK(a->tokens && a->parents && a->sampled && a->page_table && a->seq_lens && a->path && a->counts && a->next_tokens && a->new_lens && a->status_dev,
          DBT_ERR_INVALID_ARG, "NULL pointer");
    const int32_t *in[6] = {a->tokens, a->parents, a->sampled, a->page_table, a->seq_lens, a->node_counts};
    for (const int32_t *i : in)
        CHECK(!i || (i != a->path && i != a->counts && i != a->next_tokens && i != a->new_lens), DBT_ERR_INVALID_ARG, "an output is also an input");
    TreeAcceptParams p{};
    p.tokens = a->tokens;
    p.parents = a->parents;
    p.sampled = a->sampled;
    p.page_table = a->page_table;
    p.seq_lens = a->seq_lens;
    p.node_counts = a->node_counts;
    p.pool = static_cast<char *>(a->pool);
    p.path = a->path;
    p.counts = a->counts;
    p.next_tokens = a->next_tokens;
    p.new_lens = a->new_lens;
    p.status = a->status_dev;
    p.N = a->max_nodes;
    p.hkv = a->n_kv_heads;
    p.num_pages = a->num_pages;
    p.pps = a->pages_per_seq;
    p.vecs = (int)(a->head_dim * elem(a->dtype) / 16);
    p.planes = a->n_layers * 2;
    const long long vecs = (long long)p.planes * p.hkv * p.vecs;
    return launched(launch(tree_accept_kernel, dim3((unsigned)((vecs + 255) / 256), a->B), 256, 0, cuda_stream, 1, false, p), "tree_accept");
}

}  // extern "C"

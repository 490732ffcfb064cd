// Sampling a token per row of logits by temperature, top-k, top-p and min-p, from one given uniform number a row (sm_100a).
//
// With w_i = exp((z_i - max z) / T) every filter keeps a prefix of the row in falling order (ties: lower id first): top-k by
// count, top-p by mass, min-p by value; the kept set is the shortest of the three.  The token is the first one, in rising
// order of ids, at which the running sum of the kept w exceeds u times their total.
//
// A row is held by the shared memory of a cluster of 1 to 8 blocks, so the logits are read from HBM once, whatever the
// filters.  No row is sorted as a whole.  The border of a filter is found by narrowing: the row's values between two bounds
// are dropped into 16 buckets (equal steps of the float's ordered bit pattern, the last one open below), the blocks add up
// their counts and masses, and the bucket that holds the border is the next range.  As soon as what lies above the range and
// in it is at most kSmList values -- mostly after one or two rounds -- the first block gathers these, sorts them and finishes alone.
// Flat rows, whose kept set is larger, go on until the range itself is that short, or a single value; then one pass in
// the order of ids sums what is kept.
//
// Masses are 64-bit sums of 64-bit exponentials: which id a number falls on hangs on the last bits of sums over the
// vocabulary; with 128256 tokens fp32 would move the border of one row in a few hundred.  The exponential is table-driven (a
// 64-entry table of powers of two and a polynomial of degree 5 on a 128th of an octave either side; the method of P. T. P.
// Tang, ACM TOMS 15 (1989)), relative error below 1e-14.
//
// What bounds it: one row, the cluster barriers (a microsecond each); many rows, the 64-bit pipe where all of a row's
// exponentials are needed (top-p alone, no filter at all), else the passes over shared memory.
#pragma once

#include <type_traits>

#include "dbt_ptx.cuh"

namespace dbt {

constexpr int kSmThreads = 256;
constexpr int kSmWarps = kSmThreads / 32;
constexpr int kSmBuckets = 16;
constexpr int kSmList = 1024;    // values that one block sorts
constexpr int kSmMaxCluster = 8;
constexpr int kSmMaxSlice = 32768;  // values of a row per block
constexpr int kSmScratchBytes = kSmBuckets * kSmThreads * 8;  // bucket masses per thread, or the list's keys, w and sums
static_assert(3 * kSmList * 8 <= kSmScratchBytes, "the list fits the scratch area");
static_assert(kSmMaxSlice / kSmThreads <= 255, "counts of a thread fit a byte per bucket");

struct SampleParams {
    const void *logits;
    long long row_stride;
    const float *uniforms, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int32_t *tokens;
    float *logprobs;
    int vocab, slice;  // values per block, a multiple of 8
};

__device__ __forceinline__ uint32_t sm_key(float x) {
    const int b = __float_as_int(x);
    return (uint32_t)b ^ ((uint32_t)(b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float sm_value(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
constexpr uint32_t kSmKeyLowest = 0x007fffffu;  // of -inf

struct SampleShared {
    double exchange[2][kSmMaxCluster][2 * kSmBuckets];
    double local[2 * kSmBuckets];
    double table[64];  // 2^(j / 64)
    double warp_d[kSmWarps];
    int warp_i[kSmWarps];
    int counts[kSmBuckets];
    int found;
};

struct SampleRow {
    SampleShared *sh;
    float *x;        // this block's values
    double *scratch;
    int n, base;  // values held, id of the first
    uint32_t rank, cluster;
    int parity;
    double top, step;  // largest value; 64 / (T ln 2)
    bool top_inf;

    __device__ __forceinline__ double weight(float z) const {
        if (top_inf) return z == INFINITY ? 1.0 : 0.0;
        const double t = ((double)z - top) * step;  // exponent in 64ths of an octave
        if (!(t > -64000.0) || z == -INFINITY) return 0.0;  // below 2^-1000
        const double shifted = t + 6755399441055744.0;  // 1.5 * 2^52: rounds to an integer in the low bits
        const int i = __double2loint(shifted);
        const double r = t - (shifted - 6755399441055744.0);
        // e^(r ln2 / 64) = 1 + r c + (r c)^2 / 2 + ..., |r c| <= 0.00542
        constexpr double c = 0.010830424696249145;  // ln 2 / 64
        const double p = fma(fma(fma(fma(fma(c * c * c * c * c / 120.0, r, c * c * c * c / 24.0), r, c * c * c / 6.0), r, c * c / 2.0), r, c), r, 1.0);
        const double w = p * sh->table[i & 63];
        return __hiloint2double(__double2hiint(w) + (i >> 6) * (1 << 20), __double2loint(w));
    }

    // sh->local[0..nv) of every block becomes visible to all: returns the buffer [rank][2 * kSmBuckets].
    __device__ __forceinline__ const double (*share(int nv))[2 * kSmBuckets] {
        __syncthreads();
        double(*buf)[2 * kSmBuckets] = sh->exchange[parity];
        parity ^= 1;
        if (cluster == 1) {
            for (int i = threadIdx.x; i < nv; i += kSmThreads) buf[0][i] = sh->local[i];
            __syncthreads();
        } else {
            for (int i = threadIdx.x; i < nv * (int)cluster; i += kSmThreads) {
                const int to = i / nv, v = i - to * nv;
                asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(mapa_u32(smem_u32(&buf[rank][v]), to)), "d"(sh->local[v]) : "memory");
            }
            cluster_sync_all();
        }
        return buf;
    }
    __device__ __forceinline__ double block_sum_d(double v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh->warp_d[threadIdx.x >> 5] = v;
        __syncthreads();
        double t = 0.0;
#pragma unroll
        for (int w = 0; w < kSmWarps; w++) t += sh->warp_d[w];
        return t;
    }
    __device__ __forceinline__ int block_sum_i(int v) {
        v = __reduce_add_sync(0xffffffffu, v);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh->warp_i[threadIdx.x >> 5] = v;
        __syncthreads();
        int t = 0;
#pragma unroll
        for (int w = 0; w < kSmWarps; w++) t += sh->warp_i[w];
        return t;
    }
    // Sum over the cluster, in the order of the ranks.
    __device__ __forceinline__ double sum_all(double v) {
        const double s = block_sum_d(v);
        if (threadIdx.x == 0) sh->local[0] = s;
        const auto buf = share(1);
        double t = 0.0;
        for (uint32_t r = 0; r < cluster; r++) t += buf[r][0];
        return t;
    }
};

// A border in falling order: values above tau are in, of those equal to it the first `ties` by id.
struct SampleBorder {
    uint32_t tau;
    int ties;
};
// A range of ordered bit patterns, what lies above it, and what it holds.
struct SampleRange {
    uint32_t lo, hi;
    long long above_n;
    double above_w;
    long long n;
};

// How many of n equal weights it takes to reach `mass`, one at least.
__device__ __forceinline__ int sm_ties(double mass, double each, int n) {
    const double need = ceil(mass / each);
    return need >= 1.0 ? (need < (double)n ? (int)need : n) : 1;  // (0 / 0: one)
}

// One round: 16 buckets of 2^shift patterns from r.hi down, the last one open to r.lo.  MASS: by mass (goal), else by count.
// `limit`: an earlier border; values outside it do not count.  total (first round): gets the mass of the whole range times
// `share_p` as the goal.  Returns true when the border itself is found.
template <bool MASS>
__device__ __forceinline__ bool sm_round(SampleRow &row, SampleRange &r, int shift, double &goal, bool first, double share_p,
                                         const SampleBorder *limit, SampleBorder &found) {
    SampleShared &sh = *row.sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned long long c0 = 0, c1 = 0;
    if (MASS)
#pragma unroll
        for (int b = 0; b < kSmBuckets; b++) row.scratch[b * kSmThreads + tid] = 0.0;
    if (tid < kSmBuckets) sh.counts[tid] = 0;
    const uint32_t lo = limit ? max(r.lo, limit->tau + 1) : r.lo;  // the border's own ties are added below
    for (int i = tid; i < row.n; i += kSmThreads) {
        const float z = row.x[i];
        const uint32_t k = sm_key(z);
        if (k > r.hi || k < lo) continue;
        const int b = min((int)((r.hi - k) >> shift), kSmBuckets - 1);
        const unsigned long long one = 1ull << (8 * (b & 7));
        if (b < 8) c0 += one;
        else c1 += one;
        if (MASS) row.scratch[b * kSmThreads + tid] += row.weight(z);
    }
    __syncthreads();
#pragma unroll
    for (int b = 0; b < kSmBuckets; b++) {
        const int c = (int)(((b < 8 ? c0 : c1) >> (8 * (b & 7))) & 255);
        const int s = __reduce_add_sync(0xffffffffu, c);
        if (lane == b && s) atomicAdd(&sh.counts[b], s);
    }
    if (MASS)
        for (int b = warp; b < kSmBuckets; b += kSmWarps) {
            double v = 0.0;
#pragma unroll
            for (int j = 0; j < kSmThreads / 32; j++) v += row.scratch[b * kSmThreads + j * 32 + lane];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (lane == 0) sh.local[b] = v;
        }
    __syncthreads();
    if (tid < kSmBuckets) sh.local[kSmBuckets + tid] = sh.counts[tid];
    const auto buf = row.share(2 * kSmBuckets);
    // lane b: bucket b over the blocks, then the running sums
    double w = 0.0, cw;
    long long c = 0, cc;
    if (lane < kSmBuckets) {
        for (uint32_t k = 0; k < row.cluster; k++) {
            if (MASS) w += buf[k][lane];
            c += (long long)buf[k][kSmBuckets + lane];
        }
        if (limit && limit->tau <= r.hi && limit->tau >= r.lo && (int)min((r.hi - limit->tau) >> shift, (uint32_t)(kSmBuckets - 1)) == lane) {
            c += limit->ties;
            if (MASS) w += limit->ties * row.weight(sm_value(limit->tau));
        }
    }
    cw = w;
    cc = c;
#pragma unroll
    for (int o = 1; o < kSmBuckets; o <<= 1) {
        const double a = __shfl_up_sync(0xffffffffu, cw, o);
        const long long d = __shfl_up_sync(0xffffffffu, cc, o);
        if (lane >= o) {
            cw += a;
            cc += d;
        }
    }
    if (MASS && first) goal = share_p * (r.above_w + __shfl_sync(0xffffffffu, cw, kSmBuckets - 1));
    const bool reached = MASS ? r.above_w + cw >= goal : (double)(r.above_n + cc) >= goal;
    const unsigned at = __ballot_sync(0xffffffffu, lane < kSmBuckets && c > 0 && reached);
    const unsigned held = __ballot_sync(0xffffffffu, lane < kSmBuckets && c > 0);
    // (a goal that rounding puts above the total: the last bucket that holds anything; the range always holds something)
    const int j = at ? __ffs(at) - 1 : held ? 31 - __clz(held) : 0;
    r.above_w += __shfl_sync(0xffffffffu, cw - w, j);
    r.above_n += __shfl_sync(0xffffffffu, cc - c, j);
    r.n = __shfl_sync(0xffffffffu, c, j);
    const double in = __shfl_sync(0xffffffffu, w, j);
    const uint32_t hi = r.hi;
    r.hi = hi - ((uint32_t)j << shift);
    const uint32_t span = 1u << shift;  // (shift <= 28)
    if (j < kSmBuckets - 1 && r.hi - r.lo >= span) r.lo = r.hi - span + 1;
    if (r.hi != r.lo) return false;
    found.tau = r.hi;
    if (MASS) {
        found.ties = sm_ties(goal - r.above_w, in / (double)r.n, (int)r.n);
    } else {
        found.ties = (int)(goal - (double)r.above_n);
    }
    return true;
}

// Every value from pattern `lo` to `hi` into the first block's scratch as (pattern falling, id rising) keys; returns how many.
__device__ __forceinline__ int sm_gather(SampleRow &row, uint32_t lo, uint32_t hi) {
    SampleShared &sh = *row.sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int mine = 0;
    for (int i = tid; i < row.n; i += kSmThreads) {
        const uint32_t k = sm_key(row.x[i]);
        mine += k >= lo && k <= hi;
    }
    int run = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += v;
    }
    __syncthreads();
    if (lane == 31) sh.warp_i[warp] = run;
    __syncthreads();
    int at = run - mine, total = 0;
#pragma unroll
    for (int w = 0; w < kSmWarps; w++) {
        if (w < warp) at += sh.warp_i[w];
        total += sh.warp_i[w];
    }
    if (tid == 0) sh.local[0] = total;
    const auto buf = row.share(1);
    int all = 0;
    for (uint32_t r = 0; r < row.cluster; r++) {
        if (r < row.rank) at += (int)buf[r][0];
        all += (int)buf[r][0];
    }
    const uint32_t list = mapa_u32(smem_u32(row.scratch), 0);
    for (int i = tid; i < row.n; i += kSmThreads) {
        const uint32_t k = sm_key(row.x[i]);
        if (k >= lo && k <= hi) {
            if (at < kSmList)  // (the callers have counted)
                asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(list + 8 * at), "l"(((unsigned long long)~k << 32) | (uint32_t)(row.base + i)) : "memory");
            at++;
        }
    }
    if (row.cluster == 1) __syncthreads();
    else cluster_sync_all();
    return min(all, kSmList);
}

// Bitonic sort of n <= kSmList keys by one block, rising.
__device__ __forceinline__ void sm_sort(unsigned long long *key, int n) {
    int m = 1;
    while (m < n) m <<= 1;
    for (int i = n + threadIdx.x; i < m; i += kSmThreads) key[i] = ~0ull;
    __syncthreads();
    for (int k = 2; k <= m; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            for (int t = threadIdx.x; t < m / 2; t += kSmThreads) {
                const int a = 2 * t - (t & (j - 1)), b = a + j;
                const unsigned long long x = key[a], y = key[b];
                if ((x > y) == ((a & k) == 0)) {
                    key[a] = y;
                    key[b] = x;
                }
            }
            __syncthreads();
        }
}
// Running sums of v[0..n) by one block, in order; 4 values per thread.
__device__ __forceinline__ void sm_running(SampleShared &sh, const double *v, double *out, int n) {
    static_assert(kSmList == 4 * kSmThreads, "four values a thread");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    double a[4], sum = 0.0;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        a[k] = 4 * tid + k < n ? v[4 * tid + k] : 0.0;
        sum += a[k];
    }
    double run = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double x = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += x;
    }
    __syncthreads();
    if (lane == 31) sh.warp_d[warp] = run;
    __syncthreads();
    double before = __shfl_up_sync(0xffffffffu, run, 1);
    if (lane == 0) before = 0.0;
    double base = 0.0;
    for (int w = 0; w < warp; w++) base += sh.warp_d[w];
    base += before;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        base += a[k];
        if (4 * tid + k < n) out[4 * tid + k] = base;
    }
    __syncthreads();
}

struct SampleFilters {
    bool k_on, p_on, m_on;
    int k;
    double p, m, u;
};

// The first block finishes alone from the n largest values (keys in scratch).  goal: mass that top-p asks for, where it is
// known; the list holds every survivor of top-k otherwise, or the whole row.
__device__ __forceinline__ void sm_finish_list(SampleRow &row, const SampleParams &p, int r, const SampleFilters &f, int n, bool goal_known,
                                               double goal) {
    SampleShared &sh = *row.sh;
    const int tid = threadIdx.x;
    unsigned long long *key = reinterpret_cast<unsigned long long *>(row.scratch);
    double *w = row.scratch + kSmList, *run = row.scratch + 2 * kSmList;
    sm_sort(key, n);
    if (f.k_on) n = min(n, f.k);
    for (int i = tid; i < n; i += kSmThreads) w[i] = row.weight(sm_value(~(uint32_t)(key[i] >> 32)));
    __syncthreads();
    int keep = n;
    if (f.p_on || f.m_on) {
        if (f.p_on) sm_running(sh, w, run, n);
        if (f.p_on && !goal_known) goal = f.p * run[n - 1];
        int in_p = 0, in_m = 0;
        for (int i = tid; i < n; i += kSmThreads) {
            in_p += f.p_on && run[i] < goal;
            in_m += f.m_on && w[i] >= f.m;
        }
        if (f.p_on) keep = min(keep, row.block_sum_i(in_p) + 1);
        if (f.m_on) keep = min(keep, row.block_sum_i(in_m));
        keep = max(keep, 1);
    }
    // the kept ones by id, their weights' places beside
    for (int i = tid; i < keep; i += kSmThreads) {
        const unsigned long long k = key[i];
        key[i] = (k << 32) | (uint32_t)i;
    }
    __syncthreads();
    sm_sort(key, keep);
    double *wi = run;  // weights by id, then their running sums over the weights' old place
    for (int i = tid; i < keep; i += kSmThreads) wi[i] = w[(uint32_t)key[i]];
    __syncthreads();
    sm_running(sh, wi, w, keep);
    const double total = w[keep - 1], target = f.u * total;
    if (tid == 0) sh.found = kSmList;
    __syncthreads();
    int first = kSmList, last = -1;
    for (int i = tid; i < keep; i += kSmThreads) {
        if (first == kSmList && w[i] > target) first = i;
        if (wi[i] > 0.0) last = i;
    }
    if (first < kSmList) atomicMin(&sh.found, first);
    __syncthreads();
    int at = sh.found;
    if (at == kSmList) {  // u of one or more, or not a number
        __syncthreads();
        if (tid == 0) sh.found = -1;
        __syncthreads();
        atomicMax(&sh.found, last);
        __syncthreads();
        at = sh.found;
    }
    if (tid == 0) {
        p.tokens[r] = (int32_t)(key[at] >> 32);
        if (p.logprobs) p.logprobs[r] = (float)log(wi[at] / total);
    }
}

template <typename T>
__global__ void __launch_bounds__(kSmThreads) sample_kernel(const SampleParams p) {
    extern __shared__ __align__(16) uint8_t smem_b[];
    __shared__ SampleShared sh;
    SampleRow row;
    row.sh = &sh;
    row.scratch = reinterpret_cast<double *>(smem_b);
    row.x = reinterpret_cast<float *>(smem_b + kSmScratchBytes);
    row.parity = 0;
    row.rank = cluster_rank();
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(row.cluster));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int r = blockIdx.x / row.cluster;
    row.base = row.rank * p.slice;
    row.n = max(0, min(p.slice, p.vocab - row.base));

    // ---- the row into shared memory, its largest value
    const T *src = reinterpret_cast<const T *>(p.logits) + (long long)r * p.row_stride + row.base;
    float mx = -INFINITY;
    auto put = [&](int i, float v) {
        v = v != v ? -INFINITY : v + 0.f;  // NaN counts as -inf; -0 becomes +0
        row.x[i] = v;
        mx = fmaxf(mx, v);
    };
    constexpr int VN = 16 / sizeof(T);
    int head = 0;
    if ((reinterpret_cast<uintptr_t>(src) & 15) == 0) {
        head = row.n / VN * VN;
#pragma unroll 4
        for (int i = tid * VN; i < head; i += kSmThreads * VN) {
            const uint4 raw = __ldg(reinterpret_cast<const uint4 *>(src + i));
            const T *e = reinterpret_cast<const T *>(&raw);
#pragma unroll
            for (int k = 0; k < VN; k++) put(i + k, load1(e + k));
        }
    }
    for (int i = head + tid; i < row.n; i += kSmThreads) put(i, load1(src + i));
    if (tid < 64) sh.table[tid] = exp2(tid / 64.0);
    SampleFilters f;
    const float temp = p.temperature ? p.temperature[r] : 1.f;
    f.u = p.uniforms[r];
    f.k = p.top_k ? p.top_k[r] : 0;
    f.p = p.top_p ? p.top_p[r] : 1.f;
    f.m = p.min_p ? p.min_p[r] : 0.f;
    f.m_on = f.m > 0.0;
    if (f.m > 1.0) f.k = 1;  // nothing but the likeliest token reaches it
    f.k_on = f.k > 0 && f.k < p.vocab;
    f.p_on = !(f.p >= 1.0);
    if (f.p != f.p) f.p = 0.0;
    mx = block_max(mx, reinterpret_cast<float *>(sh.warp_d));
    if (tid == 0) sh.local[0] = mx;
    {
        const auto buf = row.share(1);
        for (uint32_t k = 0; k < row.cluster; k++) mx = fmaxf(mx, (float)buf[k][0]);
    }
    row.top = mx;
    row.top_inf = mx == INFINITY;
    row.step = 92.332482616893657 / (double)temp;  // 64 / ln 2
    if (mx == -INFINITY) {
        if (row.rank == 0 && tid == 0) {
            p.tokens[r] = -1;
            if (p.logprobs) p.logprobs[r] = -INFINITY;
        }
        return;
    }
    if (!(temp > 0.f)) {  // the largest logit, the lowest id of several
        int best = 0x7fffffff;
        for (int i = tid; i < row.n; i += kSmThreads)
            if (row.x[i] == mx) best = min(best, row.base + i);
        best = __reduce_min_sync(0xffffffffu, best);
        if (lane == 0) sh.warp_i[warp] = best;
        __syncthreads();
        for (int w = 0; w < kSmWarps; w++) best = min(best, sh.warp_i[w]);
        if (tid == 0) sh.local[0] = best;
        const auto buf = row.share(1);
        for (uint32_t k = 0; k < row.cluster; k++) best = min(best, (int)buf[k][0]);
        if (row.rank == 0 && tid == 0) {
            p.tokens[r] = best;
            if (p.logprobs) p.logprobs[r] = 0.f;
        }
        return;
    }

    // ---- the borders
    const uint32_t key_top = sm_key(mx);
    SampleBorder border{0, 0};  // everything
    bool bounded = false;
    auto narrow = [&](auto mass, double &goal, const SampleBorder *limit, SampleRange &range, SampleBorder &found) -> int {
        // 1: the values from range.lo up fit the list; 2: `found` is the border
        constexpr bool MASS = decltype(mass)::value;
        // The first window reaches 8 units below the largest value (counts), 8 T (masses): about where the border lies in a
        // language model's logits.  A border below it is looked for in a window 16 times as wide, then in all that is left.
        float reach = MASS ? 8.f * temp : 8.f;
        range = SampleRange{kSmKeyLowest, key_top, 0, 0.0, 0};
        for (int it = 0; it < 16; it++) {  // (two rounds of windows, then eight at most: a round takes four of 32 bits)
            const uint32_t full = range.hi - range.lo;
            uint32_t span = full;
            if (range.lo == kSmKeyLowest && it < 2) {
                const uint32_t low = sm_key(sm_value(range.hi) - reach);  // (not a number: above, the full range)
                if (low < range.hi && low > range.lo) span = range.hi - low;
                reach *= 16.f;
            }
            const int shift = 28 - __clz(span | 15);  // 16 buckets cover span + 1 patterns
            const bool exact = sm_round<MASS>(row, range, shift, goal, it == 0, f.p, limit, found);
            if (exact) return 2;
            if (!limit && range.above_n + range.n <= kSmList) return 1;
            if (range.n <= kSmList) {
                // the range alone fits the list: the first block sorts it and says where the border is (the ties of an
                // earlier border, which may be many more than count, stay outside)
                const bool ends = limit && range.lo <= limit->tau;
                const int n = sm_gather(row, ends ? limit->tau + 1 : range.lo, range.hi);
                if (row.rank == 0) {
                    unsigned long long *key = reinterpret_cast<unsigned long long *>(row.scratch);
                    double *w = row.scratch + kSmList, *run = row.scratch + 2 * kSmList;
                    sm_sort(key, n);
                    int at;  // number of values of the range above the border
                    if (MASS) {
                        for (int i = tid; i < n; i += kSmThreads) w[i] = row.weight(sm_value(~(uint32_t)(key[i] >> 32)));
                        __syncthreads();
                        sm_running(sh, w, run, n);
                        int before = 0;
                        for (int i = tid; i < n; i += kSmThreads) before += range.above_w + run[i] < goal;
                        at = row.block_sum_i(before);
                        if (!ends) at = min(at, n - 1);
                    } else {
                        at = (int)(goal - (double)range.above_n) - 1;
                    }
                    uint32_t tau;
                    int same = 0;
                    if (at < n) {
                        tau = ~(uint32_t)(key[at] >> 32);
                        for (int i = tid; i <= at; i += kSmThreads) same += (uint32_t)(key[i] >> 32) == ~tau;
                        same = row.block_sum_i(same);
                    } else {
                        tau = limit->tau;
                        same = sm_ties(goal - range.above_w - (n > 0 ? run[n - 1] : 0.0), row.weight(sm_value(tau)), limit->ties);
                    }
                    if (tid == 0) {
                        sh.local[0] = tau;
                        sh.local[1] = same;
                    }
                }
                const auto buf = row.share(2);
                found.tau = (uint32_t)buf[0][0];
                found.ties = (int)buf[0][1];
                return 2;
            }
        }
        found = SampleBorder{range.hi, 1};
        return 2;
    };

    SampleRange range{kSmKeyLowest, key_top, 0, 0.0, p.vocab};
    bool listed = p.vocab <= kSmList, goal_known = false;
    double goal = 0.0;
    if (!listed && f.k_on) {
        goal = f.k;
        if (narrow(std::false_type{}, goal, nullptr, range, border) == 1) listed = true;
        else bounded = true;
    }
    if (!listed && f.p_on) {
        SampleBorder other;
        const int how = narrow(std::true_type{}, goal, bounded ? &border : nullptr, range, other);
        goal_known = true;
        if (how == 1) {
            listed = true;
        } else {
            if (bounded && other.tau == border.tau) other.ties = min(other.ties, border.ties);
            border = other;  // (never below top-k's: masses were counted inside it)
            bounded = true;
        }
    } else if (!listed && !bounded && f.m_on) {
        // w >= m is z >= max + T ln m; a little below that, whatever the roundings: the list's own test is the exact one
        const double low = row.top + (double)temp * (log(f.m) - 1e-6);
        const uint32_t lo = row.top_inf ? key_top : max(kSmKeyLowest, sm_key(__double2float_rd(low) + 0.f));
        int c = 0;
        for (int i = tid; i < row.n; i += kSmThreads) c += sm_key(row.x[i]) >= lo;
        if (row.sum_all((double)c) <= kSmList) {
            listed = true;
            range.lo = lo;
        }
    }
    if (listed) {
        const int n = sm_gather(row, range.lo, key_top);
        if (row.rank == 0) sm_finish_list(row, p, r, f, n, goal_known, goal);
        return;
    }

    // ---- many values are kept: sums in the order of ids.  Warp w of a block has a run of consecutive values.
    const int per = ((p.slice + kSmWarps - 1) / kSmWarps + 31) & ~31, i0 = min(row.n, warp * per), i1 = min(row.n, i0 + per);
    int ties_before = 0;
    if (bounded) {
        int c = 0;
        for (int i = i0 + lane; i < i1; i += 32) c += sm_key(row.x[i]) == border.tau;
        c = __reduce_add_sync(0xffffffffu, c);
        __syncthreads();
        if (lane == 0) sh.warp_i[warp] = c;
        __syncthreads();
        int all = 0;
        for (int w = 0; w < kSmWarps; w++) {
            if (w < warp) ties_before += sh.warp_i[w];
            all += sh.warp_i[w];
        }
        if (tid == 0) sh.local[0] = all;
        const auto buf = row.share(1);
        for (uint32_t k = 0; k < row.rank; k++) ties_before += (int)buf[k][0];
    }
    // the weight of value i, zero where it is not kept; `seen` counts the border's ties before the warp's 32
    auto kept = [&](int i, int &seen) -> double {
        const float z = i < i1 ? row.x[i] : 0.f;
        const uint32_t k = sm_key(z);
        bool in = i < i1 && (!bounded || k > border.tau);
        if (bounded) {
            const bool tie = i < i1 && k == border.tau;
            const unsigned m = __ballot_sync(0xffffffffu, tie);
            in = in || (tie && seen + __popc(m & ((1u << lane) - 1)) < border.ties);
            seen += __popc(m);
        }
        if (!in) return 0.0;
        const double w = row.weight(z);
        return f.m_on && w < f.m ? 0.0 : w;
    };
    double mine = 0.0;
    int seen = ties_before;
    for (int i = i0 + lane; i - lane < i1; i += 32) mine += kept(i, seen);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    __syncthreads();
    if (lane == 0) sh.warp_d[warp] = mine;
    __syncthreads();
    double all = 0.0, total = 0.0;
    for (int w = 0; w < kSmWarps; w++) all += sh.warp_d[w];
    if (tid == 0) sh.local[0] = all;
    const auto sums = row.share(1);
    double base = 0.0, run = 0.0;
    for (uint32_t k = 0; k < row.cluster; k++) total += sums[k][0];
    const double target = f.u * total;
    // the block, then the warp in whose run the target lies; the last with any mass takes what rounding leaves over
    int owner = -1, last = 0;
    for (uint32_t k = 0; k < row.cluster && owner < 0; k++) {
        if (k == row.rank) base = run;
        run += sums[k][0];
        if (sums[k][0] > 0.0) last = k;
        if (run > target) owner = k;
    }
    if ((owner < 0 ? last : owner) != (int)row.rank) return;
    run = base;
    owner = -1;
    last = 0;
    double before = base;
    for (int w = 0; w < kSmWarps && owner < 0; w++) {
        const double next = run + sh.warp_d[w];
        if (sh.warp_d[w] > 0.0) {
            last = w;
            if (warp == w) before = run;
        }
        if (next > target) owner = w;
        run = next;
    }
    if ((owner < 0 ? last : owner) != warp) return;
    seen = ties_before;
    int token = -1;
    double share_w = 0.0;
    for (int i = i0 + lane; i - lane < i1; i += 32) {
        const double w = kept(i, seen);
        double upto = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, w > 0.0 && before + upto > target), any = __ballot_sync(0xffffffffu, w > 0.0);
        if (any) {
            const int l = hit ? __ffs(hit) - 1 : 31 - __clz(any);
            token = row.base + i - lane + l;
            share_w = __shfl_sync(0xffffffffu, w, l);
        }
        if (hit) break;
        before += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) {
        p.tokens[r] = token;
        if (p.logprobs) p.logprobs[r] = (float)log(share_w / total);
    }
}

}  // namespace dbt

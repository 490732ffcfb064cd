// Sampling a token per row of logits by temperature, top-k, top-p and min-p, from one given uniform number a row (sm_100a).
//
// With w_i = exp((z_i - max z) / T) every filter keeps a prefix of the row in falling order (ties: lower id first): top-k by
// count, top-p by mass, min-p by value; the kept set is the shortest of the three.  The token is the first one, in rising
// order of ids, at which the running sum of the kept w exceeds u times their total.
//
// A row is shared out over a cluster of 1 to 8 blocks.  Its logits come from HBM once and are read again, from L1 or L2, by the
// passes that follow (held in shared memory they left room for two blocks per SM and 256 rows of 128256 with all filters took 383 us;
// with four resident, which cover one another's barriers, 241, and 127 with the steps that came later).  No row is sorted as a whole.
//
// The short way.  Every thread knows the largest of the values it loaded, one for each place of its four-value loads; the K-th
// largest of these maxima has at least K values of the row at or above it, and seldom many more.  What lies above that bound
// (K = top_k, or 384 where top-p alone asks) is sent to the first block, which sorts it and finishes alone, if the kept set turns
// out to lie inside.
//
// The middle way, where more is kept.  The values' counts in 1024 equal steps below the largest (taken along in a pass that is made
// anyway) say in which steps the border must lie -- by count exactly, by mass up to what the steps' width leaves open --; one pass
// forms the mass above them and sends what lies in them to the first block, which sorts it and finds the border, exactly or
// not at all.
//
// The long way, for ties and whatever the others leave.  The border of a filter is found by narrowing: the row's values between
// two bounds are dropped into 16 buckets (equal steps of the float's ordered bit pattern, the last one open below), the blocks
// add up their counts and masses, and the bucket that holds the border is the next range, until what lies above the range and
// in it, or at least the range itself, is a list that one block can sort, or a single value.
//
// Where the kept set is larger than a list, a pass in the order of ids sums what is kept, 256 ids at a time.
//
// Masses are 64-bit sums of 64-bit exponentials: which id a number falls on hangs on the last bits of sums over the
// vocabulary; with 128256 tokens fp32 would move the border of one row in a few hundred.  The exponential is table-driven (16
// powers of two and a polynomial of degree 6 on a 32nd of an octave either side; the method of P. T. P. Tang, ACM TOMS 15
// (1989)), relative error below 1e-14.  16 doubles are one row of the shared-memory banks: lookups do not conflict (64 entries
// cost six cycles a warp, as much as the arithmetic).
//
// What bounds it: one row, the cluster barriers (one to two microseconds each); many rows, where all of a row's exponentials are
// needed (top-p alone, no filter at all), the latency of the 64-bit chains and of the passes over L2, else the passes.  Measured,
// fp32 logits, 128256 a row: one row 13 us without filters, 15 with top-k 50, top-p and min-p, 23 with top-p alone; 256 rows (131 MB, 20 us
// of HBM) 89, 57 and 137 to 193, with settings of all kinds 126 to 132; 64 rows without filters 28.
#pragma once

#include <type_traits>

#include "dbt_ptx.cuh"

namespace dbt {

constexpr int kSmBuckets = 16;   // of a round by count; by mass kSmMassBuckets
constexpr int kSmMassBuckets = 8;
constexpr int kSmList = 1024;    // values that one block sorts
constexpr int kSmGuess = 512;    // the largest top_k of the short way
// Values that the short way asks for where top-p alone says how many: a list of up to 512 is sorted in two thirds of the time that one
// of up to 1024 takes.  With 512, 384, 256: one row of 32000 21.0, 19.0, 18.9 us; 64 rows of 128256 114, 85, 83; 256 rows whose
// border lies below the list 295, 294, 383 (too few exact ones for the middle way).  Not measured at other widths.
constexpr int kSmNucleus = 384;
constexpr int kSmMaxBuckets = 64;  // for the threads' maxima
constexpr int kSmRun = 256;      // ids summed together by a warp on the long way
constexpr int kSmSteps = 1024;   // of the middle way
constexpr int kSmMaxCluster = 8;
constexpr int kSmMaxSlice = 32768;  // values of a row per block
// Scratch area: the list's keys, w and sums, or bucket masses per thread.
constexpr int sm_scratch_bytes(int threads) { return 8 * (3 * kSmList > kSmMassBuckets * threads ? 3 * kSmList : kSmMassBuckets * threads); }
static_assert(kSmMaxSlice / 256 <= 255, "counts of a thread fit a byte per bucket");

struct SampleParams {
    const void *logits;
    long long row_stride;
    const float *uniforms, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int32_t *tokens;
    float *logprobs;
    int vocab, slice;  // values per block, a multiple of 8
    int rows, order;   // order: long rows first
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
    double table[16];  // 2^(j / 16)
    double warp_d[32];
    int warp_i[32];
    int counts[kSmBuckets];
    int found, sent;
    unsigned slots;  // list entries handed out to the cluster (first block)
    union {
        struct {
            int local[kSmMaxBuckets], all[kSmMaxCluster][kSmMaxBuckets];  // short way: the threads' maxima by bucket
        } maxima;
        struct {
            double mass[kSmMaxSlice / kSmRun];  // where many are kept: per run of ids the kept mass, its running sum, the border's ties
            double sums[kSmMaxSlice / kSmRun];
            int ties[kSmMaxSlice / kSmRun];
        } runs;
    };
};

template <typename T, int NT>
struct SampleRow {
    static constexpr int kWarps = NT / 32;
    SampleShared *sh;
    const T *src;  // this block's values
    double *scratch;
    int n, base;  // values held, id of the first
    uint32_t rank, cluster;
    int parity;
    double top, step;  // largest value; 16 / (T ln 2)
    float zmin;        // smaller values weigh nothing: below 2^-1000, or (where the largest is infinite) not infinite

    __device__ __forceinline__ void set_scale(float mx, float temp) {
        const bool inf = mx == INFINITY;
        top = inf ? 3.402823466e38 : mx;
        step = inf ? 0.0 : 23.083120654223414 / (double)temp;  // 16 / ln 2
        zmin = inf ? INFINITY : fmaxf(__double2float_ru(top - 16000.0 / step), -3.402823466e38f);
    }
    // Without a branch, so that several values' chains overlap.
    __device__ __forceinline__ double weight(float z) const {
        const double t = ((double)fminf(fmaxf(z, zmin), 3.402823466e38f) - top) * step;  // exponent in 16ths of an octave
        const double shifted = t + 6755399441055744.0;  // 1.5 * 2^52: rounds to an integer in the low bits
        const int i = __double2loint(shifted);
        const double r = t - (shifted - 6755399441055744.0);
        // e^(r ln2 / 16) = 1 + r c + (r c)^2 / 2 + ..., |r c| <= 0.0217
        constexpr double c = 0.04332169878499658, c2 = c * c / 2.0, c3 = c2 * c / 3.0, c4 = c3 * c / 4.0, c5 = c4 * c / 5.0, c6 = c5 * c / 6.0;
        const double p = fma(fma(fma(fma(fma(fma(c6, r, c5), r, c4), r, c3), r, c2), r, c), r, 1.0);
        const double w = p * sh->table[i & 15];
        const int hi = __double2hiint(w) + (i >> 4) * (1 << 20);
        const bool any = z >= zmin;
        return __hiloint2double(any ? hi : 0, any ? __double2loint(w) : 0);
    }

    static __device__ __forceinline__ float clean(float v) { return v != v ? -INFINITY : v + 0.f; }  // NaN counts as -inf; -0 becomes +0
    __device__ __forceinline__ float at(int i) const { return clean(load1(src + i)); }
    // f(i, z, m) for this thread's share of the block's values, m neighbours z[0..m) from number i on: fours out of 16-byte vectors,
    // several in flight, and the single values before the first whole vector and after the last.
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        constexpr int VN = 16 / sizeof(T), A = 4;
        const int tid = threadIdx.x, lead = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(src) & 15)) & 15) / (int)sizeof(T));
        const int vecs = (n - lead) / VN, tail = lead + vecs * VN;
        const uint4 *v = reinterpret_cast<const uint4 *>(src + lead);
        for (int i0 = tid; i0 < vecs; i0 += A * NT) {
            uint4 raw[A];
#pragma unroll
            for (int a = 0; a < A; a++)
                if (i0 + a * NT < vecs) raw[a] = __ldg(v + i0 + a * NT);
#pragma unroll
            for (int a = 0; a < A; a++) {
                if (i0 + a * NT >= vecs) break;
                const T *e = reinterpret_cast<const T *>(&raw[a]);
#pragma unroll
                for (int k = 0; k < VN; k += 4) {
                    const float z[4] = {clean(load1(e + k)), clean(load1(e + k + 1)), clean(load1(e + k + 2)), clean(load1(e + k + 3))};
                    f(lead + (i0 + a * NT) * VN + k, z, 4);
                }
            }
        }
        for (int s = 0; s < 2; s++) {
            const int i = s == 0 ? tid : tail + tid;
            if (i < (s == 0 ? lead : n)) {
                const float z[4] = {at(i), 0.f, 0.f, 0.f};
                f(i, z, 1);
            }
        }
    }
    // A list entry: pattern falling, id rising.
    __device__ __forceinline__ void send(uint32_t addr, uint32_t k, int i) const {
        asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(((unsigned long long)~k << 32) | (uint32_t)(base + i)) : "memory");
    }

    // sh->local[0..nv) of every block becomes visible to all: returns the buffer [rank][2 * kSmBuckets].
    __device__ __forceinline__ const double (*share(int nv))[2 * kSmBuckets] {
        __syncthreads();
        double(*buf)[2 * kSmBuckets] = sh->exchange[parity];
        parity ^= 1;
        if (cluster == 1) {
            for (int i = threadIdx.x; i < nv; i += NT) buf[0][i] = sh->local[i];
            __syncthreads();
        } else {
            for (int i = threadIdx.x; i < nv * (int)cluster; i += NT) {
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
        for (int w = 0; w < NT / 32; w++) t += sh->warp_d[w];
        return t;
    }
    __device__ __forceinline__ int block_sum_i(int v) {
        v = __reduce_add_sync(0xffffffffu, v);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh->warp_i[threadIdx.x >> 5] = v;
        __syncthreads();
        int t = 0;
#pragma unroll
        for (int w = 0; w < NT / 32; w++) t += sh->warp_i[w];
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

// A border in falling order: values above tau are in, of those equal to it the first `ties` by id (all of them: `whole`).
struct SampleBorder {
    uint32_t tau;
    int ties;
    bool whole;
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

// One round: buckets of 2^shift patterns from r.hi down, the last one open to r.lo.  MASS: by mass (goal), else by count.  `limit`: an
// earlier border; values outside it do not count.  find_goal: the goal is the mass of all that lies in the range and above times share_p
// (else the open bucket's mass is not needed, and not formed).  Returns true when the border itself is found.
template <bool MASS, typename T, int NT>
__device__ __forceinline__ bool sm_round(SampleRow<T, NT> &row, SampleRange &r, int shift, double &goal, bool find_goal, double share_p,
                                         const SampleBorder *limit, SampleBorder &found) {
    constexpr int NB = MASS ? kSmMassBuckets : kSmBuckets;
    SampleShared &sh = *row.sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned long long c0 = 0, c1 = 0;
    if (MASS)
#pragma unroll
        for (int b = 0; b < NB; b++) row.scratch[b * NT + tid] = 0.0;
    if (tid < kSmBuckets) sh.counts[tid] = 0;
    const uint32_t lo = limit ? max(r.lo, limit->tau + 1) : r.lo;  // the border's own ties are added below
    const bool open = MASS && !find_goal && ((r.hi - r.lo) >> shift) >= NB;  // the last bucket's mass is not needed
    row.each([&](int, const float(&z)[4], int m) {
        int b[4];  // bucket, -1: outside
        bool any = false;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const uint32_t k = sm_key(z[e]);
            const bool in = e < m && k <= r.hi && k >= lo;
            b[e] = in ? (int)min((r.hi - k) >> shift, (uint32_t)(NB - 1)) : -1;  // (patterns may be more than 2^31 apart)
            const unsigned long long one = in ? 1ull << (8 * (b[e] & 7)) : 0ull;
            if (NB <= 8 || b[e] < 8) c0 += one;
            else c1 += one;
            any = any || (in && !(open && b[e] == NB - 1));
        }
        if (MASS && any) {
            double w[4];  // side by side, then into the buckets one after the other
#pragma unroll
            for (int e = 0; e < 4; e++) w[e] = row.weight(z[e]);
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (b[e] >= 0) row.scratch[b[e] * NT + tid] += w[e];
        }
    });
    __syncthreads();
#pragma unroll
    for (int b = 0; b < NB; b++) {
        const int c = (int)(((b < 8 ? c0 : c1) >> (8 * (b & 7))) & 255);
        const int s = __reduce_add_sync(0xffffffffu, c);
        if (lane == b && s) atomicAdd(&sh.counts[b], s);
    }
    if (MASS)
        for (int b = warp; b < NB; b += NT / 32) {
            double v = 0.0;
#pragma unroll
            for (int j = 0; j < NT / 32; j++) v += row.scratch[b * NT + j * 32 + lane];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (lane == 0) sh.local[b] = v;
        }
    __syncthreads();
    if (tid < NB) sh.local[kSmBuckets + tid] = sh.counts[tid];
    const auto buf = row.share(2 * kSmBuckets);
    // lane b: bucket b over the blocks, then the running sums
    double w = 0.0, cw;
    long long c = 0, cc;
    if (lane < NB) {
        for (uint32_t k = 0; k < row.cluster; k++) {
            if (MASS) w += buf[k][lane];
            c += (long long)buf[k][kSmBuckets + lane];
        }
        if (limit && limit->tau <= r.hi && limit->tau >= r.lo && (int)min((r.hi - limit->tau) >> shift, (uint32_t)(NB - 1)) == lane) {
            c += limit->ties;
            if (MASS) w += limit->ties * row.weight(sm_value(limit->tau));
        }
    }
    cw = w;
    cc = c;
#pragma unroll
    for (int o = 1; o < NB; o <<= 1) {
        const double a = __shfl_up_sync(0xffffffffu, cw, o);
        const long long d = __shfl_up_sync(0xffffffffu, cc, o);
        if (lane >= o) {
            cw += a;
            cc += d;
        }
    }
    if (MASS && find_goal) goal = share_p * (r.above_w + __shfl_sync(0xffffffffu, cw, NB - 1));
    const bool reached = MASS ? r.above_w + cw >= goal : (double)(r.above_n + cc) >= goal;
    const unsigned at = __ballot_sync(0xffffffffu, lane < NB && c > 0 && reached);
    const unsigned held = __ballot_sync(0xffffffffu, lane < NB && c > 0);
    // (a goal that rounding puts above the total, or in the open bucket: the last that holds anything; the range always holds something)
    const int j = at ? __ffs(at) - 1 : held ? 31 - __clz(held) : 0;
    r.above_w += __shfl_sync(0xffffffffu, cw - w, j);
    r.above_n += __shfl_sync(0xffffffffu, cc - c, j);
    r.n = __shfl_sync(0xffffffffu, c, j);
    const double in = __shfl_sync(0xffffffffu, w, j);
    const uint32_t hi = r.hi;
    r.hi = hi - ((uint32_t)j << shift);
    const uint32_t span = 1u << shift;  // (shift <= 29)
    if (j < NB - 1 && r.hi - r.lo >= span) r.lo = r.hi - span + 1;
    if (r.hi != r.lo) return false;
    found.tau = r.hi;
    if (MASS) found.ties = sm_ties(goal - r.above_w, in / (double)r.n, (int)r.n);
    else found.ties = (int)(goal - (double)r.above_n);
    found.whole = found.ties >= r.n && !(limit && limit->tau == r.hi && !limit->whole);
    return true;
}

// Every value from pattern `lo` to `hi` into the first block's scratch as (pattern falling, id rising) keys; returns how many.
template <typename T, int NT>
__device__ __forceinline__ int sm_gather(SampleRow<T, NT> &row, uint32_t lo, uint32_t hi) {
    SampleShared &sh = *row.sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int mine = 0;
    row.each([&](int, const float(&z)[4], int m) {
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const uint32_t k = sm_key(z[e]);
            mine += e < m && k >= lo && k <= hi;
        }
    });
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
    for (int w = 0; w < NT / 32; w++) {
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
    row.each([&](int i, const float(&z)[4], int m) {
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const uint32_t k = sm_key(z[e]);
            if (e < m && k >= lo && k <= hi) {
                if (at < kSmList) row.send(list + 8 * at, k, i + e);  // (the callers have counted)
                at++;
            }
        }
    });
    if (row.cluster == 1) __syncthreads();
    else cluster_sync_all();
    return min(all, kSmList);
}

// Bitonic merges inside a warp of keys that stand four to a lane (number = first + 4 lane + place): steps from distance `from` down.
__device__ __forceinline__ void sm_merge(unsigned long long (&x)[4], int first, int k, int from) {
    const int i0 = first + 4 * (threadIdx.x & 31);
    auto order = [](unsigned long long &a, unsigned long long &b, bool rising) {
        const bool swap = (a > b) == rising;
        const unsigned long long s = swap ? b : a, l = swap ? a : b;
        a = s;
        b = l;
    };
    for (int j = from; j >= 4; j >>= 1) {
        const bool least = ((i0 & j) == 0) == ((i0 & k) == 0);
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const unsigned long long y = __shfl_xor_sync(0xffffffffu, x[q], j >> 2);
            x[q] = (x[q] < y) == least ? x[q] : y;
        }
    }
    if (k >= 4) {
        const bool rising = (i0 & k) == 0;
        order(x[0], x[2], rising);
        order(x[1], x[3], rising);
        order(x[0], x[1], rising);
        order(x[2], x[3], rising);
    } else {
        order(x[0], x[1], true);
        order(x[2], x[3], false);
    }
}
__device__ __forceinline__ void sm_sort_warp(unsigned long long (&x)[4], int first) {
#pragma unroll 1
    for (int k = 2; k <= 128; k <<= 1) sm_merge(x, first, k, k >> 1);
}
// Sort of n <= kSmList keys by one block, rising: 128 keys to a warp in registers, larger distances through shared memory.
__device__ __forceinline__ void sm_sort(unsigned long long *key, int n) {
    int m = 128;
    while (m < n) m <<= 1;
    __syncthreads();
    const int i0 = 4 * (int)threadIdx.x, first = i0 & ~127;
    if (i0 < m) {
        unsigned long long x[4];
#pragma unroll
        for (int q = 0; q < 4; q++) x[q] = i0 + q < n ? key[i0 + q] : ~0ull;
        sm_sort_warp(x, first);
#pragma unroll 1
        for (int k = 256; k <= m; k <<= 1) {
#pragma unroll 1
            for (int j = k >> 1; j >= 128; j >>= 1) {
#pragma unroll
                for (int q = 0; q < 4; q++) key[i0 + q] = x[q];
                asm volatile("bar.sync 1, %0;" ::"r"(m / 4) : "memory");
                const bool least = ((i0 & j) == 0) == ((i0 & k) == 0);
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const unsigned long long y = key[(i0 ^ j) + q];
                    x[q] = (x[q] < y) == least ? x[q] : y;
                }
                asm volatile("bar.sync 1, %0;" ::"r"(m / 4) : "memory");
            }
            sm_merge(x, first, k, 64);
        }
#pragma unroll
        for (int q = 0; q < 4; q++) key[i0 + q] = x[q];
    }
    __syncthreads();
}
// Running sums of v[0..n) by one block, in order.
template <int NT>
__device__ __forceinline__ void sm_running(SampleShared &sh, const double *v, double *out, int n) {
    constexpr int E = kSmList / NT;
    static_assert(E * NT == kSmList && NT <= 1024, "the list is shared out evenly");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    double a[E], sum = 0.0;
#pragma unroll
    for (int k = 0; k < E; k++) {
        a[k] = E * tid + k < n ? v[E * tid + k] : 0.0;
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
    for (int k = 0; k < E; k++) {
        base += a[k];
        if (E * tid + k < n) out[E * tid + k] = base;
    }
    __syncthreads();
}
// Running sums of a warp's values, four to a lane in order; returns the sum before the lane's first.
__device__ __forceinline__ double sm_running_warp(const double (&a)[4]) {
    const int lane = threadIdx.x & 31;
    double run = (a[0] + a[1]) + (a[2] + a[3]);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double x = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += x;
    }
    const double before = __shfl_up_sync(0xffffffffu, run, 1);
    return lane == 0 ? 0.0 : before;
}

struct SampleFilters {
    bool k_on, p_on, m_on;
    int k;
    double p, m, u;
};

// The first block finishes alone from the n largest values (keys in scratch).  goal: mass that top-p asks for, where it is
// known; the list holds every survivor of top-k otherwise, or the whole row.  guess: the list may be too short for what
// top-p and min-p keep; false then, nothing is written, and *mass gets what the list weighs.
template <typename T, int NT>
__device__ __forceinline__ bool sm_finish_list(SampleRow<T, NT> &row, const SampleParams &p, int r, const SampleFilters &f, int n, bool goal_known,
                                               double goal, bool guess, double *mass) {
    SampleShared &sh = *row.sh;
    const int tid = threadIdx.x;
    unsigned long long *key = reinterpret_cast<unsigned long long *>(row.scratch);
    double *w = row.scratch + kSmList, *run = row.scratch + 2 * kSmList;
    if (n <= 128) {  // one warp, without barriers
        __syncthreads();
        if (tid < 32) {
            const int i0 = 4 * tid;
            unsigned long long x[4];
#pragma unroll
            for (int q = 0; q < 4; q++) x[q] = i0 + q < n ? key[i0 + q] : ~0ull;
            sm_sort_warp(x, 0);
            if (f.k_on) n = min(n, f.k);
            double v[4];
#pragma unroll
            for (int q = 0; q < 4; q++) v[q] = i0 + q < n ? row.weight(sm_value(~(uint32_t)(x[q] >> 32))) : 0.0;
            double upto = sm_running_warp(v);
            const double whole = __shfl_sync(0xffffffffu, upto + ((v[0] + v[1]) + (v[2] + v[3])), 31);
            if (f.p_on && !goal_known) goal = f.p * whole;
            int in_p = 0, in_m = 0;
#pragma unroll
            for (int q = 0; q < 4; q++) {
                upto += v[q];
                in_p += i0 + q < n && upto < goal;
                in_m += i0 + q < n && v[q] >= f.m;
            }
            in_p = f.p_on ? __reduce_add_sync(0xffffffffu, in_p) : n;
            in_m = f.m_on ? __reduce_add_sync(0xffffffffu, in_m) : n;
            const int keep = max(1, min(min(n, in_p + 1), in_m));
            const bool inside = in_p < n || in_m < n;  // the kept set ends within the list
            if (tid == 0) sh.found = !guess || inside;
            if (guess && !inside) {
                if (tid == 0) *mass = whole;
            } else {
                // the kept ones by id
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    w[i0 + q] = v[q];
                    x[q] = i0 + q < keep ? (x[q] << 32) | (uint32_t)(i0 + q) : ~0ull;
                }
                sm_sort_warp(x, 0);
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 4; q++) v[q] = i0 + q < keep ? w[(uint32_t)x[q]] : 0.0;
                double before = sm_running_warp(v);
                const double total = __shfl_sync(0xffffffffu, before + ((v[0] + v[1]) + (v[2] + v[3])), 31), target = f.u * total;
                int at = -1;  // the lane's first place past the target, or else its last with any weight
                bool past = false;
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    before += v[q];
                    if (v[q] > 0.0 && !past) {
                        at = q;
                        past = before > target;
                    }
                }
                const unsigned hit = __ballot_sync(0xffffffffu, past), any = __ballot_sync(0xffffffffu, at >= 0);
                if (tid == (hit ? __ffs(hit) - 1 : 31 - __clz(any))) {
                    unsigned long long id = x[0];
                    double mine = v[0];
#pragma unroll
                    for (int q = 1; q < 4; q++)
                        if (q == at) {
                            id = x[q];
                            mine = v[q];
                        }
                    p.tokens[r] = (int32_t)(id >> 32);
                    if (p.logprobs) p.logprobs[r] = (float)log(mine / total);
                }
            }
        }
        __syncthreads();
        return sh.found != 0;
    }
    sm_sort(key, n);
    if (f.k_on) n = min(n, f.k);
    for (int i = tid; i < n; i += NT) w[i] = row.weight(sm_value(~(uint32_t)(key[i] >> 32)));
    __syncthreads();
    int keep = n;
    if (f.p_on || f.m_on) {
        if (f.p_on) sm_running<NT>(sh, w, run, n);
        if (f.p_on && !goal_known) goal = f.p * run[n - 1];
        int in_p = 0, in_m = 0;
        for (int i = tid; i < n; i += NT) {
            in_p += f.p_on && run[i] < goal;
            in_m += f.m_on && w[i] >= f.m;
        }
        if (f.p_on) in_p = row.block_sum_i(in_p);
        if (f.m_on) in_m = row.block_sum_i(in_m);
        const bool inside = (f.p_on && in_p < n) || (f.m_on && in_m < n);  // the kept set ends within the list
        if (guess && !inside) {
            *mass = run[n - 1];
            return false;
        }
        if (f.p_on) keep = min(keep, in_p + 1);
        if (f.m_on) keep = min(keep, in_m);
        keep = max(keep, 1);
    }
    // the kept ones by id, their weights' places beside
    for (int i = tid; i < keep; i += NT) {
        const unsigned long long k = key[i];
        key[i] = (k << 32) | (uint32_t)i;
    }
    __syncthreads();
    sm_sort(key, keep);
    double *wi = run;  // weights by id, then their running sums over the weights' old place
    for (int i = tid; i < keep; i += NT) wi[i] = w[(uint32_t)key[i]];
    __syncthreads();
    sm_running<NT>(sh, wi, w, keep);
    const double total = w[keep - 1], target = f.u * total;
    if (tid == 0) sh.found = kSmList;
    __syncthreads();
    int first = kSmList, last = -1;
    for (int i = tid; i < keep; i += NT) {
        if (first == kSmList && w[i] > target && wi[i] > 0.0) first = i;
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
    return true;
}

template <typename T, int NT>
__global__ void __launch_bounds__(NT, NT == 256 ? 4 : 1) sample_kernel(const SampleParams p) {
    extern __shared__ __align__(16) uint8_t smem_b[];
    __shared__ SampleShared sh;
    SampleRow<T, NT> row;
    row.sh = &sh;
    row.scratch = reinterpret_cast<double *>(smem_b);
    row.parity = 0;
    row.rank = cluster_rank();
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(row.cluster));
    if (row.cluster > 1) cluster_arrive();  // waited for before the first store into another block's shared memory
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int r = blockIdx.x / row.cluster;
    if (p.order) {
        // Of every NT rows those that may keep most come first: with top-p, and no top-k that the short way can take.  Such a row takes two
        // to four times as long as the others, and begun last it runs alone.
        const int i = r % NT, t = r - i + tid;
        bool longer = false;
        if (t < p.rows) {
            const int k = p.top_k ? p.top_k[t] : 0;
            longer = p.top_p[t] < 1.f && (k <= 0 || k > kSmGuess);
        }
        const unsigned those = __ballot_sync(0xffffffffu, longer);
        if (lane == 0) sh.warp_i[warp] = __popc(those);
        __syncthreads();
        int before = __popc(those & ((1u << lane) - 1)), all = 0;
#pragma unroll
        for (int w = 0; w < NT / 32; w++) {
            if (w < warp) before += sh.warp_i[w];
            all += sh.warp_i[w];
        }
        if (t < p.rows && longer == (i < all) && (longer ? before == i : tid - before == i - all)) sh.found = t;
        __syncthreads();
        r = sh.found;
    }
    row.base = row.rank * p.slice;
    row.n = max(0, min(p.slice, p.vocab - row.base));
    row.src = reinterpret_cast<const T *>(p.logits) + (long long)r * p.row_stride + row.base;

    // ---- the row's largest value
    float own[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};  // by place in the fours
    row.each([&](int, const float(&z)[4], int m) {
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (e < m) own[e] = fmaxf(own[e], z[e]);
    });
    if (tid < 16) sh.table[tid] = exp2(tid / 16.0);
    SampleFilters f;
    const float temp = p.temperature ? p.temperature[r] : 1.f;
    f.u = p.uniforms[r];
    if (f.u < 0.0) f.u = 0.0;  // (below nothing: the first token of any weight)
    f.k = p.top_k ? p.top_k[r] : 0;
    f.p = p.top_p ? p.top_p[r] : 1.f;
    f.m = p.min_p ? p.min_p[r] : 0.f;
    f.m_on = f.m > 0.0;
    if (f.m > 1.0) {  // no weight reaches it: the likeliest token stays alone, and is not held against it again
        f.k = 1;
        f.m_on = false;
    }
    f.k_on = f.k > 0 && f.k < p.vocab;
    f.p_on = !(f.p >= 1.0);
    if (f.p != f.p) f.p = 0.0;
    const float own_max = fmaxf(fmaxf(own[0], own[1]), fmaxf(own[2], own[3]));
    float mx = block_max(own_max, reinterpret_cast<float *>(sh.warp_d));
    float low_max = INFINITY;  // the lowest of the maxima, without values that stand for -inf
#pragma unroll
    for (int e = 0; e < 4; e++) low_max = own[e] > -1e4f ? fminf(low_max, own[e]) : low_max;
    low_max = -block_max(-low_max, reinterpret_cast<float *>(sh.warp_d));
    if (tid == 0) {
        sh.local[0] = mx;
        sh.local[1] = low_max;
        sh.sent = 0;
        sh.slots = 0;
    }
    if (tid < kSmMaxBuckets) sh.maxima.local[tid] = 0;
    if (row.cluster > 1) cluster_wait();  // every block of the cluster runs: its shared memory may be written
    {
        const auto buf = row.share(2);
        for (uint32_t k = 0; k < row.cluster; k++) {
            mx = fmaxf(mx, (float)buf[k][0]);
            low_max = fminf(low_max, (float)buf[k][1]);
        }
    }
    row.set_scale(mx, temp);
    if (mx == -INFINITY) {
        if (row.rank == 0 && tid == 0) {
            p.tokens[r] = -1;
            if (p.logprobs) p.logprobs[r] = -INFINITY;
        }
        return;
    }
    if (!(temp > 0.f)) {  // the largest logit, the lowest id of several
        int best = 0x7fffffff;
        if (own_max == mx)  // (few threads)
            row.each([&](int i, const float(&z)[4], int m) {
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (e < m && z[e] == mx) best = min(best, row.base + i + e);
            });
        best = __reduce_min_sync(0xffffffffu, best);
        if (lane == 0) sh.warp_i[warp] = best;
        __syncthreads();
        for (int w = 0; w < NT / 32; w++) best = min(best, sh.warp_i[w]);
        if (tid == 0) sh.local[0] = best;
        const auto buf = row.share(1);
        for (uint32_t k = 0; k < row.cluster; k++) best = min(best, (int)buf[k][0]);
        if (row.rank == 0 && tid == 0) {
            p.tokens[r] = best;
            if (p.logprobs) p.logprobs[r] = 0.f;
        }
        return;
    }

    const uint32_t key_top = sm_key(mx);
    struct {
        bool on;
        double total;
        SampleRange range;
    } known{};
    // ---- the middle way's steps: this block's counts, and the cluster's in the first block, behind the list's first two places
    int *steps = reinterpret_cast<int *>(row.scratch + 2 * kSmList), *all_steps = steps + kSmSteps;
    static_assert(2 * kSmSteps * 4 <= kSmList * 8, "the counts fit the list's third place");
    const float per_step = kSmSteps / (f.k_on ? fmaxf(mx - low_max, 1e-30f) : 16.f * temp);  // (by mass 16 T: e^-16 of the largest)
    auto step_of = [&](float z) { return (int)fminf((mx - z) * per_step, (float)(kSmSteps - 1)); };  // the last one is open below
    auto clear_steps = [&]() {
        for (int i = tid; i < 2 * kSmSteps; i += NT) steps[i] = 0;
        __syncthreads();
    };
    bool counted = false;
    // ---- the short way
    const int most = min(kSmGuess, 2 * NT * (int)row.cluster);  // (at most half of the maxima: the bound stays high)
    if (p.vocab > kSmList && (f.k_on ? f.k <= most : f.p_on || f.m_on)) {
        uint32_t lo = key_top;
        bool bound = false;
        if (!f.k_on && !f.p_on) {
            // w >= m is z >= max + T ln m; a little below that, whatever the roundings: the list's own test is the exact one
            const double low = row.top + (double)temp * (log(f.m) - 1e-6);
            if (mx < INFINITY) lo = max(kSmKeyLowest, sm_key(__double2float_rd(low) + 0.f));
            bound = true;
        } else {
            // equal steps from the largest value down to the lowest of the maxima
            const float per = kSmMaxBuckets / (low_max < mx ? mx - low_max : 32.f);
#pragma unroll
            for (int e = 0; e < 4; e++) atomicAdd(&sh.maxima.local[(int)fminf((mx - own[e]) * per, (float)(kSmMaxBuckets - 1))], 1);
            __syncthreads();
            for (int i = tid; i < kSmMaxBuckets * (int)row.cluster; i += NT) {
                const int to = i / kSmMaxBuckets, b = i - to * kSmMaxBuckets;
                asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(mapa_u32(smem_u32(&sh.maxima.all[row.rank][b]), to)), "r"(sh.maxima.local[b]) : "memory");
            }
            if (row.cluster == 1) __syncthreads();
            else cluster_sync_all();
            int a = 0, b = 0;  // buckets 2 lane, 2 lane + 1
            for (uint32_t k = 0; k < row.cluster; k++) {
                a += sh.maxima.all[k][2 * lane];
                b += sh.maxima.all[k][2 * lane + 1];
            }
            int run = a + b;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += v;
            }
            const int want = f.k_on ? f.k : min(kSmNucleus, most);
            const unsigned at = __ballot_sync(0xffffffffu, run >= want);
            const int l = at ? __ffs(at) - 1 : 31, before = __shfl_sync(0xffffffffu, run - a - b, l), first = __shfl_sync(0xffffffffu, a, l);
            const int j = 2 * l + (before + first < want);
            // the bucket's lower end, and a little below that for the roundings; the last bucket is open: no bound
            bound = at && j < kSmMaxBuckets - 1 && mx < INFINITY;
            if (bound) lo = sm_key(mx - (j + 1.01f) / per + 0.f);
        }
        if (bound) {
            // what lies at or above it to the first block, a part of the list's second place for each; with top-p alone also the total
            const int part = kSmList / (int)row.cluster;
            const uint32_t list = mapa_u32(smem_u32(row.scratch + kSmList + row.rank * part), 0);
            const bool all = f.p_on && !f.k_on;
            double total = 0.0, listed = 0.0;
            const float lo_value = sm_value(lo);  // (the cleaned values are in the order of their patterns)
            auto pick = [&](int i, const float(&z)[4], int m) {
                if (m == 4 ? fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])) < lo_value : z[0] < lo_value) return;
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (e < m && z[e] >= lo_value) {
                        const int at = atomicAdd(&sh.sent, 1);
                        if (at < part) row.send(list + 8 * at, sm_key(z[e]), i + e);
                    }
            };
            if (all) {
                clear_steps();
                counted = true;
                row.each([&](int i, const float(&z)[4], int m) {
                    double w[4];
#pragma unroll
                    for (int e = 0; e < 4; e++) w[e] = e < m ? row.weight(z[e]) : 0.0;
                    total += (w[0] + w[1]) + (w[2] + w[3]);
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (e < m) {
                            atomicAdd(&steps[step_of(z[e])], 1);
                            listed += z[e] >= lo_value ? w[e] : 0.0;
                        }
                    pick(i, z, m);
                });
            } else
                row.each(pick);
            if (all) {
                total = row.block_sum_d(total);
                listed = row.block_sum_d(listed);
            }
            __syncthreads();
            if (tid == 0) {
                sh.local[0] = sh.sent;
                sh.local[1] = total;
                sh.local[2] = listed;
            }
            const auto buf = row.share(3);
            bool fits = true;
            total = listed = 0.0;
            int n = 0, from[kSmMaxCluster + 1];
#pragma unroll
            for (int k = 0; k < kSmMaxCluster; k++) {
                from[k] = n;
                if (k < (int)row.cluster) {
                    n += (int)buf[k][0];
                    total += buf[k][1];
                    listed += buf[k][2];
                    fits = fits && buf[k][0] <= part;
                }
            }
            from[kSmMaxCluster] = n;
            known.total = total;
            if (all && !f.m_on && listed < f.p * total * (1.0 - 1e-9)) {
                // top-p reaches further down for certain: no need to sort the list (7 us); the search begins below it
                known.range = SampleRange{kSmKeyLowest, lo - 1, n, listed, 0};
                known.on = lo > kSmKeyLowest;
            } else if (fits && (!f.k_on || n >= f.k)) {  // (n < k: roundings wider than the buckets)
                bool done = true;
                double mass = 0.0;
                if (row.rank == 0) {
                    unsigned long long *key = reinterpret_cast<unsigned long long *>(row.scratch), *raw = key + kSmList;
#pragma unroll
                    for (int k = 0; k < kSmMaxCluster; k++)
                        for (int i = tid; i < from[k + 1] - from[k]; i += NT) key[from[k] + i] = raw[k * part + i];
                    __syncthreads();
                    // (the list's sums would overwrite the counts: they wait in registers)
                    constexpr int KEEP = kSmSteps / NT;
                    int kept[KEEP];
#pragma unroll
                    for (int k = 0; k < KEEP; k++) kept[k] = all ? steps[k * NT + tid] : 0;
                    done = sm_finish_list(row, p, r, f, n, all, f.p * total, all, &mass);
                    if (!done) {
                        __syncthreads();
#pragma unroll
                        for (int k = 0; k < KEEP; k++) {
                            steps[k * NT + tid] = kept[k];
                            all_steps[k * NT + tid] = 0;
                        }
                    }
                }
                if (!all) return;  // (the list holds all that top-k, or min-p, keeps)
                if (tid == 0) {
                    sh.local[0] = done;
                    sh.local[1] = mass;
                }
                const auto verdict = row.share(2);
                if (verdict[0][0] != 0.0) return;
                // top-p reaches further down
                known.range = SampleRange{kSmKeyLowest, lo - 1, n, verdict[0][1], 0};
                known.on = lo > kSmKeyLowest;
            }
        }
    }

    // ---- the long way: the borders
    SampleBorder border{0, 0, true};  // everything
    bool bounded = false;
    auto narrow = [&](auto mass, double &goal, bool find_goal, const SampleBorder *limit, SampleRange &range, SampleBorder &found) -> int {
        // 1: the values from range.lo up fit the list; 2: `found` is the border
        constexpr bool MASS = decltype(mass)::value;
        constexpr int NB = MASS ? kSmMassBuckets : kSmBuckets, BITS = MASS ? 3 : 4;
        // The first window reaches 8 units below the largest value (counts), 8 T (masses): about where the border lies in a
        // language model's logits.  A border below it is looked for in a window 16 times as wide, then in all that is left.
        float reach = MASS ? 8.f * temp : 8.f;
        for (int it = 0; it < 16; it++) {  // (two rounds of windows, then eleven at most: a round takes three of 32 bits, or four)
            uint32_t span = range.hi - range.lo;
            if (range.lo == kSmKeyLowest && it < 2) {
                const uint32_t low = sm_key(sm_value(range.hi) - reach);  // (not a number: above, the full range)
                if (low < range.hi && low > range.lo) span = range.hi - low;
                reach *= 16.f;
            }
            const int shift = 32 - BITS - __clz(span | (NB - 1));  // the buckets cover span + 1 patterns
            const bool exact = sm_round<MASS>(row, range, shift, goal, find_goal && it == 0, f.p, limit, found);
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
                        for (int i = tid; i < n; i += NT) w[i] = row.weight(sm_value(~(uint32_t)(key[i] >> 32)));
                        __syncthreads();
                        sm_running<NT>(sh, w, run, n);
                        int before = 0;
                        for (int i = tid; i < n; i += NT) before += range.above_w + run[i] < goal;
                        at = row.block_sum_i(before);
                        if (!ends) at = min(at, n - 1);
                    } else {
                        at = (int)(goal - (double)range.above_n) - 1;
                    }
                    uint32_t tau;
                    int same = 0, more = 0;  // ties up to the border, and beyond it
                    if (at < n) {
                        tau = ~(uint32_t)(key[at] >> 32);
                        for (int i = tid; i < n; i += NT) {
                            const bool tie = (uint32_t)(key[i] >> 32) == ~tau;
                            same += tie && i <= at;
                            more += tie && i > at;
                        }
                        same = row.block_sum_i(same);
                        more = row.block_sum_i(more);
                    } else {
                        tau = limit->tau;
                        same = sm_ties(goal - range.above_w - (n > 0 ? run[n - 1] : 0.0), row.weight(sm_value(tau)), limit->ties);
                        more = same < limit->ties || !limit->whole;
                    }
                    if (tid == 0) {
                        sh.local[0] = tau;
                        sh.local[1] = same;
                        sh.local[2] = more;
                    }
                }
                const auto buf = row.share(3);
                found = SampleBorder{(uint32_t)buf[0][0], (int)buf[0][1], buf[0][2] == 0.0};
                return 2;
            }
        }
        found = SampleBorder{range.hi, 1, false};
        return 2;
    };

    // The middle way: false where the steps cannot tell, or told wrongly.
    auto bracket = [&](auto mass, double goal, SampleBorder &found) -> bool {
        constexpr bool MASS = decltype(mass)::value;
        row.share(1);  // (every block's counts are there, the first block's sums are clear)
        const uint32_t to = mapa_u32(smem_u32(all_steps), 0);
        for (int i = tid; i < kSmSteps; i += NT)
            if (steps[i]) asm volatile("red.shared::cluster.add.u32 [%0], %1;" ::"r"(to + 4 * i), "r"(steps[i]) : "memory");
        if (row.cluster == 1) __syncthreads();
        else cluster_sync_all();
        if (row.rank == 0) {
            // running sums over the steps, in the list's first two places (one warp alone, 32 steps a time, took 17 us of a row's 115)
            double *each = row.scratch, *run = row.scratch + kSmList;
            double base = 0.0;
            int listed = 0, from = 0;  // the first step behind the short way's list
            if (MASS && known.on) {
                // the list's own mass is exact: a few heavy values in the middle of their steps would be half a step off
                listed = step_of(sm_value(known.range.hi)) + 1;
                int seen = 0;
                for (int s = tid; s < listed; s += NT) seen += all_steps[s];
                seen = row.block_sum_i(seen);
                base = known.range.above_w + (double)(seen - known.range.above_n) * row.weight(mx - (listed - 0.5f) / per_step);
                from = base >= goal ? listed - 1 : listed;
            }
            for (int s = tid; s < kSmSteps; s += NT) {
                const int c = s >= listed ? all_steps[s] : 0;
                each[s] = MASS ? c * row.weight(mx - (s + 0.5f) / per_step) : (double)c;
            }
            __syncthreads();
            sm_running<NT>(sh, each, run, kSmSteps);
            if (tid == 0) sh.found = kSmSteps;
            __syncthreads();
            int first = kSmSteps;
            for (int s = tid; s < kSmSteps; s += NT)
                if (first == kSmSteps && s >= from && base + run[s] >= goal) first = s;
            first = __reduce_min_sync(0xffffffffu, first);
            if (lane == 0) atomicMin(&sh.found, first);
            __syncthreads();
            if (tid == 0) {
                const int at = sh.found;
                int a = at, b = at;
                // by mass the border may lie in a neighbour: both, where they fit
                if (MASS && at > 0 && at < kSmSteps - 2 && all_steps[at - 1] + all_steps[at] + all_steps[at + 1] <= kSmList) {
                    a--;
                    b++;
                }
                sh.local[0] = at < kSmSteps - 1 && all_steps[at] <= kSmList ? a : -1;
                sh.local[1] = b;
            }
        }
        const auto where = row.share(2);
        const int a = (int)where[0][0], b = (int)where[0][1];
        if (a < 0) return false;
        const uint32_t slots = mapa_u32(smem_u32(&sh.slots), 0), list = mapa_u32(smem_u32(row.scratch), 0);
        double above = 0.0;
        int above_n = 0;
        row.each([&](int i, const float(&z)[4], int m) {
            int s[4];
            bool any = false;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                s[e] = e < m ? step_of(z[e]) : kSmSteps;
                any = any || s[e] < a;
                above_n += s[e] < a;
            }
            if (MASS && any) {
                double w[4];
#pragma unroll
                for (int e = 0; e < 4; e++) w[e] = s[e] < a ? row.weight(z[e]) : 0.0;
                above += (w[0] + w[1]) + (w[2] + w[3]);
            }
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (s[e] >= a && s[e] <= b) {
                    unsigned slot;
                    asm volatile("atom.shared::cluster.add.u32 %0, [%1], 1;" : "=r"(slot) : "r"(slots) : "memory");
                    if (slot < kSmList) row.send(list + 8 * slot, sm_key(z[e]), i + e);
                }
        });
        if (MASS) above = row.block_sum_d(above);
        above_n = row.block_sum_i(above_n);
        __syncthreads();
        if (tid == 0) {
            sh.local[0] = above;
            sh.local[1] = above_n;
        }
        const auto buf = row.share(2);
        above = 0.0;
        long long before_n = 0;
        for (uint32_t k = 0; k < row.cluster; k++) {
            above += buf[k][0];
            before_n += (long long)buf[k][1];
        }
        if (row.rank == 0) {
            const int n = min((int)sh.slots, kSmList);
            unsigned long long *key = reinterpret_cast<unsigned long long *>(row.scratch);
            double *w = row.scratch + kSmList, *run = row.scratch + 2 * kSmList;
            sm_sort(key, n);
            int at;  // number of the list's values above the border
            bool good;
            if (MASS) {
                for (int i = tid; i < n; i += NT) w[i] = row.weight(sm_value(~(uint32_t)(key[i] >> 32)));
                __syncthreads();
                sm_running<NT>(sh, w, run, n);
                int before = 0;
                for (int i = tid; i < n; i += NT) before += above + run[i] < goal;
                at = row.block_sum_i(before);
                good = at < n && (above < goal || before_n == 0);
            } else {
                at = (int)(goal - (double)before_n) - 1;
                good = at >= 0 && at < n;
            }
            int same = 0, more = 0;  // ties up to the border, and beyond it
            uint32_t tau = 0;
            if (good) {
                tau = ~(uint32_t)(key[at] >> 32);
                for (int i = tid; i < n; i += NT) {
                    const bool tie = (uint32_t)(key[i] >> 32) == ~tau;
                    same += tie && i <= at;
                    more += tie && i > at;
                }
            }
            same = row.block_sum_i(same);
            more = row.block_sum_i(more);
            __syncthreads();
            if (tid == 0) {
                sh.local[0] = good;
                sh.local[1] = tau;
                sh.local[2] = same;
                sh.local[3] = more;
            }
        }
        const auto border_at = row.share(4);
        if (border_at[0][0] == 0.0) return false;
        found = SampleBorder{(uint32_t)border_at[0][1], (int)border_at[0][2], border_at[0][3] == 0.0};
        return true;
    };

    SampleRange range{kSmKeyLowest, key_top, 0, 0.0, p.vocab};
    bool listed = p.vocab <= kSmList, goal_known = false;
    double goal = 0.0;
    if (!listed && f.k_on) {
        goal = f.k;
        if (f.k > most && low_max < mx && mx < INFINITY) {  // (else the short way has looked at them, and found too many)
            clear_steps();
            row.each([&](int, const float(&z)[4], int m) {
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (e < m) atomicAdd(&steps[step_of(z[e])], 1);
            });
            bounded = bracket(std::false_type{}, goal, border);
        }
        if (!bounded) {
            listed = narrow(std::false_type{}, goal, false, nullptr, range, border) == 1;
            bounded = !listed;
        }
    }
    if (!listed && f.p_on) {
        SampleBorder other;
        range = known.on ? known.range : SampleRange{kSmKeyLowest, key_top, 0, 0.0, p.vocab};
        goal = f.p * known.total;
        if (counted && mx < INFINITY && bracket(std::true_type{}, goal, other)) {
            border = other;
            bounded = true;
        } else {
            const int how = narrow(std::true_type{}, goal, !known.on, bounded ? &border : nullptr, range, other);
            goal_known = true;
            if (how == 1) {
                listed = true;
            } else {
                if (bounded && other.tau == border.tau) other.ties = min(other.ties, border.ties);
                border = other;  // (never below top-k's: masses were counted inside it)
                bounded = true;
            }
        }
    }
    if (listed) {
        const int n = sm_gather(row, range.lo, key_top);
        if (row.rank == 0) sm_finish_list(row, p, r, f, n, goal_known, goal, false, nullptr);
        return;
    }

    // ---- many values are kept: sums in the order of ids, a warp per run of kSmRun of them, eight neighbours a lane
    const int runs = (row.n + kSmRun - 1) / kSmRun;
    const bool ranked = bounded && !border.whole;  // some of the border's ties stay out: their order counts
    const bool vectors = (reinterpret_cast<uintptr_t>(row.src) & 15) == 0;
    auto values = [&](int q, float(&z)[8]) {
        const int i = q * kSmRun + lane * 8;
        if (vectors && i + 8 <= row.n) {
            load8(row.src + i, z);
#pragma unroll
            for (int e = 0; e < 8; e++) z[e] = row.clean(z[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++) z[e] = i + e < row.n ? row.at(i + e) : -INFINITY;  // (behind the last: no weight)
        }
    };
    auto count_ties = [&](const float(&z)[8], int q) {
        int c = 0;
#pragma unroll
        for (int e = 0; e < 8; e++) c += sm_key(z[e]) == border.tau && q * kSmRun + lane * 8 + e < row.n;
        return c;
    };
    // the kept weights of a lane's eight values; `seen`: the border's ties before run q
    auto weigh = [&](int q, int seen, double(&w)[8]) {
        float z[8];
        values(q, z);
#pragma unroll
        for (int e = 0; e < 8; e++) w[e] = row.weight(z[e]);
        if (!bounded && !f.m_on) return;
        if (ranked) {
            const int mine = count_ties(z, q);
            int run = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += v;
            }
            seen += run - mine;
        }
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const uint32_t k = sm_key(z[e]);
            bool in = !bounded || k > border.tau;
            if (bounded && k == border.tau) in = border.whole || seen++ < border.ties;
            if (!in || (f.m_on && w[e] < f.m)) w[e] = 0.0;
        }
    };
    __syncthreads();
    int ties_before = 0;  // of the blocks before
    if (ranked) {
        for (int q = warp; q < runs; q += NT / 32) {
            float z[8];
            values(q, z);
            const int c = __reduce_add_sync(0xffffffffu, count_ties(z, q));
            if (lane == 0) sh.runs.ties[q] = c;
        }
        __syncthreads();
        if (warp == 0) {  // running sums, each without its own
            int base = 0;
            for (int q0 = 0; q0 < runs; q0 += 32) {
                const int mine = q0 + lane < runs ? sh.runs.ties[q0 + lane] : 0;
                int run = mine;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int v = __shfl_up_sync(0xffffffffu, run, o);
                    if (lane >= o) run += v;
                }
                if (q0 + lane < runs) sh.runs.ties[q0 + lane] = base + run - mine;
                base += __shfl_sync(0xffffffffu, run, 31);
            }
            if (lane == 0) sh.local[0] = base;
        }
        const auto buf = row.share(1);
        for (uint32_t k = 0; k < row.rank; k++) ties_before += (int)buf[k][0];
    }
    for (int q = warp; q < runs; q += NT / 32) {
        double w[8];
        weigh(q, ranked ? ties_before + sh.runs.ties[q] : 0, w);
        double mine = ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
        if (lane == 0) sh.runs.mass[q] = mine;
    }
    __syncthreads();
    if (warp == 0) {  // running sums of the runs
        double base = 0.0;
        for (int q0 = 0; q0 < runs; q0 += 32) {
            double run = q0 + lane < runs ? sh.runs.mass[q0 + lane] : 0.0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double v = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += v;
            }
            if (q0 + lane < runs) sh.runs.sums[q0 + lane] = base + run;
            base += __shfl_sync(0xffffffffu, run, 31);
        }
        if (lane == 0) sh.local[0] = base;
    }
    const auto sums = row.share(1);
    double total = 0.0, base = 0.0, upto = 0.0;
    for (uint32_t k = 0; k < row.cluster; k++) total += sums[k][0];
    const double target = f.u * total;
    // the block, then the run that the target lies in; the last with any mass takes what rounding leaves over
    int owner = -1, last = 0;
    for (uint32_t k = 0; k < row.cluster && owner < 0; k++) {
        const bool hit = upto + sums[k][0] > target;
        if (hit || sums[k][0] > 0.0) {
            last = k;
            base = upto;
        }
        if (hit) owner = k;
        upto += sums[k][0];
    }
    if (last != (int)row.rank || warp != 0) return;
    int q = -1, q_last = 0;
    for (int q0 = 0; q0 < runs && q < 0; q0 += 32) {
        const int mine = q0 + lane;
        const bool some = mine < runs && sh.runs.mass[mine] > 0.0;  // (the running sums may rise by a rounding where there is nothing)
        const unsigned hit = __ballot_sync(0xffffffffu, some && base + sh.runs.sums[mine] > target), any = __ballot_sync(0xffffffffu, some);
        if (any) q_last = q0 + 31 - __clz(any);
        if (hit) q = q0 + __ffs(hit) - 1;
    }
    if (q < 0) q = q_last;
    if (q > 0) base += sh.runs.sums[q - 1];
    double w[8];
    weigh(q, ranked ? ties_before + sh.runs.ties[q] : 0, w);
    const double mine = ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
    double run = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double v = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += v;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, mine > 0.0 && base + run > target), any = __ballot_sync(0xffffffffu, mine > 0.0);
    if (!any || lane != (hit ? __ffs(hit) - 1 : 31 - __clz(any))) return;  // (any: the run has mass)
    run += base - mine;
    int at = -1;
    double share_w = 0.0;
    bool past = false;
#pragma unroll
    for (int e = 0; e < 8; e++) {
        run += w[e];
        if (w[e] > 0.0 && !past) {
            at = e;
            share_w = w[e];
            past = run > target;
        }
    }
    p.tokens[r] = row.base + q * kSmRun + lane * 8 + at;
    if (p.logprobs) p.logprobs[r] = (float)log(share_w / total);
}

}  // namespace dbt

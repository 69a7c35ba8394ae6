// sample.hip -- sampling from logits: temperature, top-k, top-p and min-p, then
// the inverse-CDF draw with a given uniform, and the filtered distribution
// where it is asked for (the p and q that the stochastic accept rule reads,
// Sec. 2.1; the draft's own tokens).
//
// Mathematics.  For a row x with maximum m, temperature 1 / c' (c = c' log2 e):
//   w_v = 2^((x_v - m) c) in double precision (fp32's error of 1e-7 moves the
//   edges of 128 K bins past a 24-bit uniform once in some hundred rows).
//   Order the row by value, ties by index: key(v) = (order-preserving image of
//   x_v, inverted index), 64 bits, all different.  Each filter keeps a prefix of
//   that order: top-k the first k; top-p those before which less than top_p of
//   the mass that top-k left lies; min-p those with w_v >= min_p.  So a row is
//   decided by one threshold key t and the mass at and above it:
//   p_v = w_v [key(v) >= t] / mass.  The draw is the smallest v whose running
//   mass, in index order, exceeds u times the whole.
// Masses that are summed in no fixed order (histograms, by LDS atomics) are
// integers, in units of 2^-50 (2^-43 over a whole row): their sums do not depend
// on the order.
//
// Work.  Workgroup (chunk, row) of 1024 threads reads 8192 entries, 8 a thread.
//   * Rows with a small top-k (kListK): it counts its entries into 256 bins of
//     1/8 below its maximum, finds the bin that holds its k-th largest and
//     writes the entries down to it, some 1/8 more than k, to the workspace, as
//     keys.  The row's last workgroup has every candidate: it finds the k-th by
//     radix steps in LDS, sorts the k, and applies the other filters, the draw
//     and the probabilities to them.  The row is read once and nothing else of
//     V entries is touched but the zeros of the distribution.
//   * Other rows: it sums its weights, and where a filter is on, also by bin.
//     The row's last workgroup finds the bin where top-p (or a large top-k)
//     ends, gathers that bin's entries from the row (out of L2), and narrows it
//     down in LDS to the one entry where the count or mass is reached.  Where
//     distributions are asked for, a second launch writes them (and draws).
//   Whatever the bins do not resolve (values further apart than 32, thousands of
//   equal ones, huge magnitudes) is narrowed down by passes over the row, with
//   2048 buckets of the key range each.
#include "mad_device.h"
#include "mad_internal.h"

namespace mad {

constexpr int kThreads = 1024, kRun = kSampleChunk / kThreads;   // entries of a thread: consecutive
constexpr int kBins = 256, kBuckets = 2048, kList = 4096, kFinal = 64;
constexpr double kBinUnit = 0x1p-50, kRowUnit = 0x1p-43;   // 8192 and 2^20 weights of at most 1 fit 63 bits

// 2^y for y <= 0 (y > -1000): the Taylor series of 2^f, |f| <= 1/2, to 12th order: below 2e-16 relative
__device__ __forceinline__ double exp2_neg(double y) {
    const double n = rint(y), f = (y - n) * 0.6931471805599453;
    double p = 1.0 / 479001600.0;
    p = fma(p, f, 1.0 / 39916800.0);
    p = fma(p, f, 1.0 / 3628800.0);
    p = fma(p, f, 1.0 / 362880.0);
    p = fma(p, f, 1.0 / 40320.0);
    p = fma(p, f, 1.0 / 5040.0);
    p = fma(p, f, 1.0 / 720.0);
    p = fma(p, f, 1.0 / 120.0);
    p = fma(p, f, 1.0 / 24.0);
    p = fma(p, f, 1.0 / 6.0);
    p = fma(p, f, 0.5);
    p = fma(p, f, 1.0);
    p = fma(p, f, 1.0);
    return ldexp(p, (int)n);
}
// weight of x against the maximum m (+inf against +inf: 1)
__device__ __forceinline__ double weight(float x, float m, double c) {
    const double y = ((double)x - (double)m) * c;
    const double w = exp2_neg(y > -1000.0 ? y : -1000.0);
    return x == m ? 1.0 : y > -1000.0 ? w : 0.0;
}
// the value that a key holds
__device__ __forceinline__ float key_value(uint64_t k) {
    const uint32_t o = (uint32_t)(k >> 32);
    return __uint_as_float((o & 0x80000000u) ? o ^ 0x80000000u : ~o);
}

// a thread's run of kRun entries from entry e on (unaligned 16-byte loads; -inf past V)
__device__ __forceinline__ void load_run(const float *row, int e, int V, float (&x)[kRun]) {
    if (e + kRun <= V) {
        __builtin_memcpy(x, row + e, kRun * 4);
    } else {
        #pragma unroll
        for (int i = 0; i < kRun; ++i) x[i] = e + i < V ? row[e + i] : -INFINITY;
    }
}
__device__ __forceinline__ void load_run(const bf16_t *row, int e, int V, float (&x)[kRun]) {
    if (e + kRun <= V) {
        uint4 u;
        __builtin_memcpy(&u, row + e, kRun * 2);
        unpack16(u, x, bf16_t());
    } else {
        #pragma unroll
        for (int i = 0; i < kRun; ++i) x[i] = e + i < V ? bf16_to_f32(row[e + i].bits) : -INFINITY;
    }
}
// Zeros at device scope: the row's last workgroup, perhaps behind another L2, writes over some of them in this launch
// (at device scope too).
__device__ __forceinline__ void zero_run(float *row, int e, int V) {
    if (e + kRun <= V) {
        #pragma unroll
        for (int i = 0; i < kRun; i += 4) store_agent4(row + e + i, f32x4_agent{0.f, 0.f, 0.f, 0.f});
    } else {
        #pragma unroll
        for (int i = 0; i < kRun; ++i)
            if (e + i < V) store_agent(row + e + i, 0.f);
    }
}
__device__ __forceinline__ void store_run(float *row, int e, int V, const float (&x)[kRun]) {
    if (e + kRun <= V) {
        __builtin_memcpy(row + e, x, kRun * 4);
    } else {
        #pragma unroll
        for (int i = 0; i < kRun; ++i)
            if (e + i < V) row[e + i] = x[i];
    }
}

__device__ __forceinline__ void put64(void *p, uint64_t v) {
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t get64(const void *p) { return load_agent64(reinterpret_cast<const uint64_t *>(p)); }
__device__ __forceinline__ uint64_t f64_bits(double v) { return (uint64_t)__double_as_longlong(v); }
__device__ __forceinline__ double bits_f64(uint64_t v) { return __longlong_as_double((long long)v); }

// A chunk's record in the workspace: 32 bytes of header, then the candidates' keys, or the bins' masses and counts.
//   header: maximum and flags | first value that is certainly a candidate, candidates | mass of the chunk | -
struct ChunkHead {
    float max;
    uint32_t flags;   // 1: a NaN; 2: no bins; 4: candidates left out below `edge`
    float edge;
    uint32_t n;
    double mass;
};
constexpr int kHead = 32, kRecord = kHead + kBins * 12;
static_assert(kRecord <= kSampleRecord && kHead + kEmit * 8 <= kSampleRecord, "chunk record");

struct SampleLds {
    uint64_t list[kList];       // gathered keys
    uint64_t mass[kBuckets];    // histogram: masses (integers), or doubles' bits
    uint32_t cnt[kBuckets];
    double c_mass[kSampleMaxChunks];    // per chunk: mass against the row's maximum, kept mass
    float c_max[kSampleMaxChunks], c_edge[kSampleMaxChunks];
    uint32_t c_flags[kSampleMaxChunks], c_n[kSampleMaxChunks];
    double part[16], part2[16];   // one per wave
    double res[4];
    uint64_t key[4];
    int num[4];
};
static_assert(sizeof(SampleLds) <= 64 * 1024, "static LDS");

// sum over the workgroup, the same in every thread (fixed order); `part`: 16 doubles of LDS, free again behind the
// next barrier
__device__ __forceinline__ double block_sum(double v, double *part) {
    v = __longlong_as_double((long long)wave_fold_u64(f64_bits(v), add_f64_bits));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = part[0];
    #pragma unroll
    for (int k = 1; k < kThreads / 64; ++k) s += part[k];
    return s;
}
// exclusive prefix sum over the workgroup's threads
__device__ __forceinline__ double block_scan(double v, double *part) {
    const double incl = wave_scan_f64(v);
    if ((threadIdx.x & 63) == 63) part[threadIdx.x >> 6] = incl;
    __syncthreads();
    double s = incl - v;
    for (int k = 0; k < (int)(threadIdx.x >> 6); ++k) s += part[k];
    return s;
}

// One row, by one workgroup.
template <typename T> struct Row {
    const T *x;
    int V, n_chunks;
    float m;       // maximum
    double c;      // log2 e / temperature
    SampleLds *s;

    // f(value, index) for every entry; four chunks in flight
    template <typename F> __device__ __forceinline__ void each(F f) const {
        constexpr int U = 4;
        const int e0 = threadIdx.x * kRun;
        for (int c0 = 0; c0 < n_chunks; c0 += U) {
            float v[U][kRun];
            #pragma unroll
            for (int k = 0; k < U; ++k) load_run(x, (c0 + k) * kSampleChunk + e0, V, v[k]);
            #pragma unroll
            for (int k = 0; k < U; ++k) {
                const int e = (c0 + k) * kSampleChunk + e0;
                #pragma unroll
                for (int i = 0; i < kRun; ++i)
                    if (e + i < V) f(v[k][i], e + i);
            }
        }
    }
};

// Where a count or a mass is reached: the keys in [lo, hi] hold the place; `above`: what lies above hi.
struct Range {
    uint64_t lo, hi;
    double mass, count;   // above hi
};

// Finds in the histogram mass/cnt (nb buckets, highest keys last; masses as doubles' bits) the first bucket from the
// top with which `target` of the measure is reached on top of what r holds, or the last that is not empty.  Returns
// it (-1: all are empty) and adds what lies above it to r.  *n: its entries.
__device__ __forceinline__ int crossing(SampleLds &s, int nb, bool by_count, double target, Range &r, int *n) {
    const int tid = threadIdx.x, b0 = nb - 1 - 2 * tid, b1 = b0 - 1;   // two buckets a thread, from the top
    const double m0 = b0 >= 0 ? bits_f64(s.mass[b0]) : 0.0, m1 = b1 >= 0 ? bits_f64(s.mass[b1]) : 0.0;
    const double n0 = b0 >= 0 ? (double)s.cnt[b0] : 0.0, n1 = b1 >= 0 ? (double)s.cnt[b1] : 0.0;
    if (tid == 0) s.num[0] = 0x7fffffff, s.num[1] = -1;
    const double em = block_scan(m0 + m1, s.part), en = block_scan(n0 + n1, s.part2);
    const double before = by_count ? r.count + en : r.mass + em, v0 = by_count ? n0 : m0, v1 = by_count ? n1 : m1;
    int at = 0x7fffffff, some = -1;
    if (n1 > 0.0) some = 2 * tid + 1;
    else if (n0 > 0.0) some = 2 * tid;
    if (n1 > 0.0 && before + v0 + v1 >= target) at = 2 * tid + 1;
    if (n0 > 0.0 && before + v0 >= target) at = 2 * tid;
    if (at != 0x7fffffff) atomicMin(&s.num[0], at);
    if (some >= 0) atomicMax(&s.num[1], some);
    __syncthreads();
    const int pos = s.num[0] != 0x7fffffff ? s.num[0] : s.num[1];
    if (pos >= 0 && (pos >> 1) == tid) {
        const bool second = pos & 1;
        s.res[0] = em + (second ? m0 : 0.0);
        s.res[1] = en + (second ? n0 : 0.0);
        s.num[2] = (int)(second ? n1 : n0);
    }
    __syncthreads();
    if (pos < 0) return -1;
    r.mass += s.res[0];
    r.count += s.res[1];
    *n = s.num[2];
    const int b = nb - 1 - pos;
    __syncthreads();
    return b;
}

// The entry at which `target` is reached, among the keys of r (n of them in the list if in_list): its key; r.mass and
// r.count become what lies at and above it.  The row has at least one entry in the range.
template <typename T>
__device__ uint64_t select(const Row<T> &row, Range &r, bool by_count, double target, int n, bool in_list) {
    SampleLds &s = *row.s;
    const int tid = threadIdx.x;
    for (;;) {
        if (!in_list) {   // into the list, if it takes them
            if (tid == 0) s.num[3] = 0;
            __syncthreads();
            row.each([&](float x, int i) {
                const uint64_t k = argmax_key(x, i);
                if (k >= r.lo && k <= r.hi) {
                    const int p = atomicAdd(&s.num[3], 1);
                    if (p < kList) s.list[p] = k;
                }
            });
            __syncthreads();
            n = s.num[3];
            in_list = n <= kList;
            __syncthreads();
        }
        // The keys of the list that are still in the range; few enough are put in order by one wave.
        if (in_list && n <= kFinal) break;
        int sh = 64 - __clzll((long long)(r.hi - r.lo)) - 11;   // 2048 buckets (a range of one key holds one entry)
        if (sh < 0) sh = 0;
        for (int b = tid; b < kBuckets; b += kThreads) s.mass[b] = 0, s.cnt[b] = 0;
        __syncthreads();
        const double unit = in_list ? kBinUnit : kRowUnit, per = 1.0 / unit;
        auto count = [&](uint64_t k, float x) {
            if (k >= r.lo && k <= r.hi) {
                const int b = (int)((k - r.lo) >> sh);
                atomicAdd(&s.cnt[b], 1u);
                atomicAdd((unsigned long long *)&s.mass[b], (unsigned long long)(weight(x, row.m, row.c) * per + 0.5));
            }
        };
        if (in_list) {
            const int all = s.num[3];
            for (int i = tid; i < all; i += kThreads) count(s.list[i], key_value(s.list[i]));
        } else {
            row.each([&](float x, int i) { count(argmax_key(x, i), x); });
        }
        __syncthreads();
        for (int b = tid; b < kBuckets; b += kThreads) s.mass[b] = f64_bits((double)s.mass[b] * unit);
        __syncthreads();
        const int b = crossing(s, kBuckets, by_count, target, r, &n);
        const uint64_t lo = r.lo + ((uint64_t)b << sh);
        r.hi = min(r.hi, lo + (((uint64_t)1 << sh) - 1));
        r.lo = lo;
    }
    // at most 64: wave 0 orders them by rank and sums in order
    if (tid == 0) s.num[2] = 0;
    __syncthreads();
    const int all = s.num[3];
    for (int i = tid; i < all; i += kThreads)
        if (s.list[i] >= r.lo && s.list[i] <= r.hi) s.mass[atomicAdd(&s.num[2], 1)] = s.list[i];
    __syncthreads();
    const int f = s.num[2];
    if (tid < f) {
        const uint64_t mine = s.mass[tid];
        int rank = 0;
        for (int j = 0; j < f; ++j) rank += s.mass[j] > mine ? 1 : 0;
        s.mass[kFinal + rank] = mine;
    }
    if (tid == 0 && f == 0) {   // nothing there (a mass reached only but for rounding): all above the range
        s.key[0] = r.hi + 1;
        s.res[0] = r.mass;
        s.res[1] = r.count;
    }
    __syncthreads();
    if (tid < 64 && f > 0) {
        const uint64_t k = tid < f ? s.mass[kFinal + tid] : 0;
        const double w = tid < f ? weight(key_value(k), row.m, row.c) : 0.0;
        const double incl = wave_scan_f64(w);
        const bool hit = tid < f && (by_count ? r.count + tid + 1 : r.mass + incl) >= target;
        const unsigned long long hm = __ballot(hit);
        const int l = hm ? __ffsll((long long)hm) - 1 : f - 1;
        if (tid == l) {
            s.key[0] = k;
            s.res[0] = r.mass + incl;
            s.res[1] = r.count + tid + 1;
        }
    }
    __syncthreads();
    r.mass = s.res[0];
    r.count = s.res[1];
    const uint64_t t = s.key[0];
    __syncthreads();
    return t;
}

// The row's bins (against its maximum, 1/8 apart) from its chunks' records, into s.mass / s.cnt: bin 0, the one of the
// maximum, last.
__device__ __forceinline__ void merge_bins(SampleLds &s, const char *rec, int n_chunks, float m, double c) {
    const int tid = threadIdx.x, j = tid & (kBins - 1), part = tid / kBins;   // four parts of the chunks a bin
    const float mb = floorf(m * 8.f);
    double w = 0.0;
    uint32_t n = 0;
    #pragma unroll 4
    for (int k = part; k < n_chunks; k += kThreads / kBins) {
        const float cm = s.c_max[k];
        const float d = mb - floorf(cm * 8.f);   // the chunk's bin of the row's bin j is j - d
        if (cm == -INFINITY || (float)j < d) continue;
        const char *p = rec + (size_t)k * kSampleRecord + kHead;
        const int jc = j - (int)d;
        w += (double)get64(p + 8 * jc) * kBinUnit * weight(cm, m, c);
        n += __hip_atomic_load(reinterpret_cast<uint32_t *>(const_cast<char *>(p) + 8 * kBins + 4 * jc), __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
    }
    s.list[tid] = f64_bits(w);
    s.cnt[kBins + tid] = n;
    __syncthreads();
    if (tid < kBins) {
        double sum = 0.0;
        uint32_t num = 0;
        #pragma unroll
        for (int k = 0; k < kThreads / kBins; ++k) {
            sum += bits_f64(s.list[j + k * kBins]);
            num += s.cnt[kBins + j + k * kBins];
        }
        s.mass[kBins - 1 - j] = f64_bits(sum);
        s.cnt[kBins - 1 - j] = num;
    }
    __syncthreads();
}

// The range of keys that holds the place where `target` is reached, by the row's bins; whole: by none.
__device__ __forceinline__ Range by_bins(SampleLds &s, float m, bool by_count, double target) {
    Range r = {0, ~(uint64_t)0, 0.0, 0.0};
    int n;
    const double mb = (double)floorf(m * 8.f);
    // total of the bins: below them the range is open
    double tm = 0.0, tn = 0.0;
    if (threadIdx.x < kBins) {
        tm = bits_f64(s.mass[threadIdx.x]);
        tn = (double)s.cnt[threadIdx.x];
    }
    tm = block_sum(tm, s.part);
    tn = block_sum(tn, s.part2);
    __syncthreads();
    if ((by_count ? tn : tm) < target) {
        r.mass = tm;
        r.count = tn;
        r.hi = argmax_key((float)((mb - (kBins - 1)) / 8.0), -1) - 1;   // below the last bin's lower edge
        return r;
    }
    const int b = crossing(s, kBins, by_count, target, r, &n), j = kBins - 1 - b;
    // keys of values in [(mb - j) / 8, (mb - j + 1) / 8): every index (the image of an edge with the index field at 0)
    const uint64_t edge = (uint64_t)0xffffffffu << 32;
    r.lo = argmax_key((float)((mb - j) / 8.0), 0) & edge;
    r.hi = (argmax_key((float)((mb - j + 1) / 8.0), 0) & edge) - 1;
    return r;
}

// The draw: the first entry with which the running kept mass exceeds u * (sum of c_mass), c_mass[] each chunk's.
template <typename T>
__device__ int draw(const Row<T> &row, uint64_t t, double u) {
    SampleLds &s = *row.s;
    const int tid = threadIdx.x;
    if (tid < 64) {
        double z = 0.0;
        for (int k = tid; k < row.n_chunks; k += 64) z += s.c_mass[k];
        const double target = u * __longlong_as_double((long long)wave_fold_u64(f64_bits(z), add_f64_bits));
        double carry = 0.0, before = 0.0;
        int at = -1, last = 0;
        for (int k0 = 0; k0 < row.n_chunks && at < 0; k0 += 64) {
            const double w = k0 + tid < row.n_chunks ? s.c_mass[k0 + tid] : 0.0, incl = wave_scan_f64(w);
            const unsigned long long pos = __ballot(w > 0.0), hit = __ballot(w > 0.0 && carry + incl > target);
            if (pos) last = k0 + 63 - __clzll((long long)pos);
            if (hit) {
                const int l = __ffsll((long long)hit) - 1;
                at = k0 + l;
                before = carry + read_lane_f64(incl, l) - read_lane_f64(w, l);
            }
            carry += read_lane_f64(incl, 63);
        }
        if (tid == 0) {
            s.num[0] = at < 0 ? last : at;                     // rounding: the last chunk, its last entry
            s.res[0] = at < 0 ? INFINITY : target - before;
            s.num[1] = 0x7fffffff;
            s.num[2] = -1;
        }
    }
    __syncthreads();
    const int e0 = s.num[0] * kSampleChunk + tid * kRun;
    const double target = s.res[0];
    float x[kRun];
    load_run(row.x, e0, row.V, x);
    double w[kRun], sum = 0.0;
    int last = -1;
    #pragma unroll
    for (int i = 0; i < kRun; ++i) {
        w[i] = e0 + i < row.V && argmax_key(x[i], e0 + i) >= t ? weight(x[i], row.m, row.c) : 0.0;
        sum += w[i];
        if (w[i] > 0.0) last = e0 + i;
    }
    double run = block_scan(sum, s.part);
    int first = 0x7fffffff;
    #pragma unroll
    for (int i = kRun - 1; i >= 0; --i) {
        // (the run's sums from its start, each formed the same way)
        double upto = run;
        #pragma unroll
        for (int k = 0; k <= i; ++k) upto += w[k];
        if (w[i] > 0.0 && upto > target) first = e0 + i;
    }
    if (first != 0x7fffffff) atomicMin(&s.num[1], first);
    if (last >= 0) atomicMax(&s.num[2], last);
    __syncthreads();
    return s.num[1] != 0x7fffffff ? s.num[1] : s.num[2];
}

// A row with a small top-k, all candidates in the list (n of them, the k-th largest among them).
template <typename T>
__device__ void finish_list(const Row<T> &row, const SampleArgs &a, int b, size_t r, int n) {
    SampleLds &s = *row.s;
    const int tid = threadIdx.x, k = min(a.top_k[b], n);
    Range all = {0, ~(uint64_t)0, 0.0, 0.0};
    if (tid == 0) s.num[3] = n;
    __syncthreads();
    const uint64_t t = n > k ? select(row, all, true, (double)k, n, true) : 0;
    // the k kept, ordered by rank: keys to mass[], weights behind them
    if (tid == 0) s.num[2] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads)
        if (s.list[i] >= t) s.mass[atomicAdd(&s.num[2], 1)] = s.list[i];
    __syncthreads();
    uint64_t *sorted = s.mass + kListK, *ws = s.mass + 2 * kListK;
    if (tid < k) {
        const uint64_t mine = s.mass[tid];
        int rank = 0;
        for (int j = 0; j < k; ++j) rank += s.mass[j] > mine ? 1 : 0;
        sorted[rank] = mine;
        ws[rank] = f64_bits(weight(key_value(mine), row.m, row.c));
    }
    __syncthreads();
    const double w = tid < k ? bits_f64(ws[tid]) : 0.0;
    const double before = block_scan(w, s.part), total = block_sum(w, s.part2);
    const bool keep = tid < k && (a.top_p[b] >= 1.0 || before < a.top_p[b] * total) && w >= a.min_p[b];
    const int kept = __syncthreads_count(keep);   // a prefix
    const double z = block_sum(keep ? w : 0.0, s.part);
    if (tid == 0) s.num[0] = 0x7fffffff, s.num[1] = -1;
    __syncthreads();
    if (keep) {
        const int v = key_index(sorted[tid]);
        if (a.probs) store_agent(a.probs + r * row.V + v, (float)(w / z));
        if (a.tok) {
            // running mass in index order, summed in the order of the values
            double upto = 0.0;
            for (int j = 0; j < kept; ++j) upto += key_index(sorted[j]) <= v ? bits_f64(ws[j]) : 0.0;
            if (w > 0.0) {
                if (upto > (double)a.u[r] * z) atomicMin(&s.num[0], v);
                atomicMax(&s.num[1], v);
            }
        }
    }
    __syncthreads();
    if (tid == 0 && a.tok) a.tok[r] = s.num[0] != 0x7fffffff ? s.num[0] : s.num[1];
}

// kept mass of every chunk into c_mass[]; returns their sum
template <typename T>
__device__ double chunk_masses(const Row<T> &row, uint64_t t) {
    SampleLds &s = *row.s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    double *part = reinterpret_cast<double *>(s.list);   // [chunk][wave]
    static_assert(kSampleMaxChunks * 16 <= kList, "partial sums fit the list");
    __syncthreads();
    for (int c = 0; c < row.n_chunks; ++c) {
        float x[kRun];
        const int e = c * kSampleChunk + tid * kRun;
        load_run(row.x, e, row.V, x);
        double w = 0.0;
        #pragma unroll
        for (int i = 0; i < kRun; ++i)
            if (e + i < row.V && argmax_key(x[i], e + i) >= t) w += weight(x[i], row.m, row.c);
        w = __longlong_as_double((long long)wave_fold_u64(f64_bits(w), add_f64_bits));
        if (lane == 0) part[c * 16 + wave] = w;
    }
    __syncthreads();
    if (tid < row.n_chunks) {
        double w = 0.0;
        for (int k = 0; k < 16; ++k) w += part[tid * 16 + k];
        s.c_mass[tid] = w;
    }
    __syncthreads();
    double z = 0.0;
    for (int c = 0; c < row.n_chunks; ++c) z += s.c_mass[c];
    return z;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(const SampleArgs a) {
    __shared__ SampleLds s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int rows = a.B * a.T, r = blockIdx.x % rows, chunk = blockIdx.x / rows, b = r / a.T;
    const int top_k = a.top_k[b];
    const bool listed = top_k > 0 && top_k <= kListK;
    const bool binned = !listed && (top_k > 0 || a.top_p[b] < 1.0);
    Row<T> row = {reinterpret_cast<const T *>(a.logits) + (size_t)r * a.V, a.V, a.n_chunks, 0.f, a.c[b], &s};
    char *rec0 = a.records + (size_t)r * a.n_chunks * kSampleRecord, *rec = rec0 + (size_t)chunk * kSampleRecord;

    // ---- this chunk: maximum, NaN, bins ----
    const int e0 = chunk * kSampleChunk + tid * kRun;
    float x[kRun];
    load_run(row.x, e0, a.V, x);
    float m = -INFINITY;
    bool nan = false;
    #pragma unroll
    for (int i = 0; i < kRun; ++i) {
        nan |= x[i] != x[i];
        m = fmaxf(m, x[i]);
    }
    m = group_max<64>(m);
    nan = __any(nan);
    if (lane == 0) {
        s.c_max[wave] = m;
        s.c_flags[wave] = nan ? 1 : 0;
    }
    if (tid < kBins) s.mass[tid] = 0, s.cnt[tid] = 0;
    if (tid == 0) s.num[0] = 0, s.num[1] = 0;
    __syncthreads();
    m = s.c_max[0];
    uint32_t flags = s.c_flags[0];
    #pragma unroll
    for (int k = 1; k < kThreads / 64; ++k) {
        m = fmaxf(m, s.c_max[k]);
        flags |= s.c_flags[k];
    }
    const float mb = floorf(m * 8.f);
    if (!(fabsf(m) < 0x1p20f)) flags |= 2;   // (bins of 1/8 are exact below 2^21)
    float edge = INFINITY;
    uint32_t n_out = 0;
    double mass = 0.0;
    if (listed) {
        if (!(flags & 2)) {
            #pragma unroll
            for (int i = 0; i < kRun; ++i) {
                const float j = mb - floorf(x[i] * 8.f);
                if (j < (float)kBins) atomicAdd(&s.cnt[(int)j], 1u);
            }
            __syncthreads();
            if (wave == 0) {   // the bin with which top_k are reached, or the last
                double v[kBins / 64], sum = 0.0;
                #pragma unroll
                for (int i = 0; i < kBins / 64; ++i) {
                    v[i] = (double)s.cnt[lane * (kBins / 64) + i];
                    sum += v[i];
                }
                double run = wave_scan_f64(sum) - sum;
                int at = kBins - 1;
                for (int i = kBins / 64 - 1; i >= 0; --i) {
                    double upto = run;
                    for (int k = 0; k <= i; ++k) upto += v[k];
                    if (upto >= (double)top_k) at = lane * (kBins / 64) + i;
                }
                at = (int)(0xffffffffu - (uint32_t)wave_fold_u64((uint64_t)(0xffffffffu - (uint32_t)at),
                                                                 [](uint64_t p, uint64_t q) { return p > q ? p : q; }));
                if (lane == 0) s.num[2] = at;
            }
            __syncthreads();
            const int at = s.num[2];
            edge = (mb - (float)at) * 0.125f;
            bool left = false;
            #pragma unroll
            for (int i = 0; i < kRun; ++i) {
                if (x[i] >= edge) {
                    const int p = atomicAdd(&s.num[0], 1);
                    if (p < kEmit) put64(rec + kHead + 8 * p, argmax_key(x[i], e0 + i));
                } else {
                    left |= x[i] > -INFINITY && at == kBins - 1;   // a finite one below the bins
                }
            }
            if (left) s.num[1] = 1;
            __syncthreads();
            n_out = (uint32_t)s.num[0];
            if (n_out > (uint32_t)kEmit) flags |= 4, edge = INFINITY, n_out = 0;
            else if (s.num[1]) flags |= 4;
        } else if (m > -INFINITY) {
            flags |= 4;   // candidates only by the row's last workgroup
        }
        if (a.probs) zero_run(a.probs + (size_t)r * a.V, e0, a.V);
    } else {
        #pragma unroll
        for (int i = 0; i < kRun; ++i) {
            const double w = e0 + i < a.V ? weight(x[i], m, row.c) : 0.0;
            mass += m == -INFINITY ? 0.0 : w;
            if (binned && !(flags & 2)) {
                const float j = mb - floorf(x[i] * 8.f);
                if (j < (float)kBins && e0 + i < a.V) {
                    atomicAdd((unsigned long long *)&s.mass[(int)j], (unsigned long long)(w * (1.0 / kBinUnit) + 0.5));
                    atomicAdd(&s.cnt[(int)j], 1u);
                }
            }
        }
        mass = block_sum(mass, s.part);   // (its barrier stands behind the atomics)
        if (binned && tid < kBins) {
            put64(rec + kHead + 8 * tid, s.mass[tid]);
            __hip_atomic_store(reinterpret_cast<uint32_t *>(rec + kHead + 8 * kBins) + tid, s.cnt[tid], __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (tid == 0) {
        put64(rec, (uint64_t)__float_as_uint(m) | (uint64_t)flags << 32);
        put64(rec + 8, (uint64_t)__float_as_uint(edge) | (uint64_t)n_out << 32);
        put64(rec + 16, f64_bits(mass));
    }
    wait_vm_stores();
    __syncthreads();
    if (tid == 0) {
        unsigned *cnt = a.counters + (size_t)r * kCounterStride;
        const int last = arrive(cnt) == (unsigned)(a.n_chunks - 1);
        if (last) reset_counter(cnt);
        s.num[3] = last;
    }
    __syncthreads();
    if (!s.num[3]) return;

    // ---- the row's last workgroup ----
    if (tid < a.n_chunks) {
        const char *p = rec0 + (size_t)tid * kSampleRecord;
        const uint64_t h0 = get64(p), h1 = get64(p + 8), h2 = get64(p + 16);
        s.c_max[tid] = __uint_as_float((uint32_t)h0);
        s.c_flags[tid] = (uint32_t)(h0 >> 32);
        s.c_edge[tid] = __uint_as_float((uint32_t)h1);
        s.c_n[tid] = (uint32_t)(h1 >> 32);
        s.c_mass[tid] = bits_f64(h2);
    }
    __syncthreads();
    m = -INFINITY;
    flags = 0;
    int n = 0;
    for (int c = 0; c < a.n_chunks; ++c) {
        m = fmaxf(m, s.c_max[c]);
        flags |= s.c_flags[c];
        n += (int)s.c_n[c];
    }
    row.m = m;
    RowResult *out = a.rows + r;
    if ((flags & 1) || m == -INFINITY) {   // no distribution
        if (tid == 0) {
            if (a.tok) a.tok[r] = -1;
            if (!listed) *out = RowResult{~(uint64_t)0, 1.0, 0.f, 0};
        }
        return;
    }
    if (listed && n <= kList) {
        // the candidates, in whatever order: chunk by chunk, a wave each
        int at = 0;
        for (int c = 0; c < a.n_chunks; ++c) {
            const int nc = (int)s.c_n[c];
            if (c % (kThreads / 64) == wave)
                for (int i = lane; i < nc; i += 64) s.list[at + i] = get64(rec0 + (size_t)c * kSampleRecord + kHead + 8 * i);
            at += nc;
        }
        __syncthreads();
        // What a chunk left out lies below its edge: harmless where the k-th candidate does not.
        bool complete = true;
        if (flags & 4) {
            float worst = -INFINITY;
            for (int c = 0; c < a.n_chunks; ++c)
                if (s.c_flags[c] & 4) worst = fmaxf(worst, s.c_edge[c]);
            complete = false;
            if (worst < INFINITY) {
                int above = 0;
                for (int i = tid; i < n; i += kThreads) above += key_value(s.list[i]) >= worst ? 1 : 0;
                complete = block_sum((double)above, s.part) >= (double)top_k;
                __syncthreads();
            }
        }
        if (complete) {
            finish_list(row, a, b, r, n);
            return;
        }
    }
    // ---- any row: threshold and mass ----
    uint64_t t = 0;
    double kept;
    bool have = false;   // c_mass[] holds the kept masses
    if (!listed) {
        __syncthreads();
        if (tid < a.n_chunks) s.c_mass[tid] = s.c_max[tid] == -INFINITY ? 0.0 : s.c_mass[tid] * weight(s.c_max[tid], m, row.c);
        __syncthreads();
        kept = 0.0;
        for (int c = 0; c < a.n_chunks; ++c) kept += s.c_mass[c];
        have = true;
    } else {
        kept = chunk_masses(row, 0);
    }
    bool bins = binned;
    if (bins)
        for (int c = 0; c < a.n_chunks; ++c) bins = bins && (!(s.c_flags[c] & 2) || s.c_max[c] == -INFINITY);
    const Range whole = {0, ~(uint64_t)0, 0.0, 0.0};
    if (top_k > 0 && top_k < a.V) {
        if (bins) merge_bins(s, rec0, a.n_chunks, m, row.c);
        Range g = bins ? by_bins(s, m, true, (double)top_k) : whole;
        t = select(row, g, true, (double)top_k, 0, false);
        kept = g.mass;
        have = false;
    }
    if (a.top_p[b] < 1.0) {
        const double target = a.top_p[b] * kept;
        if (bins) merge_bins(s, rec0, a.n_chunks, m, row.c);
        Range g = bins ? by_bins(s, m, false, target) : whole;
        const uint64_t tp = select(row, g, false, target, 0, false);
        if (tp > t) {
            t = tp;
            kept = g.mass;
        }
        have = false;
    }
    const double min_p = a.min_p[b];
    if (min_p > 0.0 && (t == 0 || weight(key_value(t), m, row.c) < min_p)) {
        // the least value whose weight reaches min_p, by bisection over the ordered images
        uint32_t lo = 0, hi = (uint32_t)(argmax_key(m, 0) >> 32);   // hi reaches it
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2;
            const float v = key_value((uint64_t)mid << 32);
            if (v == v && weight(v, m, row.c) >= min_p) hi = mid;
            else lo = mid + 1;
        }
        t = (uint64_t)hi << 32;
        kept = chunk_masses(row, t);
        have = true;
    }
    if (a.tok && !a.probs) {
        if (!have) kept = chunk_masses(row, t);
        const int v = draw(row, t, (double)a.u[r]);
        if (tid == 0) a.tok[r] = v;
        return;
    }
    if (listed) {   // (no second launch for it) its distribution, over the zeros
        if (a.tok) {
            if (!have) kept = chunk_masses(row, t);
            const int v = draw(row, t, (double)a.u[r]);
            if (tid == 0) a.tok[r] = v;
        }
        float *p = a.probs + (size_t)r * a.V;
        row.each([&](float v, int i) {
            if (argmax_key(v, i) >= t) store_agent(p + i, (float)(weight(v, m, row.c) / kept));
        });
        return;
    }
    if (tid == 0) *out = RowResult{t, kept, m, 1};
}

// The distributions of the rows that the first launch only decided, and their draws.
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_emit_kernel(const SampleArgs a) {
    __shared__ SampleLds s;
    const int tid = threadIdx.x;
    const int rows = a.B * a.T, r = blockIdx.x % rows, chunk = blockIdx.x / rows, b = r / a.T;
    if (a.top_k[b] > 0 && a.top_k[b] <= kListK) return;
    const RowResult res = a.rows[r];
    Row<T> row = {reinterpret_cast<const T *>(a.logits) + (size_t)r * a.V, a.V, a.n_chunks, res.m, a.c[b], &s};
    const int e0 = chunk * kSampleChunk + tid * kRun;
    float x[kRun], p[kRun];
    load_run(row.x, e0, a.V, x);
    double sum = 0.0;
    #pragma unroll
    for (int i = 0; i < kRun; ++i) {
        const double w = res.valid && e0 + i < a.V && argmax_key(x[i], e0 + i) >= res.t ? weight(x[i], res.m, row.c) : 0.0;
        sum += w;
        p[i] = (float)(w / res.mass);
    }
    store_run(a.probs + (size_t)r * a.V, e0, a.V, p);
    if (!a.tok || !res.valid) return;
    sum = block_sum(sum, s.part);
    char *rec0 = a.records + (size_t)r * a.n_chunks * kSampleRecord;
    if (tid == 0) {
        put64(rec0 + (size_t)chunk * kSampleRecord + 24, f64_bits(sum));
        wait_vm_stores();
        unsigned *cnt = a.counters + (size_t)r * kCounterStride;
        const int last = arrive(cnt) == (unsigned)(a.n_chunks - 1);
        if (last) reset_counter(cnt);
        s.num[3] = last;
    }
    __syncthreads();
    if (!s.num[3]) return;
    if (tid < a.n_chunks) s.c_mass[tid] = bits_f64(get64(rec0 + (size_t)tid * kSampleRecord + 24));
    __syncthreads();
    const int v = draw(row, res.t, (double)a.u[r]);
    if (tid == 0) a.tok[r] = v;
}

// ------------------------------------------------------------------ host ----

size_t sample_ws_bytes(int B, int T, int V) {
    const size_t rows = (size_t)B * T, chunks = ((size_t)V + kSampleChunk - 1) / kSampleChunk;
    return kCounterRegionBytes + align256(rows * sizeof(RowResult)) + rows * chunks * kSampleRecord;
}

template <typename T>
static hipError_t launch_sample_t(const SampleArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.B * a.T) * (unsigned)a.n_chunks), block(kThreads);
    hipLaunchKernelGGL((sample_kernel<T>), grid, block, 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.probs) return e;
    bool emit = false;
    for (int b = 0; b < a.B; ++b) emit |= a.top_k[b] == 0 || a.top_k[b] > kListK;
    if (!emit) return e;
    hipLaunchKernelGGL((sample_emit_kernel<T>), grid, block, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_sample(const SampleArgs &a, int dtype, hipStream_t st) {
    return dtype == MAD_BF16 ? launch_sample_t<bf16_t>(a, st) : launch_sample_t<float>(a, st);
}

}  // namespace mad

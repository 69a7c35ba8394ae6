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
// integers: their sums do not depend on the order.  Entries of equal value all
// round the same way, and a filter may end among thousands of them at a tiny
// weight, so the units go down with the weights: a bin's unit with the bin, a
// list's with its largest weight, and sums over a whole row keep what the unit
// leaves in a second integer.
//
// Work.  Workgroup (chunk, row) of 1024 threads reads 8192 entries, 8 a thread.
//   * Rows with a small top-k (kListK): it finds a value that at least top_k of
//     its entries reach (from its threads' maxima, counted into bins of 1/8, and
//     where those crowd, from all of them in bins of a 256th of what is left) and
//     writes the entries down to there, somewhat more than top_k, to the
//     workspace.  The row's last workgroup then has every candidate: it sorts
//     the best and applies the filters, the draw and the probabilities to them.
//     The row is read once and nothing else of V entries is touched but the
//     zeros of the distribution.
//   * Rows with min-p alone likewise: a chunk's candidates are what min-p leaves
//     against its own maximum (the row's leaves no more of them).
//   * Other rows: it sums its weights, and where a filter is on, also by bins of
//     1/8 below its maximum.  The row's last workgroup finds the bin in which the
//     filter ends.  A second launch, over all chunks again, collects that bin's
//     entries (the mass above it is known from the bins); its last workgroup finds
//     the entry where the count or mass is reached, and draws.  Where distributions
//     are asked for, a third launch writes them.
//   * Rows with a large top-k and a top-p: top-p's bin is known only behind the k-th
//     entry, so the row's last workgroup collects both bins' entries itself.
//   What none of these holds (thousands of entries to a bin, values further apart
//   than 32, huge magnitudes) one workgroup narrows down in passes over the row, with
//   2048 buckets of the key range each, from what is known.
//
// Bound.  Small calls: one launch's chain of round trips (with time stamps in the
// kernel, 12.2 us in all: loads 2.7, bins and candidates 2.8, arrival 0.9, the records
// 2.4, the list's end 3.4): a row of 50257 11.2 us, 20 rows with their distributions
// 13.1.  Large ones: 80 rows of 128256 fp32 with top-p and distributions (82 MB read and
// written once) 68.3 us: 24.4 for the weights (two workgroups per CU load, then compute,
// in step: 1.8 TB/s, and the vector ALU is busy 86 % of the time: 60 instructions an
// entry, 31 of them its weight, the others its bin's), 29 for the cut (a read at 4 TB/s,
// then 5 - 14 us for a row's last workgroup), 16.5 for the distributions (5 TB/s, a copy's
// rate).  64 rows of 128256 with settings of their own, tokens only, 47.5 us.  A top-k of
// 200 with top-p, tokens only: a row of 50257 64 us, 16 rows of 128256 83; min-p alone
// 14.8 and 16.4 (by the bins 23 and 24).  Rows that go by passes: 77 - 163 for top-p in a
// crowded body, 49 - 76 for min-p there, 91 - 306 for the other filters where all entries
// are within 1/8 (the same sizes).
//   The bins' own units cost the first launch two instructions an entry (weights all
// in 2^-50 of the largest: 67.9 us for the 80 rows, 46.1 for the 64, and wrong ends
// among tiny weights).
//   Not kept: several chunks to a workgroup of the first launch, the next one's loads
// in flight (its 64 registers do not hold the loop and the row's end: 33 us against
// 26.5 of one to each); the row's end as a function that is not inlined (75).
#include "mad_device.h"
#include "mad_internal.h"

#include <algorithm>

namespace mad {

constexpr int kThreads = 1024, kRun = kSampleChunk / kThreads;   // entries of a thread: consecutive
constexpr int kBins = 256, kBuckets = 2048, kList = 4096, kFinal = 128, kSort = 512;
constexpr int kResident = 512;   // workgroups at a time: two for each of the 256 CUs (64 KB of LDS, 2048 threads)
constexpr int kUnknown = 0x7fffffff;
// 8192 weights of at most 1 in units of 2^-50, and 2^20 in units of 2^-43, come to 2^63 at most.  Weights of a whole row
// may lie far below its largest, and equal ones are all rounded the same way, so what a unit of 2^-43 leaves of each is
// counted too, in units of 2^-86 (signed, 2^62 at most): a sum is exact to 2^-67, far below a double's step.
constexpr double kBinUnit = 0x1p-50, kRowUnit = 0x1p-43, kRestUnit = 0x1p-86;

// 2^(j / 256), 0 <= j < 256, from the Taylor series at compile time (below 2e-16 relative)
constexpr int kTable = 256;
struct Exp2Table {
    double v[kTable];
    constexpr Exp2Table() : v() {
        for (int j = 0; j < kTable; ++j) {
            const double f = 0.6931471805599453 * j / kTable;   // 0 <= f < ln 2
            double p = 1.0;
            for (int k = 20; k > 0; --k) p = 1.0 + p * f / k;
            v[j] = p;
        }
    }
};
__constant__ const Exp2Table kExp2 = Exp2Table();

// The weight of x against the maximum m, c = 256 log2 e / temperature: with (x - m) c = n + f, |f| <= 1/2, it is
// 2^(n / 256) from the table and 2^(f / 256) by its series (to f^4: 4e-17 relative).  In double, at half the operations
// of a series alone; the coefficients are in scalar registers, formed where they are used: the compiler would keep a
// copy of each in vector registers all through the kernel, of which there are 64, and have them spilled.
struct Series {
    double k1, k2, k3, k4;
};
__device__ __forceinline__ Series series() {
    constexpr double k1 = 0.6931471805599453 / kTable, k2 = k1 * k1 / 2, k3 = k2 * k1 / 3, k4 = k3 * k1 / 4;
    Series s = {k1, k2, k3, k4};
    asm volatile("" : "+s"(s.k1), "+s"(s.k2), "+s"(s.k3), "+s"(s.k4));
    return s;
}
// m finite, x not above it (a NaN or -inf: 2^-1000)
__device__ __forceinline__ double weight_finite(float x, double m, double c, const double *table, const Series &s) {
    const double y = fmax(((double)x - m) * c, -1000.0 * kTable);
    const double t = y + 0x1.8p52;   // n in the low bits
    const double f = y - (t - 0x1.8p52);
    double p = fma(s.k4, f, s.k3);
    p = fma(p, f, s.k2);
    p = fma(p, f, s.k1);
    p = fma(p, f, 1.0);
    const uint32_t n = (uint32_t)__double_as_longlong(t);
    const uint64_t w = (uint64_t)__double_as_longlong(p * table[n & (kTable - 1)]);
    const uint32_t hi = (uint32_t)(w >> 32) + ((n & ~(uint32_t)(kTable - 1)) << 12);   // times 2^(n >> 8)
    return __longlong_as_double((long long)((uint64_t)hi << 32 | (uint32_t)w));
}
// any m and x (+inf against +inf: 1; below 2^-1000: 0)
__device__ __forceinline__ double weight(float x, float m, double c, const double *table) {
    const double y = ((double)x - (double)m) * c;
    return x == m ? 1.0 : y > -1000.0 * kTable ? weight_finite(x, (double)m, c, table, series()) : 0.0;
}
// w (<= 1) as an integer of 1 / per, to nearest; per a power of two up to 2^50: from the low mantissa bits of a sum with 2^52
__device__ __forceinline__ unsigned long long units(double w, double per) {
    return (unsigned long long)__double_as_longlong(fma(w, per, 0x1p52)) - (unsigned long long)__double_as_longlong(0x1p52);
}
// what units(w, per) leaves of w, in its 2^43rd part (signed)
__device__ __forceinline__ long long rest_units(double w, double per) {
    const double whole = fma(w, per, 0x1p52) - 0x1p52;
    return __double_as_longlong(fma(fma(w, per, -whole), 0x1p43, 0x1.8p52)) - __double_as_longlong(0x1.8p52);
}
// The bins' masses, each in a unit of its own.  With k = c / 2048, the binades of weight that a bin of 1/8 spans, an entry
// of bin j has a weight of at most 2^-e, e = floor((j - 1) k), and of at least 2^-(j + 1) k; it is counted in 2^-(50 + e),
// that is to 2^-(50 - 2 k) of itself (2^-49 at temperature 1), where 8192 of one value all round the same way.  k is cut
// off at 3 1/2 (temperature 0.0515), where a bin's weights are gone within 15 bins.  `step` is k with 20 bits behind the
// point, so that 2^(50 + e) is a multiply-add and a mask on a double's high word.
__device__ __forceinline__ uint32_t bin_step(double c) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)(fmin(c, 3.5 * 2048) * 512.0)); }
__device__ __forceinline__ uint32_t bin_per_high(int j, uint32_t step) {
    return (__umul24((uint32_t)j, step) + ((1073u << 20) - step)) & 0xfff00000u;
}
__device__ __forceinline__ double bin_per(int j, uint32_t step) {
    return __longlong_as_double((long long)((uint64_t)bin_per_high(j, step) << 32));
}
__device__ __forceinline__ double bin_unit(int j, uint32_t step) {
    return __longlong_as_double((long long)((uint64_t)((2046u << 20) - bin_per_high(j, step)) << 32));
}
// the value that a key holds
__device__ __forceinline__ float key_value(uint64_t k) {
    const uint32_t o = (uint32_t)(k >> 32);
    return __uint_as_float((o & 0x80000000u) ? o ^ 0x80000000u : ~o);
}

// A thread's run of kRun entries from entry e on (unaligned 16-byte loads; -inf past V), as it is loaded: the next
// chunk's is in flight while this one's is worked on.
template <typename T> struct Run;
template <> struct Run<float> {
    float v[kRun];
    __device__ __forceinline__ void load(const float *row, int e, int V) {
        if (e + kRun <= V) {
            __builtin_memcpy(v, row + e, kRun * 4);
        } else {
            #pragma unroll
            for (int i = 0; i < kRun; ++i) v[i] = e + i < V ? row[e + i] : -INFINITY;
        }
    }
    __device__ __forceinline__ void unpack(float (&x)[kRun]) const {
        #pragma unroll
        for (int i = 0; i < kRun; ++i) x[i] = v[i];
    }
};
template <> struct Run<bf16_t> {
    uint4 v;
    __device__ __forceinline__ void load(const bf16_t *row, int e, int V) {
        if (e + kRun <= V) {
            __builtin_memcpy(&v, row + e, kRun * 2);
        } else {
            uint32_t w[kRun / 2];
            #pragma unroll
            for (int i = 0; i < kRun / 2; ++i) {
                const uint32_t lo = e + 2 * i < V ? row[e + 2 * i].bits : 0xff80u, hi = e + 2 * i + 1 < V ? row[e + 2 * i + 1].bits : 0xff80u;
                w[i] = lo | hi << 16;
            }
            v = uint4{w[0], w[1], w[2], w[3]};
        }
    }
    __device__ __forceinline__ void unpack(float (&x)[kRun]) const { unpack16(v, x, bf16_t()); }
};
template <typename T>
__device__ __forceinline__ void load_run(const T *row, int e, int V, float (&x)[kRun]) {
    Run<T> run;
    run.load(row, e, V);
    run.unpack(x);
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
__device__ __forceinline__ uint32_t get32(const void *p) {
    return __hip_atomic_load(reinterpret_cast<uint32_t *>(const_cast<void *>(p)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t f64_bits(double v) { return (uint64_t)__double_as_longlong(v); }
__device__ __forceinline__ double bits_f64(uint64_t v) { return __longlong_as_double((long long)v); }

// what is the same in every lane, in scalar registers (64 vector registers are all that two workgroups per CU leave)
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(uniform(__float_as_uint(v))); }
__device__ __forceinline__ uint64_t uniform(uint64_t v) { return (uint64_t)uniform((uint32_t)(v >> 32)) << 32 | uniform((uint32_t)v); }
__device__ __forceinline__ double uniform(double v) { return bits_f64(uniform(f64_bits(v))); }

// A chunk's record in the workspace: a header of 32 bytes, then keys, or the bins' masses and counts.
//   first launch:  maximum, flags | edge, keys | mass          second: count and keys | mass above the range
constexpr int kHead = 32;
static_assert(kHead + kBins * 12 <= (int)kSampleRecord && kHead + kEmit * 8 <= (int)kSampleRecord, "chunk record");
// flags: a NaN; magnitudes beyond the bins; candidates left out below `edge` (min-p's: up to it)
constexpr uint32_t kNaN = 1, kNoBins = 2, kLeft = 4;

struct SampleLds {
    uint64_t list[kList];       // gathered keys
    uint64_t mass[kBuckets];    // histogram: masses (integers), or doubles' bits
    uint32_t cnt[kBuckets];
    double exp2[kTable];   // kExp2
    double bucket_mass[kBins];
    uint32_t bucket_cnt[kBins];
    double c_mass[kSampleMaxChunks];    // per chunk: kept mass; against the row's maximum
    double c_unit[kSampleMaxChunks];    // the weight of its maximum: what its bins' masses are against the row's
    float c_max[kSampleMaxChunks];      // its maximum; or where its keys begin in the list
    double part[16];   // one per wave
    double res[4];
    uint64_t key[4];
    float fmx[16];
    uint32_t flag[16];
    int num[4];
};
static_assert(sizeof(SampleLds) <= 64 * 1024, "static LDS");
static_assert(kBuckets <= kList && 2 * kSampleMaxChunks <= kBuckets, "second sums");
__device__ __forceinline__ SampleLds &lds() {
    __shared__ SampleLds s;
    return s;
}

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

// The workgroup's least `first` and greatest `last`, where both rise with the thread (0x7fffffff, -1: none): one lane of
// a wave for each (an LDS atomic of 64 lanes on one word takes as long as 64).
__device__ __forceinline__ void first_and_last(int first, int last, int *least, int *greatest) {
    const int lane = threadIdx.x & 63;
    const unsigned long long f = __ballot(first != 0x7fffffff), l = __ballot(last >= 0);
    if (f && lane == __ffsll((long long)f) - 1) atomicMin(least, first);
    if (l && lane == 63 - __clzll((long long)l)) atomicMax(greatest, last);
}

// One row, by one workgroup.
template <typename T> struct Row {
    const T *x;
    int V, n_chunks;
    float m;       // maximum
    double c;      // 256 log2 e / temperature

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

// Finds in the histogram mass/cnt (256 buckets of 8 parts each, the highest keys last; masses as integers of `unit`)
// the first bucket from the top with which `target` of the measure is reached on top of what r holds, or the last that
// is not empty.  PARTS: the part of it, with what the masses leave in the list's place (integers of kRestUnit).  Returns
// its number and adds what lies above it to r; *n: its entries.
template <bool PARTS>
__device__ __forceinline__ int crossing(SampleLds &s, double unit, bool by_count, double target, Range &r, int *n) {
    constexpr int P = kBuckets / kBins, Q = kBins / 64;
    const int tid = threadIdx.x;
    if (tid < kBins) {
        uint64_t m = 0, rest = 0;
        uint32_t c = 0;
        #pragma unroll
        for (int p = 0; p < P; ++p) {
            m += s.mass[tid * P + p], c += s.cnt[tid * P + p];
            if constexpr (PARTS) rest += s.list[tid * P + p];
        }
        s.bucket_mass[kBins - 1 - tid] = (double)m * unit + (double)(int64_t)rest * kRestUnit;
        s.bucket_cnt[kBins - 1 - tid] = c;
    }
    __syncthreads();
    if (tid < 64) {   // four buckets a lane, from the top
        double m[Q], c[Q], sm = 0.0, sc = 0.0;
        #pragma unroll
        for (int q = 0; q < Q; ++q) {
            m[q] = s.bucket_mass[tid * Q + q];
            c[q] = (double)s.bucket_cnt[tid * Q + q];
            sm += m[q];
            sc += c[q];
        }
        double um = r.mass + (wave_scan_f64(sm) - sm), uc = r.count + (wave_scan_f64(sc) - sc);   // above lane's first
        double hm = 0.0, hc = 0.0, lm = 0.0, lc = 0.0;
        int hit = -1, last = -1;
        #pragma unroll
        for (int q = 0; q < Q; ++q) {
            if (c[q] > 0.0) {
                last = q, lm = um, lc = uc;
                if (hit < 0 && (by_count ? uc + c[q] : um + m[q]) >= target) hit = q, hm = um, hc = uc;
            }
            um += m[q];
            uc += c[q];
        }
        const unsigned long long hits = __ballot(hit >= 0), some = __ballot(last >= 0);
        const int l = hits ? __ffsll((long long)hits) - 1 : some ? 63 - __clzll((long long)some) : 0;
        if (tid == l) {
            int at = kBins - 1 - (tid * Q + (hits ? hit : max(last, 0)));
            double am = hits ? hm : lm, ac = hits ? hc : lc;
            int in = (int)s.bucket_cnt[kBins - 1 - at];
            if constexpr (PARTS) {
                int part = -1;
                double pm = 0.0, pc = 0.0;
                for (int p = P - 1; p >= 0; --p) {
                    const double xc = (double)s.cnt[at * P + p], xm = (double)s.mass[at * P + p] * unit + (double)(int64_t)s.list[at * P + p] * kRestUnit;
                    if (xc > 0.0) {
                        part = p, pm = am, pc = ac;
                        if ((by_count ? ac + xc : am + xm) >= target) break;
                    }
                    am += xm;
                    ac += xc;
                }
                at = at * P + max(part, 0);
                am = pm;
                ac = pc;
                in = (int)s.cnt[at];
            }
            s.num[0] = at;
            s.num[2] = in;
            s.res[0] = am;
            s.res[1] = ac;
        }
    }
    __syncthreads();
    r.mass = uniform(s.res[0]);
    r.count = uniform(s.res[1]);
    *n = uniform(s.num[2]);
    return uniform(s.num[0]);   // (what follows writes none of these before a barrier)
}

// n different keys (512 at most) into descending order: each counts the larger ones, by 8 threads or 2
__device__ __forceinline__ void sort_down(const uint64_t *from, uint64_t *to, int n) {
    static_assert(kFinal * 8 <= kThreads && kSort * 2 <= kThreads, "threads for each key");
    const int sh = n <= kFinal ? 3 : 1, e = threadIdx.x >> sh, part = threadIdx.x & ((1 << sh) - 1);
    const uint64_t mine = e < n ? from[e] : 0;
    int rank = 0;
    for (int j = part; j < n; j += 1 << sh) rank += from[j] > mine ? 1 : 0;
    rank += __shfl_xor(rank, 1);
    if (sh == 3) {
        rank += __shfl_xor(rank, 2);
        rank += __shfl_xor(rank, 4);
    }
    if (e < n && part == 0) to[rank] = mine;
}

// The entry at which `target` is reached, among the keys of r: its key (or the end of r, where rounding leaves
// nothing in it); r.mass and r.count become what lies at and above it.  r holds n keys (or as many as there are, where
// that is not known).  STREAM: out of the row, through the list as soon as that takes them; else out of the list.
template <bool STREAM, typename T>
__device__ __forceinline__ uint64_t select(const Row<T> &row, Range &r, bool by_count, double target, int n) {
    SampleLds &s = lds();
    const int tid = threadIdx.x;
    bool in_list = !STREAM;
    for (;;) {
        if constexpr (STREAM) if (!in_list && n <= kList) {   // into the list
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
            n = uniform(s.num[3]);
            in_list = true;
            __syncthreads();
        }
        // The keys of the list that are still in the range: few enough are put in order.
        if (in_list && n <= kFinal) break;
        for (int b = tid; b < kBuckets; b += kThreads) {
            s.mass[b] = 0, s.cnt[b] = 0;
            if constexpr (STREAM) if (!in_list) s.list[b] = 0;
        }
        if (tid == 0) s.key[0] = ~(uint64_t)0, s.key[1] = 0;
        __syncthreads();
        int sh, at;
        if (in_list) {
            // To the keys that are there: equal values differ in a few bits of their indices only.  Then 256 buckets,
            // each in 8 parts by lane: equal values go to one bucket.
            const int all = uniform(s.num[3]);
            uint64_t lo = ~(uint64_t)0, hi = 0;
            #pragma unroll 1
            for (int i = tid; i < all; i += kThreads) {
                const uint64_t k = s.list[i];
                if (k >= r.lo && k <= r.hi) lo = min(lo, k), hi = max(hi, k);
            }
            lo = wave_fold_u64(lo, [](uint64_t x, uint64_t y) { return x < y ? x : y; });
            hi = wave_fold_u64(hi, [](uint64_t x, uint64_t y) { return x > y ? x : y; });
            if ((tid & 63) == 0 && lo <= hi) {
                atomicMin((unsigned long long *)&s.key[0], (unsigned long long)lo);
                atomicMax((unsigned long long *)&s.key[1], (unsigned long long)hi);
            }
            __syncthreads();
            r.lo = uniform(s.key[0]);
            r.hi = uniform(s.key[1]);
            sh = max(64 - __clzll((long long)(r.hi - r.lo)) - 8, 0);
            // in 2^-50 of the power of two above the largest weight here (2^-900 at least, which none is near)
            const double top = fmax(((double)key_value(r.hi) - (double)row.m) * row.c, -900.0 * kTable);
            const int e = key_value(r.hi) == row.m ? 0 : (int)floor(top * (1.0 / kTable)) + 1;
            const double unit = bits_f64((uint64_t)(1023 - 50 + e) << 52);
            const double per = 1.0 / unit;
            #pragma unroll 1
            for (int i = tid; i < all; i += kThreads) {
                const uint64_t k = s.list[i];
                if (k >= r.lo && k <= r.hi) {
                    const int b = (int)((k - r.lo) >> sh) * (kBuckets / kBins) + (tid & 7);
                    atomicAdd(&s.cnt[b], 1u);
                    atomicAdd((unsigned long long *)&s.mass[b], units(weight(key_value(k), row.m, row.c, s.exp2), per));
                }
            }
            __syncthreads();
            at = crossing<false>(s, unit, by_count, target, r, &n);
        } else {
            sh = max(64 - __clzll((long long)(r.hi - r.lo)) - 11, 0);   // 2048 buckets (a range of one key holds one entry)
            if constexpr (STREAM)
                row.each([&](float x, int i) {
                    const uint64_t k = argmax_key(x, i);
                    if (k >= r.lo && k <= r.hi) {
                        const int b = (int)((k - r.lo) >> sh);
                        const double w = weight(x, row.m, row.c, s.exp2);
                        atomicAdd(&s.cnt[b], 1u);
                        atomicAdd((unsigned long long *)&s.mass[b], units(w, 1.0 / kRowUnit));
                        atomicAdd((unsigned long long *)&s.list[b], (unsigned long long)rest_units(w, 1.0 / kRowUnit));
                    }
                });
            __syncthreads();
            at = crossing<true>(s, kRowUnit, by_count, target, r, &n);
        }
        const uint64_t lo = r.lo + ((uint64_t)at << sh);
        r.hi = lo + min(r.hi - lo, ((uint64_t)1 << sh) - 1);   // (no sum past 64 bits)
        r.lo = lo;
    }
    // at most 128: ordered by rank, then wave 0 sums them in order, two a lane
    if (tid == 0) s.num[1] = 0;
    __syncthreads();
    const int all = uniform(s.num[3]);
    #pragma unroll 1
    for (int i = tid; i < all; i += kThreads)
        if (s.list[i] >= r.lo && s.list[i] <= r.hi) s.mass[atomicAdd(&s.num[1], 1)] = s.list[i];
    __syncthreads();
    const int f = uniform(s.num[1]);
    sort_down(s.mass, s.mass + kSort, f);
    if (tid == 0 && f == 0) {   // nothing there (a mass reached only but for rounding): all above the range
        s.key[0] = r.hi + 1;
        s.res[0] = r.mass;
        s.res[1] = r.count;
    }
    __syncthreads();
    if (tid < 64 && f > 0) {
        uint64_t k[2];
        double w[2];
        #pragma unroll
        for (int i = 0; i < 2; ++i) {
            k[i] = 2 * tid + i < f ? s.mass[kSort + 2 * tid + i] : 0;
            w[i] = 2 * tid + i < f ? weight(key_value(k[i]), row.m, row.c, s.exp2) : 0.0;
        }
        const double incl1 = wave_scan_f64(w[0] + w[1]), incl0 = incl1 - w[1];
        auto reached = [&](int i, double incl) {
            return 2 * tid + i < f && (by_count ? r.count + (2 * tid + i + 1) : r.mass + incl) >= target;
        };
        const bool hit0 = reached(0, incl0), hit = hit0 || reached(1, incl1);
        const unsigned long long hm = __ballot(hit);
        const int l = hm ? __ffsll((long long)hm) - 1 : (f - 1) >> 1, i = hm ? !hit0 : (f - 1) & 1;
        if (tid == l) {
            s.key[0] = i ? k[1] : k[0];
            s.res[0] = r.mass + (i ? incl1 : incl0);
            s.res[1] = r.count + (2 * tid + i + 1);
        }
    }
    __syncthreads();
    r.mass = uniform(s.res[0]);
    r.count = uniform(s.res[1]);
    const uint64_t t = uniform(s.key[0]);
    __syncthreads();
    return t;
}

// The first of the 256 values v(0), v(1), .. with which `target` is reached, by one wave (four a lane): its index (the
// last that is not 0 where none is), and the sum before it.
template <typename F>
__device__ __forceinline__ int first_reaching(F v, double target, double *before) {
    const int lane = threadIdx.x & 63;
    double x[kBins / 64], sum = 0.0;
    #pragma unroll
    for (int i = 0; i < kBins / 64; ++i) {
        x[i] = v(lane * (kBins / 64) + i);
        sum += x[i];
    }
    const double run = wave_scan_f64(sum) - sum;
    int at = -1;
    double pre = 0.0;
    #pragma unroll
    for (int i = kBins / 64 - 1; i >= 0; --i) {
        double upto = run;
        #pragma unroll
        for (int k = 0; k < i; ++k) upto += x[k];
        if (x[i] > 0.0 && upto + x[i] >= target) at = i, pre = upto;
    }
    const unsigned long long hit = __ballot(at >= 0), some = __ballot(sum > 0.0);
    const int l = hit ? __ffsll((long long)hit) - 1 : some ? 63 - __clzll((long long)some) : 0;
    if (!hit) {
        #pragma unroll
        for (int i = 0; i < kBins / 64; ++i) {
            if (x[i] > 0.0) at = i;
        }
        at = max(at, 0);
        pre = run;
        for (int k = 0; k < at; ++k) pre += x[k];
    }
    *before = read_lane_f64(pre, l);
    return l * (kBins / 64) + __builtin_amdgcn_readlane(at, l);
}

// The row's last workgroup: every chunk's header, lane c of each wave has chunks c and c + 64.
struct Heads {
    float max[2], edge[2];
    uint32_t flags[2], n[2];
    double mass[2];
    // over the row
    float m, worst;    // maximum; the highest edge below which candidates were left out
    bool nan, no_bins, left;
    int total;
};
__device__ __forceinline__ Heads load_heads(const char *rec0, int n_chunks) {
    Heads h;
    const int lane = threadIdx.x & 63;
    uint64_t w[2][3];
    #pragma unroll
    for (int i = 0; i < 2; ++i)
        #pragma unroll
        for (int k = 0; k < 3; ++k) w[i][k] = lane + 64 * i < n_chunks ? get64(rec0 + (size_t)(lane + 64 * i) * kSampleRecord + 8 * k) : 0;
    float m = -INFINITY, worst = -INFINITY, total = 0.f;
    uint32_t all = 0;
    #pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool in = lane + 64 * i < n_chunks;
        h.max[i] = in ? __uint_as_float((uint32_t)w[i][0]) : -INFINITY;
        h.flags[i] = (uint32_t)(w[i][0] >> 32);
        h.edge[i] = __uint_as_float((uint32_t)w[i][1]);
        h.n[i] = (uint32_t)(w[i][1] >> 32);
        h.mass[i] = bits_f64(w[i][2]);
        m = fmaxf(m, h.max[i]);
        if (h.flags[i] & kLeft) worst = fmaxf(worst, h.edge[i]);
        if ((h.flags[i] & kNoBins) && h.max[i] == -INFINITY) h.flags[i] &= ~kNoBins;   // nothing to count there
        all |= h.flags[i];
        total += (float)h.n[i];
    }
    h.m = uniform(group_max<64>(m));
    h.worst = uniform(group_max<64>(worst));
    h.nan = __any(all & kNaN);
    h.no_bins = __any(all & kNoBins);
    h.left = __any(all & kLeft);
    h.total = uniform((int)group_sum<64>(total));   // (exact: at most 2^16)
    return h;
}
// the listed keys of all chunks into LDS, a wave a chunk (n[], offset by the sums before); f(key) for each
template <typename F>
__device__ __forceinline__ void load_list(SampleLds &s, const char *rec0, int n_chunks, const uint32_t (&n)[2], F f) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int off[2];
    const double i0 = wave_scan_f64((double)n[0]), i1 = wave_scan_f64((double)n[1]);
    off[0] = (int)(i0 - (double)n[0]);
    off[1] = (int)(i1 - (double)n[1]) + (int)read_lane_f64(i0, 63);
    for (int c = wave; c < n_chunks; c += kThreads / 64) {
        const int nc = __builtin_amdgcn_readlane((int)(c < 64 ? n[0] : n[1]), c & 63);
        const int at = __builtin_amdgcn_readlane(c < 64 ? off[0] : off[1], c & 63);
        if (lane == 0) s.c_max[c] = (float)at;
        for (int i = lane; i < nc; i += 64) {
            const uint64_t k = get64(rec0 + (size_t)c * kSampleRecord + kHead + 8 * i);
            s.list[at + i] = k;
            f(k);
        }
    }
}

// The draw: the first entry with which the running kept mass exceeds u * (sum of c_mass), c_mass[] each chunk's.
template <typename T>
__device__ __forceinline__ int draw(const Row<T> &row, uint64_t t, double u) {
    SampleLds &s = lds();
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
    const int e0 = uniform(s.num[0]) * kSampleChunk + tid * kRun;
    const double target = uniform(s.res[0]);
    float x[kRun];
    load_run(row.x, e0, row.V, x);
    double w[kRun], sum = 0.0;
    int last = -1;
    const bool finite = row.m < INFINITY;
    const Series terms = series();
    #pragma unroll
    for (int i = 0; i < kRun; ++i) {
        const bool in = e0 + i < row.V && argmax_key(x[i], e0 + i) >= t && (finite ? x[i] > -INFINITY : x[i] == row.m);
        w[i] = 0.0;
        if (__any(in)) {
            const double y = finite ? weight_finite(x[i], (double)row.m, row.c, s.exp2, terms) : 1.0;
            w[i] = in && y > 0x1p-999 ? y : 0.0;
        }
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
    first_and_last(first, last, &s.num[1], &s.num[2]);
    __syncthreads();
    return s.num[1] != 0x7fffffff ? s.num[1] : s.num[2];
}

// the k-th key of the list of n (seldom asked for: kept out of its callers' registers)
__device__ __noinline__ uint64_t nth_of_list(float m, double c, int k, int n) {
    const Row<float> row = {nullptr, 0, 0, m, c};
    Range all = {0, ~(uint64_t)0, 0.0, 0.0};
    return select<false>(row, all, true, (double)k, n);
}

// A row with a small top-k, all candidates in the list (n of them, the k-th largest among them), and counted in cnt[]
// by bins of 1/8 below the maximum, the last bin open.
template <typename T>
__device__ __forceinline__ void finish_list(const Row<T> &row, const SampleArgs &a, int b, size_t r, int n) {
    SampleLds &s = lds();
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, k = min(a.top_k[b], n);
    uint64_t *some = s.mass, *sorted = s.mass + kSort;
    // down to few: the bins that hold k, or, where those hold too many, down to the k-th itself
    if (wave == 0) {
        double before;
        const int j = first_reaching([&](int i) { return (double)s.cnt[i]; }, (double)k, &before);
        if (lane == 0) {
            s.num[0] = j;
            s.num[1] = (int)before + (int)s.cnt[j];
            s.num[2] = 0;
            s.num[3] = n;
        }
    }
    __syncthreads();
    uint64_t t = 0;
    if (s.num[0] < kBins - 1) t = argmax_key((floorf(row.m * 8.f) - (float)s.num[0]) * 0.125f, 0) & ((uint64_t)0xffffffffu << 32);
    if (s.num[1] > kSort) {
        __syncthreads();
        t = n > k ? nth_of_list(row.m, row.c, k, n) : 0;
        if (tid == 0) s.num[2] = 0;
        __syncthreads();
    }
    for (int i = tid; i < n; i += kThreads)
        if (s.list[i] >= t) some[atomicAdd(&s.num[2], 1)] = s.list[i];
    __syncthreads();
    sort_down(some, sorted, s.num[2]);   // k of them at least, 512 at most
    __syncthreads();
    // one wave applies the filters, two entries a lane in order
    static_assert(kListK <= 128, "two a lane");
    if (wave == 0) {
        uint64_t key[2];
        double w[2];
        #pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bool in = 2 * lane + i < k;
            key[i] = in ? sorted[2 * lane + i] : 0;
            w[i] = in ? weight(key_value(key[i]), row.m, row.c, s.exp2) : 0.0;
        }
        const double incl = wave_scan_f64(w[0] + w[1]), total = read_lane_f64(incl, 63);
        const double before[2] = {incl - (w[0] + w[1]), incl - w[1]};
        bool keep[2];
        #pragma unroll
        for (int i = 0; i < 2; ++i) {
            keep[i] = 2 * lane + i < k && (a.top_p[b] >= 1.0 || before[i] < a.top_p[b] * total) && w[i] >= a.min_p[b];
            w[i] = keep[i] ? w[i] : 0.0;
        }
        const double z = __longlong_as_double((long long)wave_fold_u64(f64_bits(w[0] + w[1]), add_f64_bits));
        const int kept = (int)__popcll(__ballot(keep[0])) + (int)__popcll(__ballot(keep[1]));   // a prefix
        const double inv = 1.0 / z;
        #pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (keep[i] && a.probs) store_agent(a.probs + r * row.V + key_index(key[i]), (float)(w[i] * inv));
            s.list[2 * lane + i] = f64_bits(w[i]);
            s.cnt[2 * lane + i] = (uint32_t)key_index(key[i]);
        }
        if (lane == 0) {
            s.num[0] = kept;
            s.num[1] = 0x7fffffff;
            s.num[2] = -1;
            s.res[0] = a.tok ? (double)a.u[r] * z : 0.0;
        }
    }
    if (!a.tok) return;
    __syncthreads();
    // the running mass up to each entry in index order, eight threads an entry
    const int kept = s.num[0], e = tid >> 3, part = tid & 7;
    const uint32_t v = s.cnt[e];
    double upto = 0.0;
    for (int j = part; j < kept; j += 8) upto += s.cnt[j] <= v ? bits_f64(s.list[j]) : 0.0;
    upto += __shfl_xor(upto, 1);
    upto += __shfl_xor(upto, 2);
    upto += __shfl_xor(upto, 4);
    if (e < kept && part == 0 && s.list[e] != 0) {
        if (upto > s.res[0]) atomicMin(&s.num[1], (int)v);
        atomicMax(&s.num[2], (int)v);
    }
    __syncthreads();
    if (tid == 0) a.tok[r] = s.num[1] != 0x7fffffff ? s.num[1] : s.num[2];
}

// The listed entries that stay (n[]: a chunk's, as in load_list) to their chunks' masses, a wave a chunk; returns the
// sum over the row.
template <typename T>
__device__ __forceinline__ double add_listed(const Row<T> &row, const uint32_t (&n)[2], uint64_t t) {
    SampleLds &s = lds();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int c = wave; c < row.n_chunks; c += kThreads / 64) {
        const int nc = __builtin_amdgcn_readlane((int)(c < 64 ? n[0] : n[1]), c & 63), at = (int)s.c_max[c];
        unsigned long long sum = 0, rest = 0;   // (at most 4096 entries)
        #pragma unroll 1
        for (int i = lane; i < nc; i += 64) {
            const uint64_t k = s.list[at + i];
            const double w = k >= t ? weight(key_value(k), row.m, row.c, s.exp2) : 0.0;
            sum += units(w, 1.0 / kBinUnit);
            rest += (unsigned long long)rest_units(w, 1.0 / kBinUnit);
        }
        sum = wave_fold_u64(sum, [](uint64_t x, uint64_t y) { return x + y; });
        rest = wave_fold_u64(rest, [](uint64_t x, uint64_t y) { return x + y; });
        if (lane == 0) s.c_mass[c] += (double)sum * kBinUnit + (double)(int64_t)rest * (kBinUnit * 0x1p-43);
    }
    __syncthreads();
    double kept = 0.0;
    #pragma unroll
    for (int i = 0; i < 2; ++i)
        if (lane + 64 * i < row.n_chunks) kept += s.c_mass[lane + 64 * i];
    return uniform(__longlong_as_double((long long)wave_fold_u64(f64_bits(kept), add_f64_bits)));
}

// kept mass of every chunk into c_mass[]; returns their sum.  (Not inlined into the passes over a row, whose registers it
// would share: 48 us a row of 50257 with min-p among near-equal entries, 58 inlined.)
template <typename T>
__device__ __noinline__ double chunk_masses(const Row<T> row, uint64_t t) {
    SampleLds &s = lds();
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
            if (e + i < row.V && argmax_key(x[i], e + i) >= t) w += weight(x[i], row.m, row.c, s.exp2);
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

// The least key whose value's weight reaches p (0 < p <= 1): 64 places at a time, by every wave.
__device__ __forceinline__ uint64_t least_weight(float m, double c, double p) {
    SampleLds &s = lds();
    uint32_t lo = 0, hi = (uint32_t)(argmax_key(m, 0) >> 32);   // hi reaches it; the answer is in [lo, hi]
    while (lo < hi) {
        const uint32_t span = hi - lo, step = span / 64 + 1;
        const uint32_t at = lo + min(span, (uint32_t)(threadIdx.x & 63) * step);
        const float v = key_value((uint64_t)at << 32);
        const unsigned long long ok = __ballot(v == v && weight(v, m, c, s.exp2) >= p);   // (images below -inf's are NaN)
        const int l = ok ? __ffsll((long long)ok) - 1 : 64;
        const uint32_t was = lo;
        if (l > 0) lo = was + min(span, (uint32_t)(l - 1) * step) + 1;
        if (l < 64) hi = was + min(span, (uint32_t)l * step);
        else lo = min(lo, hi);
    }
    return (uint64_t)lo << 32;
}

template <typename T>
__device__ __forceinline__ Row<T> row_of(const SampleArgs &a, int r) {
    return Row<T>{reinterpret_cast<const T *>(a.logits) + (size_t)r * a.V, a.V, a.n_chunks, 0.f, a.c[r / a.T]};
}
// whether this workgroup is the row's last to get here; what it stored at device scope is visible then
__device__ __forceinline__ bool row_last(const SampleArgs &a, int r, int groups, SampleLds &s) {
    wait_vm_stores();
    __syncthreads();
    if (threadIdx.x == 0) {
        unsigned *cnt = a.counters + (size_t)r * kCounterStride;
        const int last = arrive(cnt) == (unsigned)(groups - 1);
        if (last) reset_counter(cnt);
        s.num[3] = last;
    }
    __syncthreads();
    const bool last = s.num[3];
    __syncthreads();
    return last;
}

// A row by passes over it, by one workgroup: what the bins or the lists did not hold.  Not inlined: the kernels keep
// their registers (64, for two workgroups per CU) and its spills stay in it.
template <typename T> struct SolveJob {
    Row<T> row;
    double top_p, min_p, u;
    int32_t *tok;     // or null
    float *over;      // the row's distribution, zeros so far, where no other launch writes it
    RowResult *out;
    int top_k;
    // where the first filter (top-k, else top-p) ends, as far as it is known: `n` keys, none to search for where
    // target < 0; and min-p's bound
    Range range;
    double target;
    uint64_t least;
    int n;
    const char *rec0;   // the row's records
};
template <typename T>
__device__ __noinline__ void solve_row(const SolveJob<T> j) {
    SampleLds &s = lds();
    const int tid = threadIdx.x;
    __syncthreads();
    const Row<T> row = j.row;
    uint64_t t = 0;
    bool known = j.n < kUnknown;
    if (!known || j.target >= 0.0) {
        for (int pass = 0; pass < 2; ++pass) {   // top-k, then top-p of its mass
            const bool by_count = pass == 0;
            if (by_count ? j.top_k == 0 : j.top_p >= 1.0) continue;
            Range g = known ? j.range : Range{0, ~(uint64_t)0, 0.0, 0.0};
            const double target = known ? j.target : by_count ? (double)j.top_k : j.top_p * chunk_masses(row, t);
            t = max(t, select<true>(row, g, by_count, target, known ? j.n : kUnknown));
            known = false;   // (the other filter's place is not)
        }
    }
    if (j.least > 0) t = max(t, j.least);
    else if (j.min_p > 0.0) t = max(t, least_weight(row.m, row.c, j.min_p));
    const double kept = chunk_masses(row, t);
    if (j.tok) {
        const int v = draw(row, t, j.u);
        if (tid == 0) *j.tok = v;
    }
    if (j.over)
        row.each([&](float v, int i) {
            if (argmax_key(v, i) >= t) store_agent(j.over + i, (float)(weight(v, row.m, row.c, s.exp2) * (1.0 / kept)));
        });
    if (tid == 0) *j.out = RowResult{t, kept, 0.0, 0.f, 0.f, row.m, kRowDone};
}
template <typename T>
__device__ __forceinline__ SolveJob<T> solve_job(const SampleArgs &a, const Row<T> &row, int r) {
    const int b = r / a.T, k = a.top_k[b];
    return SolveJob<T>{row, a.top_p[b], a.min_p[b], a.tok ? (double)a.u[r] : 0.0, a.tok ? a.tok + r : nullptr,
                       a.probs && k > 0 && k <= kListK ? a.probs + (size_t)r * a.V : nullptr, a.rows + r, k,
                       Range{0, 0, 0.0, 0.0}, -1.0, 0, kUnknown, a.records + (size_t)r * a.n_chunks * kSampleRecord};
}

// A row with a large top-k and a top-p (whose target is known only behind top-k), from its chunks' bins (c_max and
// c_unit are set), by its last workgroup: for each filter the bin in which it ends, that bin's entries from the row, and
// among them the place; then the draw.
template <typename T>
__device__ __noinline__ void cut_row(const SolveJob<T> job) {
    SampleLds &s = lds();
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Row<T> row = job.row;
    const char *rec0 = job.rec0;
    const uint64_t least = job.least;
    double total = 0.0;
    const float rb = floorf(row.m * 8.f), low = (rb - (float)(kBins - 1)) * 0.125f;   // low: the bins' end
    const uint64_t bits = (uint64_t)0xffffffffu << 32;
    uint64_t t = least;
    float lo, hi = -INFINITY;   // the values listed
    int all = 0;
    for (int pass = 0; pass < 3; ++pass) {   // top-k, top-p of its mass, and where another key than top-p's is the end, its bin
        const bool by_count = pass == 0;
        double target = -1.0;
        if (pass < 2) {
            target = by_count ? (double)job.top_k : job.top_p * total;
            // the row's bins: bin j of a chunk whose maximum lies d bins lower is the row's j + d
            const int j = tid & (kBins - 1);
            double w = 0.0;
            uint32_t n = 0;
            #pragma unroll 4
            for (int k = tid / kBins; k < row.n_chunks; k += kThreads / kBins) {
                const float top = s.c_max[k], d = rb - floorf(top * 8.f);
                const bool in = top > -INFINITY && (float)j >= d;
                const char *q = rec0 + (size_t)k * kSampleRecord + kHead;
                const int jc = in ? j - (int)d : 0;
                if (by_count) n += in ? get32(q + 8 * kBins + 4 * jc) : 0;
                else w += in ? bits_f64(get64(q + 8 * jc)) * s.c_unit[k] : 0.0;
            }
            s.list[tid] = f64_bits(by_count ? (double)n : w);
            __syncthreads();
            if (wave == 0) {
                auto bin = [&](int i) {
                    return bits_f64(s.list[i]) + bits_f64(s.list[i + kBins]) + bits_f64(s.list[i + 2 * kBins]) + bits_f64(s.list[i + 3 * kBins]);
                };
                double before;
                const int i = first_reaching(bin, target, &before);
                if (lane == 0) s.num[0] = before + bin(i) >= target ? i : kBins;   // kBins: reached below the last bin
            }
            __syncthreads();
            const int i = uniform(s.num[0]);
            lo = i < kBins ? (rb - (float)i) * 0.125f : -3.402823466e38f;   // (an entry of -inf has no mass)
            hi = (rb - (float)(i - 1)) * 0.125f;
            // where min-p ends above top-p's bin, only that counts
            if (key_value(least) >= hi && !by_count) continue;
        } else {
            const float tv = key_value(t);
            if (tv < hi) break;
            lo = tv;
            hi = fmaxf((floorf(tv * 8.f) + 1.f) * 0.125f, low);
        }
        // what lies above the range, chunk by chunk (a wave a chunk), and the entries in it
        __syncthreads();
        if (tid == 0) s.num[1] = 0, s.num[3] = 0;
        __syncthreads();
        for (int c = wave; c < row.n_chunks; c += kThreads / 64) {
            const float ups = floorf(s.c_max[c] * 8.f) - hi * 8.f;   // the last bin above
            const char *q = rec0 + (size_t)c * kSampleRecord + kHead;
            double sum = 0.0;
            uint32_t n = 0;
            #pragma unroll
            for (int i = 0; i < kBins / 64; ++i) {
                const bool up = (float)(lane + 64 * i) <= ups;
                const double y = bits_f64(get64(q + 8 * (lane + 64 * i)));
                sum += up ? y : 0.0;
                if (by_count) {
                    const uint32_t z = get32(q + 8 * kBins + 4 * (lane + 64 * i));
                    n += up ? z : 0;
                }
            }
            sum = wave_sum_f64(sum);
            if (by_count) n = (uint32_t)group_sum<64>((float)n);   // (exact: at most 8192)
            if (lane == 0) {
                s.c_mass[c] = sum * s.c_unit[c];
                if (by_count) atomicAdd(&s.num[1], (int)n);
            }
        }
        row.each([&](float x, int i) {
            if (x >= lo && x < hi) {
                const int p = atomicAdd(&s.num[3], 1);
                if (p < kList) s.list[p] = argmax_key(x, i);
            }
        });
        __syncthreads();
        all = uniform(s.num[3]);
        double above = 0.0;
        #pragma unroll
        for (int i = 0; i < 2; ++i)
            if (lane + 64 * i < row.n_chunks) above += s.c_mass[lane + 64 * i];
        above = uniform(__longlong_as_double((long long)wave_fold_u64(f64_bits(above), add_f64_bits)));
        Range g = {argmax_key(lo, 0) & bits, (argmax_key(hi, 0) & bits) - 1, above, (double)uniform(s.num[1])};
        if (all > kList) {
            SolveJob<T> rest = job;
            if (pass == 0) rest.range = g, rest.target = target, rest.n = all;   // (else top-k's place is behind)
            solve_row<T>(rest);
            return;
        }
        if (target >= 0.0) {
            t = max(t, select<false>(row, g, by_count, target, all));
            if (by_count) total = g.mass;   // at and above the k-th
        }
    }
    // each chunk's kept mass: above the range, and the listed entries that stay
    uint64_t *fix = s.mass, *rest = s.mass + kSampleMaxChunks;   // (the search's, which is over)
    __syncthreads();
    if (tid < 2 * kSampleMaxChunks) fix[tid] = 0;
    __syncthreads();
    #pragma unroll 1
    for (int i = tid; i < all; i += kThreads) {
        const uint64_t k = s.list[i];
        if (k >= t) {
            const double w = weight(key_value(k), row.m, row.c, s.exp2);
            atomicAdd((unsigned long long *)&fix[key_index(k) / kSampleChunk], units(w, 1.0 / kBinUnit));
            atomicAdd((unsigned long long *)&rest[key_index(k) / kSampleChunk], (unsigned long long)rest_units(w, 1.0 / kBinUnit));
        }
    }
    __syncthreads();
    if (tid < row.n_chunks) s.c_mass[tid] += (double)fix[tid] * kBinUnit + (double)(int64_t)rest[tid] * (kBinUnit * 0x1p-43);
    __syncthreads();
    double kept = 0.0;
    #pragma unroll
    for (int i = 0; i < 2; ++i)
        if (lane + 64 * i < row.n_chunks) kept += s.c_mass[lane + 64 * i];
    kept = uniform(__longlong_as_double((long long)wave_fold_u64(f64_bits(kept), add_f64_bits)));
    if (job.tok) {
        const int v = draw(row, t, job.u);
        if (tid == 0) *job.tok = v;
    }
    if (tid == 0) *job.out = RowResult{t, kept, 0.0, 0.f, 0.f, row.m, kRowDone};
}

// rows whose one filter is min-p: what stays is known from the maximum
__host__ __device__ inline bool min_p_only(int top_k, double top_p, double min_p) { return top_k == 0 && top_p >= 1.0 && min_p > 0.0; }
// rows that the first launch ends though their candidates are not listed
__host__ __device__ inline bool both_filters(int top_k, double top_p) { return top_k > kListK && top_p < 1.0; }

template <typename T>
__global__ __launch_bounds__(kThreads, 8) void sample_kernel(const SampleArgs a) {
    SampleLds &s = lds();
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int rows = a.B * a.T, chunk = blockIdx.x / rows, r = blockIdx.x - chunk * rows, b = r / a.T;
    const int top_k = a.top_k[b];
    const bool listed = top_k > 0 && top_k <= kListK;
    const bool floored = min_p_only(top_k, a.top_p[b], a.min_p[b]);
    const bool binned = !listed && !floored && (top_k > 0 || a.top_p[b] < 1.0);
    Row<T> row = row_of<T>(a, r);
    char *rec0 = a.records + (size_t)r * a.n_chunks * kSampleRecord, *rec = rec0 + (size_t)chunk * kSampleRecord;

    // ---- this chunk: maximum, NaN ----
    const int e0 = chunk * kSampleChunk + tid * kRun;
    float x[kRun];
    load_run(row.x, e0, a.V, x);
    if (tid < kTable) s.exp2[tid] = kExp2.v[tid];
    float mine = -INFINITY;
    bool nan = false;
    #pragma unroll
    for (int i = 0; i < kRun; ++i) {
        nan |= x[i] != x[i];
        mine = fmaxf(mine, x[i]);
    }
    float m = group_max<64>(mine);
    nan = __any(nan);
    if (lane == 0) {
        s.fmx[wave] = m;
        s.flag[wave] = nan ? kNaN : 0;
    }
    if (tid < kBins) s.mass[tid] = 0, s.cnt[tid] = 0;
    if (tid == 0) s.num[0] = 0, s.num[1] = 0;
    if (listed && a.probs) zero_run(a.probs + (size_t)r * a.V, e0, a.V);
    __syncthreads();
    m = uniform(group_max<16>(s.fmx[lane & 15]));
    uint32_t flags = __any(s.flag[lane & 15] != 0) ? kNaN : 0;
    const float mb = floorf(m * 8.f);
    if (!(fabsf(m) < 0x1p20f)) flags |= kNoBins;   // (bins of 1/8 are exact below 2^21)
    float edge = INFINITY;
    uint32_t n_out = 0;
    double mass = 0.0;
    if (listed) {
        if (!(flags & kNoBins)) {
            // the threads' maxima by bins; where fewer than top_k of them are in the bins, every entry
            int at;
            for (int every = 0;; every = 1) {
                if (!every) {
                    const float j = mb - floorf(mine * 8.f);
                    if (j < (float)kBins) atomicAdd(&s.cnt[(int)j], 1u);
                } else {
                    #pragma unroll
                    for (int i = 0; i < kRun; ++i) {
                        const float j = mb - floorf(x[i] * 8.f);
                        if (j < (float)kBins && x[i] != mine) atomicAdd(&s.cnt[(int)j], 1u);   // (fewer than there are: harmless)
                    }
                }
                __syncthreads();
                if (wave == 0) {
                    double before;
                    const int j = first_reaching([&](int i) { return (double)s.cnt[i]; }, (double)top_k, &before);
                    if (lane == 0) s.num[2] = before + (double)s.cnt[j] >= (double)top_k ? j : kBins;
                }
                __syncthreads();
                at = s.num[2];
                if (at < kBins || every) break;
            }
            at = min(at, kBins - 1);   // fewer than top_k in the bins: all of them
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
            if (n_out > (uint32_t)kEmit && m - edge > 0x1p-100f) {
                // too many (a flat distribution): by 256 bins from there to the maximum, all entries counted
                wait_vm_stores();   // (other threads write over these keys)
                __syncthreads();
                const float per = 256.f / (m - edge);
                auto place = [&](float v) { return kBins - 1 - min((int)((v - edge) * per), kBins - 1); };   // (falls with v)
                if (tid < kBins) s.cnt[tid] = 0;
                if (tid == 0) s.num[0] = 0;
                __syncthreads();
                #pragma unroll
                for (int i = 0; i < kRun; ++i)
                    if (x[i] >= edge) atomicAdd(&s.cnt[place(x[i])], 1u);
                __syncthreads();
                if (wave == 0) {
                    double before;
                    const int j = first_reaching([&](int i) { return (double)s.cnt[i]; }, (double)top_k, &before);
                    if (lane == 0) s.num[2] = j;
                }
                __syncthreads();
                #pragma unroll
                for (int i = 0; i < kRun; ++i)
                    if (x[i] >= edge && place(x[i]) <= s.num[2]) {
                        const int p = atomicAdd(&s.num[0], 1);
                        if (p < kEmit) put64(rec + kHead + 8 * p, argmax_key(x[i], e0 + i));
                    }
                __syncthreads();
                n_out = (uint32_t)s.num[0];
            }
            if (n_out > (uint32_t)kEmit) flags |= kLeft, edge = INFINITY, n_out = 0;
            else if (s.num[1]) flags |= kLeft;
        } else if (m > -INFINITY) {
            flags |= kLeft;   // (edge +inf) candidates only by the row's last workgroup
        }
    } else if (floored) {
        // what min-p leaves against this chunk's maximum (the row's leaves no more), with a margin for the roundings here
        const double bound = (double)m + a.drop[b];
        edge = (float)(bound - 1e-6 * (fabs((double)m) + fabs(a.drop[b])) - 1e-40);
        if (fabsf(m) < 1e30f && edge > -1e30f) {
            #pragma unroll
            for (int i = 0; i < kRun; ++i)
                if (x[i] >= edge) {
                    const int p = atomicAdd(&s.num[0], 1);
                    if (p < kEmit) put64(rec + kHead + 8 * p, argmax_key(x[i], e0 + i));
                }
            __syncthreads();
            n_out = (uint32_t)s.num[0];
            if (n_out > (uint32_t)kEmit) flags |= kLeft, edge = m, n_out = 0;   // (none of them may stay in the row)
        } else if (m > -INFINITY) {
            flags |= kLeft, edge = INFINITY;   // by the row's last workgroup
        }
    } else {
        if (m == INFINITY) {
            #pragma unroll
            for (int i = 0; i < kRun; ++i) mass += x[i] == m ? 1.0 : 0.0;
        } else if (m > -INFINITY) {   // (what is past the row's end is -inf: as good as 0)
            const Series terms = series();
            double md = (double)m, c = row.c;
            asm volatile("" : "+v"(md), "+v"(c));   // (kept at hand)
            const uint32_t step = bin_step(row.c);
            auto weigh = [&](auto bins, auto count) {
                #pragma unroll
                for (int i = 0; i < kRun; ++i) {
                    const double w = weight_finite(x[i], md, c, s.exp2, terms);
                    mass += w;
                    if constexpr (bins.value) {
                        const float below = mb - floorf(x[i] * 8.f);
                        if (below < (float)kBins) {   // (not -inf)
                            const int j = (int)below;
                            atomicAdd((unsigned long long *)&s.mass[j], units(w, bin_per(j, step)));
                            if constexpr (count.value) atomicAdd(&s.cnt[j], 1u);
                        }
                    }
                    if (i % 2 == 1) __builtin_amdgcn_sched_barrier(0);   // (few temporaries at a time)
                }
            };
            using Yes = std::true_type;
            using No = std::false_type;
            if (!binned || (flags & kNoBins)) weigh(No(), No());
            else if (top_k > 0) weigh(Yes(), Yes());
            else weigh(Yes(), No());
        }
        // (wave 0 alone needs the sum)
        mass = __longlong_as_double((long long)wave_fold_u64(f64_bits(mass), add_f64_bits));
        if (lane == 0) s.part[wave] = mass;
        __syncthreads();
        if (wave == 0) mass = __longlong_as_double((long long)wave_fold_u64(lane < 16 ? f64_bits(s.part[lane]) : 0, add_f64_bits));
        if (binned && tid < kBins) {
            put64(rec + kHead + 8 * tid, f64_bits((double)s.mass[tid] * bin_unit(tid, bin_step(row.c))));
            if (top_k > 0)
                __hip_atomic_store(reinterpret_cast<uint32_t *>(rec + kHead + 8 * kBins) + tid, s.cnt[tid], __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (tid == 0) {
        put64(rec, (uint64_t)__float_as_uint(m) | (uint64_t)flags << 32);
        put64(rec + 8, (uint64_t)__float_as_uint(edge) | (uint64_t)n_out << 32);
        put64(rec + 16, f64_bits(mass));
    }
    if (listed && tid < kBins) s.cnt[tid] = 0;   // (its last reader is behind a barrier)
    if (!row_last(a, r, a.n_chunks, s)) return;

    // ---- the row's last workgroup ----
    const Heads h = load_heads(rec0, a.n_chunks);
    m = row.m = h.m;
    RowResult out = {0, 0, 0.0, 0.f, 0.f, m, kRowDone};
    if (h.nan || m == -INFINITY) {   // no distribution
        if (tid == 0) {
            if (a.tok) a.tok[r] = -1;
            out.mode = kRowNone;
            a.rows[r] = out;
        }
        return;
    }
    if (listed) {
        // What a chunk left out lies below its edge: harmless where the k-th candidate does not.
        bool complete = h.total <= kList && !(h.worst == INFINITY);
        if (complete) {
            const float rb = floorf(m * 8.f);
            load_list(s, rec0, a.n_chunks, h.n, [&](uint64_t k) {
                atomicAdd(&s.cnt[(int)fminf(rb - floorf(key_value(k) * 8.f), kBins - 1)], 1u);
            });
            __syncthreads();
            if (h.left) {
                int above = 0;
                for (int i = tid; i < h.total; i += kThreads) above += key_value(s.list[i]) >= h.worst ? 1 : 0;
                complete = block_sum((double)above, s.part) >= (double)top_k;
            }
        }
        if (complete) {
            if (tid == 0) a.rows[r] = out;
            finish_list(row, a, b, r, h.total);
            return;
        }
        solve_row<T>(solve_job(a, row, r));
        return;
    } else if (floored) {
        out.t = least_weight(m, row.c, a.min_p[b]);
        if (h.total > kList || (h.left && h.worst >= key_value(out.t))) {
            SolveJob<T> job = solve_job(a, row, r);
            job.least = out.t;
            solve_row<T>(job);
            return;
        }
        load_list(s, rec0, a.n_chunks, h.n, [](uint64_t) {});
        if (tid < a.n_chunks) s.c_mass[tid] = 0.0;
        __syncthreads();
        out.mass = add_listed(row, h.n, out.t);
        if (a.tok) {
            const int v = draw(row, out.t, (double)a.u[r]);
            if (tid == 0) a.tok[r] = v;
        }
    } else {
        // the chunks' masses against the row's maximum
        double cm[2];
        #pragma unroll
        for (int i = 0; i < 2; ++i) cm[i] = h.max[i] == -INFINITY ? 0.0 : h.mass[i] * weight(h.max[i], m, row.c, s.exp2);
        if (wave == 0) {
            #pragma unroll
            for (int i = 0; i < 2; ++i)
                if (lane + 64 * i < a.n_chunks) {
                    s.c_mass[lane + 64 * i] = cm[i];
                    s.c_max[lane + 64 * i] = h.max[i];
                    s.c_unit[lane + 64 * i] = h.max[i] == -INFINITY ? 0.0 : weight(h.max[i], m, row.c, s.exp2);
                }
        }
        out.mass = __longlong_as_double((long long)wave_fold_u64(f64_bits(cm[0] + cm[1]), add_f64_bits));
        __syncthreads();
        const double min_p = a.min_p[b];
        if (min_p > 0.0) out.t = least_weight(m, row.c, min_p);   // so far: no entry below it stays
        if (binned) {
            if (both_filters(top_k, a.top_p[b])) {
                SolveJob<T> job = solve_job(a, row, r);
                job.least = out.t;
                if (h.no_bins) solve_row<T>(job);
                else cut_row<T>(job);
                return;
            }
            if (h.no_bins) {
                out.mode = kRowSlow;
            } else {
                out.mode = kRowCut;
                const float rb = floorf(m * 8.f), low = (rb - (float)(kBins - 1)) * 0.125f;   // low: the bins' end
                out.target = top_k > 0 ? (double)top_k : a.top_p[b] * out.mass;
                // the row's bins: bin j of a chunk whose maximum lies d bins lower is the row's j + d
                const int j = tid & (kBins - 1);
                double w = 0.0;
                uint32_t n = 0;
                #pragma unroll 4
                for (int k = tid / kBins; k < a.n_chunks; k += kThreads / kBins) {
                    const float top = s.c_max[k], d = rb - floorf(top * 8.f);
                    const bool in = top > -INFINITY && (float)j >= d;
                    const char *q = rec0 + (size_t)k * kSampleRecord + kHead;
                    const int jc = in ? j - (int)d : 0;
                    const double x = bits_f64(get64(q + 8 * jc));
                    w += in ? x * s.c_unit[k] : 0.0;
                    if (top_k > 0) {
                        const uint32_t y = __hip_atomic_load(reinterpret_cast<uint32_t *>(const_cast<char *>(q) + 8 * kBins + 4 * jc),
                                                             __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        n += in ? y : 0;
                    }
                }
                s.list[tid] = f64_bits(top_k > 0 ? (double)n : w);
                __syncthreads();
                if (wave != 0) return;
                auto bin = [&](int i) {
                    return bits_f64(s.list[i]) + bits_f64(s.list[i + kBins]) + bits_f64(s.list[i + 2 * kBins]) + bits_f64(s.list[i + 3 * kBins]);
                };
                double before;
                const int i = first_reaching(bin, out.target, &before);
                const bool in = before + bin(i) >= out.target;   // else it is reached below the last bin
                out.lo = in ? (rb - (float)i) * 0.125f : -3.402823466e38f;   // (an entry of -inf has no mass)
                out.hi = in ? (rb - (float)(i - 1)) * 0.125f : low;
                // where min-p ends above it, only that counts: its bin's entries down to it
                const float tv = key_value(out.t);
                if (out.t > 0 && tv >= out.hi) {
                    out.lo = tv;
                    out.hi = fmaxf((floorf(tv * 8.f) + 1.f) * 0.125f, low);
                    out.target = -1.0;
                }
            }
        } else if (a.tok) {
            const int v = draw(row, 0, (double)a.u[r]);
            if (tid == 0) a.tok[r] = v;
        }
    }
    if (tid == 0) a.rows[r] = out;
}

// The second launch: the entries of each undecided row's range, the mass above it, the cut, and the draw.
template <typename T>
__global__ __launch_bounds__(kThreads, 8) void sample_cut_kernel(const SampleArgs a) {
    SampleLds &s = lds();
    const int tid = threadIdx.x, lane = tid & 63;
    const int rows = a.n_cut * a.T, part = blockIdx.x / rows, i_cut = blockIdx.x - part * rows, b = a.cut[i_cut / a.T];
    const int r = b * a.T + i_cut % a.T, chunk0 = part * a.cut_per_group, chunk1 = min(chunk0 + a.cut_per_group, a.n_chunks);
    RowResult res = a.rows[r];
    res.t = uniform(res.t), res.target = uniform(res.target), res.lo = uniform(res.lo), res.hi = uniform(res.hi);
    res.m = uniform(res.m), res.mode = uniform(res.mode);
    if (res.mode != kRowCut && (res.mode != kRowSlow || part > 0)) return;
    Row<T> row = row_of<T>(a, r);
    row.m = res.m;
    if (tid < kTable) s.exp2[tid] = kExp2.v[tid];
    if (res.mode == kRowSlow) {
        solve_row<T>(solve_job(a, row, r));
        return;
    }
    char *rec0 = a.records + (size_t)r * a.n_chunks * kSampleRecord;
    Run<T> next;
    next.load(row.x, chunk0 * kSampleChunk + tid * kRun, a.V);
    for (int chunk = chunk0; chunk < chunk1; ++chunk) {
        const int e0 = chunk * kSampleChunk + tid * kRun;
        float x[kRun];
        next.unpack(x);
        if (chunk + 1 < chunk1) next.load(row.x, e0 + kSampleChunk, a.V);   // in flight meanwhile
        char *rec = rec0 + (size_t)chunk * kSampleRecord;
        // what lies above the range: the chunk's bins up to there (read before the keys take their place)
        double q = 0.0;
        uint32_t n_above = 0;
        float top = 0.f;
        if (tid < 64) {
            top = __uint_as_float((uint32_t)get64(rec));
            const float ups = floorf(top * 8.f) - res.hi * 8.f;   // the last bin above
            #pragma unroll
            for (int i = 0; i < kBins / 64; ++i) {
                const double y = bits_f64(get64(rec + kHead + 8 * (lane + 64 * i)));
                const bool up = (float)(lane + 64 * i) <= ups;
                q += up ? y : 0.0;
                if (a.top_k[b] > 0) {
                    const uint32_t z = __hip_atomic_load(reinterpret_cast<uint32_t *>(rec + kHead + 8 * kBins) + lane + 64 * i, __ATOMIC_RELAXED,
                                                         __HIP_MEMORY_SCOPE_AGENT);
                    n_above += up ? z : 0;
                }
            }
            q = wave_sum_f64(q);
            n_above = (uint32_t)group_sum<64>((float)n_above);   // (exact: at most 8192)
        }
        if (tid == 0) s.num[0] = 0;
        __syncthreads();
        #pragma unroll
        for (int i = 0; i < kRun; ++i)
            if (x[i] < res.hi && x[i] >= res.lo && e0 + i < a.V) {
                const int p = atomicAdd(&s.num[0], 1);
                if (p < kEmit) put64(rec + kHead + 8 * p, argmax_key(x[i], e0 + i));
            }
        __syncthreads();
        if (tid == 0) {
            put64(rec, (uint64_t)(uint32_t)s.num[0] | (uint64_t)n_above << 32);
            put64(rec + 16, f64_bits(q > 0.0 ? q * weight(top, res.m, row.c, s.exp2) : 0.0));
        }
        __syncthreads();   // (the count is read)
    }
    if (!row_last(a, r, a.cut_groups, s)) return;

    // ---- the row's last workgroup ----
    uint32_t n[2];
    float total = 0.f;
    double mass = 0.0, count = 0.0;
    bool over = false;
    #pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool in = lane + 64 * i < a.n_chunks;
        const uint64_t h0 = in ? get64(rec0 + (size_t)(lane + 64 * i) * kSampleRecord) : 0;
        const double up = in ? bits_f64(get64(rec0 + (size_t)(lane + 64 * i) * kSampleRecord + 16)) : 0.0;
        n[i] = (uint32_t)h0;
        over |= n[i] > (uint32_t)kEmit;
        total += (float)n[i];
        mass += up;
        count += (double)(uint32_t)(h0 >> 32);
        if (tid < 64 && in) {
            s.c_mass[lane + 64 * i] = up;
        }
    }
    const int all = uniform((int)group_sum<64>(total));
    mass = uniform(__longlong_as_double((long long)wave_fold_u64(f64_bits(mass), add_f64_bits)));
    count = uniform(__longlong_as_double((long long)wave_fold_u64(f64_bits(count), add_f64_bits)));
    const uint64_t bits = (uint64_t)0xffffffffu << 32;
    Range g = {argmax_key(res.lo, 0) & bits, (argmax_key(res.hi, 0) & bits) - 1, mass, count};
    if (__any(over) || all > kList) {
        SolveJob<T> job = solve_job(a, row, r);
        job.range = g;
        job.target = res.target;
        job.least = res.t;
        job.n = all;
        solve_row<T>(job);
        return;
    }
    load_list(s, rec0, a.n_chunks, n, [](uint64_t) {});
    if (tid == 0) s.num[3] = all;
    __syncthreads();
    uint64_t t = res.t;
    if (res.target >= 0.0) {
        t = max(t, select<false>(row, g, a.top_k[b] > 0, res.target, all));
    }
    const double kept = add_listed(row, n, t);   // (above the range, and the listed entries that stay)
    if (a.tok) {
        const int v = draw(row, t, (double)a.u[r]);
        if (tid == 0) a.tok[r] = v;
    }
    if (tid == 0) {
        RowResult out = res;
        out.t = t;
        out.mass = kept;
        out.mode = kRowDone;
        a.rows[r] = out;
    }
}

// The third launch: the distributions of the rows that were not finished from their list.
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_emit_kernel(const SampleArgs a) {
    const int tid = threadIdx.x;
    const int rows = a.n_emit * a.T, chunk = blockIdx.x / rows, i_emit = blockIdx.x - chunk * rows, b = a.emit[i_emit / a.T];
    const int r = b * a.T + i_emit % a.T;
    const int e0 = chunk * kSampleChunk + tid * kRun;
    const RowResult res = a.rows[r];
    float x[kRun], p[kRun];
    load_run(reinterpret_cast<const T *>(a.logits) + (size_t)r * a.V, e0, a.V, x);
    __shared__ double table[kTable];
    if (tid < kTable) table[tid] = kExp2.v[tid];
    __syncthreads();
    const float tv = key_value(res.t);   // the row has no NaN
    const uint32_t ti = (uint32_t)key_index(res.t);   // (a bound of values: past every index)
    const bool any = res.mode == kRowDone;
    const double c = a.c[b], inv = 1.0 / res.mass;
    #pragma unroll
    for (int i = 0; i < kRun; ++i) {
        const bool stays = any && (res.t == 0 || x[i] > tv || (x[i] == tv && (uint32_t)(e0 + i) <= ti));
        p[i] = 0.f;
        if (__any(stays)) p[i] = stays ? (float)(weight(x[i], res.m, c, table) * inv) : 0.f;
    }
    store_run(a.probs + (size_t)r * a.V, e0, a.V, p);
}

// ------------------------------------------------------------------ host ----

size_t sample_ws_bytes(int B, int T, int V) {
    const size_t rows = (size_t)B * T, chunks = ((size_t)V + kSampleChunk - 1) / kSampleChunk;
    return kCounterRegionBytes + align256(rows * sizeof(RowResult)) + rows * chunks * kSampleRecord;
}

template <typename T>
static hipError_t launch_sample_t(const SampleArgs &a, hipStream_t st) {
    const unsigned T_ = (unsigned)a.T;
    hipLaunchKernelGGL((sample_kernel<T>), dim3(a.B * T_ * a.n_chunks), dim3(kThreads), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.n_cut > 0) {
        hipLaunchKernelGGL((sample_cut_kernel<T>), dim3(a.n_cut * T_ * a.cut_groups), dim3(kThreads), 0, st, a);
        e = hipGetLastError();
    }
    if (e == hipSuccess && a.n_emit > 0) {
        hipLaunchKernelGGL((sample_emit_kernel<T>), dim3(a.n_emit * T_ * a.n_chunks), dim3(kThreads), 0, st, a);
        e = hipGetLastError();
    }
    return e;
}

// The second launch's chunks to a workgroup: as many as leave every workgroup resident at once, so that one's loads run
// under another's emission (28 rows of 16 chunks 28.8 -> 25.6 us, 80 rows 28.7 -> 27.5).
static void split_rows(int rows, int n_chunks, int *per_group, int *groups) {
    *per_group = std::min((int)(((int64_t)rows * n_chunks + kResident - 1) / kResident), n_chunks);
    *groups = (n_chunks + *per_group - 1) / *per_group;
}

hipError_t launch_sample(const SampleArgs &args, int dtype, hipStream_t st) {
    SampleArgs a = args;
    // rows with a small top-k, with top-k and top-p, or with min-p alone are finished in the first launch; plain ones have
    // nothing to cut
    a.n_cut = a.n_emit = 0;
    for (int b = 0; b < a.B; ++b) {
        if (a.top_k[b] > 0 && a.top_k[b] <= kListK) continue;
        if ((a.top_k[b] > 0 || a.top_p[b] < 1.0) && !both_filters(a.top_k[b], a.top_p[b])) a.cut[a.n_cut++] = (uint8_t)b;
        if (a.probs) a.emit[a.n_emit++] = (uint8_t)b;
    }
    split_rows(std::max(a.n_cut, 1) * a.T, a.n_chunks, &a.cut_per_group, &a.cut_groups);
    return dtype == MAD_BF16 ? launch_sample_t<bf16_t>(a, st) : launch_sample_t<float>(a, st);
}

}  // namespace mad

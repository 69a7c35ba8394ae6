// logprobs.hip -- log probabilities of given tokens, ranks, entropies and the
// most probable alternatives, from the logits in one read.
//
// Mathematics, for a row's logits x, c = log2 e / temperature, M near max x c:
//   d_v = x_v c - M,  e_v = 2^d_v,  s = sum e,  u = sum e d
//   log p_v = ln 2 * (d_v - log2 s);   entropy = ln 2 * (log2 s - u / s)
//   rank = entries above the token's logit, and equal ones before it.
// M is max x times c as fp32 rounds it, so that d is one fused operation with one
// rounding whatever the logits' offset.  A thread keeps M, s and u of what it has
// seen, raises M at most once per step of 16 entries, and sums within a step in
// fp32, over steps and threads in fp64.
//
// The first top_n of the order: each wave keeps its largest 64 keys (value, then
// index) sorted, one to a lane.  An entry above the wave's top_n-th, and above what
// any wave of the workgroup has as its top_n-th, is put in by a ballot (its place)
// and a shift by one lane; few entries of a row come that far.  Before there are
// top_n: the top_n-th largest of 64 maxima of disjoint groups (lane l of every
// wave), which top_n entries at least reach.  The same bound, of the lanes' maxima,
// thins a step in which many entries are above the list (a rising row).  At the end an entry's place
// among the waves' lists is counted by binary searches.
//
// Work: a workgroup takes a run of a row's chunks of 8192, its waves 1024 of each
// and no barrier between the first chunk and the last; with few rows, more
// workgroups to a row, whose results the last of them to arrive joins.
#include "mad_device.h"
#include "mad_internal.h"

namespace mad {

namespace {

constexpr int kWg = 512, kEntries = 16;   // threads, entries of a thread and step
static_assert(kWg * kEntries == kLogprobChunk, "");
constexpr int kMany = 64;                 // entries of a step above the list that are thinned first
constexpr float kNear = 0x1p26f;          // |m| c below which M is m c as rounded

// Sums relative to M, which m alone tells: below kNear m c as fp32 rounds it (within 2 of m c: d <= 2), else m c exactly, formed
// in differences only.
struct Stats {
    double s, u;
    float m;        // the largest entry
};
// M of a less M of b (a <= b)
__device__ __forceinline__ float lower(float a, float b, float c) {
    #pragma clang fp contract(off)   // each M as it was rounded
    const float ma = a * c, mb = b * c;
    if (!(fabsf(ma) < kNear)) return (a - b) * c;   // (far below any near b)
    return fabsf(mb) < kNear ? ma - mb : fmaf(-b, c, ma);
}

__device__ __forceinline__ uint32_t order_of(float x) { return (uint32_t)(argmax_key(x, 0) >> 32); }
__device__ __forceinline__ float value_of(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint64_t read_lane_u64(uint64_t v, int l) {
    return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), l) << 32) |
           (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, l);
}
__device__ __forceinline__ uint64_t max_u64(uint64_t a, uint64_t b) { return a > b ? a : b; }

// the n-th largest of the lanes' values
__device__ __forceinline__ uint32_t nth_of_lanes(uint32_t g, int n) {
    int above = 0;
    #pragma unroll 8
    for (int l = 0; l < 64; ++l) {
        const uint32_t o = __builtin_amdgcn_readlane(g, l);
        above += o > g || (o == g && l < (int)(threadIdx.x & 63)) ? 1 : 0;
    }
    return __builtin_amdgcn_readlane(g, __builtin_ctzll(__ballot(above == n - 1)));
}

// the lanes' sums together, in every lane
__device__ __forceinline__ Stats wave_join(Stats a, float c) {
    const float m = group_max<64>(a.m);
    const float d = a.m == m ? 0.f : fmaxf(lower(a.m, m, c), -3000.f);
    const double f = (double)__builtin_amdgcn_exp2f(d);
    a.u = wave_sum_f64(f * (a.u + (double)d * a.s));
    a.s = wave_sum_f64(f * a.s);
    a.m = m;
    return a;
}

// the place of x in a list of n keys, the largest first: how many are above
__device__ __forceinline__ int place(const uint64_t *list, int n, uint64_t x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        const bool up = list[mid] > x;
        lo = up ? mid + 1 : lo;
        hi = up ? hi : mid;
    }
    return lo;
}

struct Shared {
    uint64_t list[kLogprobSplits][MAD_MAX_TOP], best[MAD_MAX_TOP];
    uint64_t bound;
    uint32_t group[8][64];
    double s[8], u[8];
    float m[8];
    int above[8], inf[8];
    int last;
};
static_assert(kLogprobSplits >= 8, "a list for each wave");

// The first n of the order among `lists` lists of up to n sorted keys (0: none) into best.
__device__ __forceinline__ void join_lists(Shared &sh, int lists, int n) {
    for (int i = threadIdx.x; i < lists * n; i += kWg) {
        const int l = i / n, k = i - l * n;
        const uint64_t x = sh.list[l][k];
        int at = k;
        for (int o = 0; o < lists; ++o) at += o == l ? 0 : place(sh.list[o], n, x);
        if (x != 0 && at < n) sh.best[at] = x;   // (keys differ: their index is in them)
    }
}

}  // namespace

template <typename T, bool TOP>
__global__ __launch_bounds__(kWg, 6) void logprobs_kernel(const LogprobArgs a) {
    constexpr int VEC = Elem<T>::VEC, NV = kEntries / VEC;
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = blockIdx.x / a.splits, split = blockIdx.x - row * a.splits;
    const int b = row / a.T, t = row - b * a.T, n = a.top_n, V = a.V;
    const T *x0 = reinterpret_cast<const T *>(a.logits) + b * a.seq + t * a.row;
    const int skew = (int)((uintptr_t)x0 & 15) / (int)sizeof(T);   // entries of another row in the first 16 bytes
    const uint4 *base = reinterpret_cast<const uint4 *>(x0 - skew);
    const int vecs = (V + skew + VEC - 1) / VEC;
    const float c = a.c[b];
    const int chunk0 = (int)((int64_t)a.n_chunks * split / a.splits), chunk1 = (int)((int64_t)a.n_chunks * (split + 1) / a.splits);

    uint4 raw[NV];
    auto load = [&](int chunk) {
        #pragma unroll
        for (int j = 0; j < NV; ++j) raw[j] = base[min((chunk * NV + j) * kWg + tid, vecs - 1)];
    };
    load(chunk0);
    const int tok = a.tok ? a.tok[row] : -1;
    const bool has = tok >= 0 && tok < V;
    const float xt = has ? Elem<T>::load1(x0 + tok) : INFINITY;

    Stats st = {0.0, 0.0, -INFINITY};
    int above = 0, inf = 0;      // (of the wave)
    uint64_t key = 0;            // lane i: the wave's i-th largest
    uint64_t bound = 0;          // only keys above it count
    if (TOP && tid == 0) sh.bound = 0;

    for (int chunk = chunk0; chunk < chunk1; ++chunk) {
        float x[kEntries];
        #pragma unroll
        for (int j = 0; j < NV; ++j) {
            float f[VEC];
            unpack16(raw[j], f, T());
            #pragma unroll
            for (int e = 0; e < VEC; ++e) x[j * VEC + e] = f[e];
        }
        if (chunk + 1 < chunk1) load(chunk + 1);
        const int first = chunk * kLogprobChunk - skew;   // the chunk's first entry
        const bool edge = first < 0 || first + kLogprobChunk > V;
        auto index = [&](int i) { return first + ((i / VEC) * kWg + tid) * VEC + i % VEC; };
        auto inside = [&](int i) { return !edge || (uint32_t)index(i) < (uint32_t)V; };
        if (edge) {
            #pragma unroll
            for (int i = 0; i < kEntries; ++i) x[i] = inside(i) ? x[i] : -INFINITY;
        }
        float m = x[0];
        #pragma unroll
        for (int i = 1; i < kEntries; ++i) m = fmaxf(m, x[i]);

        const float mn = fmaxf(st.m, m), M = mn * c;
        float s = 0.f, u = 0.f;
        if (fabsf(M) < kNear) {
            #pragma unroll
            for (int i = 0; i < kEntries; ++i) {
                const float d = fmaf(x[i], c, -M), e = __builtin_amdgcn_exp2f(d);
                s += e;
                u = fmaf(e, d, u);
            }
            if (!(u == u)) {   // an e of 0 with a d of -inf, or a NaN (which s has too)
                u = 0.f;
                #pragma unroll
                for (int i = 0; i < kEntries; ++i) {
                    const float d = fmaf(x[i], c, -M);
                    u = fmaf(__builtin_amdgcn_exp2f(d), fmaxf(d, -200.f), u);
                }
            }
        } else if (fabsf(mn) < INFINITY) {
            #pragma unroll
            for (int i = 0; i < kEntries; ++i) {
                const float d = (x[i] - mn) * c, e = __builtin_amdgcn_exp2f(d);
                s += e;
                u = fmaf(e, fmaxf(d, -200.f), u);
            }
        }
        if (__any(!(fabsf(mn) < INFINITY))) {   // nothing but -inf, a +inf, or NaN alone
            #pragma unroll
            for (int i = 0; i < kEntries; ++i) {
                inf += __popcll(__ballot(x[i] == INFINITY));
                s = x[i] != x[i] ? __builtin_nanf("") : s;
            }
        }
        if (st.m < mn && mn < INFINITY) {
            const float d = fmaxf(lower(st.m, mn, c), -3000.f), f = __builtin_amdgcn_exp2f(d);
            st.u = (double)f * (st.u + (double)d * st.s);
            st.s *= (double)f;
            st.m = mn;
        }
        st.s += (double)s;
        st.u += (double)u;

        if (has && __any(m >= xt)) {
            #pragma unroll
            for (int i = 0; i < kEntries; ++i)
                above += __popcll(__ballot(x[i] > xt || (x[i] == xt && index(i) < tok && inside(i))));
        }
        if constexpr (TOP) {
            if (chunk == chunk0) {
                sh.group[wave][lane] = order_of(m);
                __syncthreads();
                uint32_t g = 0;
                #pragma unroll
                for (int k = 0; k < 8; ++k) g = max(g, sh.group[k][lane]);
                bound = ((uint64_t)nth_of_lanes(g, n) << 32) - 1;   // (no order is 0)
            } else {
                bound = max_u64(bound, *reinterpret_cast<volatile uint64_t *>(&sh.bound));
            }
            // entries of the bound's value and above (some of that value are not above it); a bound among the NaNs' keys: all
            float xb = value_of(bound);
            if (__any(!(m < xb))) {
                int many = 0;
                #pragma unroll
                for (int i = 0; i < kEntries; ++i) many += __popcll(__ballot(!(x[i] < xb)));
                if (many > kMany && chunk > chunk0) {
                    const uint32_t o = nth_of_lanes(order_of(m), n);
                    bound = max_u64(bound, ((uint64_t)o << 32) - 1);
                    xb = value_of(bound);
                }
                const int at0 = here(tid);   // (the keys are made where they are needed)
                #pragma unroll
                for (int i = 0; i < kEntries; ++i) {
                    if (!__any(!(x[i] < xb))) continue;
                    const int at_i = first + ((i / VEC) * kWg + at0) * VEC + i % VEC;
                    const uint64_t mine = !edge || (uint32_t)at_i < (uint32_t)V ? argmax_key(x[i], at_i) : 0;
                    for (uint64_t left = __ballot(mine > bound); left; left = __ballot(mine > bound) & left & (left - 1)) {
                        const uint64_t y = read_lane_u64(mine, __builtin_ctzll(left));
                        const int at = __popcll(__ballot(key > y));
                        const uint64_t before = dpp_u64<0x138>(key);   // the lane below's (wave_shr 1)
                        key = lane < at ? key : lane == at ? y : before;
                        bound = max_u64(bound, read_lane_u64(key, n - 1));
                    }
                }
                if (lane == 0 && chunk + 1 < chunk1) atomicMax((unsigned long long *)&sh.bound, (unsigned long long)bound);
            }
        }
    }

    // ---- the workgroup's waves together ----
    st = wave_join(st, c);
    if (TOP) sh.list[wave][lane] = key;
    if (lane == 0) {
        sh.s[wave] = st.s;
        sh.u[wave] = st.u;
        sh.m[wave] = st.m;
        sh.above[wave] = above;
        sh.inf[wave] = inf;
    }
    __syncthreads();
    if (TOP) {
        if (tid < n) sh.best[tid] = 0;
        __syncthreads();
        join_lists(sh, 8, n);
        __syncthreads();
    }
    const LogprobRecord *rec = a.records + (size_t)row * a.splits;
    if (wave == 0) {
        st = lane < 8 ? Stats{sh.s[lane & 7], sh.u[lane & 7], sh.m[lane & 7]} : Stats{0.0, 0.0, -INFINITY};
        st = wave_join(st, c);
        above = inf = 0;
        for (int k = 0; k < 8; ++k) {
            above += sh.above[k];
            inf += sh.inf[k];
        }
    }

    if (a.splits > 1) {
        // a record for each workgroup of the row; the last to arrive joins them
        if (wave == 0) {
            LogprobRecord *mine = const_cast<LogprobRecord *>(rec + split);
            if (TOP && lane < n) __hip_atomic_store(&mine->best[lane], sh.best[lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (lane == 0) {
                const uint64_t w[4] = {(uint64_t)__double_as_longlong(st.s), (uint64_t)__double_as_longlong(st.u),
                                       (uint64_t)__float_as_uint(st.m) | (uint64_t)(uint32_t)above << 32, (uint64_t)(uint32_t)inf};
                #pragma unroll
                for (int k = 0; k < 4; ++k)
                    __hip_atomic_store(reinterpret_cast<uint64_t *>(mine) + k, w[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            asm volatile("s_waitcnt vmcnt(0)" : : : "memory");   // the record is out before the arrival
            if (lane == 0) {
                unsigned *cnt = a.counters + (size_t)row * kCounterStride;
                sh.last = arrive(cnt) == (unsigned)a.splits - 1;
                if (sh.last) reset_counter(cnt);
            }
        }
        __syncthreads();
        if (!sh.last) return;
        if (TOP) {
            if (tid < n) sh.best[tid] = 0;
            for (int i = tid; i < a.splits * n; i += kWg) sh.list[i / n][i % n] = load_agent64(&rec[i / n].best[i % n]);
            __syncthreads();
            join_lists(sh, a.splits, n);
            __syncthreads();
        }
        if (wave == 0) {
            uint64_t w[4] = {0, 0, 0xff800000u, 0};
            if (lane < a.splits)
                for (int k = 0; k < 4; ++k) w[k] = load_agent64(reinterpret_cast<const uint64_t *>(rec + lane) + k);
            st = wave_join(Stats{__longlong_as_double((long long)w[0]), __longlong_as_double((long long)w[1]), __uint_as_float((uint32_t)w[2])}, c);
            above = inf = 0;
            for (int k = 0; k < a.splits; ++k) {
                above += __builtin_amdgcn_readlane((int)(w[2] >> 32), k);
                inf += __builtin_amdgcn_readlane((int)(uint32_t)w[3], k);
            }
        }
    }

    // ---- the row's end ----
    if (wave != 0) return;
    const bool none = !(st.s == st.s) || (inf == 0 && st.m == -INFINITY);
    const double ln2 = 0.6931471805599453, nan = __builtin_nan("");
    const double ls = none ? nan : inf > 0 ? log((double)inf) : log(st.s);
    const bool near = fabsf(st.m * c) < kNear;
    auto log_p = [&](float v) {
        if (none) return (float)nan;
        if (inf > 0) return v == INFINITY ? (float)-ls : -INFINITY;
        const double d = near ? (double)v * (double)c - (double)(st.m * c) : ((double)v - (double)st.m) * (double)c;
        return (float)(d * ln2 - ls);
    };
    if (lane == 0) {
        if (a.logp) a.logp[row] = none ? (float)nan : has ? log_p(xt) : -INFINITY;
        if (a.rank) a.rank[row] = none ? -1 : has ? above : V;
        if (a.entropy) a.entropy[row] = (float)(none || inf > 0 ? ls : ls - ln2 * (st.u / st.s));
    }
    if (TOP && lane < n) {
        const uint64_t k = sh.best[lane];
        a.top_tok[(int64_t)row * n + lane] = none ? -1 : key_index(k);
        a.top_logp[(int64_t)row * n + lane] = log_p(value_of(k));
    }
}

size_t logprobs_ws_bytes(int rows, int V) {
    const int splits = logprob_splits(rows, V);
    return kCounterRegionBytes + (splits > 1 ? align256((size_t)rows * splits * sizeof(LogprobRecord)) : 0);
}

template <typename T>
static hipError_t launch_t(const LogprobArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.rows * a.splits)), wg(kWg);
    if (a.top_n > 0) hipLaunchKernelGGL((logprobs_kernel<T, true>), grid, wg, 0, st, a);
    else hipLaunchKernelGGL((logprobs_kernel<T, false>), grid, wg, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_logprobs(const LogprobArgs &a, int dtype, hipStream_t st) {
    return dtype == MAD_BF16 ? launch_t<bf16_t>(a, st) : launch_t<float>(a, st);
}

}  // namespace mad

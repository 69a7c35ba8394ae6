// logprobs.hip -- log probabilities of given tokens, ranks, entropies and the
// most probable alternatives, from the logits in one read.
//
// Mathematics, for a row's logits x, c = log2 e / temperature, M not far from max x c:
//   d_v = x_v c - M,  e_v = 2^d_v,  s = sum e,  u = sum e d
//   log p_v = ln 2 * (d_v - log2 s);   entropy = ln 2 * (log2 s - u / s)
//   rank = entries above the token's logit, and equal ones before it.
// M is some entry times c as fp32 rounds it, so that d is one fused operation with
// one rounding whatever the logits' offset.  A thread keeps M, s and u of what it
// has seen, raises M where a step of 16 (32) entries exceeds it by more than 8 (log2
// units: few steps do), and sums within a step in fp32, over steps and threads in
// fp64.
//
// The first top_n of the order: entries (keys of value, then index) above a bound go
// into their wave's list in LDS.  The first bound is a value that top_n entries of the
// workgroup's first chunk reach: the top_n-th largest of 64 maxima of disjoint
// groups.  A list that grows beyond about 1.5 top_n is cut to its first top_n by
// counting what is above each key; the last that stays is a bound for every wave of
// the workgroup.  A step in which many lanes have entries above the bound (a rising
// row) is thinned first by the bound of its lanes' maxima.  At the end what the lists
// hold above the largest bound is put in order, again by counting.
//
// Work: a workgroup takes a run of a row's chunks of 4096 (8192), its waves a quarter
// of each and no barrier between the first chunk and the last; with few rows, more
// workgroups to a row, whose results the last of them to arrive joins.
//
// What bounds it: many rows, the vector ALU (85 % busy; an entry takes about 7
// instructions, one of them an exponential at half rate, and 3 more where it may be
// above the token's logit); few rows, the chain load - first bound - sums - lists -
// arrival - join, 0.4 to 3.6 us each.
// Rows of which a mask leaves little are slower: a bound that is the mask's value lets
// every lane's equal entries through to the lists' test, and entries of -inf have a
// step's entropy formed again (2048 rows of 128256 with 100 live tokens, bf16: top 1
// 165 - 194 us, top 20 823 - 847, where dense rows take 105 and 128).
// Measured: 2048 rows of 128256, bf16, top 1: 103 - 106 us (5.0 TB/s; from about the
// 20th of calls one behind the other 120), fp32 182 us (5.8 TB/s); 4096 rows of 2000,
// top 5: 29 us, of 12000 41, fp32 46; 80 rows of 128256, fp32, top 5: 19.7 us; one row
// of 50257, top 20: 12.2 us.
#include "mad_device.h"
#include "mad_internal.h"

namespace mad {

namespace {

constexpr int kWg = 256, kWaves = kWg / 64;
constexpr int kMany = 24;                 // lanes with entries above the bound from which on a step is thinned first
constexpr int kFewGroups = 32;            // top_n up to which 64 groups give the first bound, else 256 (fewer entries pass, longer to find)
constexpr int kOwn = 128;                 // a wave's list while it grows
static_assert(MAD_MAX_TOP + 64 <= kOwn, "what a cut leaves, and an entry of each lane");
constexpr int kRecs = (kLogprobSplits + kWaves - 1) / kWaves;   // records that a wave joins
constexpr int kList = kRecs * MAD_MAX_TOP > kOwn ? kRecs * MAD_MAX_TOP : kOwn;
constexpr float kLag = 8.f;               // M is raised where a step's largest x c is above it by more (log2 units)
constexpr float kNear = 0x1p26f;          // |m| c below which M is m c as rounded

// Sums relative to M, which m alone tells: below kNear m c as fp32 rounds it (within 2 of it), else m c exactly, formed
// in differences only.
struct Stats {
    double s, u;
    float m;        // -inf: nothing yet
};
// M of a less M of b (a <= b), one of them rounded where only it is near: logits next to each other lie on both sides of
// the border
__device__ __forceinline__ float lower(float a, float b, float c) {
    #pragma clang fp contract(off)   // each M as it was rounded
    const float ma = a * c, mb = b * c;
    const bool near_a = fabsf(ma) < kNear, near_b = fabsf(mb) < kNear;
    if (near_a) return near_b ? ma - mb : fmaf(-b, c, ma);
    return near_b ? fmaf(a, c, -mb) : (a - b) * c;
}

// the next number below (-inf: itself)
__device__ __forceinline__ float next_below(float x) {
    const uint32_t u = __float_as_uint(x);
    return x == 0.f ? __uint_as_float(0x80000001u) : x == -INFINITY ? x : __uint_as_float(x > 0.f ? u - 1 : u + 1);
}
__device__ __forceinline__ uint32_t order_of(float x) { return (uint32_t)(argmax_key(x, 0) >> 32); }
__device__ __forceinline__ float value_of(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint64_t max_u64(uint64_t a, uint64_t b) { return a > b ? a : b; }

// A value that n of the lanes' values g (G to a lane) reach, n of them at least: the n-th largest but for its low 16 bits
// (for bf16 entries it is that one), bit by bit over the values that still share its upper bits.
template <int G>
__device__ __forceinline__ uint32_t reached_by(const uint32_t (&g)[G], int n) {
    uint64_t in[G];
    #pragma unroll
    for (int k = 0; k < G; ++k) in[k] = ~0ull;
    uint32_t value = 0;
    #pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        uint64_t up[G];
        int many = 0;
        #pragma unroll
        for (int k = 0; k < G; ++k) {
            up[k] = __ballot(g[k] >> bit & 1) & in[k];
            many += __popcll(up[k]);
        }
        const bool has = many >= n;
        value |= has ? 1u << bit : 0u;
        #pragma unroll
        for (int k = 0; k < G; ++k) in[k] = has ? up[k] : in[k] ^ up[k];
        n -= has ? 0 : many;
    }
    return value;
}
__device__ __forceinline__ uint64_t below_order(uint32_t order) { return order == 0 ? 0 : ((uint64_t)order << 32) - 1; }

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

struct Shared {
    uint64_t own[kWaves][kList + 8], best[MAD_MAX_TOP];
    uint64_t bound;
    int place[kWaves * kList];
    float entries[kWaves][64];
    uint32_t group[kWaves][64];
    double s[kWaves], u[kWaves];
    float m[kWaves];
    int above[kWaves], inf[kWaves], held[kWaves];
    int last;
};

// The first n of the order among the waves' lists (held[w] keys each) into best: a key's place is the number of keys above
// it (keys differ: their index is in them), each wave counting in its own list.  Begins and ends at a barrier.
__device__ __forceinline__ void join_lists(Shared &sh, int wave, int lane, int held, int n) {
    for (int i = threadIdx.x; i < kWaves * kList; i += kWg) sh.place[i] = 0;
    if (lane < 8) sh.own[wave][held + lane] = 0;   // (read, and above nothing)
    if (lane == 0) sh.held[wave] = held;
    if ((int)threadIdx.x < n) sh.best[threadIdx.x] = 0;
    __syncthreads();
    int from[kWaves + 1] = {0};
    #pragma unroll
    for (int w = 0; w < kWaves; ++w) from[w + 1] = from[w] + sh.held[w];
    auto key_of = [&](int i) {
        int w = 0;
        #pragma unroll
        for (int k = 1; k < kWaves; ++k) w += i >= from[k] ? 1 : 0;
        int start = 0;
        #pragma unroll
        for (int k = 1; k < kWaves; ++k) start = w == k ? from[k] : start;
        return sh.own[w][i - start];
    };
    const uint64_t *own = sh.own[wave];
    for (int i = lane; i < from[kWaves]; i += 64) {
        const uint64_t x = key_of(i);
        int above = 0;
        for (int k = 0; k < held; k += 8) {
            ulonglong2 y[4];
            #pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = reinterpret_cast<const ulonglong2 *>(own + k)[q];
            #pragma unroll
            for (int q = 0; q < 4; ++q) above += (y[q].x > x ? 1 : 0) + (y[q].y > x ? 1 : 0);
        }
        if (above > 0) atomicAdd(&sh.place[i], above);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < from[kWaves]; i += kWg) {
        const int at = sh.place[i];
        if (at < n) sh.best[at] = key_of(i);
    }
    __syncthreads();
}

}  // namespace

// E: entries of a thread and step
template <typename T, int E, bool TOP>
__global__ __launch_bounds__(kWg, 4) void logprobs_kernel(const LogprobArgs a) {
    constexpr int VEC = Elem<T>::VEC, NV = E / VEC, CHUNK = kWg * E;
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

    // 16 bytes a lane and piece; pieces past the run's or the row's last: the last one again
    uint4 raw[NV];
    const uint32_t end = (uint32_t)min(vecs, chunk1 * NV * kWg) - 1;
    auto load = [&](int chunk) {
        #pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t at = min((uint32_t)((chunk * NV + j) * kWg + tid), end) * 16u;
            raw[j] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(base) + at);
        }
    };
    load(chunk0);
    const int tok = a.tok ? a.tok[row] : -1;
    const bool has = tok >= 0 && tok < V;
    const float xt = has ? Elem<T>::load1(x0 + tok) : INFINITY;
    const float below = next_below(xt);

    Stats st = {0.0, 0.0, -INFINITY};
    int above = 0, inf = 0;      // (of the wave)
    uint64_t *own = sh.own[wave];
    int held = 0;                // keys in it
    uint64_t bound = 0;          // only keys above it count
    // the wave's list to its first n, the last of which is a bound
    auto cut = [&]() {
        const uint64_t k0 = lane < held ? own[lane] : 0, k1 = 64 + lane < held ? own[64 + lane] : 0;
        int a0 = 0, a1 = 0;
        #pragma unroll 4
        for (int i = 0; i < held; ++i) {
            const uint64_t x = own[i];
            a0 += x > k0 ? 1 : 0;
            a1 += x > k1 ? 1 : 0;
        }
        if (k0 != 0 && a0 < n) own[a0] = k0;
        if (k1 != 0 && a1 < n) own[a1] = k1;
        if (held >= n) bound = max_u64(bound, own[n - 1]);
        held = min(held, n);
    };
    if (TOP && tid == 0) sh.bound = 0;

    for (int chunk = chunk0; chunk < chunk1; ++chunk) {
        float x[E];
        #pragma unroll
        for (int j = 0; j < NV; ++j) {
            float f[VEC];
            unpack16(raw[j], f, T());
            #pragma unroll
            for (int e = 0; e < VEC; ++e) x[j * VEC + e] = f[e];
        }
        load(chunk + 1);
        const int first = chunk * CHUNK - skew;   // the chunk's first entry
        const bool edge = first < 0 || first + CHUNK > V;
        auto index = [&](int i) { return first + ((i / VEC) * kWg + tid) * VEC + i % VEC; };
        if (edge) {   // what is not the row's: -inf
            #pragma unroll
            for (int i = 0; i < E; ++i) x[i] = (uint32_t)index(i) < (uint32_t)V ? x[i] : -INFINITY;
        }
        float mj[NV], m = -INFINITY;   // the pieces' largest
        #pragma unroll
        for (int j = 0; j < NV; ++j) {
            mj[j] = x[j * VEC];
            #pragma unroll
            for (int e = 1; e < VEC; ++e) mj[j] = fmaxf(mj[j], x[j * VEC + e]);
            m = fmaxf(m, mj[j]);
        }

        if (__any(!((m - st.m) * c <= kLag))) {   // (nothing yet: inf or NaN)
            const float mn = (m - st.m) * c > kLag && m < INFINITY ? m : st.m;
            if (st.m < mn) {
                const float d = fmaxf(lower(st.m, mn, c), -3000.f), f = __builtin_amdgcn_exp2f(d);
                st.u = (double)f * (st.u + (double)d * st.s);
                st.s *= (double)f;
                st.m = mn;
            }
        }
        const float M = st.m * c;
        float s = 0.f, u = 0.f;
        if (fabsf(M) < kNear && m < INFINITY) {
            float s1 = 0.f, u1 = 0.f;   // every other entry's
            #pragma unroll
            for (int i = 0; i < E; i += 2) {
                const float d = fmaf(x[i], c, -M), e = __builtin_amdgcn_exp2f(d);
                const float d1 = fmaf(x[i + 1], c, -M), e1 = __builtin_amdgcn_exp2f(d1);
                s += e;
                u = fmaf(e, d, u);
                s1 += e1;
                u1 = fmaf(e1, d1, u1);
            }
            s += s1;
            u += u1;
            if (!(u == u)) {   // an e of 0 with a d of -inf, or a NaN (which s has too)
                u = 0.f;
                const float again = __int_as_float(here(__float_as_int(M)));   // (no registers held for this)
                #pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float d = fmaf(x[i], c, -again), e = __builtin_amdgcn_exp2f(d);
                    u = fmaf(e, fmaxf(d, -200.f), u);
                }
            }
        } else if (fabsf(st.m) < INFINITY && m < INFINITY) {
            #pragma unroll
            for (int i = 0; i < E; ++i) {
                const float d = (x[i] - st.m) * c, e = __builtin_amdgcn_exp2f(d);
                s += e;
                u = fmaf(e, fmaxf(d, -200.f), u);
            }
        }
        st.s += (double)s;
        st.u += (double)u;
        if (__any(!(fabsf(m) < INFINITY))) {   // a +inf, nothing but -inf, or NaN alone
            #pragma unroll
            for (int i = 0; i < E; ++i) {
                inf += __popcll(__ballot(x[i] == INFINITY));
                if (x[i] != x[i]) st.s = __builtin_nan("");
            }
        }

        if (has && __any(m >= xt)) {
            // above the token's logit; in pieces before the token's, equal to it too: above the next number below
            #pragma unroll
            for (int j = 0; j < NV; ++j) {
                const float y = index(j * VEC) + VEC <= tok ? below : xt;
                #pragma unroll
                for (int e = 0; e < VEC; ++e) above += __popcll(__ballot(x[j * VEC + e] > y));
            }
            if (xt == -INFINITY) {   // (nothing is below)
                #pragma unroll
                for (int i = 0; i < E; ++i)
                    above += __popcll(__ballot(x[i] == xt && index(i) >= 0 && index((i / VEC) * VEC) + VEC <= tok));
            }
        }
        if constexpr (TOP) {
            if (chunk == chunk0) {
                sh.group[wave][lane] = order_of(m);
                __syncthreads();
                uint32_t g[kWaves], all[1] = {0};
                #pragma unroll
                for (int k = 0; k < kWaves; ++k) {
                    g[k] = sh.group[k][lane];
                    all[0] = max(all[0], g[k]);
                }
                bound = below_order(n > kFewGroups ? reached_by(g, n) : reached_by(all, n));
            } else {
                bound = max_u64(bound, *reinterpret_cast<volatile uint64_t *>(&sh.bound));
            }
            // lanes with entries of the bound's value and above (some of that value are not above it)
            auto lanes_above = [&]() { return __ballot(!(m < value_of(bound))); };
            uint64_t lanes = lanes_above();
            if (lanes) {
                if (chunk > chunk0 && __popcll(lanes) > kMany) {
                    const uint32_t g[1] = {order_of(m)};
                    bound = max_u64(bound, below_order(reached_by(g, n)));
                    lanes = lanes_above();
                }
                while (lanes) {
                    // 64 / E of these lanes spread their entries over the wave
                    int from = -1, slot = -1;   // whose entry this lane takes, where this lane's go
                    #pragma unroll
                    for (int k = 0; k < 64 / E; ++k) {
                        const int l = lanes ? __builtin_ctzll(lanes) : -1;
                        lanes &= lanes - 1;
                        from = lane / E == k ? l : from;
                        slot = lane == l ? k : slot;
                    }
                    if (slot >= 0) {
                        #pragma unroll
                        for (int q = 0; q < E / 4; ++q)
                            reinterpret_cast<float4 *>(sh.entries[wave])[slot * (E / 4) + q] = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
                    }
                    const float v = sh.entries[wave][lane];
                    const int e = lane % E, i = first + ((e / VEC) * kWg + wave * 64 + from) * VEC + e % VEC;
                    const uint64_t mine = from >= 0 && (uint32_t)i < (uint32_t)V ? argmax_key(v, i) : 0;
                    uint64_t in = __ballot(mine > bound);
                    if (held + __popcll(in) > kOwn) {
                        cut();
                        in = __ballot(mine > bound);
                        lanes &= lanes_above();
                    }
                    if (mine > bound) own[held + __popcll(in & ((1ull << lane) - 1))] = mine;
                    held += __popcll(in);
                }
                if (chunk + 1 < chunk1 && held > n + max(n >> 1, 4)) {
                    cut();
                    if (lane == 0) atomicMax((unsigned long long *)&sh.bound, (unsigned long long)bound);
                }
            }
        }
    }

    // ---- the workgroup's waves together ----
    st = wave_join(st, c);
    if (lane == 0) {
        sh.s[wave] = st.s;
        sh.u[wave] = st.u;
        sh.m[wave] = st.m;
        sh.above[wave] = above;
        sh.inf[wave] = inf;
    }
    if (TOP) join_lists(sh, wave, lane, held, n);
    else __syncthreads();
    if (wave == 0) {
        st = lane < kWaves ? Stats{sh.s[lane & (kWaves - 1)], sh.u[lane & (kWaves - 1)], sh.m[lane & (kWaves - 1)]} : Stats{0.0, 0.0, -INFINITY};
        st = wave_join(st, c);
        above = inf = 0;
        for (int k = 0; k < kWaves; ++k) {
            above += sh.above[k];
            inf += sh.inf[k];
        }
    }

    if (a.splits > 1) {
        // a record for each workgroup of the row; the last to arrive joins them
        LogprobRecord *rec = a.records + (size_t)row * a.splits;
        if (wave == 0) {
            LogprobRecord *mine = rec + split;
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
        // everything that is read of the records, at once
        uint64_t w[4] = {0, 0, 0xff800000u, 0}, part[kRecs];
        uint32_t nth[1] = {0};
        const int half = (a.splits + 1) / 2, deep = (n + half - 1) / half;   // some half of the lists, this deep, hold top_n
        if (lane < a.splits) {
            #pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = load_agent64(reinterpret_cast<const uint64_t *>(rec + lane) + k);
            if (TOP) nth[0] = (uint32_t)(load_agent64(&rec[lane].best[deep - 1]) >> 32);
        }
        if (TOP) {
            #pragma unroll
            for (int k = 0; k < kRecs; ++k)
                part[k] = k * kWaves + wave < a.splits && lane < n ? load_agent64(&rec[k * kWaves + wave].best[lane]) : 0;
            const uint64_t least = below_order(reached_by(nth, (n + deep - 1) / deep));
            held = 0;
            #pragma unroll
            for (int k = 0; k < kRecs; ++k) {
                const bool in = part[k] > least;
                const uint64_t all = __ballot(in);
                if (in) own[held + __popcll(all & ((1ull << lane) - 1))] = part[k];
                held += __popcll(all);
            }
            join_lists(sh, wave, lane, held, n);
        }
        if (wave == 0) {
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
    // equal entries before the token in its own 16-byte piece
    if (has) {
        const int piece = (tok + skew) & ~(VEC - 1), i = piece - skew + lane;
        above += __popcll(__ballot(lane < VEC && i >= 0 && i < tok && Elem<T>::load1(x0 + max(i, 0)) == xt));
    }
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

// Few rows: as many workgroups to a row as the CUs hold at once, so that a call is one round (80 rows of 128256, fp32, in 1280
// places 24.2 us for 20.3 in 1024).  In 512 -> 1024 places, us: 80 rows of 128256, bf16, top 20, 23.6 -> 21.4, top 5 18.8 -> 18.4,
// fp32 19.4 -> 19.8; 256 rows 30.6 -> 27.8; 320 of 50257 23.3 -> 21.7; only two workgroups to a row do not pay (512 of 128256
// 34.4 -> 37.1, 500 of 32000, fp32, 17.2 -> 20.9).  Else a workgroup to a row.
LogprobPlan plan_logprobs(int rows, int V) {
    LogprobPlan p;
    constexpr int chunk = kWg * 16;
    p.n_chunks = (V + 7 + chunk - 1) / chunk;   // (a row may begin up to 7 entries into its first 16 bytes)
    const int want = rows > kCounterLines / 4 ? 1 : kLogprobWgs / rows < kLogprobSplits ? kLogprobWgs / rows : kLogprobSplits;
    const int each = want < 1 ? p.n_chunks : (p.n_chunks + want - 1) / want;
    p.splits = (p.n_chunks + each - 1) / each;
    return p;
}

// The counters, and a record for each workgroup of a row that has several: at most kLogprobWgs in all, and a chunk each.  A
// workspace holds every call of at most these sizes, so that fewer rows count, which take more workgroups each, and shorter ones,
// whose chunks may divide into more: never less where a size grows.
size_t logprobs_ws_bytes(int rows, int V) {
    const int chunks = plan_logprobs(rows, V).n_chunks, most = chunks < kLogprobSplits ? chunks : kLogprobSplits;
    const int64_t records = (int64_t)rows * most < kLogprobWgs ? (int64_t)rows * most : kLogprobWgs;
    return kCounterRegionBytes + (most > 1 ? align256((size_t)records * sizeof(LogprobRecord)) : 0);
}

template <typename T, int E>
static hipError_t launch_t(const LogprobArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.rows * a.splits)), wg(kWg);
    if (a.top_n > 0) hipLaunchKernelGGL((logprobs_kernel<T, E, true>), grid, wg, 0, st, a);
    else hipLaunchKernelGGL((logprobs_kernel<T, E, false>), grid, wg, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_logprobs(const LogprobArgs &a, int dtype, hipStream_t st) {
    if (dtype != MAD_BF16) return launch_t<float, 16>(a, st);
    if (a.splits > 1 || a.V < kLogprobLong) return launch_t<bf16_t, 16>(a, st);
    LogprobArgs x = a;
    x.n_chunks = (a.V + 7 + kWg * 32 - 1) / (kWg * 32);
    return launch_t<bf16_t, 32>(x, st);
}

}  // namespace mad

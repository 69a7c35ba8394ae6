// logprobs.hip -- log probabilities of given tokens, ranks, entropies and the
// most probable alternatives, from the logits in one read.
//
// Mathematics, for a row's logits x, c = log2 e / temperature, m = max x:
//   d_v = (x_v - m) c,  e_v = 2^d_v,  s = sum e,  u = sum e d
//   log p_v = ln 2 * (d_v - log2 s);   entropy = ln 2 * (log2 s - u / s)
//   rank = entries above the token's logit, and equal ones before it.
// (x - m is formed before the product: the fused form's rounding of m c would
// shift every term alike.)  A thread keeps m, s and u of what it has seen, raises
// m once per chunk of 16 entries, and sums within a chunk in fp32, over chunks
// and threads in fp64.
//
// The first top_n of the order: the entries that reach a bound go into a list in
// LDS, the list is cut to its first top_n by counting, and from then on the last of those
// is the bound, which few entries of the later chunks pass.  The first chunk's
// bound: the top_n-th largest of 64 maxima of disjoint groups (lane l of every
// wave); top_n entries at least reach it, and some top_n more by chance.  Where
// that bound lets too many through (a row of few different values), the chunk's
// entries are taken largest by largest.
//
// Work: a workgroup takes a run of a row's chunks of 8192; with few rows, more
// workgroups to a row, whose results the last of them to arrive joins.  Bound: bytes, 10
// vector instructions an entry close behind.
#include "mad_device.h"
#include "mad_internal.h"

namespace mad {

namespace {

constexpr int kWg = 512, kEntries = 16;              // threads, entries of a thread and chunk
static_assert(kWg * kEntries == kLogprobChunk, "");
constexpr int kList = 1024;                          // list of entries that reached the bound
constexpr int kCut = 256;                            // the list is cut where it holds more
static_assert(kLogprobSplits * MAD_MAX_TOP <= kList && kCut + MAD_MAX_TOP <= kList, "");

struct Stats {
    double s, u;
    float m;
    int above, inf;
};

// a's and b's entries together (s, u relative to m; c as above)
__device__ __forceinline__ Stats join(const Stats &a, const Stats &b, float c) {
    Stats r;
    r.m = fmaxf(a.m, b.m);
    const float da = a.m == r.m ? 0.f : fmaxf((a.m - r.m) * c, -3000.f), db = b.m == r.m ? 0.f : fmaxf((b.m - r.m) * c, -3000.f);
    const double fa = (double)__builtin_amdgcn_exp2f(da), fb = (double)__builtin_amdgcn_exp2f(db);
    r.s = fa * a.s + fb * b.s;
    r.u = fa * (a.u + (double)da * a.s) + fb * (b.u + (double)db * b.s);
    r.above = a.above + b.above;
    r.inf = a.inf + b.inf;
    return r;
}

__device__ __forceinline__ uint32_t order_of(float x) { return (uint32_t)(argmax_key(x, 0) >> 32); }
__device__ __forceinline__ float value_of(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint64_t max_u64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t wave_max_u64(uint64_t v) {
    return wave_fold_u64(v, [](uint64_t a, uint64_t b) { return max_u64(a, b); });
}

struct Shared {
    uint64_t list[kList], best[MAD_MAX_TOP], wave_best[8];
    uint32_t group[8][64];
    Stats st[8];
    int count, last;
};

// the first n of the order among best[0 .. nb) and list[0 .. count): into best
__device__ void cut(Shared &sh, int nb, int count, int n) {
    const int total = nb + count;
    uint64_t key[3];
    int at[3];
    auto entry = [&](int i) { return i < nb ? sh.best[i] : sh.list[i - nb]; };
    #pragma unroll
    for (int k = 0; k < 3; ++k) {   // total <= kList + MAD_MAX_TOP < 3 kWg
        const int i = threadIdx.x + k * kWg;
        key[k] = i < total ? entry(i) : 0;
        at[k] = 0;
    }
    for (int i = 0; i < nb; ++i) {
        const uint64_t x = sh.best[i];
        #pragma unroll
        for (int k = 0; k < 3; ++k) at[k] += x > key[k] ? 1 : 0;
    }
    for (int i = 0; i < count; ++i) {
        const uint64_t x = sh.list[i];
        #pragma unroll
        for (int k = 0; k < 3; ++k) at[k] += x > key[k] ? 1 : 0;
    }
    __syncthreads();
    #pragma unroll
    for (int k = 0; k < 3; ++k)   // (keys differ: their index is in them)
        if (threadIdx.x + k * kWg < total && at[k] < n) sh.best[at[k]] = key[k];
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
}

}  // namespace

template <typename T, bool TOP>
__global__ __launch_bounds__(kWg) void logprobs_kernel(const LogprobArgs a) {
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
    const int tok = a.tok ? a.tok[row] : -1;
    const bool has = tok >= 0 && tok < V;
    const float xt = has ? Elem<T>::load1(x0 + tok) : INFINITY;
    const int chunk0 = (int)((int64_t)a.n_chunks * split / a.splits), chunk1 = (int)((int64_t)a.n_chunks * (split + 1) / a.splits);

    Stats st = {0.0, 0.0, -INFINITY, 0, 0};
    int nb = 0;              // entries of best
    uint32_t least = 0;      // ... the last one's order, once there are top_n
    if (TOP && tid == 0) sh.count = 0;
    if (TOP) __syncthreads();

    uint4 raw[NV];
    auto load = [&](int chunk) {
        #pragma unroll
        for (int j = 0; j < NV; ++j) raw[j] = base[min((chunk * NV + j) * kWg + tid, vecs - 1)];
    };
    load(chunk0);
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
        if (fabsf(m) < INFINITY) {
            const float mn = fmaxf(st.m, m);
            float s = 0.f, u = 0.f;
            #pragma unroll
            for (int i = 0; i < kEntries; ++i) {
                const float d = (x[i] - mn) * c, e = __builtin_amdgcn_exp2f(d);
                s += e;
                u = fmaf(e, fmaxf(d, -200.f), u);   // (an e of 0 with a d of -inf)
            }
            if (st.m < mn) {
                const float d = fmaxf((st.m - mn) * c, -3000.f), f = __builtin_amdgcn_exp2f(d);
                st.u = (double)f * (st.u + (double)d * st.s);
                st.s *= (double)f;
                st.m = mn;
            }
            st.s += (double)s;
            st.u += (double)u;
        } else {   // nothing but -inf, a +inf, or a NaN
            #pragma unroll
            for (int i = 0; i < kEntries; ++i) {
                st.inf += x[i] == INFINITY ? 1 : 0;
                if (x[i] != x[i]) st.s = __builtin_nan("");
            }
        }
        if (has) {
            #pragma unroll
            for (int i = 0; i < kEntries; ++i) st.above += x[i] > xt || (x[i] == xt && index(i) < tok && inside(i)) ? 1 : 0;
        }
        if constexpr (TOP) {
            const uint32_t mo = order_of(m);   // (a chunk without an entry: -inf's)
            // entries that reach `bound` into the list; their number, which may be more than it holds
            const int before = sh.count;   // (the same for all: read behind a barrier)
            auto put = [&](uint32_t bound) {
                __syncthreads();
                if (mo >= bound) {
                    #pragma unroll
                    for (int i = 0; i < kEntries; ++i)
                        if (inside(i) && order_of(x[i]) >= bound) {
                            const int at = atomicAdd(&sh.count, 1);
                            if (at < kList) sh.list[at] = argmax_key(x[i], index(i));
                        }
                }
                __syncthreads();
                return sh.count;
            };
            auto group_bound = [&]() {   // the n-th largest of 64 groups' maxima
                sh.group[wave][lane] = mo;
                __syncthreads();
                uint32_t g = 0;
                #pragma unroll
                for (int k = 0; k < 8; ++k) g = max(g, sh.group[k][lane]);
                int above = 0;
                for (int l = 0; l < 64; ++l) {
                    const uint32_t o = __builtin_amdgcn_readlane(g, l);
                    above += o > g || (o == g && l < lane) ? 1 : 0;
                }
                const uint64_t mine = __ballot(above == n - 1);
                return (uint32_t)__builtin_amdgcn_readlane(g, __builtin_ctzll(mine));
            };
            int count = put(nb < n ? group_bound() : least + 1);
            if (count > kList && nb == n) {
                __syncthreads();   // (every thread has read the count)
                if (tid == 0) sh.count = before;
                count = put(max(group_bound(), least + 1));
            }
            if (count > kList) {
                // largest by largest: the list's part from `before` on again
                uint64_t under = ~0ull;
                int got = before;
                for (int k = 0; k < n; ++k) {
                    uint64_t mine = 0;
                    #pragma unroll
                    for (int i = 0; i < kEntries; ++i) {
                        const uint64_t key = inside(i) ? argmax_key(x[i], index(i)) : 0;
                        mine = key < under ? max_u64(mine, key) : mine;
                    }
                    mine = wave_max_u64(mine);
                    if (lane == 0) sh.wave_best[wave] = mine;
                    __syncthreads();
                    uint64_t top = 0;
                    #pragma unroll
                    for (int w = 0; w < 8; ++w) top = max_u64(top, sh.wave_best[w]);
                    __syncthreads();
                    if (top == 0) break;
                    if (tid == 0) sh.list[got] = top;
                    ++got;
                    under = top;
                }
                if (tid == 0) sh.count = got;
                __syncthreads();
                count = got;
            }
            if (nb < n || count > kCut || chunk + 1 == chunk1) {
                cut(sh, nb, count, n);
                nb = min(nb + count, n);
                if (nb == n) least = (uint32_t)(sh.best[n - 1] >> 32);
            }
        }
    }

    // ---- the workgroup's threads together ----
    auto fold = [&](Stats &v, int width) {
        for (int k = 1; k < width; k <<= 1) {
            Stats o;
            o.m = __shfl_xor(v.m, k);
            o.s = __shfl_xor(v.s, k);
            o.u = __shfl_xor(v.u, k);
            o.above = __shfl_xor(v.above, k);
            o.inf = __shfl_xor(v.inf, k);
            v = join(v, o, c);
        }
    };
    fold(st, 64);
    if (lane == 0) sh.st[wave] = st;
    __syncthreads();
    st = sh.st[lane & 7];
    fold(st, 8);

    if (a.splits > 1) {
        // a record for each workgroup of the row; the last to arrive joins them
        LogprobRecord *rec = a.records + (size_t)row * a.splits;
        if (TOP && tid < nb) __hip_atomic_store(&rec[split].best[tid], sh.best[tid], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (tid == 0) {
            uint64_t *p = reinterpret_cast<uint64_t *>(&rec[split]);
            const uint64_t w[4] = {(uint64_t)__double_as_longlong(st.s), (uint64_t)__double_as_longlong(st.u),
                                   (uint64_t)__float_as_uint(st.m) | (uint64_t)(uint32_t)st.above << 32,
                                   (uint64_t)(uint32_t)st.inf | (uint64_t)(uint32_t)nb << 32};
            for (int k = 0; k < 4; ++k) __hip_atomic_store(p + k, w[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        wait_vm_stores();
        __syncthreads();
        if (tid == 0) {
            unsigned *cnt = a.counters + (size_t)row * kCounterStride;
            sh.last = arrive(cnt) == (unsigned)a.splits - 1;
            if (sh.last) reset_counter(cnt);
            sh.count = 0;
        }
        __syncthreads();
        if (!sh.last) return;
        const int from = lane & (kLogprobSplits - 1);
        st = {0.0, 0.0, -INFINITY, 0, 0};
        int has_best = 0;
        if (from < a.splits) {
            const uint64_t *p = reinterpret_cast<const uint64_t *>(&rec[from]);
            const uint64_t w0 = load_agent64(p), w1 = load_agent64(p + 1), w2 = load_agent64(p + 2), w3 = load_agent64(p + 3);
            st = {__longlong_as_double((long long)w0), __longlong_as_double((long long)w1), __uint_as_float((uint32_t)w2), (int)(w2 >> 32), (int)(uint32_t)w3};
            has_best = (int)(w3 >> 32);
        }
        if (TOP) {
            for (int k = wave; k < a.splits; k += 8) {
                const int nk = __builtin_amdgcn_readlane(has_best, k);
                if (lane < nk) {
                    const uint64_t key = load_agent64(&rec[k].best[lane]);
                    sh.list[atomicAdd(&sh.count, 1)] = key;
                }
            }
            __syncthreads();
            const int count = sh.count;
            __syncthreads();
            cut(sh, 0, count, n);
        }
        fold(st, kLogprobSplits);
    }

    // ---- the row's end ----
    if (wave != 0) return;
    const bool none = !(st.s == st.s) || (st.inf == 0 && st.m == -INFINITY);
    const double ln2 = 0.6931471805599453, nan = __builtin_nan("");
    const double ls = none ? nan : st.inf > 0 ? log((double)st.inf) : log(st.s);
    auto log_p = [&](float v) {
        if (none) return (float)nan;
        if (st.inf > 0) return v == INFINITY ? (float)-ls : -INFINITY;
        return (float)(((double)v - (double)st.m) * (double)c * ln2 - ls);
    };
    if (lane == 0) {
        if (a.logp) a.logp[row] = none ? (float)nan : has ? log_p(xt) : -INFINITY;
        if (a.rank) a.rank[row] = none ? -1 : has ? st.above : V;
        if (a.entropy) a.entropy[row] = (float)(none || st.inf > 0 ? ls : ls - ln2 * (st.u / st.s));
    }
    if (TOP && lane < n) {
        const uint64_t key = sh.best[lane];
        a.top_tok[(int64_t)row * n + lane] = none ? -1 : key_index(key);
        a.top_logp[(int64_t)row * n + lane] = log_p(value_of(key));
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

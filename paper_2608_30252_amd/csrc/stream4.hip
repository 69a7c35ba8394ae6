// stream4.hip -- the target's verify attention (Sec. 2.1, Sec. 3.3; T = 1: a
// single token's) over a 4-bit cache: e2m1 codes, a power-of-two scale for each
// row and 32 features.
//
// Mathematics.  With key j's rows k_j, v_j (code times scale) and row r's query q
// (cs = softmax scale * log2 e):
//   x_j = (q . k_j) * cs,   p_j = 2^(x_j - m),   o = sum p_j v_j
// A code times its scale is exact in bf16, and one instruction
// (v_cvt_scalef32_pk_bf16_fp4) makes two of them, scale included: it takes the
// scale from an fp32's exponent field, which the scale's byte is, shifted.
//   S^T = K Q^T   bf16 x bf16; an fp32 query is split into three bf16 terms
//                 (24 bits), three products to the same accumulator.
//   O^T = V^T P^T bf16 x bf16: a probability is rounded to bf16 (2^-8 relative,
//                 the output's own rounding); V's values keep bf16's range, so keys
//                 of any size meet in one sum.  fp32: three bf16 terms.
// m is raised, and the sums scaled, only where a score exceeds it by more than 4
// (log2 units; p <= 2^4 loses nothing): some row's maximum grows in most steps, by
// little.
//
// Operands without a transposition.  A matrix step takes 32 keys in any order that
// both operands share; here key 4 e + lg of the step is element e of lane group
// lg (lane = 16 lg + lr).
//   K: lane (lr, lg) reads a quarter of one key's row (features D/4 * lg ..),
//      which one scale covers, and the queries' fragments hold the same features.
//   V: lane (lr, lg) reads, for its eight keys, the D/16 features that start at
//      D/16 * lr: a matrix row is a lane's j-th feature.  The conversion gives
//      pairs of features of a key; a byte permute of two keys' pairs gives two
//      features' pairs of keys.
//
// Work decomposition: stream8.hip's.  Units (sequence, KV head) are cut into slabs
// that are dealt to one workgroup per CU (plan_stream); inside it the eight waves
// take chunks of 4 KB (32 keys at d 128, 64 at d 64) in turn, each through its
// own ring of LDS stages, for every query row, and merge at a unit's end.
//
// What a row does not see is left out whatever it holds: scores by selection, rows
// past the length are never read, and where a step with hidden keys has a NaN
// scale in V (0 * NaN is NaN) its keys are taken out and NaN given to the rows that
// see them.
#include "stream_device.h"

namespace mad {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_v;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2_v;

constexpr float kLazy4 = 4.f;      // the maximum is raised where a score exceeds it by more (log2 units)

// T: bf16_t or float (queries and output)
template <int D, int NB, typename T>
struct Stream4Cfg {
    static constexpr bool F32 = std::is_same<T, float>::value;
    static constexpr int NWV = 8;                          // waves
    static constexpr int RB = D / 2;                       // bytes per K (and V) row
    static constexpr int CPR = D / 32;                     // 16-byte pieces, and scales, per row
    static constexpr int CHUNK = 4096;                     // K, then V
    static constexpr int KPC = 2048 / RB;                  // keys per chunk
    static constexpr int SCALES = 2 * KPC * 4;             // a chunk's scales: a dword per K row, then per V row
    static constexpr int LOADS = 4 + SCALES / 256;         // direct loads per chunk: 2 + 2 of 1 KB, and the scales
    static constexpr int KST = D / 32, DB = D / 16, NQ = F32 ? 3 : 1;
    static constexpr int RP = NB * 16;                     // padded query rows
    // query fragments (1 KB each), in registers where they and the accumulators leave room for the rest
    static constexpr int QBYTES = NB * KST * NQ * 1024;
    static constexpr bool QREG = NB * (KST * NQ + DB) * 4 < 120;
    static constexpr int REST = NWV * RP * 8 + QBYTES, STAGES = NWV * (CHUNK + SCALES);
    static constexpr int NST = 4 * STAGES + REST + 1536 <= 160 * 1024 ? 4 : 3;   // stages per wave
    static constexpr int PRE = NST - 2;                    // ... that the waves' exchange leaves alone
    static constexpr int RING = NST * NWV * CHUNK;         // stage 0 of every wave, then stage 1, ..
    static constexpr int OFF_S = RING;                     // scales, likewise
    static constexpr int OFF_ML = OFF_S + NST * NWV * SCALES;   // the waves' (maximum, sum) per row
    static constexpr int OFF_Q = OFF_ML + NWV * RP * 8;
    static constexpr int USED = OFF_Q + QBYTES;
    static constexpr int SMEM = USED > kMergeBytes ? USED : kMergeBytes;
    // the waves' exchange goes through the last two stages of all of them, XD feature blocks at a time
    static constexpr int OFF_X = PRE * NWV * CHUNK;
    static constexpr int XD = NB * DB <= 8 ? DB : NB == 2 ? 4 : NB == 1 ? 8 : 2;
    static_assert(SMEM + 2 * MAD_MAX_VERIFY_ROWS * 4 + 64 <= 160 * 1024, "LDS, with the kernel's static arrays");
    static_assert(NWV * NB * XD * 1024 <= 2 * NWV * CHUNK && NB * XD <= NWV && DB % XD == 0, "exchange");
};

// A direct load of one dword, one half-word (zero-extended) per lane; lanes of a wave: consecutive dwords at lds.
__device__ __forceinline__ void lds_stream4(const void *src, uint32_t lds) {
    const uint32_t m = __builtin_amdgcn_readfirstlane(lds);
    uint32_t saved;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved) : "v"(src), "s"(m) : "memory");
}
__device__ __forceinline__ void lds_stream2(const void *src, uint32_t lds) {
    const uint32_t m = __builtin_amdgcn_readfirstlane(lds);
    uint32_t saved;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_ushort %1, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved) : "v"(src), "s"(m) : "memory");
}

// 16-byte piece c of K row k sits at piece c ^ k4_swz(k), so that a pass of the operand reads finds its 16 rows (every
// fourth, four of them offset) in different banks.  V rows lie as they are: a read takes whole rows side by side.
template <int D> __device__ __forceinline__ int k4_swz(int k) { return D == 128 ? (k >> 2) & 3 : (k >> 3) & 1; }

// a pair of features (byte B of w) of a key to bf16, times the scale in s's exponent field (exact)
template <int B> __device__ __forceinline__ uint32_t pair_bf16(uint32_t w, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, B));
}
__device__ __forceinline__ bf16x8_v codes_bf16(uint32_t w, float s) {   // 8 features of a key
    return __builtin_bit_cast(bf16x8_v, (u32x4_v{pair_bf16<0>(w, s), pair_bf16<1>(w, s), pair_bf16<2>(w, s), pair_bf16<3>(w, s)}));
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

struct Kv4Scales {
    uint64_t k, v;
    int64_t seq, head;
};

template <int D, int NB, typename T>
__global__ __launch_bounds__(512, 1) void stream4_kernel(const Stream4Args args) {
    using C = Stream4Cfg<D, NB, T>;
    constexpr int KST = C::KST, DB = C::DB, NQ = C::NQ, SLAB = stream8_slab(D);
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int s_last[2];
    const StreamCtx a = load_ctx(args);
    Kv4Scales sc = {ptr_bits(args.k_scale), ptr_bits(args.v_scale), args.s_seq, args.s_head};
    asm volatile("" : "+s"(sc.k), "+s"(sc.v), "+s"(sc.seq), "+s"(sc.head));

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lr = lane & 15, lg = lane >> 4;
    const int w = blockIdx.x;
    const int TT = a.T, G = a.G, R = TT * G, Hkv = a.Hkv;

    // ---- this workgroup's run of slabs: the first one's unit (b, c) and slab t, and their number ----
    int b, c, t, left, piece = w;   // piece: this run's number within its unit's pieces, less the unit's
    if (a.by_unit) {
        b = __popcll(__ballot(Hkv * a.rec.z <= w)) - 1;   // records past the last row hold the end
        const int k = a.splits(b), rel = w - Hkv * a.wg0(b), n0 = a.slabs(b);
        const bool turn = a.by_unit == 1;   // neighbouring workgroups take the row's units in turn
        const int m = turn ? Hkv : k, x0 = rel / m, x1 = rel - x0 * m;
        c = turn ? x1 : x0;
        const int part = turn ? x0 : x1;
        piece = w - rel + c * k + part;
        const int lo = n0 / k, hi = n0 - lo * k;   // hi pieces of lo + 1 slabs, then of lo
        t = part * lo + min(part, hi);
        left = lo + (part < hi ? 1 : 0);
    } else {
        const int g0 = stream_first(w, a.base, a.rem);
        left = stream_first(w + 1, a.base, a.rem) - g0;
        b = __popcll(__ballot(Hkv * a.rec.w <= g0)) - 1;
        const int n0 = a.slabs(b), rel = g0 - Hkv * a.tile0(b);
        c = rel / n0;
        t = rel - c * n0;
    }

    // ---- loads: lane l of load j (j = 0, 1 for K, and for V) fetches LDS slot cidx % CPR of the chunk's row cidx / CPR
    // (cidx = 64 j + l): for K the row's piece slot ^ swizzle(row).  The second load of a pair adds 1024 to both of its
    // addresses (an instruction offset). ----
    uint32_t koff[2], voff[2];
    #pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int cidx = 64 * j + lane, kr = cidx / C::CPR, slot = cidx % C::CPR;
        koff[j] = kr * C::RB + ((slot ^ k4_swz<D>(kr)) << 4) - 1024 * j;
        voff[j] = lane * 16;
    }
    constexpr int STAGE = C::NWV * C::CHUNK, SSTAGE = C::NWV * C::SCALES;   // from a wave's stage to its next
    unsigned char *ring = smem + wave * C::CHUNK;
    unsigned char *ring_s = smem + C::OFF_S + wave * C::SCALES;
    const uint32_t lds_k = lds_addr(ring), lds_s = lds_addr(ring_s);
    const float cs = a.cs;
    float *lse = bits_ptr<float>(a.lse);
    int pu0 = -1, pu1 = -1;   // units of which this run holds a piece: begun by an earlier workgroup, begun here

    // ---- a segment of the run: slabs t .. t1 - 1 of unit (b, c), keys [key0, key1) ----
    struct Segment {
        int b, c, t, t1, nt, len;
        int64_t key0, key1;
        const uint8_t *k, *v, *ks, *vs;
    };
    auto segment = [&](int b, int c, int t, int left) {
        Segment x;
        x.b = b; x.c = c; x.t = t;
        x.nt = a.slabs(b);
        x.len = a.len(b);
        x.t1 = min(x.nt, t + left);
        x.key0 = (int64_t)t * SLAB;
        x.key1 = min((int64_t)x.len, (int64_t)x.t1 * SLAB);
        x.k = bits_ptr<const uint8_t>(a.k) + b * a.seq + c * a.head;
        x.v = bits_ptr<const uint8_t>(a.v) + b * a.seq + c * a.head;
        x.ks = bits_ptr<const uint8_t>(sc.k) + b * sc.seq + c * sc.head;
        x.vs = bits_ptr<const uint8_t>(sc.v) + b * sc.seq + c * sc.head;
        return x;
    };
    auto issue = [&](const Segment &g, int64_t key, int stage) {
        const uint32_t at = lds_k + stage * STAGE, at_s = lds_s + stage * SSTAGE;
        const uint8_t *k0 = g.k + key * C::RB, *v0 = g.v + key * C::RB;
        const int last = (int)min(g.key1 - key, (int64_t)C::KPC) - 1;   // the chunk's last key
        if constexpr (D == 128) {
            const int ln = here(lane), row = min(ln & 31, last);
            lds_stream4((ln < 32 ? g.ks : g.vs) + (key + row) * 4, at_s);
        } else {
            const int row = min(here(lane), last);
            lds_stream2(g.ks + (key + row) * 2, at_s);
            lds_stream2(g.vs + (key + row) * 2, at_s + 256);
        }
        if (last == C::KPC - 1) {
            lds_stream16_x2<true>(k0, koff[0], koff[1], at);
            lds_stream16_x2<true>(v0, voff[0], voff[1], at + 2048);
        } else {
            const int ln = here(lane);
            #pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int cidx = 64 * j + ln, kr = cidx / C::CPR, slot = cidx % C::CPR;
                const int row = min(kr, last);   // rows past the last: the last one again, hidden
                lds_stream16_nt(k0 + row * C::RB + (slot ^ k4_swz<D>(kr)) * 16, ring + stage * STAGE + j * 1024);
                lds_stream16_nt(v0 + row * C::RB + slot * 16, ring + stage * STAGE + 2048 + j * 1024);
            }
        }
    };
    // ---- a unit's queries: fragment (nb, ks) holds feature D/4 * lg + 8 ks + e of row 16 nb + lr; rows past R repeat
    // the last.  Wave w loads fragments w, w + 8, .. into LDS, 1 KB each as they are used (bf16); fp32 ones as 2 KB that
    // split_q turns into their three bf16 terms, each what the ones before leave. ----
    auto fetch_q = [&](const Segment &g) {
        const int ln = here(lane), q_lr = ln & 15, q_lg = ln >> 4;
        for (int f = wave; f < KST * NB; f += C::NWV) {
            const int ks = f % KST, row = min(f / KST * 16 + q_lr, R - 1), rt = row / G;
            const T *src = bits_ptr<const T>(a.q) + (((size_t)g.b * TT + rt) * a.Hq + (size_t)g.c * G + (row - rt * G)) * D +
                           D / 4 * q_lg + 8 * ks;
            unsigned char *dst = smem + C::OFF_Q + f * NQ * 1024;
            lds_stream16(src, dst);
            if constexpr (C::F32) lds_stream16(src + 4, dst + 1024);
        }
    };
    auto split_q = [&]() {   // (a lane reads its own 32 bytes and writes over them)
        for (int f = wave; f < KST * NB; f += C::NWV) {
            u32x4_v *p = reinterpret_cast<u32x4_v *>(smem + C::OFF_Q + f * NQ * 1024) + here(lane);
            f32x4_v x[2] = {__builtin_bit_cast(f32x4_v, p[0]), __builtin_bit_cast(f32x4_v, p[64])};
            #pragma unroll
            for (int n = 0; n < NQ; ++n) {
                bf16x8_v h;
                #pragma unroll
                for (int e = 0; e < 8; ++e) {
                    h[e] = (__bf16)x[e >> 2][e & 3];
                    x[e >> 2][e & 3] -= (float)h[e];
                }
                p[n * 64] = __builtin_bit_cast(u32x4_v, h);
            }
        }
    };
    auto q_frag = [&](int nb, int ks, int i) {
        return *reinterpret_cast<const bf16x8_v *>(smem + C::OFF_Q + (((nb * KST + ks) * NQ + i) * 64 + lane) * 16);
    };

    constexpr int STEP = C::NWV * C::KPC;
    Segment g = segment(b, c, t, left);
    int64_t key = g.key0 + wave * C::KPC;   // this wave's next chunk
    fetch_q(g);
    #pragma unroll
    for (int s = 0; s < C::PRE; ++s)
        if (key + s * STEP < g.key1) issue(g, key + s * STEP, s);
    // the wave's oldest chunk (and queries) have landed; the loads of up to `ahead` later chunks may be on their way
    auto landed = [&](int ahead) {
        static_assert(C::LOADS == 5 || C::LOADS == 6, "");
        if (ahead >= 3) {
            if constexpr (C::LOADS == 5) asm volatile("s_waitcnt vmcnt(15)" : : : "memory");
            else asm volatile("s_waitcnt vmcnt(18)" : : : "memory");
        } else if (ahead == 2) {
            if constexpr (C::LOADS == 5) asm volatile("s_waitcnt vmcnt(10)" : : : "memory");
            else asm volatile("s_waitcnt vmcnt(12)" : : : "memory");
        } else if (ahead == 1) {
            if constexpr (C::LOADS == 5) asm volatile("s_waitcnt vmcnt(5)" : : : "memory");
            else asm volatile("s_waitcnt vmcnt(6)" : : : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        }
    };
    // this wave's chunks from `key` on: behind the first, at most `most`
    auto later = [&](int64_t key, int most) { return key < g.key1 ? (int)min((g.key1 - 1 - key) / STEP, (int64_t)most) : 0; };
    for (bool first = true;; first = false) {
        const int u = g.b * Hkv + g.c;
        // the stages that the exchange held; the queries are older than these loads
        #pragma unroll
        for (int s = C::PRE; s < C::NST; ++s)
            if (key + s * STEP < g.key1) issue(g, key + s * STEP, s);
        landed(max(later(key, C::NST - 1) - (C::PRE - 1), 0));
        if constexpr (C::F32) split_q();
        __syncthreads();
        bf16x8_v qf[C::QREG ? NB : 1][KST][NQ];
        if constexpr (C::QREG) {
            #pragma unroll
            for (int nb = 0; nb < NB; ++nb)
                #pragma unroll
                for (int ks = 0; ks < KST; ++ks)
                    #pragma unroll
                    for (int i = 0; i < NQ; ++i) qf[nb][ks][i] = q_frag(nb, ks, i);
        }

        f32x4_v o[NB][DB];   // o[nb][j][i]: feature D/16 * (4 lg + i) + j of row 16 nb + lr
        float m_run[NB], l_run[NB];   // m in log2 units; sum of p
        int lim[NB];                          // the last key that row 16 nb + lr sees
        #pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            m_run[nb] = -INFINITY;
            l_run[nb] = 0.f;
            lim[nb] = g.len - TT + min(16 * nb + lr, R - 1) / G;
            #pragma unroll
            for (int db = 0; db < DB; ++db) o[nb][db] = f32x4_v{0.f, 0.f, 0.f, 0.f};
        }
        const int open_to = g.len - TT;   // keys up to here are seen by every row

        for (int stage = 0; key < g.key1; key += STEP, stage = stage == C::NST - 1 ? 0 : stage + 1) {
            landed(later(key, C::NST - 1));
            const unsigned char *st = ring + stage * STAGE, *ss = ring_s + stage * SSTAGE;
            #pragma unroll
            for (int kh = 0; kh < C::KPC / 32; ++kh) {
                // accumulator element i of block blk is key 32 kh + 4 (4 blk + i) + lg: A row 4 lg' + i of it is that key
                uint32_t kc[2][KST], vc[8];
                float ksc[2], vsc[8];
                #pragma unroll
                for (int blk = 0; blk < 2; ++blk) {
                    const int kr = 32 * kh + 16 * blk + 4 * (lr & 3) + (lr >> 2);
                    if constexpr (D == 128) {
                        const u32x4_v x = *reinterpret_cast<const u32x4_v *>(st + kr * C::RB + ((lg ^ k4_swz<D>(kr)) << 4));
                        #pragma unroll
                        for (int ks = 0; ks < KST; ++ks) kc[blk][ks] = x[ks];
                        ksc[blk] = scale_of(ss[kr * 4 + lg]);
                    } else {
                        const u32x2_v x = *reinterpret_cast<const u32x2_v *>(st + kr * C::RB + (((lg >> 1) ^ k4_swz<D>(kr)) << 4) + 8 * (lg & 1));
                        #pragma unroll
                        for (int ks = 0; ks < KST; ++ks) kc[blk][ks] = x[ks];
                        ksc[blk] = scale_of(ss[kr * 4 + (lg >> 1)]);
                    }
                }
                #pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int vr = 32 * kh + 4 * e + lg;
                    const unsigned char *p = st + 2048 + vr * C::RB + lr * (D / 32);
                    if constexpr (D == 128) vc[e] = *reinterpret_cast<const uint32_t *>(p);
                    else vc[e] = *reinterpret_cast<const uint16_t *>(p);
                    vsc[e] = scale_of(ss[C::KPC * 4 + vr * 4 + lr * C::CPR / 16]);
                }
                bf16x8_v qc[NB];
                if constexpr (!C::QREG) {
                    #pragma unroll
                    for (int nb = 0; nb < NB; ++nb) qc[nb] = q_frag(nb, 0, 0);
                }
                if (kh == C::KPC / 32 - 1) {
                    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");   // the stage is read
                    if (key + C::NST * STEP < g.key1) issue(g, key + C::NST * STEP, stage);
                }

                f32x4_v sacc[NB][2];
                bf16x8_v kf[2];
                #pragma unroll
                for (int n = 0; n < KST * NQ; ++n) {   // step ks = n / NQ, query term n % NQ
                    const int ks = n / NQ;
                    bf16x8_v qn[NB];   // the next term's, on their way from LDS
                    if constexpr (!C::QREG) {
                        if (n + 1 < KST * NQ) {
                            #pragma unroll
                            for (int nb = 0; nb < NB; ++nb) qn[nb] = q_frag(nb, (n + 1) / NQ, (n + 1) % NQ);
                        }
                    }
                    if (n % NQ == 0) {
                        #pragma unroll
                        for (int blk = 0; blk < 2; ++blk) kf[blk] = codes_bf16(kc[blk][ks], ksc[blk]);
                    }
                    #pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        #pragma unroll
                        for (int blk = 0; blk < 2; ++blk) {
                            const f32x4_v acc = n == 0 ? f32x4_v{0.f, 0.f, 0.f, 0.f} : sacc[nb][blk];
                            if constexpr (C::QREG) sacc[nb][blk] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[blk], qf[nb][ks][n % NQ], acc, 0, 0, 0);
                            else sacc[nb][blk] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[blk], qc[nb], acc, 0, 0, 0);
                        }
                    if constexpr (!C::QREG) {
                        #pragma unroll
                        for (int nb = 0; nb < NB; ++nb) qc[nb] = qn[nb];
                    }
                    if (n % 2 == 1 || !C::QREG) __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_sched_barrier(0);
                const bool open = key + C::KPC - 1 <= open_to;   // every row sees the whole chunk
                u32x4_v pk[NB][NQ];   // the probabilities' bf16 terms
                #pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    // the lane's largest score (hidden ones -inf from here on)
                    if (!open) {
                        const int seen = lim[nb] - (int)key - 32 * kh - lg;   // element e is key 4 e + lg
                        #pragma unroll
                        for (int e = 0; e < 8; ++e) sacc[nb][e >> 2][e & 3] = 4 * e <= seen ? sacc[nb][e >> 2][e & 3] : -INFINITY;
                    }
                    float mt = sacc[nb][0][0];
                    #pragma unroll
                    for (int e = 1; e < 8; ++e) mt = fmaxf(mt, sacc[nb][e >> 2][e & 3]);
                    mt *= cs;
                    if (__any(mt > m_run[nb] + kLazy4)) {
                        // the four lanes of a row agree on its maximum; rows that stay have a factor of 1
                        mt = max_over_row_lanes(mt);
                        const float mn = mt > m_run[nb] + kLazy4 ? mt : m_run[nb];
                        const float alpha = mn == m_run[nb] ? 1.f : __builtin_amdgcn_exp2f(m_run[nb] - mn);
                        l_run[nb] *= alpha;
                        m_run[nb] = mn;
                        #pragma unroll
                        for (int db = 0; db < DB; ++db) o[nb][db] *= alpha;
                    }
                    const float ms = m_run[nb] == -INFINITY ? 0.f : m_run[nb];
                    float ps = 0.f;
                    #pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        float p0 = __builtin_amdgcn_exp2f(fmaf(sacc[nb][h >> 1][2 * (h & 1)], cs, -ms));
                        float p1 = __builtin_amdgcn_exp2f(fmaf(sacc[nb][h >> 1][2 * (h & 1) + 1], cs, -ms));
                        ps += p0 + p1;
                        #pragma unroll
                        for (int n = 0; n < NQ; ++n) {
                            const uint32_t r = cvt_pk_bf16(p0, p1);
                            pk[nb][n][h] = r;
                            if (n + 1 < NQ) {
                                p0 -= bf16_lo(r);
                                p1 -= bf16_hi(r);
                            }
                        }
                    }
                    l_run[nb] += ps;
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (!open) {
                    // NaN scales in V at keys that some row does not see: out of the product, and into the rows that see them
                    uint32_t any = 0;
                    #pragma unroll
                    for (int e = 0; e < 8; ++e) any |= __float_as_uint(vsc[e]) == 0x7f800000u ? 1u : 0u;
                    if (__any(any != 0)) {
                        bf16x8_v is_nan;
                        #pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const bool nan = __float_as_uint(vsc[e]) == 0x7f800000u;
                            is_nan[e] = nan ? (__bf16)1.f : (__bf16)0.f;
                            vsc[e] = nan ? 1.f : vsc[e];
                            vc[e] = nan ? 0u : vc[e];
                        }
                        #pragma unroll
                        for (int nb = 0; nb < NB; ++nb) {
                            bf16x8_v seen;
                            #pragma unroll
                            for (int e = 0; e < 8; ++e) seen[e] = 32 * kh + 4 * e + lg <= lim[nb] - (int)key ? (__bf16)1.f : (__bf16)0.f;
                            const f32x4_v hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(is_nan, seen, f32x4_v{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                            #pragma unroll
                            for (int db = 0; db < DB; ++db)
                                #pragma unroll
                                for (int i = 0; i < 4; ++i) o[nb][db][i] = hit[i] > 0.f ? __builtin_nanf("") : o[nb][db][i];
                        }
                    }
                }
                #pragma unroll
                for (int h = 0; h < DB / 2; ++h) {   // the lane's features 2 h, 2 h + 1
                    u32x4_v f0, f1;
                    #pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        uint32_t y0, y1;
                        if (h == 0) { y0 = pair_bf16<0>(vc[2 * x], vsc[2 * x]); y1 = pair_bf16<0>(vc[2 * x + 1], vsc[2 * x + 1]); }
                        else if (h == 1) { y0 = pair_bf16<1>(vc[2 * x], vsc[2 * x]); y1 = pair_bf16<1>(vc[2 * x + 1], vsc[2 * x + 1]); }
                        else if (h == 2) { y0 = pair_bf16<2>(vc[2 * x], vsc[2 * x]); y1 = pair_bf16<2>(vc[2 * x + 1], vsc[2 * x + 1]); }
                        else { y0 = pair_bf16<3>(vc[2 * x], vsc[2 * x]); y1 = pair_bf16<3>(vc[2 * x + 1], vsc[2 * x + 1]); }
                        f0[x] = __builtin_amdgcn_perm(y1, y0, 0x05040100u);
                        f1[x] = __builtin_amdgcn_perm(y1, y0, 0x07060302u);
                    }
                    #pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        #pragma unroll
                        for (int n = 0; n < NQ; ++n) {
                            const bf16x8_v p = __builtin_bit_cast(bf16x8_v, pk[nb][n]);
                            o[nb][2 * h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_v, f0), p, o[nb][2 * h], 0, 0, 0);
                            o[nb][2 * h + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_v, f1), p, o[nb][2 * h + 1], 0, 0, 0);
                        }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }

        // ---- the segment's end.  The next one's first chunks (into the stages that the exchange leaves) and queries
        // are on their way while the waves' results are added up ----
        left -= g.t1 - g.t;
        const bool whole = g.t == 0 && g.t1 == g.nt;   // every slab of the unit ran here
        if (!whole) {
            if (first) pu0 = u;   // the run's first unit; another one that does not end here is its last
            else pu1 = u;
        }
        const bool more = left > 0;
        if (more) {
            const bool wrap = g.c + 1 == Hkv;
            g = segment(wrap ? g.b + 1 : g.b, wrap ? 0 : g.c + 1, 0, left);
            key = g.key0 + wave * C::KPC;
            #pragma unroll
            for (int s = 0; s < C::PRE; ++s)
                if (key + s * STEP < g.key1) issue(g, key + s * STEP, s);
        }
        // each wave's (max, sum of p) per row, in log2 units, and from all of them its factor
        const int x_lane = here(lane), x_lr = x_lane & 15, x_lg = x_lane >> 4;
        float2 *xml = reinterpret_cast<float2 *>(smem + C::OFF_ML);   // [8][RP]
        #pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const float lt = sum_over_row_lanes(l_run[nb]);
            if (x_lg == 0) xml[wave * C::RP + 16 * nb + x_lr] = make_float2(m_run[nb], lt);
        }
        __syncthreads();   // (also: every wave is done with its stages and the queries)
        if (more) fetch_q(g);
        float M[NB], L[NB];
        #pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            float2 ml[C::NWV];
            M[nb] = -INFINITY;
            L[nb] = 0.f;
            #pragma unroll
            for (int k = 0; k < C::NWV; ++k) {
                ml[k] = xml[k * C::RP + 16 * nb + x_lr];
                M[nb] = fmaxf(M[nb], ml[k].x);
            }
            const float mr = M[nb] == -INFINITY ? 0.f : M[nb];
            #pragma unroll
            for (int k = 0; k < C::NWV; ++k) L[nb] = fmaf(__builtin_amdgcn_exp2f(ml[k].x - mr), ml[k].y, L[nb]);
            const float wt = __builtin_amdgcn_exp2f(m_run[nb] - mr);
            #pragma unroll
            for (int db = 0; db < DB; ++db) o[nb][db] *= wt;
        }
        // the sums, XD feature quads at a time: every wave's fragments to LDS as they are (1 KB each), wave w adds up
        // the w-th of them.  Quad q is features D/4 * lg + 4 q .. + 3: o[nb][4 q % DB + e][4 q / DB].
        f32x4_v *xo = reinterpret_cast<f32x4_v *>(smem + C::OFF_X) + x_lane;
        #pragma unroll
        for (int d0 = 0; d0 < DB; d0 += C::XD) {
            if (d0 > 0) __syncthreads();
            #pragma unroll
            for (int nb = 0; nb < NB; ++nb)
                #pragma unroll
                for (int db = 0; db < C::XD; ++db) {
                    const int j = 4 * (d0 + db) % DB, i = 4 * (d0 + db) / DB;
                    xo[((nb * C::XD + db) * C::NWV + wave) * 64] = f32x4_v{o[nb][j][i], o[nb][j + 1][i], o[nb][j + 2][i], o[nb][j + 3][i]};
                }
            __syncthreads();
            if (wave < NB * C::XD) {
                const int nb = wave / C::XD, db = d0 + wave % C::XD, r = 16 * nb + x_lr;
                f32x4_v y = xo[wave * C::NWV * 64];
                #pragma unroll
                for (int k = 1; k < C::NWV; ++k) y += xo[(wave * C::NWV + k) * 64];
                float mr = M[0], lr_ = L[0];
                #pragma unroll
                for (int n = 1; n < NB; ++n) {
                    mr = nb == n ? M[n] : mr;
                    lr_ = nb == n ? L[n] : lr_;
                }
                const int f = D / 4 * x_lg + 4 * db;   // this lane's four features
                if (r < R) {
                    if (whole) {
                        const size_t head = out_head(a, u, r);
                        const float inv = lr_ == 0.f ? 0.f : 1.f / lr_;
                        store_quad(bits_ptr<T>(a.out) + head * D + f, y * inv);
                        if (lse && f == 0) lse[head] = lr_ == 0.f ? -INFINITY : (mr + log2f(lr_)) * kLn2;
                    } else {
                        // runs and units both advance in slab order, so piece + u numbers the pieces one after the other
                        float *pp = bits_ptr<float>(a.part) + (size_t)(piece + u) * piece_floats(R, D);
                        store_agent4(pp + r * D + f, y);
                        if (f == 0) store_agent2(pp + R * D + 2 * r, mr, lr_);
                    }
                }
            }
        }
        if (!more) break;
        __syncthreads();   // the exchange area is the last two stages
    }
    if ((pu0 < 0 && pu1 < 0) || a.merge2) return;

    // ---- arrivals; the last workgroup at a unit merges its pieces (stream.hip) ----
    const UnitPieces up0 = unit_pieces(a, max(pu0, 0)), up1 = unit_pieces(a, max(pu1, 0));
    wait_vm_stores();
    __syncthreads();
    if (tid == 0 || tid == 64) {
        const int u = tid == 0 ? pu0 : pu1;
        int last = 0;
        if (u >= 0) {
            unsigned *cnt = bits_ptr<unsigned>(a.counters) + (size_t)u * kCounterStride;
            last = arrive(cnt) == (unsigned)((tid == 0 ? up0.np : up1.np) - 1);
            if (last) reset_counter(cnt);
        }
        s_last[tid >> 6] = last;
    }
    __syncthreads();
    const int pf = piece_floats(R, D);
    const float *part = bits_ptr<const float>(a.part);
    const int last = (s_last[0] ? 1 : 0) + (s_last[1] ? 2 : 0);
    if (last == 0) return;
    const int bytes0 = (last & 1) ? up0.np * pf * 4 : 0, bytes1 = (last & 2) ? up1.np * pf * 4 : 0;
    const int at1 = (bytes0 + 1023) & ~1023;
    __shared__ float sinv[2 * MAD_MAX_VERIFY_ROWS];
    auto merge = [&](bool first_unit, bool second_unit, int at) {
        if (first_unit) load_pieces(part + (size_t)up0.p0 * pf, bytes0, smem);
        if (second_unit) load_pieces(part + (size_t)up1.p0 * pf, bytes1, smem + at);
        const MergeJob<D, T, true> j0 = {pu0, up0.np, R, smem, smem + R * D * 4, pf * 4, sinv};
        const MergeJob<D, T, true> j1 = {pu1, up1.np, R, smem + at, smem + at + R * D * 4, pf * 4, sinv + R};
        wait_vm(0);
        __syncthreads();
        if (first_unit) j0.weights(a);
        if (second_unit) j1.weights(a);
        __syncthreads();
        if (first_unit) j0.sums(a);
        if (second_unit) j1.sums(a);
    };
    if (at1 + bytes1 <= kMergeBytes) {
        merge(last & 1, last & 2, at1);
    } else {   // one after the other (each fits: plan_stream)
        merge(true, false, 0);
        __syncthreads();
        merge(false, true, 0);
    }
}

// ------------------------------------------------------------------ host ----

template <int D, int NB, typename T>
static hipError_t launch_nb(const Stream4Args &a, hipStream_t st) {
    using C = Stream4Cfg<D, NB, T>;
    hipLaunchKernelGGL((stream4_kernel<D, NB, T>), dim3((unsigned)a.n_wg), dim3(64 * C::NWV), C::SMEM, st, a);
    return hipGetLastError();
}

template <int D, typename T>
static hipError_t launch_d(const Stream4Args &a, hipStream_t st) {
    hipError_t e = hipErrorInvalidValue;
    switch ((a.T * a.G + 15) / 16) {
        case 1: e = launch_nb<D, 1, T>(a, st); break;
        case 2: e = launch_nb<D, 2, T>(a, st); break;
        case 3: e = launch_nb<D, 3, T>(a, st); break;
        case 4: e = launch_nb<D, 4, T>(a, st); break;
    }
    if (e != hipSuccess || a.merge2 == 0) return e;
    hipLaunchKernelGGL((stream_merge_kernel<D, T, true>), dim3((unsigned)(a.B * a.Hkv), (unsigned)(a.T * a.G)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_stream4(const Stream4Args &a, int dtype, int d, hipStream_t st) {
    if (dtype == MAD_BF16) return d == 64 ? launch_d<64, bf16_t>(a, st) : launch_d<128, bf16_t>(a, st);
    return d == 64 ? launch_d<64, float>(a, st) : launch_d<128, float>(a, st);
}

}  // namespace mad

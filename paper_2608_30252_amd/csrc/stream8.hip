// stream8.hip -- the target's verify attention (Sec. 2.1, Sec. 3.3; T = 1: a
// single token's) over an 8-bit cache: e4m3 codes with one scale per block of
// tokens and KV head.
//
// Mathematics.  With key j's code row kc_j, its block's scales ks_j, vs_j and
// row r's query q (cs = softmax scale * log2 e):
//   x_j = (q . kc_j) * cs * ks_j,   p_j = 2^(x_j - m),   o = sum p_j vs_j vc_j
// Codes go into the matrix products as they are: an e4m3 code is exact in bf16
// and in fp16 (one conversion instruction for two).  The K scale multiplies the
// scores; a lane's 8 scores of a 32-key step are 8 consecutive keys, so they
// share one block: one factor per step.  The V scale multiplies the
// probabilities before they are rounded.
//   S^T = K Q^T   bf16 x bf16; an fp32 query is split into three bf16 terms
//                 (24 bits), three products to the same accumulator.
//   O^T = V^T P^T fp16 x fp16.  fp16 keeps 3 bits more of a probability than
//                 bf16 (2^-12 against 2^-9 relative, which against the output's own
//                 2^-9 is nothing); its range is made up for by p' = 2^11 p vs 2^(m - y),
//                 y a row's largest x_j + log2 vs_j so far: V scales of any size meet
//                 in one sum, each row's against what that row sees.  m and y are
//                 whole numbers, so 2^(m - y) goes onto vs exactly (v_ldexp), and the
//                 running maxima to within 2^4 (2^3): m is raised, and the sum of p
//                 scaled, only where a score exceeds it by more, y, and o scaled,
//                 likewise (with 16 rows to a wave some row's maximum grows in most
//                 steps, by little), so p' <= 2^15, and fp16's precision holds down
//                 to 2^-24 of the largest p vs.  fp32: a second fp16 term holds what
//                 the first leaves (22 bits).
//
// Work decomposition.  As in stream.hip a unit is one (sequence, KV head) with
// its T * G query rows, its keys are cut into slabs (16 KB of codes), and the
// slabs of all units are dealt to one workgroup per CU (plan_stream).  Inside a
// workgroup the eight waves take chunks of 8 KB (32 keys at d 128, 64 at d 64)
// in turn, each on its own: a wave loads its chunks into its own two LDS stages,
// reads a chunk's operands into registers, issues the chunk after next into the
// place and computes, for every query row.  A code is converted once per chunk,
// no wave waits for another inside a unit, and 64 - 128 KB per CU are in flight.
// With slabs that eight waves shared, row block by row block (stream.hip's
// way), every row block's wave converted the codes again and the vector ALU was the
// bound: 16 sequences of 600 .. 12000 keys (210 MB), 64/8 heads, 6 queries 86 us.
// At a unit's end the waves' results are merged through the stages.
//   Now such batches take 59 - 71 us by their lengths (216 MB counted in 65, 3.3 TB/s;
// the chunks themselves arrive at 5.9), one sequence of 32773 keys (68 MB), 40 query
// rows, 22.5 and 4.5 for the merge, 317 keys 7.1 (kernel times; calls back to back are
// 0.5 - 1.5 shorter).  The vector ALU is busy 50 - 57 % of the time in the long ones.
// What is left beside the stream: some 5 us until every CU's first chunks are there,
// 3.6 for a unit's exchange (48 rows: 200 KB through LDS), the pieces' merge, and
// workgroups with up to a fifth more slabs than the mean.  Four waves a workgroup,
// two workgroups per CU, when V scales counted against the largest: 58.3 against 58.9
// for one such batch, but 27.8 against 25.6 for 32773 keys and 7.9 against 6.9 for 317.
//   The rows' own V reference (m, y above) takes 7 % more vector instructions than one
// for the wave, 2 % of the long calls' time, and 0.1 us off the short ones, where it
// spares the exchange between lanes for the largest scale.
//   A K row's 16-byte chunk holds features 16 c .. 16 c + 15: the first 8 are one
// 32-feature step's, the rest the next one's; the query fragments are read in
// the same order.  V^T fragments (8 keys of one feature) come from transposing
// byte reads (ds_read_b64_tr_b8).
//
// What a row does not see is left out whatever it holds: scores by selection,
// and where a step with hidden keys has NaN codes in V (0 * NaN is NaN) those are
// taken out and given back to the rows that see them.
#include "stream_device.h"

namespace mad {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_v;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_v;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_v;
typedef __attribute__((ext_vector_type(2))) float f32x2_v;
typedef int v2i_t __attribute__((ext_vector_type(2)));

constexpr float kPShift = 11.f;   // the running sums are of 2^11 p
constexpr float kLazy = 4.f;      // the maximum is raised where a score exceeds it by more (log2 units)
constexpr float kLazyV = 3.f;     // likewise that of the scores with their V scale's exponent (a scale is below 2 of those)

// T: bf16_t or float (queries and output)
template <int D, int NB, typename T>
struct Stream8Cfg {
    static constexpr bool F32 = std::is_same<T, float>::value;
    static constexpr int NWV = 8;                          // waves
    static constexpr int RB = D;                           // bytes per K (and V) row
    static constexpr int CPR = D / 16;                     // 16-byte pieces per row
    static constexpr int KPC = 4096 / D;                   // keys per chunk
    static constexpr int CHUNK = 8192;                     // K, then V
    static constexpr int LOADS = 9;                        // direct loads per chunk: 4 + 4 of 1 KB, and the scales
    static constexpr int KST = D / 32, DB = D / 16, NQ = F32 ? 3 : 1;
    static constexpr int RP = NB * 16;                     // padded query rows
    // query fragments (1 KB each), in registers where they and the accumulators leave room for the rest
    static constexpr int QBYTES = NB * KST * NQ * 1024;
    static constexpr bool QREG = NB * (KST * NQ + DB) * 4 < 120;
    static constexpr bool LATE_V = NB * DB * 4 > 96;       // V's codes are read behind the softmax, for the same reason
    static constexpr int REST = NWV * 2 * 64 + NWV * RP * 8 + QBYTES;
    static constexpr int NST = NWV * 2 * CHUNK + REST + 1536 <= 160 * 1024 ? 2 : 1;   // stages per wave
    static constexpr int RING = NWV * NST * CHUNK;         // stage 0 of every wave, then stage 1
    static constexpr int OFF_S = RING;                     // scales: 16 floats per wave and stage
    static constexpr int OFF_ML = OFF_S + NWV * 2 * 64;    // the waves' (maximum, sum) per row
    static constexpr int OFF_Q = OFF_ML + NWV * RP * 8;
    static constexpr int USED = OFF_Q + QBYTES;
    static constexpr int SMEM = USED > kMergeBytes ? USED : kMergeBytes;
    // the waves' exchange goes through the last stage of all of them, XD feature blocks at a time
    static constexpr int OFF_X = RING - NWV * CHUNK;
    static constexpr int XD = NB * DB <= 8 ? DB : NB == 2 ? 4 : NB == 1 ? 8 : 2;
    static_assert(SMEM + 2 * MAD_MAX_VERIFY_ROWS * 4 + 64 <= 160 * 1024, "LDS, with the kernel's static arrays");
    static_assert(NWV * NB * XD * 1024 <= NWV * CHUNK && NB * XD <= NWV && DB % XD == 0, "exchange");
};

// Swizzles: 16-byte chunk c of key row k sits at chunk c ^ swz(k).
//   K, ds_read_b128 (a pass: 16 lanes, rows 8 (lr / 4) + lr % 4 of two lg): at D
//   128 the rows are as long as stream.hip's at d 64; at D 64 four rows share
//   256 bytes and the rows 8 apart that a pass adds need four chunks apart.
//   V, ds_read_b64_tr_b8: a pass of 32 lanes reads one chunk of 16 consecutive
//   rows: 8 (D 128) or 4 (D 64) of them share a bank's place without it.
template <int D> __device__ __forceinline__ int k8_swz(int k) { return D == 128 ? k_swz<64>(k) : (-(k >> 3)) & 3; }
template <int D> __device__ __forceinline__ int v8_swz(int k) { return D == 128 ? (k >> 1) & 7 : (k >> 2) & 3; }

// a direct load of one dword per lane (lanes of a wave: consecutive dwords at lds)
__device__ __forceinline__ void lds_stream4(const void *src, uint32_t lds) {
    const uint32_t m = __builtin_amdgcn_readfirstlane(lds);
    uint32_t saved;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved) : "v"(src), "s"(m) : "memory");
}

__device__ __forceinline__ v2i_t lds_read_tr8(const unsigned char *p) {
    return __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) v2i_t *)(p));
}
// 8 codes in two words to bf16 / fp16 (exact)
__device__ __forceinline__ bf16x8_v codes_bf16(uint32_t lo, uint32_t hi) {
    const bf16x2_v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2_v c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return __builtin_shufflevector(__builtin_shufflevector(a, b, 0, 1, 2, 3), __builtin_shufflevector(c, d, 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ f16x8_v codes_f16(uint32_t lo, uint32_t hi) {
    const f16x2_v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
    const f16x2_v c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
    return __builtin_shufflevector(__builtin_shufflevector(a, b, 0, 1, 2, 3), __builtin_shufflevector(c, d, 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7);
}
// 0x80 in every byte that is a NaN code
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

struct KvScales {
    uint64_t k, v;
    int64_t seq, head;
    int shift;
};

template <int D, int NB, typename T>
__global__ __launch_bounds__(512, 1) void stream8_kernel(const Stream8Args args) {
    using C = Stream8Cfg<D, NB, T>;
    constexpr int KST = C::KST, DB = C::DB, NQ = C::NQ, SLAB = stream8_slab(D);
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int s_last[2];
    const StreamCtx a = load_ctx(args);
    KvScales sc = {ptr_bits(args.k_scale), ptr_bits(args.v_scale), args.s_seq, args.s_head, args.log2_block};
    asm volatile("" : "+s"(sc.k), "+s"(sc.v), "+s"(sc.seq), "+s"(sc.head), "+s"(sc.shift));

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

    // ---- loads: lane l of load j (j = 0 .. 3 for K, and for V) fetches LDS slot cidx % CPR of the chunk's row
    // cidx / CPR (cidx = 64 j + l), which holds the row's piece slot ^ swizzle(row).  The second load of a pair adds
    // 1024 to both of its addresses (an instruction offset). ----
    struct Offsets {
        uint32_t k[4], v[4];
    };
    auto offsets = [](int ln) {
        Offsets x;
        #pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int cidx = 64 * j + ln, kr = cidx / C::CPR, slot = cidx % C::CPR;
            x.k[j] = kr * C::RB + ((slot ^ k8_swz<D>(kr)) << 4) - 1024 * (j & 1);
            x.v[j] = kr * C::RB + ((slot ^ v8_swz<D>(kr)) << 4) - 1024 * (j & 1);
        }
        return x;
    };
    const Offsets kept = offsets(lane);
    constexpr int NG = C::KPC / 8;   // scales of a chunk: K's of keys 8 e .., then V's (NG each), a lane each
    constexpr int STAGE = C::NWV * C::CHUNK;   // from a wave's stage to its next
    unsigned char *ring = smem + wave * C::CHUNK;
    float *ring_s = reinterpret_cast<float *>(smem + C::OFF_S) + wave * 32;
    const uint32_t lds_k = lds_addr(ring), lds_s = lds_addr(ring_s);
    const float cs = a.cs;
    float *lse = bits_ptr<float>(a.lse);
    int pu0 = -1, pu1 = -1;   // units of which this run holds a piece: begun by an earlier workgroup, begun here

    // ---- a segment of the run: slabs t .. t1 - 1 of unit (b, c), keys [key0, key1) ----
    struct Segment {
        int b, c, t, t1, nt, len;
        int64_t key0, key1;
        const uint8_t *k, *v;
        const float *s;   // lane < NG: the K scales, else the V scales
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
        x.s = bits_ptr<const float>(lane < NG ? sc.k : sc.v) + b * sc.seq + c * sc.head;
        return x;
    };
    auto issue = [&](const Segment &g, int64_t key, int stage) {
        const uint32_t at = lds_k + stage * STAGE;
        const uint8_t *k0 = g.k + key * D, *v0 = g.v + key * D;
        const int last = (int)min(g.key1 - key, (int64_t)C::KPC) - 1;   // the chunk's last key
        const int in_block = (int)(key & ((1 << sc.shift) - 1));
        if (lane < 2 * NG)   // (the block of a key past the last: the last one's)
            lds_stream4(g.s + (key >> sc.shift) + ((in_block + min((lane & (NG - 1)) * 8, last)) >> sc.shift), lds_s + stage * 64);
        if (last == C::KPC - 1) {
            const Offsets x = C::LATE_V ? offsets(here(lane)) : kept;   // (no registers to keep them in)
            lds_stream16_x2<true>(k0, x.k[0], x.k[1], at);
            lds_stream16_x2<true>(k0, x.k[2], x.k[3], at + 2048);
            lds_stream16_x2<true>(v0, x.v[0], x.v[1], at + 4096);
            lds_stream16_x2<true>(v0, x.v[2], x.v[3], at + 6144);
        } else {
            const int ln = here(lane);
            #pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int cidx = 64 * j + ln, kr = cidx / C::CPR, slot = cidx % C::CPR;
                const int row = min(kr, last);   // rows past the last: the last one again, hidden
                lds_stream16_nt(k0 + row * D + (slot ^ k8_swz<D>(kr)) * 16, ring + stage * STAGE + j * 1024);
                lds_stream16_nt(v0 + row * D + (slot ^ v8_swz<D>(kr)) * 16, ring + stage * STAGE + 4096 + j * 1024);
            }
        }
    };
    // ---- a unit's queries: fragment (nb, ks) holds feature 16 lg + 64 (ks / 2) + 8 (ks % 2) + e of row 16 nb + lr;
    // rows past R repeat the last.  Wave w loads fragments w, w + 8, .. into LDS, 1 KB each as they are used (bf16);
    // fp32 ones as 2 KB that split_q turns into their three bf16 terms, each what the ones before leave. ----
    auto fetch_q = [&](const Segment &g) {
        const int ln = here(lane), q_lr = ln & 15, q_lg = ln >> 4;
        for (int f = wave; f < KST * NB; f += C::NWV) {
            const int ks = f % KST, row = min(f / KST * 16 + q_lr, R - 1), rt = row / G;
            const T *src = bits_ptr<const T>(a.q) + (((size_t)g.b * TT + rt) * a.Hq + (size_t)g.c * G + (row - rt * G)) * D +
                           16 * q_lg + 64 * (ks >> 1) + 8 * (ks & 1);
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
    if (key < g.key1) issue(g, key, 0);
    // the wave's oldest chunk and queries have landed, the next chunk's loads (LOADS of them) may be on their way
    auto landed = [&]() {
        static_assert(C::LOADS == 9, "");
        if (C::NST == 2 && key + STEP < g.key1) asm volatile("s_waitcnt vmcnt(9)" : : : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    };
    for (bool first = true;; first = false) {
        const int u = g.b * Hkv + g.c;
        if (C::NST == 2 && key + STEP < g.key1) issue(g, key + STEP, 1);
        landed();
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

        f32x4_v o[NB][DB];
        float m_run[NB], l_run[NB], y_run[NB];   // m in log2 units; sum of 2^11 p; y
        int lim[NB];                          // the last key that row 16 nb + lr sees
        #pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            m_run[nb] = y_run[nb] = -INFINITY;
            l_run[nb] = 0.f;
            lim[nb] = g.len - TT + min(16 * nb + lr, R - 1) / G;
            #pragma unroll
            for (int db = 0; db < DB; ++db) o[nb][db] = f32x4_v{0.f, 0.f, 0.f, 0.f};
        }
        const int open_to = g.len - TT;   // keys up to here are seen by every row

        for (int stage = 0; key < g.key1; key += STEP, stage ^= C::NST - 1) {
            landed();
            const unsigned char *st = ring + stage * STAGE;
            const float *ss = ring_s + stage * 16;
            #pragma unroll
            for (int kh = 0; kh < C::KPC / 32; ++kh) {
                // A row m of block blk is key 32 kh + 8(m/4) + 4 blk + m%4 of the chunk, so
                // accumulator element e&3 of block e>>2 is key 32 kh + 8 lg + e
                u32x4_v kc[2][KST / 2];
                v2i_t vc[DB];
                #pragma unroll
                for (int blk = 0; blk < 2; ++blk) {
                    const int kr = 32 * kh + 8 * (lr >> 2) + 4 * blk + (lr & 3);
                    #pragma unroll
                    for (int j = 0; j < KST / 2; ++j)
                        kc[blk][j] = *reinterpret_cast<const u32x4_v *>(st + kr * C::RB + (((4 * j + lg) ^ k8_swz<D>(kr)) << 4));
                }
                bf16x8_v qc[NB];
                if constexpr (!C::QREG) {
                    #pragma unroll
                    for (int nb = 0; nb < NB; ++nb) qc[nb] = q_frag(nb, 0, 0);
                }
                const float ksc = ss[4 * kh + lg], vsc = ss[NG + 4 * kh + lg];
                auto read_v = [&]() {
                    const int ln = here(lane), vr = 32 * kh + 8 * (ln >> 4) + ((ln & 15) >> 1);
                    #pragma unroll
                    for (int db = 0; db < DB; ++db)   // features db*16 + lr, keys 32 kh + 8 lg .. +7
                        vc[db] = lds_read_tr8(st + 4096 + vr * C::RB + ((db ^ v8_swz<D>(vr)) << 4) + 8 * (ln & 1));
                    if (kh == C::KPC / 32 - 1) {
                        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");   // the stage is read
                        if (key + C::NST * STEP < g.key1) issue(g, key + C::NST * STEP, stage);
                    }
                };
                if constexpr (!C::LATE_V) read_v();

                // (The scheduling fences keep one row block's, one fragment's temporaries from living beside the next's:
                // without them the kernel spills from 32 rows on.)
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
                        for (int blk = 0; blk < 2; ++blk)
                            kf[blk] = codes_bf16(kc[blk][ks >> 1][2 * (ks & 1)], kc[blk][ks >> 1][2 * (ks & 1) + 1]);
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
                const float csk = cs * ksc;
                const float v_exp = (float)((int)(__float_as_uint(vsc) >> 23) - 127);   // (0: -127)
                const int kg0 = 32 * kh + 8 * lg;   // this lane's first key of the chunk
                const bool open = key + C::KPC - 1 <= open_to;   // every row sees the whole chunk
                u32x4_v pk[NB], pl[C::F32 ? NB : 1];
                #pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    // the lane's largest score (hidden ones -inf from here on)
                    if (!open) {
                        const int seen = lim[nb] - (int)key - kg0;   // (from -63 on: a key of the unit is in the chunk)
                        #pragma unroll
                        for (int j = 0; j < 8; ++j) sacc[nb][j >> 2][j & 3] = j <= seen ? sacc[nb][j >> 2][j & 3] : -INFINITY;
                    }
                    float mt = sacc[nb][0][0];
                    #pragma unroll
                    for (int j = 1; j < 8; ++j) mt = fmaxf(mt, sacc[nb][j >> 2][j & 3]);
                    mt = mt == -INFINITY ? mt : mt * csk;   // (csk may be 0)
                    if (__any(mt > fminf(m_run[nb] + kLazy, y_run[nb] + kLazyV - v_exp))) {
                        // the four lanes of a row agree on its maxima; rows that stay have factors of 1
                        const float yt = max_over_row_lanes(mt + v_exp);
                        mt = max_over_row_lanes(mt);
                        const float mn = mt > m_run[nb] + kLazy ? ceilf(mt) : m_run[nb], yn = yt > y_run[nb] + kLazyV ? ceilf(yt) : y_run[nb];
                        const float alpha = yn == y_run[nb] ? 1.f : __builtin_amdgcn_exp2f(y_run[nb] - yn);
                        l_run[nb] *= mn == m_run[nb] ? 1.f : __builtin_amdgcn_exp2f(m_run[nb] - mn);
                        m_run[nb] = mn;
                        y_run[nb] = yn;
                        #pragma unroll
                        for (int db = 0; db < DB; ++db) o[nb][db] *= alpha;
                    }
                    // (a whole number within some 140 of 0, or a NaN before the row's first key; where rv would pass 2^100, p
                    // is below 2^-80)
                    const float rv = fminf(__builtin_amdgcn_ldexpf(vsc, (int)fmaxf(m_run[nb] - y_run[nb], -1000.f)), 0x1p100f);
                    const float ms = m_run[nb] == -INFINITY ? -kPShift : m_run[nb] - kPShift;
                    float x[8];
                    #pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = fmaf(sacc[nb][j >> 2][j & 3], csk, -ms);
                    if (!open) {   // (-inf * 0 is NaN)
                        #pragma unroll
                        for (int j = 0; j < 8; ++j) x[j] = sacc[nb][j >> 2][j & 3] == -INFINITY ? -INFINITY : x[j];
                    }
                    float ps = 0.f;
                    #pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float p0 = __builtin_amdgcn_exp2f(x[2 * e]), p1 = __builtin_amdgcn_exp2f(x[2 * e + 1]);
                        ps += p0 + p1;
                        p0 *= rv;
                        p1 *= rv;
                        const f16x2_v h = __builtin_convertvector((f32x2_v{p0, p1}), f16x2_v);
                        pk[nb][e] = __builtin_bit_cast(uint32_t, h);
                        if constexpr (C::F32)
                            pl[nb][e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_v{p0 - (float)h[0], p1 - (float)h[1]}), f16x2_v));
                    }
                    l_run[nb] += ps;
                    __builtin_amdgcn_sched_barrier(0);
                }
                if constexpr (C::LATE_V) read_v();
                if (!open) {
                    // NaN codes that some row does not see: out of the product, and into the rows that see them
                    uint32_t any = 0;
                    #pragma unroll
                    for (int db = 0; db < DB; ++db) any |= nan_codes(vc[db][0]) | nan_codes(vc[db][1]);
                    if (__any(any != 0)) {
                        #pragma unroll
                        for (int db = 0; db < DB; ++db) {
                            const uint32_t n0 = nan_codes(vc[db][0]) >> 7, n1 = nan_codes(vc[db][1]) >> 7;   // 1 in each such byte
                            const f16x8_v is_nan = codes_f16(n0 * 0x38u, n1 * 0x38u);                        // 0x38: 1.0
                            #pragma unroll
                            for (int nb = 0; nb < NB; ++nb) {
                                f16x8_v seen;
                                #pragma unroll
                                for (int j = 0; j < 8; ++j) seen[j] = kg0 + j <= lim[nb] - (int)key ? (_Float16)1.f : (_Float16)0.f;
                                const f32x4_v hit = __builtin_amdgcn_mfma_f32_16x16x32_f16(is_nan, seen, f32x4_v{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                                #pragma unroll
                                for (int e = 0; e < 4; ++e) o[nb][db][e] = hit[e] > 0.f ? __builtin_nanf("") : o[nb][db][e];
                            }
                            vc[db][0] &= ~(n0 * 0xffu);
                            vc[db][1] &= ~(n1 * 0xffu);
                        }
                    }
                }
                #pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const f16x8_v vf = codes_f16(vc[db][0], vc[db][1]);
                    #pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, __builtin_bit_cast(f16x8_v, pk[nb]), o[nb][db], 0, 0, 0);
                        if constexpr (C::F32)
                            o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, __builtin_bit_cast(f16x8_v, pl[nb]), o[nb][db], 0, 0, 0);
                    }
                    if (db & 1) __builtin_amdgcn_sched_barrier(0);
                }
            }
        }

        // ---- the segment's end.  The next one's first chunks (into stage 0, which this wave has read) and queries
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
            if (C::NST == 2 && key < g.key1) issue(g, key, 0);
        }
        // each wave's (max, sum of p) per row, in log2 units, and from all of them its factor.  (The 2^11 of the running sums
        // goes here: the values' sums need fp32's range.)
        const int x_lane = here(lane), x_lr = x_lane & 15, x_lg = x_lane >> 4;
        float2 *xml = reinterpret_cast<float2 *>(smem + C::OFF_ML);   // [8][RP]
        #pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const float lt = sum_over_row_lanes(l_run[nb]);
            if (x_lg == 0) xml[wave * C::RP + 16 * nb + x_lr] = make_float2(m_run[nb], lt * 0x1p-11f);
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
            const float wt = __builtin_amdgcn_exp2f(y_run[nb] - kPShift - mr);
            #pragma unroll
            for (int db = 0; db < DB; ++db) o[nb][db] *= wt;
        }
        // the sums, XD feature blocks at a time: every wave's fragments to LDS as they are (1 KB each), wave w adds up
        // the w-th of them
        f32x4_v *xo = reinterpret_cast<f32x4_v *>(smem + C::OFF_X) + x_lane;
        #pragma unroll
        for (int d0 = 0; d0 < DB; d0 += C::XD) {
            if (d0 > 0) __syncthreads();
            #pragma unroll
            for (int nb = 0; nb < NB; ++nb)
                #pragma unroll
                for (int db = 0; db < C::XD; ++db) xo[((nb * C::XD + db) * C::NWV + wave) * 64] = o[nb][d0 + db];
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
                const int f = db * 16 + 4 * x_lg;   // this lane's four features
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
        __syncthreads();   // the exchange area is stage NST - 1
        if (C::NST == 1 && key < g.key1) issue(g, key, 0);
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
static hipError_t launch_nb(const Stream8Args &a, hipStream_t st) {
    using C = Stream8Cfg<D, NB, T>;
    hipLaunchKernelGGL((stream8_kernel<D, NB, T>), dim3((unsigned)a.n_wg), dim3(64 * C::NWV), C::SMEM, st, a);
    return hipGetLastError();
}

template <int D, typename T>
static hipError_t launch_d(const Stream8Args &a, hipStream_t st) {
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

hipError_t launch_stream8(const Stream8Args &a, int dtype, int d, hipStream_t st) {
    if (dtype == MAD_BF16) return d == 64 ? launch_d<64, bf16_t>(a, st) : launch_d<128, bf16_t>(a, st);
    return d == 64 ? launch_d<64, float>(a, st) : launch_d<128, float>(a, st);
}

}  // namespace mad

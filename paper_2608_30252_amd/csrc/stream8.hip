// stream8.hip -- the target's verify attention (Sec. 2.1, Sec. 3.3; T = 1: a
// single token's) over an 8-bit cache: e4m3 codes with one scale per block of
// tokens and KV head.  Decomposition, ring and merge are stream.hip's; a slab is
// again 32 KB of K + V, here of twice the keys.
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
//                 2^-9 is nothing); its range is made up for by p' = 2^15 p vs / vref,
//                 vref the largest V scale the wave has met in the unit: p' <= 2^15, and
//                 its precision holds down to p vs / vref = 2^-29.  fp32: a second
//                 fp16 term holds what the first leaves (22 bits).
// A K row's 16-byte chunk holds features 16 c .. 16 c + 15: the first 8 are one
// 32-feature step's, the rest the next one's; the query fragments are read in
// the same order.  V^T fragments (8 keys of one feature) come from transposing
// byte reads (ds_read_b64_tr_b8).
//
// What a row does not see is left out whatever it holds: scores by selection,
// and where a slab with hidden keys has NaN codes in V (0 * NaN is NaN) those are
// taken out and given back to the rows that see them.
#include "stream_device.h"

namespace mad {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_v;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_v;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_v;
typedef __attribute__((ext_vector_type(2))) float f32x2_v;
typedef int v2i_t __attribute__((ext_vector_type(2)));

constexpr float kPShift = 15.f;   // p' = 2^15 p

// T: bf16_t or float (queries and output)
template <int D, int NB, typename T>
struct Stream8Cfg {
    static constexpr bool F32 = std::is_same<T, float>::value;
    static constexpr int SLAB = 2 * stream_slab(D);        // keys per slab
    static constexpr int RB = D;                           // bytes per K (and V) row
    static constexpr int CPR = D / 16;                     // 16-byte chunks per row
    static constexpr int KBYTES = SLAB * RB;               // K bytes per slab (= V bytes)
    static constexpr int STAGE = 2 * KBYTES;
    static constexpr int NST = 4;                          // ring stages
    static constexpr int NWV = 8;                          // waves
    static constexpr int IPW = STAGE / 1024 / NWV + 1;     // direct loads per wave per slab: codes, and 8 scales
    static constexpr int RP = NB * 16;                     // padded query rows
    static constexpr int KS = NB == 1 ? (SLAB / 32 < 8 ? SLAB / 32 : 8) : NB == 2 ? 4 : 2;   // key groups of a slab
    static constexpr int KPG = SLAB / KS;                  // keys per group, in steps of 32
    static constexpr int QRB = D * (F32 ? 4 : 2);          // bytes per query row
    static constexpr int QBYTES = RP * QRB;
    // query areas: 2 where they are small, none (queries straight from memory) where LDS has no room
    static constexpr int QSLOTS = QBYTES <= 12288 ? 2 : QBYTES <= 24576 ? 1 : 0;
    static constexpr int OFF_S = NST * STAGE;              // scales: 64 floats per stage
    static constexpr int OFF_Q = OFF_S + NST * 256;
    static constexpr int OFF_ML = OFF_Q + QSLOTS * QBYTES;
    static constexpr int SMEM = OFF_ML + KS * RP * 8;
    static constexpr int XPASS = KS * RP * D * 4 > STAGE ? 2 : 1;   // passes of the key groups' exchange through one stage
    static_assert(STAGE == 32768 && IPW == 5 && KS * NB <= NWV && KPG % 32 == 0 && SLAB / 4 <= 64, "waves");
    static_assert(KS * RP * D * 4 <= XPASS * STAGE, "the key groups' exchange fits one stage");
    static_assert(SMEM + 2 * MAD_MAX_VERIFY_ROWS * 4 + 64 <= 160 * 1024, "LDS, with the kernel's static arrays");
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
    constexpr int KST = D / 32, DB = D / 16, NQ = C::F32 ? 3 : 1;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int s_last[2];
    const StreamCtx a = load_ctx(args);
    KvScales sc = {ptr_bits(args.k_scale), ptr_bits(args.v_scale), args.s_seq, args.s_head, args.log2_block};
    asm volatile("" : "+s"(sc.k), "+s"(sc.v), "+s"(sc.seq), "+s"(sc.head), "+s"(sc.shift));

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
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

    // ---- issue side: the next slab to load is slab i_t of unit (i_b, i_c) ----
    const int wv = __builtin_amdgcn_readfirstlane(wave);
    int i_b = b, i_c = c, i_t = t, i_left = left, i_nt = 0;
    int issued = 0, q_issued = 0, q_done = 0;   // slabs; query areas filled, and copied to registers
    int i_stage = 0;                            // stage of the slab
    int64_t i_keys = 0;                         // the unit's keys from the slab on
    const uint8_t *i_k = nullptr, *i_v = nullptr;   // the slab's K and V rows
    const float *i_s = nullptr;                     // lane < 8: the unit's K or V scales, as this lane loads them
    // scale entry e = 8 wave + lane of a stage: K's of keys 8 e .., then V's (NG each)
    constexpr int NG = C::SLAB / 8;
    const int s_e = (wave * 8 + (lane & 7)) & (2 * NG - 1), s_key = (s_e & (NG - 1)) * 8;
    auto i_unit = [&]() {
        i_nt = a.slabs(i_b);
        i_keys = a.len(i_b) - (int64_t)i_t * C::SLAB;
        i_k = bits_ptr<const uint8_t>(a.k) + i_b * a.seq + i_c * a.head + (int64_t)i_t * C::SLAB * D;
        i_v = bits_ptr<const uint8_t>(a.v) + i_b * a.seq + i_c * a.head + (int64_t)i_t * C::SLAB * D;
        i_s = bits_ptr<const float>(s_e < NG ? sc.k : sc.v) + i_b * sc.seq + i_c * sc.head;
    };
    i_unit();
    // lane l of wave load inst fetches row cidx / CPR (cidx = 64 inst + l) of the slab; LDS slot cidx % CPR of
    // the row holds its chunk slot ^ swizzle(row).  A wave's load j adds 1024 j to both of its addresses.
    constexpr int LPW = (C::IPW - 1) / 2;   // K (and V) loads per wave
    static_assert(LPW == 2, "lds_stream16_x2");
    uint32_t k_off[LPW], v_off[LPW];
    #pragma unroll
    for (int j = 0; j < LPW; ++j) {
        const int cidx = (wave * LPW + j) * 64 + lane, kr = cidx / C::CPR, slot = cidx % C::CPR;
        k_off[j] = kr * C::RB + ((slot ^ k8_swz<D>(kr)) << 4) - 1024 * j;
        v_off[j] = kr * C::RB + ((slot ^ v8_swz<D>(kr)) << 4) - 1024 * j;
    }
    const uint32_t lds_base = __builtin_amdgcn_readfirstlane(lds_addr(smem));
    const uint32_t lds0 = lds_base + wv * LPW * 1024;
    // the first slab of a unit (or of the run) needs a free query area
    auto can_issue = [&]() {
        return i_left > 0 && (C::QSLOTS == 0 || (i_t > 0 && issued > 0) || q_issued - q_done < C::QSLOTS);
    };
    auto issue = [&]() {
        if (C::QSLOTS > 0 && (i_t == 0 || issued == 0)) {
            // the unit's query rows, 1 KB per wave load; lanes past them fetch the last chunk again
            constexpr int QC = C::QRB / 16;
            unsigned char *qa = smem + C::OFF_Q + (C::QSLOTS == 2 ? (q_issued & 1) * C::QBYTES : 0);
            const T *qb = bits_ptr<const T>(a.q) + ((size_t)i_b * TT * a.Hq + (size_t)i_c * G) * D;
            for (int p = wv; p * 1024 < R * C::QRB; p += C::NWV) {
                const int ch = min(p * 64 + lane, R * QC - 1), r = ch / QC, tt = r / G;
                lds_stream16(reinterpret_cast<const unsigned char *>(qb + ((size_t)tt * a.Hq + (r - tt * G)) * D) + (ch % QC) * 16,
                             qa + p * 1024);
            }
            ++q_issued;
        }
        if (lane < 8) {   // every wave 8 of the stage's scales (the block of a key past the last: the last one's)
            const int64_t key = (int64_t)i_t * C::SLAB + min((int64_t)s_key, max(i_keys - 1, (int64_t)0));
            lds_stream4(i_s + (key >> sc.shift), lds_base + C::OFF_S + i_stage * 256 + wv * 32);
        }
        const uint32_t st = i_stage * C::STAGE;
        if (i_keys >= C::SLAB) {
            lds_stream16_x2<true>(i_k, k_off[0], k_off[1], lds0 + st);
            lds_stream16_x2<true>(i_v, v_off[0], v_off[1], lds0 + st + C::KBYTES);
        } else {
            const int last = max((int)i_keys - 1, 0);   // an empty row reads the cache's first, hidden
            #pragma unroll
            for (int j = 0; j < LPW; ++j) {
                const int inst = wv * LPW + j;
                const int cidx = inst * 64 + lane, kr = cidx / C::CPR, slot = cidx % C::CPR;
                const int key = min(kr, last);   // rows past len: the last one again, hidden
                lds_stream16_nt(i_k + key * D + (slot ^ k8_swz<D>(kr)) * 16, smem + st + inst * 1024);
                lds_stream16_nt(i_v + key * D + (slot ^ v8_swz<D>(kr)) * 16, smem + st + C::KBYTES + inst * 1024);
            }
        }
        ++issued;
        --i_left;
        i_stage = (i_stage + 1) & (C::NST - 1);
        i_keys -= C::SLAB;
        i_k += C::SLAB * D;
        i_v += C::SLAB * D;
        if (++i_t == i_nt && i_left > 0) {
            i_t = 0;
            if (++i_c == Hkv) {
                i_c = 0;
                ++i_b;
            }
            i_unit();
        }
    };

    // ---- compute side: row block rbw, key group kg of every slab ----
    const int rbw = wave % NB, kg = wave / NB, row = rbw * 16 + lr;
    const bool active = kg < C::KS;
    const int row_q = min(row, R - 1), row_t = row_q / G;   // this row's query index t
    bf16x8_v qf[NQ][KST];
    int len = 0, lim = 0, nt = 0;
    f32x4_v o[DB];
    float m_run = -INFINITY, l_run = 0.f;   // in log2 units; sum of p'
    float vref = 0.f, inv_vref = 0.f;       // the largest V scale so far (the same in every lane)
    const float cs = a.cs;

    auto start_unit = [&]() {
        nt = a.slabs(b);
        len = a.len(b);
        lim = len - TT + row_t;
        const unsigned char *qa;
        if constexpr (C::QSLOTS > 0)
            qa = smem + C::OFF_Q + (C::QSLOTS == 2 ? (q_done & 1) * C::QBYTES : 0) + row_q * C::QRB;
        else
            qa = reinterpret_cast<const unsigned char *>(bits_ptr<const T>(a.q) + (((size_t)b * TT + row_t) * a.Hq + (size_t)c * G + (row_q - row_t * G)) * D);
        #pragma unroll
        for (int ks = 0; ks < KST; ++ks) {
            const int f0 = 16 * lg + 64 * (ks >> 1) + 8 * (ks & 1);   // chunk lg + 4 (ks / 2) of the row, its half ks % 2
            if constexpr (!C::F32) {
                qf[0][ks] = *reinterpret_cast<const bf16x8_v *>(qa + f0 * 2);
            } else {
                // three bf16 terms: each what the ones before leave, to nearest
                float x[8];
                *reinterpret_cast<f32x4_v *>(x) = *reinterpret_cast<const f32x4_v *>(qa + f0 * 4);
                *reinterpret_cast<f32x4_v *>(x + 4) = *reinterpret_cast<const f32x4_v *>(qa + f0 * 4 + 16);
                #pragma unroll
                for (int i = 0; i < NQ; ++i)
                    #pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const __bf16 h = (__bf16)x[e];
                        qf[i][ks][e] = h;
                        x[e] -= (float)h;
                    }
            }
        }
        m_run = -INFINITY;
        l_run = 0.f;
        vref = inv_vref = 0.f;
        #pragma unroll
        for (int db = 0; db < DB; ++db) o[db] = f32x4_v{0.f, 0.f, 0.f, 0.f};
    };

    // 32 keys of the slab, from key 32 kh of it
    auto compute = [&](const unsigned char *st, const float *ss, int kb, int kh) {
        // A row m of block blk is key 32 kh + 8(m/4) + 4 blk + m%4 of the slab, so
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
        const float ksc = ss[4 * kh + lg], vsc = ss[NG + 4 * kh + lg];
        const int vr = 32 * kh + 8 * lg + (lr >> 1);
        #pragma unroll
        for (int db = 0; db < DB; ++db)   // features db*16 + lr, keys 32 kh + 8 lg .. +7
            vc[db] = lds_read_tr8(st + C::KBYTES + vr * C::RB + ((db ^ v8_swz<D>(vr)) << 4) + 8 * (lr & 1));
        f32x4_v sacc[2];
        #pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
            sacc[blk] = f32x4_v{0.f, 0.f, 0.f, 0.f};
            #pragma unroll
            for (int ks = 0; ks < KST; ++ks) {
                const bf16x8_v kf = codes_bf16(kc[blk][ks >> 1][2 * (ks & 1)], kc[blk][ks >> 1][2 * (ks & 1) + 1]);
                #pragma unroll
                for (int i = 0; i < NQ; ++i)
                    sacc[blk] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[i][ks], sacc[blk], 0, 0, 0);
            }
        }
        float x[8];
        float mt = -INFINITY;
        const float csk = cs * ksc;
        const int kg0 = kb + 32 * kh + 8 * lg;
        const bool open = __all(kb + C::SLAB - 1 <= lim);   // every row sees the whole slab
        #pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = sacc[j >> 2][j & 3] * csk;
        if (!open) {
            #pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = kg0 + j <= lim ? x[j] : -INFINITY;
        }
        #pragma unroll
        for (int j = 0; j < 8; ++j) mt = fmaxf(mt, x[j]);
        mt = max_over_row_lanes(mt);
        const float vm = max_over_row_lanes(vsc);
        const float mn = fmaxf(m_run, mt);
        const bool same = mn == m_run;
        const float ms = (mn == -INFINITY) ? 0.f : mn - kPShift;
        float alpha = same ? 1.f : __builtin_amdgcn_exp2f(m_run - mn);
        m_run = mn;
        const float l_alpha = alpha;
        const bool vgrew = vm > vref;   // the same in every lane
        if (vgrew) {
            inv_vref = 1.f / vm;
            alpha *= vref * inv_vref;
            vref = vm;
        }
        const float rv = vsc * inv_vref;
        float ps = 0.f;
        uint32_t pk[4], pl[4];
        #pragma unroll
        for (int e = 0; e < 4; ++e) {
            float p0 = __builtin_amdgcn_exp2f(x[2 * e] - ms), p1 = __builtin_amdgcn_exp2f(x[2 * e + 1] - ms);
            ps += p0 + p1;
            p0 *= rv;
            p1 *= rv;
            const f16x2_v h = __builtin_convertvector((f32x2_v{p0, p1}), f16x2_v);
            pk[e] = __builtin_bit_cast(uint32_t, h);
            if constexpr (C::F32)
                pl[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_v{p0 - (float)h[0], p1 - (float)h[1]}), f16x2_v));
        }
        const f16x8_v pf = __builtin_bit_cast(f16x8_v, u32x4_v{pk[0], pk[1], pk[2], pk[3]});
        l_run = fmaf(l_run, l_alpha, ps);
        if (!__all(same && !vgrew)) {
            #pragma unroll
            for (int db = 0; db < DB; ++db) o[db] *= alpha;
        }
        if (!open) {
            // NaN codes that some row does not see: out of the product, and into the rows that see them
            uint32_t any = 0;
            #pragma unroll
            for (int db = 0; db < DB; ++db) any |= nan_codes(vc[db][0]) | nan_codes(vc[db][1]);
            if (__any(any != 0)) {
                f16x8_v seen;
                #pragma unroll
                for (int j = 0; j < 8; ++j) seen[j] = kg0 + j <= lim ? (_Float16)1.f : (_Float16)0.f;
                #pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const uint32_t n0 = nan_codes(vc[db][0]) >> 7, n1 = nan_codes(vc[db][1]) >> 7;   // 1 in each such byte
                    const f32x4_v hit = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16(n0 * 0x38u, n1 * 0x38u), seen, f32x4_v{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);   // 0x38: 1.0
                    #pragma unroll
                    for (int e = 0; e < 4; ++e) o[db][e] = hit[e] > 0.f ? __builtin_nanf("") : o[db][e];
                    vc[db][0] &= ~(n0 * 0xffu);
                    vc[db][1] &= ~(n1 * 0xffu);
                }
            }
        }
        #pragma unroll
        for (int db = 0; db < DB; ++db) {
            const f16x8_v vf = codes_f16(vc[db][0], vc[db][1]);
            o[db] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf, o[db], 0, 0, 0);
            if constexpr (C::F32)
                o[db] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, __builtin_bit_cast(f16x8_v, u32x4_v{pl[0], pl[1], pl[2], pl[3]}), o[db], 0, 0, 0);
        }
    };

    // ---- end of a unit's run in this workgroup: the key groups' results are exchanged through the stage just
    // read and every thread merges whole 16-byte chunks, the unit's result or its piece (stream.hip) ----
    int pu0 = -1, pu1 = -1;   // units of which this run holds a piece: begun by an earlier workgroup, begun here
    float *lse = bits_ptr<float>(a.lse);
    auto flush = [&](unsigned char *st, bool from0) {
        const bool whole = from0 && t == nt;   // every slab of the unit ran here
        const int u = b * Hkv + c;
        if (!from0) pu0 = u;
        else if (!whole) pu1 = u;
        constexpr int DP = D / C::XPASS, QP = DP / 4;                 // features, chunks of a row per pass
        float2 *xml = reinterpret_cast<float2 *>(smem + C::OFF_ML);   // [KS][RP]
        const float lt = sum_over_row_lanes(l_run);
        #pragma unroll
        for (int ps = 0; ps < C::XPASS; ++ps) {
            __syncthreads();   // every wave is done with the stage
            if (active) {
                #pragma unroll
                for (int db = 0; db < DP / 16; ++db)
                    *reinterpret_cast<f32x4_v *>(st + ((kg * C::RP + row) * QP + ((db * 4 + lg) ^ (row & (QP - 1) & 15))) * 16) =
                        o[ps * (DP / 16) + db] * vref;
                // (max, sum of p) in log2 units: the sum is of p' = 2^15 p
                if (ps == 0 && lg == 0) xml[kg * C::RP + row] = make_float2(m_run - kPShift, lt);
            }
            __syncthreads();
            for (int x = tid; x < R * QP; x += 512) {
                const int r = x / QP, ch = x % QP;
                float m[C::KS], M = -INFINITY, L = 0.f;
                f32x4_v y = f32x4_v{0.f, 0.f, 0.f, 0.f};
                #pragma unroll
                for (int k = 0; k < C::KS; ++k) {
                    m[k] = xml[k * C::RP + r].x;
                    M = fmaxf(M, m[k]);
                }
                #pragma unroll
                for (int k = 0; k < C::KS; ++k) {
                    const float wt = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[k] - M);
                    const f32x4_v v = *reinterpret_cast<const f32x4_v *>(st + ((k * C::RP + r) * QP + (ch ^ (r & (QP - 1) & 15))) * 16);
                    L = fmaf(wt, xml[k * C::RP + r].y, L);
                    #pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = fmaf(wt, v[e], y[e]);
                }
                if (whole) {
                    const size_t head = out_head(a, u, r);
                    const float inv = L == 0.f ? 0.f : 1.f / L;
                    store_quad(bits_ptr<T>(a.out) + head * D + ps * DP + ch * 4, y * inv);
                    if (lse && ps == 0 && ch == 0) lse[head] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
                } else {
                    // runs and units both advance in slab order, so piece + u numbers the pieces one after the other
                    float *pp = bits_ptr<float>(a.part) + (size_t)(piece + u) * piece_floats(R, D);
                    store_agent4(pp + r * D + ps * DP + ch * 4, y);
                    if (ps == 0 && ch == 0) store_agent2(pp + R * D + 2 * r, M, L);
                }
            }
        }
    };

    while (issued < C::NST - 1 && can_issue()) issue();
    bool first = true;   // the run's first unit
    int c_stage = 0;
    for (int i = 0; i < left; ++i) {
        if (issued <= i) {   // the slab waited for a query area, which every wave has read by now
            __syncthreads();
            issue();
        }
        wait_vm(C::IPW * (issued - 1 - i));   // slab i has landed (this wave's part; newer query loads only make it stricter)
        __syncthreads();                      // ... every wave's part; stage (i-1) % NST is free
        while (issued < i + C::NST && can_issue()) issue();
        if (t == 0 || i == 0) {
            start_unit();
            ++q_done;
        }
        unsigned char *st = smem + c_stage * C::STAGE;
        const float *ss = reinterpret_cast<const float *>(smem + C::OFF_S + c_stage * 256);
        c_stage = (c_stage + 1) & (C::NST - 1);
        if (active) {
            #pragma unroll
            for (int h = 0; h < C::KPG / 32; ++h) compute(st, ss, t * C::SLAB, kg * (C::KPG / 32) + h);
        }
        ++t;
        if (t == nt || i == left - 1) {
            flush(st, !first || i + 1 == t);
            first = false;
            if (t == nt) {
                t = 0;
                if (++c == Hkv) {
                    c = 0;
                    ++b;
                }
            }
        }
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
    static_assert(kMergeBytes <= C::OFF_S, "the pieces lie in the ring");
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

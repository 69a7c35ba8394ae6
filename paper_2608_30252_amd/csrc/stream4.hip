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
//   O = P V       bf16 x bf16: a probability is rounded to bf16 (2^-8 relative,
//                 the output's own rounding); V's values keep bf16's range, so keys
//                 of any size meet in one sum.  fp32: three bf16 terms.
// The sum of the probabilities, and lse, take them unrounded, so an output that few keys
// dominate carries the rounding of their weights beside its own.  Root mean square error
// against 64 bits, keys and values with a few large channels: 317 keys 8.0e-4, with fp32
// probabilities 7.8e-4; 32773 keys 9.6e-4 either way.
// m is raised, and the sums scaled, only where a score exceeds it by more than 4
// (log2 units; p <= 2^4 loses nothing): some row's maximum grows in most steps, by
// little.
//
// Operands without a transposition.  A matrix step takes 32 keys in any order that
// both operands share.
//   K: lane (lr, lg) (lane = 16 lg + lr) reads a quarter of one key's row (features
//      D/4 * lg ..), which one scale covers, and the queries' fragments hold the
//      same features.
//   V: lane (lr, lg) reads, for its eight keys, the D/16 features that start at
//      D/16 * lr.  The conversion gives pairs of features of a key, where a product
//      over keys wants pairs of keys of a feature.  The sparse product (A has two of
//      every four entries of a row) takes them as they are: its 64 entries are (key,
//      feature of the pair), and A's index keeps the even or the odd ones, so that
//      the probabilities meet one feature of each pair.  Two of them cost what two
//      dense ones do, and the byte permutes that would form pairs of keys are not
//      there (16 sequences, 48 rows: 47 us with them, 44).
// The order of the keys follows from the sparse operand's: accumulator element i of
// the scores' block blk in lane group lg is key 16 (lg / 2) + 4 i + (lg ^ 2 blk), and
// that is how the K rows are laid out and the V rows are read.
//
// Work decomposition.  Units (sequence, KV head) are cut into pieces, one to a
// workgroup (plan_stream4); inside it the eight waves (or four: two workgroups to a
// CU) take chunks of 4 KB (32 keys at d 128, 64 at d 64) in turn, each through its
// own ring of LDS stages, for every query row, and add up at the end.  No run of
// slabs crosses from one unit to the next (plan_stream's do where that balances
// better): the code for it took registers from the loop and the runs themselves cost
// more than they balanced (16 sequences of 600 .. 12000 keys: 60 us against 47 by
// unit; 40 such, 32 rows: 83 against 45).  The unit's pieces are merged by its last workgroup, or by
// a second launch.
//
// What bounds it: its waves' chains of instructions.  A chunk of 32 keys by 48 rows
// takes a wave about 64 conversions, 24 dense and 24 sparse products, 24 exponentials
// and some 190 others, scores, exponentials, conversions and products one after the
// other, with two waves to a SIMD to fill each other's gaps: the vector ALU is 58 %
// busy, the matrix cores 24 %, neither the limit; without its loads the kernel takes
// nearly as long.
// Beside that a start of 5 us, 3.5 for the waves' exchange at 48 rows, and, with
// ragged lengths, pieces up to a third longer than the mean.  Waves with more chunks
// ahead of them go first (s_setprio), so that the workgroup's waves end together:
// 2 - 6 us of 47.
// Measured (us, d 128 unless given): 16 sequences of 600 .. 12000 keys, 64/8 heads,
// 6 queries: 40 - 47 by the lengths (2.6 - 3.0 TB/s), 1 query 25 (4.2 TB/s); one of
// 32773 keys, 5 queries, 21 - 22; one of 131072 keys, 1 query 31 (4.6 TB/s); 64 of
// 2000, 1 query 28 (4.9 TB/s); one of 317 keys, d 64, 6.0.  fp32: four of 32773 keys,
// 32/8 heads, 5 queries, 55 (2.6 TB/s); 16 of 600 .. 12000, d 64, 3 queries, 26.
//
// What a row does not see is left out whatever it holds: scores by selection, rows
// past the length are never read, and where a step with hidden keys has a NaN
// scale in V (0 * NaN is NaN) its keys are taken out and NaN given to the rows that
// see them.
#include "stream_device.h"

namespace mad {

typedef __attribute__((ext_vector_type(2))) unsigned int u32x2_v;

constexpr int kLeast4 = 4;             // slabs of a piece, at least (of eight waves each takes a chunk)
constexpr int kMergeFew4 = 64 << 10;   // pieces of a unit that are merged in the launch where the units are few
constexpr int merge4_bytes(int waves) { return kMergeBytes * waves / 8; }   // ... at most: what a workgroup of that many waves has in LDS
static_assert(kMergeInLaunch <= merge4_bytes(4) && kMergeFew4 <= merge4_bytes(4), "the pieces that plan_stream4 has merged in the launch fit");
constexpr float kLazy4 = 4.f;      // the maximum is raised where a score exceeds it by more (log2 units)

// T: bf16_t or float (queries and output); W: waves of a workgroup, 8 or 4 (two workgroups to a CU)
template <int D, int NB, typename T, int W>
struct Stream4Cfg {
    static constexpr bool F32 = std::is_same<T, float>::value;
    static constexpr int NWV = W, NT = 64 * W;
    static constexpr int LDS = (160 * 1024) * W / 8;       // a workgroup's share
    static constexpr int RB = D / 2;                       // bytes per K (and V) row
    static constexpr int CPR = D / 32;                     // 16-byte pieces, and scales, per row
    static constexpr int CHUNK = 4096;                     // K, then V
    static constexpr int KPC = 2048 / RB;                  // keys per chunk
    static constexpr int SCALES = 2 * KPC * 4;             // a chunk's scales: a dword per K row, then per V row
    static constexpr int LOADS = 4 + SCALES / 256;         // direct loads per chunk: 2 + 2 of 1 KB, and the scales
    static constexpr int KST = D / 32, DB = D / 16, NQ = F32 ? 3 : 1;
    static constexpr int RP = NB * 16;                     // padded query rows
    // query fragments (1 KB each), in registers where those, the accumulators, scores and probabilities leave room for the
    // rest (two waves to a SIMD have 256 each): 48 rows, 16 sequences of 600 .. 12000 keys, 48.0 us from LDS, 46.9; of 4000
    // keys each 29.4, 28.7
    static constexpr int QBYTES = NB * KST * NQ * 1024;
    static constexpr bool QREG = NB * (KST * NQ + DB + 2 + NQ) * 4 <= 200;
    static constexpr int REST = NWV * RP * 8 + QBYTES, STAGES = NWV * (CHUNK + SCALES);
    static constexpr int NST = 4 * STAGES + REST + 1024 <= LDS ? 4 : 3;   // stages per wave
    static constexpr int RING = NST * NWV * CHUNK;         // stage 0 of every wave, then stage 1, ..
    static constexpr int OFF_S = RING;                     // scales, likewise
    static constexpr int OFF_ML = OFF_S + NST * NWV * SCALES;   // the waves' (maximum, sum) per row
    static constexpr int OFF_Q = OFF_ML + NWV * RP * 8;
    static constexpr int USED = OFF_Q + QBYTES;
    static constexpr int MERGE = merge4_bytes(W);          // pieces that are merged in the launch
    static constexpr int SMEM = USED > MERGE ? USED : MERGE;
    // the waves' exchange goes through the stages, XD feature quads of a lane at a time
    static constexpr int XD = NB * DB <= 4 * NST ? DB : NB * 4 <= 4 * NST ? 4 : 2;
    static_assert(SMEM + MAD_MAX_VERIFY_ROWS * 4 + 64 <= LDS, "LDS, with the kernel's static arrays");
    static_assert(NB * XD <= 4 * NST && DB % XD == 0, "exchange");
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

// P V for one feature of every pair: A is the 16 rows' probabilities of 32 keys, taken as the two kept of every four entries
// (2:4 sparse) of 64 that are (key, feature of a pair): the even or the odd ones; B the keys' pairs as the conversion makes
// them.  Element t of A's lane group g meets pair t of B's group 2 (g % 2) + t / 4 (t < 4 and up alike), its second four
// pairs for g >= 2.
typedef __attribute__((ext_vector_type(8))) unsigned int u32x8_v;
typedef __attribute__((ext_vector_type(16))) __bf16 bf16x16_v;
constexpr int kEven = 0x8888, kOdd = 0xdddd;
template <int FEATURE> __device__ __forceinline__ f32x4_v smfma(bf16x8_v p, u32x8_v v, f32x4_v c) {
    return __builtin_amdgcn_smfmac_f32_16x16x64_bf16(p, __builtin_bit_cast(bf16x16_v, v), c, FEATURE, 0, 0);
}

template <typename V> __device__ __forceinline__ V lds_at(uint32_t at) {
    return *(const __attribute__((address_space(3))) V *)(uintptr_t)at;
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

template <int D, int NB, typename T, int W>
__global__ __launch_bounds__(64 * W, 2) void stream4_kernel(const Stream4Args args) {
    using C = Stream4Cfg<D, NB, T, W>;
    constexpr int KST = C::KST, DB = C::DB, NQ = C::NQ, SLAB = stream8_slab(D);
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int s_last;
    const StreamCtx a = load_ctx(args);
    Kv4Scales sc = {ptr_bits(args.k_scale), ptr_bits(args.v_scale), args.s_seq, args.s_head};
    asm volatile("" : "+s"(sc.k), "+s"(sc.v), "+s"(sc.seq), "+s"(sc.head));

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lr = lane & 15, lg = lane >> 4;
    const int w = blockIdx.x;
    const int TT = a.T, G = a.G, R = TT * G, Hkv = a.Hkv;

    // ---- this workgroup's piece: slabs t .. t1 - 1 of the unit u = (b, c), keys [key0, key1) ----
    const int b = __popcll(__ballot(Hkv * a.rec.z <= w)) - 1;   // records past the last row hold the end
    const int len = a.len(b), nt = len > 0 ? (len - 1) / SLAB + 1 : 1;
    const int np = a.splits(b), rel = w - Hkv * a.wg0(b);
    const bool turn = a.by_unit == 1;   // neighbouring workgroups take the row's units in turn
    const int div = turn ? Hkv : np, x0 = rel / div, x1 = rel - x0 * div;
    const int c = turn ? x1 : x0, part = turn ? x0 : x1;
    const int u = b * Hkv + c;
    const int lo = nt / np, hi = nt - lo * np;   // hi pieces of lo + 1 slabs, then of lo
    const int t = part * lo + min(part, hi), t1 = t + lo + (part < hi ? 1 : 0);
    const int64_t key0 = (int64_t)t * SLAB, key1 = min((int64_t)len, (int64_t)t1 * SLAB);
    const uint8_t *k_base = bits_ptr<const uint8_t>(a.k) + b * a.seq + c * a.head, *v_base = bits_ptr<const uint8_t>(a.v) + b * a.seq + c * a.head;
    const uint8_t *ks_base = bits_ptr<const uint8_t>(sc.k) + b * sc.seq + c * sc.head, *vs_base = bits_ptr<const uint8_t>(sc.v) + b * sc.seq + c * sc.head;

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
    // V operand: keys 4 e + v_row (e < 4), 4 e + (v_row ^ 2) of a step
    const int v_row = (lg >> 1) | ((lg & 1) << 1);
    const uint32_t v_at = lds_k + 2048 + v_row * C::RB + lr * (D / 32), vs_at = lds_s + C::KPC * 4 + v_row * 4 + lr * C::CPR / 16;
    const uint32_t v_at2 = lds_k + 2048 + (v_row ^ 2) * C::RB + lr * (D / 32), vs_at2 = lds_s + C::KPC * 4 + (v_row ^ 2) * 4 + lr * C::CPR / 16;
    const float cs = a.cs;
    float *lse = bits_ptr<float>(a.lse);
    auto issue = [&](int64_t key, int stage) {
        const uint32_t at = lds_k + stage * STAGE, at_s = lds_s + stage * SSTAGE;
        const uint8_t *k0 = k_base + key * C::RB, *v0 = v_base + key * C::RB;
        const int last = (int)min(key1 - key, (int64_t)C::KPC) - 1;   // the chunk's last key
        if constexpr (D == 128) {
            const int ln = here(lane), row = min(ln & 31, last);
            lds_stream4((ln < 32 ? ks_base : vs_base) + (key + row) * 4, at_s);
        } else {
            const int row = min(here(lane), last);
            lds_stream2(ks_base + (key + row) * 2, at_s);
            lds_stream2(vs_base + (key + row) * 2, at_s + 256);
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
    // ---- the unit's queries: fragment (nb, ks) holds feature D/4 * lg + 8 ks + e of row 16 nb + lr; rows past R repeat
    // the last.  Wave w loads fragments w, w + W, .. into LDS, 1 KB each as they are used (bf16); fp32 ones as 2 KB that
    // split_q turns into their three bf16 terms, each what the ones before leave. ----
    auto fetch_q = [&]() {
        const int ln = here(lane), q_lr = ln & 15, q_lg = ln >> 4;
        for (int f = wave; f < KST * NB; f += C::NWV) {
            const int ks = f % KST, row = min(f / KST * 16 + q_lr, R - 1), rt = row / G;
            const T *src = bits_ptr<const T>(a.q) + (((size_t)b * TT + rt) * a.Hq + (size_t)c * G + (row - rt * G)) * D +
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
    int64_t key = key0 + wave * C::KPC;   // this wave's next chunk
    fetch_q();
    #pragma unroll
    for (int s = 0; s < C::NST; ++s)
        if (key + s * STEP < key1) issue(key + s * STEP, s);
    // the wave's oldest chunk (and queries) have landed; the loads of up to `ahead` later chunks may be on their way
    auto landed = [&](int ahead) {
        static_assert(C::LOADS == 5 || C::LOADS == 6, "");
        if (ahead >= 4) {
            if constexpr (C::LOADS == 5) asm volatile("s_waitcnt vmcnt(20)" : : : "memory");
            else asm volatile("s_waitcnt vmcnt(24)" : : : "memory");
        } else if (ahead == 3) {
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
    // this wave's chunks, and those at their end that some row does not see whole
    const int chunks = key < key1 ? (int)((key1 - 1 - key) / STEP) + 1 : 0;
    const int64_t open_key = (int64_t)len - TT - (C::KPC - 1);   // chunks up to this key: seen by every row
    const int shut = chunks - (key <= open_key ? min((int)((open_key - key) / STEP) + 1, chunks) : 0);
    // (the queries are older than the chunks)
    landed(min(chunks, C::NST));
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

    f32x4_v o[NB][DB];   // o[nb][j][i]: feature D/16 * lr + j of row 16 nb + 4 lg + i
    float m_run[NB], l_run[NB];   // m in log2 units; sum of p
    // the last key that row 16 nb + lr sees (G is a power of two)
    auto lim = [&](int nb, int lr) { return len - TT + (min(16 * nb + lr, R - 1) >> __builtin_ctz(G)); };
    #pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        m_run[nb] = -INFINITY;
        l_run[nb] = 0.f;
        #pragma unroll
        for (int db = 0; db < DB; ++db) o[nb][db] = f32x4_v{0.f, 0.f, 0.f, 0.f};
    }
    int stage = 0;
    if (chunks > 6) __builtin_amdgcn_s_setprio(3);
    for (int rest = chunks - 1; rest >= 0; --rest, key += STEP, stage = stage == C::NST - 1 ? 0 : stage + 1) {
        if (rest >= 6) {
            landed(C::NST - 1);
        } else {
            if (rest >= 4) __builtin_amdgcn_s_setprio(2);
            else if (rest >= 2) __builtin_amdgcn_s_setprio(1);
            else __builtin_amdgcn_s_setprio(0);
            landed(min(rest, C::NST - 1));
        }
        const unsigned char *st = ring + stage * STAGE, *ss = ring_s + stage * SSTAGE;
        #pragma unroll
        for (int kh = 0; kh < C::KPC / 32; ++kh) {
            // accumulator element i of block blk is key 32 kh + 16 (lg / 2) + 4 i + (lg ^ 2 blk): A row 4 lg' + i of it is that key
            uint32_t kc[2][KST], vc[8];
            float ksc[2], vsc[8];
            #pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                const int kr = 32 * kh + 16 * (lr >> 3) + 4 * (lr & 3) + ((lr >> 2) ^ (2 * blk));
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
            uint32_t at_v[2] = {v_at + stage * STAGE, v_at2 + stage * STAGE}, at_s[2] = {vs_at + stage * SSTAGE, vs_at2 + stage * SSTAGE};
            asm volatile("" : "+v"(at_v[0]), "+v"(at_v[1]), "+v"(at_s[0]), "+v"(at_s[1]));   // (the rest of an address in its instruction)
            #pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (D == 128) vc[e] = lds_at<uint32_t>(at_v[e >> 2] + (32 * kh + 4 * e) * C::RB);
                else vc[e] = lds_at<uint16_t>(at_v[e >> 2] + (32 * kh + 4 * e) * C::RB);
                vsc[e] = scale_of(lds_at<uint8_t>(at_s[e >> 2] + (32 * kh + 4 * e) * 4));
            }
            bf16x8_v qc[NB];
            if constexpr (!C::QREG) {
                #pragma unroll
                for (int nb = 0; nb < NB; ++nb) qc[nb] = q_frag(nb, 0, 0);
            }
            if (kh == C::KPC / 32 - 1) {
                asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");   // the stage is read
                if (rest >= C::NST) issue(key + C::NST * STEP, stage);
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
            }
            const bool open = rest >= shut;   // every row sees the whole chunk
            if (!open) {   // hidden scores are -inf from here on
                const int ln = here(lane), lr = ln & 15, lg = ln >> 4;
                #pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    #pragma unroll
                    for (int blk = 0; blk < 2; ++blk) {
                        const int seen = lim(nb, lr) - (int)key - 32 * kh - 16 * (lg >> 1) - (lg ^ 2 * blk);
                        #pragma unroll
                        for (int i = 0; i < 4; ++i) sacc[nb][blk][i] = 4 * i <= seen ? sacc[nb][blk][i] : -INFINITY;
                    }
                }
            }
            float mt[NB];   // the lane's largest score
            bool grows = false;
            #pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                mt[nb] = sacc[nb][0][0];
                #pragma unroll
                for (int e = 1; e < 8; ++e) mt[nb] = fmaxf(mt[nb], sacc[nb][e >> 2][e & 3]);
                mt[nb] *= cs;
                grows |= mt[nb] > m_run[nb] + kLazy4;
            }
            if (__any(grows)) {
                const int lg = here(lane) >> 4;
                #pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    // the four lanes of a row agree on its maximum; rows that stay have a factor of 1
                    const float m4 = max_over_row_lanes(mt[nb]);
                    const float mn = m4 > m_run[nb] + kLazy4 ? m4 : m_run[nb];
                    const float alpha = mn == m_run[nb] ? 1.f : __builtin_amdgcn_exp2f(m_run[nb] - mn);
                    l_run[nb] *= alpha;
                    m_run[nb] = mn;
                    f32x4_v ar;   // of the rows that this lane accumulates
                    #pragma unroll
                    for (int i = 0; i < 4; ++i) ar[i] = __shfl(alpha, 4 * lg + i);
                    #pragma unroll
                    for (int db = 0; db < DB; ++db) o[nb][db] *= ar;
                }
            }
            u32x4_v pk[NB][NQ];   // the probabilities' bf16 terms
            #pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const float ms = m_run[nb] == -INFINITY ? 0.f : m_run[nb];
                float ps[4];
                #pragma unroll
                for (int h = 0; h < 4; ++h) {
                    float p0 = __builtin_amdgcn_exp2f(fmaf(sacc[nb][h >> 1][2 * (h & 1)], cs, -ms));
                    float p1 = __builtin_amdgcn_exp2f(fmaf(sacc[nb][h >> 1][2 * (h & 1) + 1], cs, -ms));
                    ps[h] = p0 + p1;
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
                l_run[nb] += (ps[0] + ps[1]) + (ps[2] + ps[3]);
            }
            if (!open) {
                // NaN scales in V at keys that some row does not see: out of the product, and into the rows that see them
                uint32_t any = 0;
                #pragma unroll
                for (int e = 0; e < 8; ++e) any |= __float_as_uint(vsc[e]) == 0x7f800000u ? 1u : 0u;
                if (__any(any != 0)) {
                    const int ln = here(lane), lr = ln & 15, lg = ln >> 4;
                    u32x8_v is_nan;
                    #pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const bool nan = __float_as_uint(vsc[e]) == 0x7f800000u;
                        is_nan[e] = nan ? 0x3f803f80u : 0u;   // 1.0 for both features of a pair
                        vsc[e] = nan ? 1.f : vsc[e];
                        vc[e] = nan ? 0u : vc[e];
                    }
                    #pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        bf16x8_v seen;
                        #pragma unroll
                        for (int e = 0; e < 8; ++e)
                            seen[e] = 32 * kh + 16 * (lg >> 1) + 4 * (e & 3) + (lg ^ 2 * (e >> 2)) <= lim(nb, lr) - (int)key ? (__bf16)1.f : (__bf16)0.f;
                        const f32x4_v hit = smfma<kEven>(seen, is_nan, f32x4_v{0.f, 0.f, 0.f, 0.f});
                        #pragma unroll
                        for (int db = 0; db < DB; ++db)
                            #pragma unroll
                            for (int i = 0; i < 4; ++i) o[nb][db][i] = hit[i] > 0.f ? __builtin_nanf("") : o[nb][db][i];
                    }
                }
            }
            #pragma unroll
            for (int h = 0; h < DB / 2; ++h) {   // the lane's features 2 h, 2 h + 1
                u32x8_v v2;
                #pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (h == 0) v2[e] = pair_bf16<0>(vc[e], vsc[e]);
                    else if (h == 1) v2[e] = pair_bf16<1>(vc[e], vsc[e]);
                    else if (h == 2) v2[e] = pair_bf16<2>(vc[e], vsc[e]);
                    else v2[e] = pair_bf16<3>(vc[e], vsc[e]);
                }
                #pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    #pragma unroll
                    for (int n = 0; n < NQ; ++n) {
                        const bf16x8_v p = __builtin_bit_cast(bf16x8_v, pk[nb][n]);
                        o[nb][2 * h] = smfma<kEven>(p, v2, o[nb][2 * h]);
                        o[nb][2 * h + 1] = smfma<kOdd>(p, v2, o[nb][2 * h + 1]);
                    }
            }
        }
    }

    // each wave's (max, sum of p) per row, in log2 units, and from all of them its factor
    const int x_lane = here(lane), x_lr = x_lane & 15, x_lg = x_lane >> 4;
    float2 *xml = reinterpret_cast<float2 *>(smem + C::OFF_ML);   // [W][RP]
    #pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const float lt = sum_over_row_lanes(l_run[nb]);
        if (x_lg == 0) xml[wave * C::RP + 16 * nb + x_lr] = make_float2(m_run[nb], lt);
    }
    __syncthreads();   // (also: every wave is done with its stages)
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
        f32x4_v wr;
        #pragma unroll
        for (int i = 0; i < 4; ++i) wr[i] = __shfl(wt, 4 * x_lg + i);
        #pragma unroll
        for (int db = 0; db < DB; ++db) o[nb][db] *= wr;
    }
    // the sums, some feature quads at a time: every wave's fragments to LDS as they are (1 KB each), wave w adds up every
    // W-th of them.  Quad q is features D/16 * lr + 4 (q % (D/64)) .. + 3 of row 4 lg + q / (D/64) of a block.
    const UnitPieces up = unit_pieces(a, u);
    f32x4_v *xo = reinterpret_cast<f32x4_v *>(smem) + x_lane;
    #pragma unroll
    for (int d0 = 0; d0 < DB; d0 += C::XD) {
        if (d0 > 0) __syncthreads();
        #pragma unroll
        for (int nb = 0; nb < NB; ++nb)
            #pragma unroll
            for (int db = 0; db < C::XD; ++db) {
                const int j = 4 * ((d0 + db) % (D / 64)), i = (d0 + db) / (D / 64);
                xo[((nb * C::XD + db) * C::NWV + wave) * 64] = f32x4_v{o[nb][j][i], o[nb][j + 1][i], o[nb][j + 2][i], o[nb][j + 3][i]};
            }
        __syncthreads();
        for (int x = wave; x < NB * C::XD; x += C::NWV) {
            const int nb = x / C::XD, db = d0 + x % C::XD, row = 4 * x_lg + db / (D / 64), r = 16 * nb + row;
            f32x4_v y = xo[x * C::NWV * 64];
            #pragma unroll
            for (int k = 1; k < C::NWV; ++k) y += xo[(x * C::NWV + k) * 64];
            float mr = M[0], lr_ = L[0];
            #pragma unroll
            for (int n = 1; n < NB; ++n) {
                mr = nb == n ? M[n] : mr;
                lr_ = nb == n ? L[n] : lr_;
            }
            mr = __shfl(mr, row);
            lr_ = __shfl(lr_, row);
            const int f = D / 16 * x_lr + 4 * (db % (D / 64));   // this lane's four features
            if (r < R) {
                if (np == 1) {
                    const size_t head = out_head(a, u, r);
                    const float inv = lr_ == 0.f ? 0.f : 1.f / lr_;
                    store_quad(bits_ptr<T>(a.out) + head * D + f, y * inv);
                    if (lse && f == 0) lse[head] = lr_ == 0.f ? -INFINITY : (mr + log2f(lr_)) * kLn2;
                } else {
                    float *pp = bits_ptr<float>(a.part) + (size_t)(up.p0 + part) * piece_floats(R, D);
                    store_agent4(pp + r * D + f, y);
                    if (f == 0) store_agent2(pp + R * D + 2 * r, mr, lr_);
                }
            }
        }
    }
    if (np == 1 || a.merge2) return;

    // ---- arrivals; the last workgroup at a unit merges its pieces ----
    wait_vm_stores();
    __syncthreads();
    if (tid == 0) {
        unsigned *cnt = bits_ptr<unsigned>(a.counters) + (size_t)u * kCounterStride;
        s_last = arrive(cnt) == (unsigned)(np - 1);
        if (s_last) reset_counter(cnt);
    }
    __syncthreads();
    if (!s_last) return;
    const int pf = piece_floats(R, D);
    __shared__ float sinv[MAD_MAX_VERIFY_ROWS];
    load_pieces<C::NT>(bits_ptr<const float>(a.part) + (size_t)up.p0 * pf, np * pf * 4, smem);   // (they fit: plan_stream4)
    const MergeJob<D, T, true, C::NT> job = {u, np, R, smem, smem + R * D * 4, pf * 4, sinv};
    wait_vm(0);
    __syncthreads();
    job.weights(a);
    __syncthreads();
    job.sums(a);
}

// ------------------------------------------------------------------ host ----

template <int D, int NB, typename T, int W>
static hipError_t launch_w(const Stream4Args &a, hipStream_t st) {
    using C = Stream4Cfg<D, NB, T, W>;
    hipLaunchKernelGGL((stream4_kernel<D, NB, T, W>), dim3((unsigned)a.n_wg), dim3(C::NT), C::SMEM, st, a);
    return hipGetLastError();
}
template <int D, int NB, typename T>
static hipError_t launch_nb(const Stream4Args &a, hipStream_t st) {
    if constexpr (!std::is_same<T, float>::value) {
        if (a.waves == 4) return launch_w<D, NB, T, 4>(a, st);
    }
    return launch_w<D, NB, T, 8>(a, st);
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

// The pieces: every workgroup one of at most `share` slabs, the smallest share whose pieces find a workgroup's place each
// (a second round of workgroups costs its start and its end again: 16 sequences of 600 .. 12000 keys, 48 rows, 43 us in 512
// places, 54 with pieces for 768).
//
// Eight waves, one workgroup to a CU, while every unit has a CU; above, four waves and two workgroups to a CU (bf16; in fp32
// the queries' three terms leave no room for a second one).  Eight -> four, us, d 128: up to 256 units, 20 sequences of 2000
// keys, 8 KV heads, 15.8 -> 17.5; 32 of 300 .. 6000, 64 rows, 57 -> 62; one of 32773, 40 rows, 23.2 -> 24.1; more units: 40
// sequences of 1000 keys, 20.4 -> 15.5; 40 of 300 .. 6000, 32 rows, 57 -> 44; 64 of 2000, 33 -> 29.
void plan_stream4(Stream4Args &a, int B, int Hkv, int d, int dtype, const int *n_keys) {
    const int slab = stream8_slab(d);
    const int64_t units = (int64_t)B * Hkv;
    int64_t total = 0;
    int nt[kMaxB], nt_max = 1;
    for (int b = 0; b < B; ++b) {
        nt[b] = n_keys[b] > 0 ? (n_keys[b] - 1) / slab + 1 : 1;
        a.row[b].x = n_keys[b];
        total += (int64_t)nt[b] * Hkv;
        nt_max = nt[b] > nt_max ? nt[b] : nt_max;
    }
    a.B = B;
    a.Hkv = Hkv;
    a.waves = units > kStreamWGs && dtype == MAD_BF16 ? 4 : 8;
    const int64_t places = kStreamWGs * 8 / a.waves;
    int np_max;
    auto deal = [&](int64_t share) {   // -> workgroups
        a.wgs = 0;
        np_max = 1;
        for (int b = 0; b < B; ++b) {
            const int k = (int)((nt[b] - 1) / share + 1);
            a.row[b].z = a.wgs;
            a.wgs += k;
            np_max = k > np_max ? k : np_max;
        }
        for (int b = B; b < kMaxB; ++b) a.row[b].z = a.wgs;
        return (int64_t)a.wgs * Hkv;
    };
    int64_t share = units >= places ? nt_max : (total + places - 1) / places;   // (no more places than units: whole ones)
    if (share < kLeast4) share = kLeast4;
    while (deal(share) > places && share < nt_max) share += 1 + share / 64;
    a.n_wg = a.wgs * Hkv;
    // Neighbouring workgroups take the row's units in turn, each XCD its own (plan_stream), where the pieces are short; else a
    // unit's pieces, us: pieces of 16 slabs, 48 rows, 8 sequences of 4000 keys 23.0 -> 21.6, 16 of 2000 21.9 -> 21.3; of 8, 32
    // rows, 16 of 1000, 13.5 -> 13.1.  Of 16, 4 rows, 4 of 8000, 13.5 -> 14.1, 8 rows, 8 of 4000, 13.6 -> 13.8; of 60 and more no
    // difference (16 of 600 .. 12000 keys, 48 rows, 43.7 -> 43.6).
    a.by_unit = Hkv % 8 == 0 && share <= (a.T * a.G >= 32 ? 16 : a.T * a.G > 16 ? 3 : 0) ? 1 : 2;
    // Merged by a unit's last workgroup or by a second launch, of what LDS there is.  Second launch -> in the launch, us, 8 KV
    // heads: up to 48 KB, 8 sequences of 1000 keys, 42 KB, 11.7 -> 11.1, one of 1000 10.9 -> 10.3, 4 of 8000, 17 KB, 14.1 -> 13.5;
    // many units, 16 of 600 .. 12000, 75 KB, 49.1 -> 43.6, 8 of 4000, 100 KB, 22.6 -> 21.6; few units and more, one of 32773, 129
    // KB, 14.8 -> 15.9, 4 of 1500, 125 KB, 13.1 -> 14.2, 4 of 2000, 83 KB, 11.4 -> 12.0.
    const int64_t bytes = (int64_t)np_max * piece_floats(a.T * a.G, d) * 4;
    const bool in_launch = bytes <= kMergeInLaunch || (units >= 64 && bytes <= merge4_bytes(a.waves)) ||
                           (units >= 32 && np_max <= 4 && bytes <= kMergeFew4);
    a.merge2 = np_max > 1 && !in_launch ? 1 : 0;
}

// The counters, and the pieces of units that are not whole: a piece's number is its workgroup's and its unit's, and from as
// many units as places on all are whole.  A workspace holds every call of at most these sizes, so that fewer units (B of 64
// whole ones, then B of 1) and fewer KV heads of larger groups count: never less where a size grows.
size_t verify4_ws_bytes(int B, int Hq, int Hkv, int d, int T) {
    constexpr int64_t places = 2 * kStreamWGs;
    const int64_t units = (int64_t)B * Hkv, most = (units < places ? units : places - 1) + places;
    const int rows = query_rows(T, Hq < kMaxGroup ? Hq : kMaxGroup);
    return kCounterRegionBytes + align256((size_t)most * piece_floats(rows, d) * 4);
}

hipError_t launch_stream4(const Stream4Args &a, int dtype, int d, hipStream_t st) {
    if (dtype == MAD_BF16) return d == 64 ? launch_d<64, bf16_t>(a, st) : launch_d<128, bf16_t>(a, st);
    return d == 64 ? launch_d<64, float>(a, st) : launch_d<128, float>(a, st);
}

}  // namespace mad

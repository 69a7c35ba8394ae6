// stream_device.h -- what the attention kernels over long key streams share
// (stream.hip: bf16 caches; stream8.hip: 8-bit caches): their kernel arguments,
// the numbering of a unit's pieces, and the merge of pieces in the launch and
// as a launch of its own.
#pragma once
#include <type_traits>

#include "mad_device.h"
#include "mad_internal.h"

namespace mad {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_v;
typedef __attribute__((ext_vector_type(4))) float f32x4_v;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4_v;

// Lanes l, l^16, l^32, l^48 hold the same query row: two lane swaps reduce over the four.
__device__ __forceinline__ float max_over_row_lanes(float v) { return pair_max<32>(pair_max<16>(v)); }
__device__ __forceinline__ float sum_over_row_lanes(float v) { return pair_sum<32>(pair_sum<16>(v)); }

// The kernel arguments, read at entry in one batch (one wait) and kept: left to
// the compiler they are read in dependent rounds where they are used, each a
// miss to host memory once the key stream has swept the L2.  The row records
// come in the same batch, one per lane, and are taken from there by readlane.
struct StreamCtx {
    uint64_t q, k, v, out, lse, part, counters;
    int64_t seq, head;
    float cs;
    int cap, Hq, Hkv, G, T, base, rem, by_unit, merge2, rows, wgs;   // rows, wgs: slabs and (by_unit) workgroups of one KV head over all rows
    int4 rec;   // lane b: row b's record
    __device__ __forceinline__ int tile0(int b) const { return __builtin_amdgcn_readlane(rec.w, b); }
    __device__ __forceinline__ int slabs(int b) const { return (b == kMaxB - 1 ? rows : tile0(b + 1)) - tile0(b); }
    __device__ __forceinline__ int wg0(int b) const { return __builtin_amdgcn_readlane(rec.z, b); }
    __device__ __forceinline__ int splits(int b) const { return (b == kMaxB - 1 ? wgs : wg0(b + 1)) - wg0(b); }
    __device__ __forceinline__ int len(int b) const { return __builtin_amdgcn_readlane(rec.x, b); }
};
__device__ __forceinline__ StreamCtx load_ctx(const StreamArgs &a) {
    StreamCtx x;
    x.rec = a.row[threadIdx.x & 63];
    x.q = ptr_bits(a.q); x.k = ptr_bits(a.k); x.v = ptr_bits(a.v); x.out = ptr_bits(a.out); x.lse = ptr_bits(a.lse);
    x.part = ptr_bits(a.part); x.counters = ptr_bits(a.counters);
    x.seq = a.seq; x.head = a.head;
    x.cs = a.scale_log2;
    x.cap = a.cap; x.Hq = a.Hq; x.Hkv = a.Hkv; x.G = a.G; x.T = a.T; x.base = a.base; x.rem = a.rem;
    x.by_unit = a.by_unit; x.merge2 = a.merge2; x.rows = a.rows; x.wgs = a.wgs;
    asm volatile("" : "+s"(x.q), "+s"(x.k), "+s"(x.v), "+s"(x.out), "+s"(x.lse), "+s"(x.part),
                 "+s"(x.counters), "+s"(x.seq), "+s"(x.head), "+s"(x.cs));
    asm volatile("" : "+s"(x.cap), "+s"(x.Hq), "+s"(x.Hkv), "+s"(x.G), "+s"(x.T), "+s"(x.base), "+s"(x.rem),
                 "+s"(x.by_unit), "+s"(x.merge2), "+s"(x.rows), "+s"(x.wgs));
    return x;
}

// where unit u's pieces are: np of them, the first numbered p0
struct UnitPieces {
    int p0, np;
};
__device__ __forceinline__ UnitPieces unit_pieces(const StreamCtx &a, int u) {
    const int b = u / a.Hkv, c = u - b * a.Hkv;
    if (a.by_unit) {
        const int k = a.splits(b);
        return {a.Hkv * a.wg0(b) + c * k + u, k};
    }
    const int nt = a.slabs(b), s0 = a.Hkv * a.tile0(b) + c * nt, w0 = stream_owner(s0, a.base, a.rem);
    return {w0 + u, stream_owner(s0 + nt - 1, a.base, a.rem) - w0 + 1};
}

// A piece in the workspace: [R][D] unnormalised o, [R] (max in log2 units, sum),
// padded to 16 bytes.
__host__ __device__ constexpr int piece_floats(int R, int d) { return (R * (d + 2) + 3) & ~3; }

__device__ __forceinline__ size_t out_head(const StreamCtx &a, int u, int row) {
    const int b = u / a.Hkv, c = u - b * a.Hkv, tt = row / a.G;
    return ((size_t)b * a.T + tt) * a.Hq + (size_t)c * a.G + (row - tt * a.G);
}

// four adjacent features of an output row
__device__ __forceinline__ void store_quad(bf16_t *p, f32x4_v y) {
    *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
}
__device__ __forceinline__ void store_quad(float *p, f32x4_v y) { *reinterpret_cast<f32x4_v *>(p) = y; }

// NAN_LSE: a row that saw NaN has an lse of NaN (else -inf).
// Log-sum-exp merge of the nr rows of unit u from its np pieces as they lie in
// LDS, by a workgroup of 512 threads: eight lanes per row turn the pieces'
// (max, sum) into weights, then (behind a barrier) one thread per feature quad.
// Piece p's o rows are at so + p * po bytes, its (max, sum) pairs at sm + p * po.
template <int D, typename T, bool NAN_LSE = false>
struct MergeJob {
    int u, np, nr;
    unsigned char *so, *sm;
    int po;
    float *sinv;   // [nr]

    __device__ __forceinline__ void weights(const StreamCtx &a) const {
        for (int r = threadIdx.x >> 3; r < nr; r += 64) {
            const int l8 = threadIdx.x & 7;
            float M = -INFINITY, L = 0.f;
            for (int p = l8; p < np; p += 8) M = fmaxf(M, reinterpret_cast<const float2 *>(sm + p * po)[r].x);
            M = group_max<8>(M);
            const float mr = M == -INFINITY ? 0.f : M;
            for (int p = l8; p < np; p += 8) {
                float2 *v = reinterpret_cast<float2 *>(sm + p * po) + r;
                const float wt = __builtin_amdgcn_exp2f(v->x - mr);
                L = fmaf(wt, v->y, L);
                v->x = wt;
            }
            L = group_sum<8>(L);
            if (l8 == 0) {
                sinv[r] = L > 0.f ? 1.f / L : 0.f;
                if (a.lse)
                    bits_ptr<float>(a.lse)[out_head(a, u, r)] = (NAN_LSE ? L != 0.f : L > 0.f) ? (M + log2f(L)) * kLn2 : -INFINITY;
            }
        }
    }
    __device__ __forceinline__ void sums(const StreamCtx &a) const {
        for (int x = threadIdx.x; x < nr * (D / 4); x += 512) {   // feature quad x % (D / 4) of row x / (D / 4)
            const int r = x / (D / 4);
            f32x4_v y = f32x4_v{0.f, 0.f, 0.f, 0.f};
            #pragma unroll 8
            for (int p = 0; p < np; ++p) {
                const f32x4_v v = *reinterpret_cast<const f32x4_v *>(so + p * po + x * 16);
                const float wt = reinterpret_cast<const float2 *>(sm + p * po)[r].x;
                #pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = fmaf(wt, v[e], y[e]);
            }
            const float inv = sinv[r];
            store_quad(bits_ptr<T>(a.out) + out_head(a, u, r) * D + (x % (D / 4)) * 4, y * inv);
        }
    }
};

// `bytes` (a multiple of 16) of pieces straight into LDS, whole; lanes past the end read its last 16 bytes
// again.  The LDS behind is padded to 1 KB.
__device__ __forceinline__ void load_pieces(const float *src, int bytes, unsigned char *lds) {
    for (int x = (threadIdx.x >> 6) * 1024; x < bytes; x += 8192)
        lds_stream16_coherent(reinterpret_cast<const unsigned char *>(src) + min(x + (int)(threadIdx.x & 63) * 16, bytes - 16), lds + x);
}

// The merge as a launch of its own, one workgroup per unit and query row: NG
// groups of D/4 threads, a feature quad each, take every NG-th piece.  A thread
// issues the loads of up to U pieces with their (max, sum) at once and folds
// them on its own, so the chain is one round trip, an exponential per piece
// and one exchange between the groups.
template <int D, typename T, bool NAN_LSE = false>
__global__ __launch_bounds__(256) void stream_merge_kernel(const StreamArgs args) {
    constexpr int FQ = D / 4, NG = 256 / FQ;
    __shared__ f32x4_v s_y[NG][FQ];
    __shared__ float2 s_ml[NG];
    const StreamCtx a = load_ctx(args);
    const int u = blockIdx.x, r = blockIdx.y, R = a.T * a.G;
    const UnitPieces up = unit_pieces(a, u);
    if (up.np == 1) return;   // finished by its workgroup
    const int fq = threadIdx.x % FQ, grp = threadIdx.x / FQ, pf = piece_floats(R, D);
    const float *po = bits_ptr<const float>(a.part) + (size_t)up.p0 * pf + r * D + fq * 4;
    const float *pm = bits_ptr<const float>(a.part) + (size_t)up.p0 * pf + R * D + r * 2;
    float M = -INFINITY, L = 0.f;
    f32x4_v y = f32x4_v{0.f, 0.f, 0.f, 0.f};
    auto fold = [&](int p0, auto n_const) {
        constexpr int U = decltype(n_const)::value;
        f32x4_v v[U];
        float2 ml[U];
        #pragma unroll
        for (int k = 0; k < U; ++k) {   // past the unit's pieces: the last one again, not used
            const size_t at = (size_t)min(p0 + k * NG, up.np - 1) * pf;
            ml[k] = *reinterpret_cast<const float2 *>(pm + at);
            v[k] = *reinterpret_cast<const f32x4_v *>(po + at);
        }
        float mn = M;
        #pragma unroll
        for (int k = 0; k < U; ++k) mn = fmaxf(mn, ml[k].x);
        const float mr = mn == -INFINITY ? 0.f : mn, c = __builtin_amdgcn_exp2f(M - mr);
        L *= c;
        y *= c;
        #pragma unroll
        for (int k = 0; k < U; ++k) {
            const bool in = p0 + k * NG < up.np;   // (a weight of 0 would make NaN of an infinite value)
            const float wt = in ? __builtin_amdgcn_exp2f(ml[k].x - mr) : 0.f;
            L = fmaf(wt, ml[k].y, L);
            #pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = fmaf(wt, in ? v[k][e] : 0.f, y[e]);
        }
        M = mn;
    };
    if (up.np <= NG) {
        fold(grp, std::integral_constant<int, 1>());
    } else if (up.np <= 4 * NG) {
        fold(grp, std::integral_constant<int, 4>());
    } else {
        for (int p = grp; p < up.np; p += 8 * NG) fold(p, std::integral_constant<int, 8>());
    }
    s_y[grp][fq] = y;
    if (fq == 0) s_ml[grp] = make_float2(M, L);
    __syncthreads();
    if (threadIdx.x >= FQ) return;
    float w[NG];
    M = s_ml[0].x;
    #pragma unroll
    for (int k = 1; k < NG; ++k) M = fmaxf(M, s_ml[k].x);
    const float mr = M == -INFINITY ? 0.f : M;
    L = 0.f;
    y = f32x4_v{0.f, 0.f, 0.f, 0.f};
    #pragma unroll
    for (int k = 0; k < NG; ++k) {
        w[k] = __builtin_amdgcn_exp2f(s_ml[k].x - mr);
        L = fmaf(w[k], s_ml[k].y, L);
        #pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = fmaf(w[k], s_y[k][fq][e], y[e]);
    }
    const float inv = L > 0.f ? 1.f / L : 0.f;
    const size_t head = out_head(a, u, r);
    store_quad(bits_ptr<T>(a.out) + head * D + fq * 4, y * inv);
    if (a.lse && fq == 0)
        bits_ptr<float>(a.lse)[head] = (NAN_LSE ? L != 0.f : L > 0.f) ? (M + log2f(L)) * kLn2 : -INFINITY;
}

}  // namespace mad

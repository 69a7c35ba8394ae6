// kv4.hip -- new K/V rows into the 4-bit cache: e2m1 codes, one power-of-two
// scale per row and 32 features, K and V apart.
//
// For 32 consecutive features x of a row:
//   scale = the least 2^k, -100 <= k <= 125, with max |x| <= 6 * 2^k
//   code  = e2m1(x / scale), to nearest even; what is beyond 6 (|x| > 1.5 * 2^127) as 6
//   a group with an element that is not finite: the scale's byte 255 (NaN), codes 0
// The exponent comes from the maximum's bits (6 = 1.5 * 2^2); dividing by a power
// of two is exact, so a code is x rounded once (v_cvt_scalef32_pk_fp4).  A row
// depends on no other row: nothing that is cached is written again.
//
// Bound: bytes (read 2 or 4, write 17/32 per element, and 2 or 4 where the values
// held are asked for).  A thread takes 8 features (a 16-byte load and one dword of
// codes), four lanes a group, 8 or 16 a row.  A wave holds consecutive rows of one
// head, whose codes and scales lie side by side; the heads are neighbours in the
// grid, since a token's heads lie side by side in the rows that are read (dealt so
// that an XCD takes neighbours: 7 % slower).  Large calls: four pieces to a thread
// (kKv4WideTiles).
// Measured: 18000 rows of 8 heads of d 128, K and V, bf16, with the values held, 37 -
// 39 us (4.5 TB/s read and written; a copy reaches 5.1), without them 19 - 21 (4.5 -
// 5.0 TB/s); fp32 64 and 34 (4.9 TB/s); 80 rows 4.4 us (a launch).
#include "mad_device.h"
#include "mad_internal.h"

namespace mad {

typedef float f32x2_v __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t or_dpp4(uint32_t v) { return v | (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true); }
__device__ __forceinline__ uint32_t or_dpp8(uint32_t v) { return v | (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xF, 0xF, true); }

// the scale's byte for a group whose largest finite |x| is m (least 2^k, -100 <= k <= 125, with m <= 6 * 2^k)
__device__ __forceinline__ uint32_t scale_byte(float m) {
    const uint32_t u = __float_as_uint(m);
    const int k = (int)(u >> 23) - 127 - 2 + ((u & 0x7fffffu) > 0x400000u ? 1 : 0);
    return (uint32_t)(min(max(k, -100), 125) + 127);
}

// N: pieces of 8 features per thread
template <typename T, int D, int N>
__global__ __launch_bounds__(256) void kv4_append_kernel(const Kv4AppendArgs a) {
    constexpr int LPR = D / 8, RPW = 256 / LPR;   // lanes per row, rows of a workgroup's pass
    const int tid = threadIdx.x, lane = tid & 63;
    const int4 rec = a.row[lane];   // tiles before row b, len, n
    const int per = 2 * a.Hkv, tile = blockIdx.x / per, hv = blockIdx.x - tile * per;
    const int b = __popcll(__ballot(rec.x <= tile)) - 1;   // rows past the last hold the end
    const int i0 = (tile - __builtin_amdgcn_readlane(rec.x, b)) * (RPW * N);   // the tile's first new row
    const int len = __builtin_amdgcn_readlane(rec.y, b), n = __builtin_amdgcn_readlane(rec.z, b);
    const bool is_v = hv >= a.Hkv;
    const int h = is_v ? hv - a.Hkv : hv;
    const RowsArg &in = is_v ? a.v_new : a.k_new, &held = is_v ? a.v_held : a.k_held;
    const int f = (tid & (LPR - 1)) * 8;   // this thread's first feature
    const T *src = reinterpret_cast<const T *>(in.p) + b * in.seq + (int64_t)h * D + f;
    T *back = reinterpret_cast<T *>(held.p) + b * held.seq + (int64_t)h * D + f;
    uint8_t *codes = reinterpret_cast<uint8_t *>(is_v ? a.v : a.k) + b * a.seq + h * a.head + (int64_t)len * (D / 2) + f / 2;
    uint8_t *scale = reinterpret_cast<uint8_t *>(is_v ? a.v_scale : a.k_scale) + b * a.s_seq + h * a.s_head + (int64_t)len * (D / 32);

    float x[N][8];
    #pragma unroll
    for (int j = 0; j < N; ++j) load8(src + min(i0 + j * RPW + tid / LPR, n - 1) * in.row, x[j]);   // past the end: the last row again
    #pragma unroll
    for (int j = 0; j < N; ++j) {
        const int i = i0 + j * RPW + tid / LPR;
        float m = 0.f, odd = 0.f;
        #pragma unroll
        for (int e = 0; e < 8; ++e) {
            m = fmaxf(m, fabsf(x[j][e]));
            odd = fmaf(x[j][e], 0.f, odd);   // a NaN where an element is not finite
        }
        m = group_max<4>(m);
        odd = group_sum<4>(odd);
        const bool fine = odd == 0.f;
        const uint32_t byte = fine ? scale_byte(m) : 255u;
        const float unit = __uint_as_float(byte << 23);
        uint32_t w = 0;
        #pragma unroll
        for (int e = 0; e < 8; ++e) x[j][e] = fminf(fmaxf(x[j][e], -0x1.8p127f), 0x1.8p127f);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[j][0], x[j][1], unit, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[j][2], x[j][3], unit, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[j][4], x[j][5], unit, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[j][6], x[j][7], unit, 3);
        w = fine ? w : 0u;
        uint32_t all = byte << (f / 32 * 8);   // the row's scales: a byte for each group
        all = or_dpp4(all);
        if constexpr (D == 128) all = or_dpp8(all);
        if (i < n) {
            *reinterpret_cast<uint32_t *>(codes + (int64_t)i * (D / 2)) = w;
            if (f == 0) {
                if constexpr (D == 128) *reinterpret_cast<uint32_t *>(scale + (int64_t)i * 4) = all;
                else *reinterpret_cast<uint16_t *>(scale + (int64_t)i * 2) = (uint16_t)all;
            }
            if (held.p) {
                const f32x2_v p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 1);
                const f32x2_v p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 3);
                const float y[8] = {p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
                store8(back + i * held.row, y);   // (exact: values of a code and a scale)
            }
        }
    }
}

template <typename T, int D>
static hipError_t launch_append_t(const Kv4AppendArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)a.tiles * 2 * a.Hkv), wg(256);
    if (a.pieces == 1) hipLaunchKernelGGL((kv4_append_kernel<T, D, 1>), grid, wg, 0, st, a);
    else hipLaunchKernelGGL((kv4_append_kernel<T, D, 4>), grid, wg, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_kv4_append(const Kv4AppendArgs &a, int dtype, int d, hipStream_t st) {
    if (dtype == MAD_BF16) return d == 64 ? launch_append_t<bf16_t, 64>(a, st) : launch_append_t<bf16_t, 128>(a, st);
    return d == 64 ? launch_append_t<float, 64>(a, st) : launch_append_t<float, 128>(a, st);
}

}  // namespace mad

// kv8.hip -- new K/V rows into the 8-bit cache: e4m3 codes with one scale per
// block of tokens and KV head, K and V apart.
//
// For each block that new rows of a sequence touch, with s_old the block's
// scale where it holds earlier rows (0 where it starts here):
//   need = the least 2^k (k >= -100) with max |x| <= 448 * 2^k over the block's
//          new elements x that are finite
//   s    = max(s_old, need);   code = e4m3(x / s), to nearest even
//   and where s > s_old the earlier rows are written again: e4m3(code * s_old / s).
// With scales that are powers of two dividing is exact, and so is writing a row
// again, but for codes that get into e4m3's subnormal range (below 2^-6): there
// a code loses a bit for each doubling, half a step of 2^-9 each time.  The
// power costs no precision against max / 448 (the codes' own exponent takes the
// factor up); it leaves up to one of their 15 binades unused.  The smallest
// 2^k comes from the exponent and mantissa bits of the maximum, without a
// logarithm: 448 = 1.75 * 2^8.
//
// Bound: bytes (read 2 or 4, write 1 per element).  One workgroup per (block,
// KV head, K or V); its elements are loaded once, in 16-byte pieces that are all
// in flight together, and stay in registers from the maximum to the codes.
// Heads are neighbours in the grid: a token's heads lie side by side in the
// rows that are read.  Measured: two prompts of up to 16384 tokens, 8 heads of
// 128, bf16, blocks of 128 (122 MB counted, two thirds of it reads): 25 us, 4.9
// TB/s (a copy's rate is 4.8 - 5.1); a token, or five for each of 16 sequences:
// 2.7 - 3.1 us, a launch and two dependent loads (the sequence's record, then its
// rows and the scale).
#include "mad_device.h"
#include "mad_internal.h"

namespace mad {

typedef float f32x2_v __attribute__((ext_vector_type(2)));

// 4 values to 4 e4m3 codes, nearest even (the callers' values are within 448 or NaN)
__device__ __forceinline__ uint32_t e4m3_x4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ bool f32_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// least 2^k, k >= -100, with m <= 448 * 2^k (m finite, >= 0)
__device__ __forceinline__ float scale_for(float m) {
    const uint32_t u = __float_as_uint(m);
    const int k = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return __uint_as_float((uint32_t)(max(k, -100) + 127) << 23);
}

// NC: 8-element pieces per thread, NC * 256 * 8 >= block * d
template <typename T, int NC>
__global__ __launch_bounds__(256) void kv8_append_kernel(const Kv8AppendArgs a) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // work item -> sequence b, its touched block j, head h, K or V
    const int4 rec = a.row[lane];   // items before row b (of one head and tensor), len, n
    const int per = 2 * a.Hkv, blk_i = blockIdx.x / per, hv = blockIdx.x - blk_i * per;
    const int b = __popcll(__ballot(rec.x <= blk_i)) - 1;   // rows past the last hold the end
    const int item0 = __builtin_amdgcn_readlane(rec.x, b), len = __builtin_amdgcn_readlane(rec.y, b);
    const int n = __builtin_amdgcn_readlane(rec.z, b);
    const bool is_v = hv >= a.Hkv;
    const int h = is_v ? hv - a.Hkv : hv;
    const int block = 1 << a.log2_block, d8 = a.d >> 3;
    const int j = (len >> a.log2_block) + blk_i - item0;
    const int64_t row0 = (int64_t)j << a.log2_block;                  // the block's first row
    const int r0 = (int)max((int64_t)len - row0, (int64_t)0);         // its new rows: [r0, r1)
    const int r1 = (int)min((int64_t)len + n - row0, (int64_t)block);
    const T *src = reinterpret_cast<const T *>(is_v ? a.v_new : a.k_new) + (((int64_t)b * a.n_cap + (row0 - len)) * a.Hkv + h) * a.d;
    uint8_t *dst = reinterpret_cast<uint8_t *>(is_v ? a.v : a.k) + b * a.seq + h * a.head + row0 * a.d;
    float *scale = (is_v ? a.v_scale : a.k_scale) + b * a.s_seq + h * a.s_head + j;
    const float s_old = r0 > 0 ? *scale : 0.f;

    // piece c = tid + 256 i of the new rows: row r0 + c / d8, features 8 (c % d8) ..
    const int pieces = (r1 - r0) * d8, sh = a.d == 64 ? 3 : 4;
    float x[NC][8];
    #pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = min(tid + 256 * i, pieces - 1);   // past the end: the last piece again
        load8(src + (int64_t)(r0 + (c >> sh)) * a.Hkv * a.d + ((c & (d8 - 1)) << 3), x[i]);
    }
    float m = 0.f;
    #pragma unroll
    for (int i = 0; i < NC; ++i)
        #pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, f32_finite(x[i][e]) ? fabsf(x[i][e]) : 0.f);
    m = group_max<64>(m);
    __shared__ float s_m[4];
    if (lane == 0) s_m[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    const float need = scale_for(m);
    const float s = s_old >= need ? s_old : need;   // (a NaN left in an unwritten scale gives way)
    // A power of two is divided by exactly with a product; another writer's scale may be anything.
    const uint32_t su = __builtin_amdgcn_readfirstlane(__float_as_uint(s)), ex = su >> 23;
    const bool pow2 = (su & 0x7fffffu) == 0 && ex >= 1 && ex <= 253;
    const float inv = __uint_as_float((254u - ex) << 23);
    #pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = tid + 256 * i;
        if (c >= pieces) continue;
        float y[8];
        if (pow2) {
            #pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = x[i][e] * inv;
        } else {
            #pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = x[i][e] / s;
        }
        #pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = f32_finite(x[i][e]) ? y[e] : __uint_as_float(0x7fc00000u);
        *reinterpret_cast<uint2 *>(dst + (int64_t)(r0 + (c >> sh)) * a.d + ((c & (d8 - 1)) << 3)) =
            make_uint2(e4m3_x4(y[0], y[1], y[2], y[3]), e4m3_x4(y[4], y[5], y[6], y[7]));
    }
    if (r0 > 0 && !(s_old >= need)) {
        // the scale grew (to a power of two): the block's earlier rows again.  (The quotient of the scales first: it is
        // exact, and code times old scale may be beyond fp32.)
        const int old = r0 * d8;
        const float down = s_old * inv;
        for (int c = tid; c < old; c += 256) {
            uint2 *p = reinterpret_cast<uint2 *>(dst + (c >> sh) * a.d + ((c & (d8 - 1)) << 3));
            const uint2 u = *p;
            uint32_t w[2] = {u.x, u.y};
            #pragma unroll
            for (int k = 0; k < 2; ++k) {
                const f32x2_v lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[k], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[k], true);
                w[k] = e4m3_x4(lo.x * down, lo.y * down, hi.x * down, hi.y * down);
            }
            *p = make_uint2(w[0], w[1]);
        }
    }
    if (tid == 0) *scale = s;
}

template <typename T>
static hipError_t launch_append_t(const Kv8AppendArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)a.blocks * 2 * a.Hkv), wg(256);
    const int nc = ((a.d << a.log2_block) + 2047) / 2048;
    if (nc <= 1) hipLaunchKernelGGL((kv8_append_kernel<T, 1>), grid, wg, 0, st, a);
    else if (nc <= 2) hipLaunchKernelGGL((kv8_append_kernel<T, 2>), grid, wg, 0, st, a);
    else if (nc <= 4) hipLaunchKernelGGL((kv8_append_kernel<T, 4>), grid, wg, 0, st, a);
    else hipLaunchKernelGGL((kv8_append_kernel<T, 8>), grid, wg, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_kv8_append(const Kv8AppendArgs &a, int dtype, hipStream_t st) {
    return dtype == MAD_BF16 ? launch_append_t<bf16_t>(a, st) : launch_append_t<float>(a, st);
}

}  // namespace mad

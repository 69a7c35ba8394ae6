// rope.hip -- each head's RMS norm of new queries and keys and the rotation at
// their positions, in one pass: what a target's fused projection leaves turns
// into what the cache's append and the verify attention take.
//
// Mathematics, for a head's d elements x at position p, h = d / 2:
//   y_j = x_j / sqrt(mean x^2 + eps) * gamma_j
//   (z_j, z_j+h) = (y_j, y_j+h) turned by p * base^(-2 j / d)     (rotate-half pairs)
// The angle is formed and reduced modulo 2 pi in double precision (mad_device.h),
// everything else is fp32, rounded to the output's type once.
//
// Bound: bytes (every element read and written once).  A wave takes 8 (d 128) or 16
// (d 64) heads of a token at a time: a lane makes one angle's cosine and sine (d / 2
// of them serve every head of the token, and are the only transcendental work), the
// wave exchanges them through LDS, and a lane holds 8 elements of a head's first half
// and the 8 that they pair with, so the norm's sum is an exchange among 8 or 4 lanes
// and the rotation is within a lane.  A wave takes two such rounds of its token where
// the call has more waves than the chip holds, else one: making the angles again
// costs less than waiting for them in longer waves does (64 + 8 heads of d 128, one
// round -> two -> all nine: 64 tokens 4.8 us -> 5 -> 9.2; 2048 tokens 15.6 -> 14.2 ->
// 16.8; 14000 tokens 105 -> 99 -> 111).
// Measured: 14000 tokens, 64 + 8 heads of d 128, bf16, 95 - 101 us (5.1 - 5.4 TB/s, a
// copy's rate), fp32 189 (5.5 TB/s); 80 tokens 4.7 us, fp32 too, one token of 32 + 8
// heads of d 64 4.4 (a launch).
#include "mad_device.h"
#include "mad_internal.h"

namespace mad {

template <typename T, int D>
__global__ __launch_bounds__(256) void norm_rope_kernel(const NormRopeArgs a) {
    constexpr int H = D / 2, LPH = D / 16, HPW = 64 / LPH;   // lanes per head, heads per wave and round
    __shared__ __align__(16) float2 s_cs[4][H];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // wave item -> token, and its rounds of heads [r0, r1)
    const int4 rec = a.row[lane];   // tokens before row b, first position
    const int want = (int)blockIdx.x * 4 + wave, item = min(want, a.items - 1);
    const int tk = item / a.groups, grp = item - tk * a.groups;
    const int b = __popcll(__ballot(rec.x <= tk)) - 1;   // rows past the last hold the end
    const int i = tk - __builtin_amdgcn_readlane(rec.x, b);
    // (the last workgroup's spare waves have no round: in place, the last item's rows must not be read after they are written)
    const int r0 = grp * a.rounds, r1 = want == item ? min(r0 + a.rounds, (a.Hq + a.Hkv + HPW - 1) / HPW) : r0;
    const int sub = lane & (LPH - 1);
    float c[8], s[8];
    if (a.rotate) {
        const int pos = a.pos ? a.pos[(int64_t)b * a.n_cap + i] : __builtin_amdgcn_readlane(rec.y, b) + i;
        if (lane < H) {
            float2 cs;
            rope_cs(pos, a.theta[lane], &cs.x, &cs.y);
            s_cs[wave][lane] = cs;
        }
    }
    __syncthreads();
    if (a.rotate) {
        #pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 cs = s_cs[wave][8 * sub + e];
            c[e] = cs.x;
            s[e] = cs.y;
        }
    }
    for (int r = r0; r < r1; ++r) {
        const int head = r * HPW + lane / LPH;
        if (head >= a.Hq + a.Hkv) continue;
        const bool is_k = head >= a.Hq;
        const int h = is_k ? head - a.Hq : head;
        const RowsArg &in = is_k ? a.k : a.q, &out = is_k ? a.k_out : a.q_out;
        const T *src = reinterpret_cast<const T *>(in.p) + b * in.seq + i * in.row + h * D + 8 * sub;
        T *dst = reinterpret_cast<T *>(out.p) + b * out.seq + i * out.row + h * D + 8 * sub;
        const T *gamma = reinterpret_cast<const T *>(is_k ? a.k_gamma : a.q_gamma);
        float x[8], y[8];
        load8(src, x);
        load8(src + H, y);
        if (gamma) {
            float g0[8], g1[8], ss = 0.f;
            load8(gamma + 8 * sub, g0);
            load8(gamma + 8 * sub + H, g1);
            #pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], fmaf(y[e], y[e], ss));
            ss = group_sum<LPH>(ss);
            const float inv = 1.f / sqrtf(fmaf(ss, 1.f / D, a.eps));
            #pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = x[e] * inv * g0[e];
                y[e] = y[e] * inv * g1[e];
            }
        }
        if (a.rotate) {
            #pragma unroll
            for (int e = 0; e < 8; ++e) rope_apply(x[e], y[e], c[e], s[e], &x[e], &y[e]);
        }
        store8(dst, x);
        store8(dst + H, y);
    }
}

template <typename T>
static hipError_t launch_t(const NormRopeArgs &a, int d, hipStream_t st) {
    const dim3 grid((unsigned)((a.items + 3) / 4)), wg(256);
    if (d == 64) hipLaunchKernelGGL((norm_rope_kernel<T, 64>), grid, wg, 0, st, a);
    else hipLaunchKernelGGL((norm_rope_kernel<T, 128>), grid, wg, 0, st, a);
    return hipGetLastError();
}

// a.row and a.tokens are set; the waves' shares here
hipError_t launch_norm_rope(NormRopeArgs &a, int dtype, int d, hipStream_t st) {
    const int per = 64 / (d / 16), rounds = (a.Hq + a.Hkv + per - 1) / per;
    a.rounds = (int64_t)a.tokens * rounds > kRopeWaves ? 2 : 1;
    while ((int64_t)a.tokens * ((rounds + a.rounds - 1) / a.rounds) > 1 << 25) a.rounds *= 2;   // (a launch has fewer than 2^32 threads)
    a.groups = (rounds + a.rounds - 1) / a.rounds;
    a.items = a.tokens * a.groups;
    return dtype == MAD_BF16 ? launch_t<bf16_t>(a, d, st) : launch_t<float>(a, d, st);
}

}  // namespace mad

// Norms of queries and keys for each head, and their rotation by the tokens' positions, between a projection and the cache:
//     x' = g x / sqrt(mean x^2 + eps)   over the channels of a token's head,
//     (a, b) -> (a cos p f_i - b sin p f_i, b cos p f_i + a sin p f_i)   for pair i < R / 2 of its first R channels.
// One pass: a lane holds 16 channels of a head, both halves of its pairs among them, so the rotation moves nothing between lanes and the norm is a sum
// over D / 16 of them.  Statistics and rotation are fp32 (64 bits where squares leave its range), the result is rounded once.  Angles are taken in turns, p f_i / 2 pi in 64 bits
// of which the whole turns are dropped: fp32 angles of far positions are off by p 2^-24, here it is p 2^-53.
// Sines and cosines are the same for all heads of a token: a wave computes each of them once and passes them on through LDS.
// Bound by memory: 16384 tokens of 32 + 8 heads of 128 channels 68 us, 4.9 TB/s there and back (a copy of 1 GiB 5.0); one token 2.6 us.
#include <algorithm>

#include "gemm_core.h"
#include "kernels.h"

namespace moin {

namespace {

constexpr int WAVES = 4;   // of a workgroup; each has work of its own

// Eight channels as fp32.
template <bool F32>
__device__ __forceinline__ void load8(const char *p, float (&x)[8])
{
    if constexpr (F32) {
        const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 16);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bits_f32(w[i] << 16);
            x[2 * i + 1] = bits_f32(w[i] & 0xFFFF0000u);
        }
    }
}
__device__ __forceinline__ void store8(char *p, const float (&x)[8])
{
    *reinterpret_cast<uint4 *>(p) =
        make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// A wave takes `per` groups of heads of one token, 64 * 16 / D heads a group.
template <int D, bool F32, bool NEIGHBOURS>
__global__ __launch_bounds__(64 * WAVES) void qk_norm_rope_kernel(RotateArgs a, int groups, int per, int parts)
{
    constexpr int LPH = D / 16, HPW = 64 / LPH, EB = F32 ? 4 : 2;
    __shared__ float2 lds_turn[WAVES][D / 2];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int64_t item = (int64_t)blockIdx.x * WAVES + wave;
    const int64_t t = item / parts;
    if (t >= a.T) return;
    const int g0 = (int)(item - t * parts) * per, g1 = min(g0 + per, groups);
    const int u = lane % LPH, hw = lane / LPH, R = a.rot, heads = a.n_heads + a.n_kv;
    // this lane's two runs of eight channels: halves of its pairs, or what is not rotated
    const bool turns = u * 16 < R;
    const int c0 = (NEIGHBOURS || !turns) ? u * 16 : u * 8, c1 = (NEIGHBOURS || !turns) ? u * 16 + 8 : u * 8 + R / 2;
    auto row = [&](int hh, const char *q, const char *k, int64_t qs, int64_t ks, int eb) {
        return hh < a.n_heads ? q + (t * qs + (int64_t)hh * D) * eb : k + (t * ks + (int64_t)(hh - a.n_heads) * D) * eb;
    };
    float x0[8], x1[8];
    auto load = [&](int grp) {
        const char *src = row(min(grp * HPW + hw, heads - 1), static_cast<const char *>(a.q), static_cast<const char *>(a.k), a.q_stride, a.k_stride, EB);
        load8<F32>(src + c0 * EB, x0);
        load8<F32>(src + c1 * EB, x1);
    };
    load(g0);
    float cs[8], sn[8];   // of pairs: 8 u + i, whose halves are x0[i] and x1[i]; or of the neighbours of both runs
    if (R > 0) {
        const double p = (double)a.positions[t];
        for (int i = lane; i < R / 2; i += 64) {
            const double turn = p * (a.freqs[i] * 0.15915494309189533577);
            float s, c;
            sincospif(2.f * (float)(turn - rint(turn)), &s, &c);
            lds_turn[wave][i] = make_float2(c, s);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 z = turns ? lds_turn[wave][u * 8 + i] : make_float2(1.f, 0.f);
            cs[i] = z.x;
            sn[i] = z.y;
        }
    }
    for (int grp = g0; grp < g1; ++grp) {
        const int hh = grp * HPW + hw;
        if (grp > g0) load(grp);
        if (a.norm) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(x0[i], x0[i], fmaf(x1[i], x1[i], sum));
#pragma unroll
            for (int d = 1; d < LPH; d <<= 1) sum += __shfl_xor(sum, d);
            float r = rsqrtf(sum * (1.f / D) + a.eps);
            const bool beyond = !(sum < 1e36f) || (sum < 1e-30f && a.eps < 1e-25f);
            if (__ballot(beyond)) {   // squares that fp32 does not hold
                double wide = 0.0;
#pragma unroll
                for (int i = 0; i < 8; ++i) wide = fma((double)x0[i], (double)x0[i], fma((double)x1[i], (double)x1[i], wide));
#pragma unroll
                for (int d = 1; d < LPH; d <<= 1) wide += __shfl_xor(wide, d);
                if (beyond) r = (float)(1.0 / sqrt(wide * (1.0 / D) + (double)a.eps));   // (the wave's other heads: as they would be without this one)
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x0[i] *= r;
                x1[i] *= r;
            }
            const char *gain = static_cast<const char *>(hh < a.n_heads ? a.q_gain : a.k_gain);
            if (gain) {
                float w0[8], w1[8];
                load8<false>(gain + c0 * 2, w0);
                load8<false>(gain + c1 * 2, w1);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x0[i] *= w0[i];
                    x1[i] *= w1[i];
                }
            }
        }
        if (R > 0 && turns) {
            if constexpr (NEIGHBOURS) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a0 = x0[2 * i], b0 = x0[2 * i + 1], a1 = x1[2 * i], b1 = x1[2 * i + 1];
                    x0[2 * i] = a0 * cs[i] - b0 * sn[i];
                    x0[2 * i + 1] = b0 * cs[i] + a0 * sn[i];
                    x1[2 * i] = a1 * cs[4 + i] - b1 * sn[4 + i];
                    x1[2 * i + 1] = b1 * cs[4 + i] + a1 * sn[4 + i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float p = x0[i], q = x1[i];
                    x0[i] = p * cs[i] - q * sn[i];
                    x1[i] = q * cs[i] + p * sn[i];
                }
            }
        }
        if (hh < heads) {
            char *dst = const_cast<char *>(row(hh, static_cast<const char *>(a.q_out), static_cast<const char *>(a.k_out), a.q_out_stride, a.k_out_stride, 2));
            store8(dst + c0 * 2, x0);
            store8(dst + c1 * 2, x1);
        }
    }
}

template <int D, bool F32>
hipError_t launch(const RotateArgs &a, hipStream_t stream)
{
    constexpr int HPW = 64 * 16 / D;
    const int groups = (a.n_heads + a.n_kv + HPW - 1) / HPW;
    // A wave takes all heads of a token where there are tokens enough to fill the chip, else a group: its sines are then the group's own.
    const int parts = a.T * groups <= 16 * compute_units() ? groups : 1, per = (groups + parts - 1) / parts;
    const dim3 grid((unsigned)((a.T * parts + WAVES - 1) / WAVES));
    if (a.neighbours)
        hipLaunchKernelGGL((qk_norm_rope_kernel<D, F32, true>), grid, dim3(64 * WAVES), 0, stream, a, groups, per, parts);
    else
        hipLaunchKernelGGL((qk_norm_rope_kernel<D, F32, false>), grid, dim3(64 * WAVES), 0, stream, a, groups, per, parts);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_qk_norm_rope(const RotateArgs &all, hipStream_t stream)
{
    RotateArgs a = all;
    constexpr int64_t AT_ONCE = 1 << 24;   // tokens of a launch, whose threads number less than 2^32
    for (; a.T > AT_ONCE; a.T -= AT_ONCE) {
        RotateArgs part = a;
        part.T = AT_ONCE;
        const hipError_t e = launch_qk_norm_rope(part, stream);
        if (e != hipSuccess) return e;
        auto on = [](const void *p, int64_t elements) { return static_cast<const char *>(p) + AT_ONCE * elements; };
        const int eb = a.x_f32 ? 4 : 2;
        if (a.q) a.q = on(a.q, a.q_stride * eb), a.q_out = const_cast<char *>(on(a.q_out, a.q_out_stride * 2));
        if (a.k) a.k = on(a.k, a.k_stride * eb), a.k_out = const_cast<char *>(on(a.k_out, a.k_out_stride * 2));
        if (a.positions) a.positions += AT_ONCE;
    }
    switch (a.D) {
    case 64: return a.x_f32 ? launch<64, true>(a, stream) : launch<64, false>(a, stream);
    case 128: return a.x_f32 ? launch<128, true>(a, stream) : launch<128, false>(a, stream);
    case 256: return a.x_f32 ? launch<256, true>(a, stream) : launch<256, false>(a, stream);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace moin

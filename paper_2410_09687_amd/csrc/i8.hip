// Matrix product in 8-bit integers: rows of x [T, d_in] and of the weight [d_out, d_in] have a scale each,
//     s = max(amax / 127 in fp32, 2^-126),   code = x / s to the nearest, ties to even,   y = s_t s_o sum_c xq_c wq_c,
// sums in int32, exact; one rounding to fp32, two for the scales.  A row with an infinity or a NaN has a scale of NaN and codes of 0.
// This file: the quantiser, and the product of up to 64 tokens, bound by the weight's bytes.  Larger ones run on the
// streams of tiles of mx.hip.
#include <algorithm>

#include "gemm_core.h"
#include "kernels.h"

namespace moin {

namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t bf16x8_amax(const uint4 &v)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, max((word(v, i) << 16) & 0x7FFF0000u, word(v, i) & 0x7FFF0000u));
    return m;
}
// Scale of a row whose largest magnitude has these fp32 bits.  (A division rounded to nearest, so that the scale is what the definition says.)
__device__ __forceinline__ float i8_scale_of(uint32_t amax)
{
    if (amax >= 0x7F800000u) return bits_f32(0x7FC00000u);
    return fmaxf(__fdiv_rn(bits_f32(amax), 127.f), bits_f32(0x00800000u));
}
// x / s to the nearest.  The product with the reciprocal may land on the wrong side of a midpoint; what it leaves, x - q s, is exact in fp32 (x
// has 8 bits, s 24, q 7, and x's last bit lies above s's) and shows it.
__device__ __forceinline__ int i8_code(float x, float s, float inv)
{
    float q = rintf(x * inv);
    const float left = fmaf(-q, s, x), half = 0.5f * s;
    if (fabsf(left) > half || (fabsf(left) == half && ((int)q & 1))) q += copysignf(1.f, left);
    return (int)fminf(fmaxf(q, -127.f), 127.f);
}
__device__ __forceinline__ uint2 i8_codes(const uint4 &v, float s, float inv)
{
    if (!(s == s)) return make_uint2(0, 0);   // (the scale alone says so)
    uint32_t c[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        c[i] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t w = word(v, 2 * i + e / 2);
            c[i] |= (uint32_t)(i8_code(bits_f32(e & 1 ? w & 0xFFFF0000u : w << 16), s, inv) & 255) << 8 * e;
        }
    }
    return make_uint2(c[0], c[1]);
}

// A row to WAVES waves (one of four rows a workgroup, or all four of one): its largest magnitude, then its codes, zeros up to the pitch.  Rows of up to
// KEEP chunks of 8 a lane stay in registers between the two.
template <int WAVES>
__global__ __launch_bounds__(256) void i8_quantize_kernel(const char *__restrict__ src, int64_t rows, int cols, int pitch, char *__restrict__ codes,
                                                          float *__restrict__ scales)
{
    constexpr int N = WAVES * 64, KEEP = 4;
    __shared__ uint32_t lds_amax[4];
    const int wave = uniform(threadIdx.x >> 6), tid = threadIdx.x % N;
    const int64_t row = (int64_t)blockIdx.x * (4 / WAVES) + (WAVES == 4 ? 0 : wave);
    if (row >= rows) return;
    const char *x = src + row * cols * 2;
    const int n8 = cols / 8;
    uint4 kept[KEEP];
    uint32_t amax = 0;
#pragma unroll
    for (int u = 0; u < KEEP; ++u) {
        const int c = u * N + tid;
        kept[u] = c < n8 ? *reinterpret_cast<const uint4 *>(x + (int64_t)c * 16) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < KEEP; ++u) amax = max(amax, bf16x8_amax(kept[u]));
    for (int c = KEEP * N + tid; c < n8; c += N) amax = max(amax, bf16x8_amax(*reinterpret_cast<const uint4 *>(x + (int64_t)c * 16)));
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, d));
    if constexpr (WAVES == 4) {
        if ((tid & 63) == 0) lds_amax[wave] = amax;
        lds_barrier();
        amax = max(max(lds_amax[0], lds_amax[1]), max(lds_amax[2], lds_amax[3]));
    }
    const float s = i8_scale_of(amax), inv = 1.f / s;
    if (tid == 0) scales[row] = s;
    char *out = codes + row * pitch;
#pragma unroll
    for (int u = 0; u < KEEP; ++u) {
        const int c = u * N + tid;
        if (c < pitch / 8) *reinterpret_cast<uint2 *>(out + c * 8) = i8_codes(kept[u], s, inv);   // (zeros beyond the columns)
    }
    for (int c = KEEP * N + tid; c < pitch / 8; c += N)
        *reinterpret_cast<uint2 *>(out + c * 8) = c < n8 ? i8_codes(*reinterpret_cast<const uint4 *>(x + (int64_t)c * 16), s, inv) : make_uint2(0, 0);
}

struct FewArgs {
    const char *x, *xq;    // bf16 tokens (FUSED) or their codes
    const float *xs;
    const char *W;
    const float *ws;
    char *y;
    int T, d_in, pitch, d_out, y_f32;
};

// 16 outputs a workgroup, all tokens; its KW waves take the 128-byte blocks of the contraction in turn and add their sums at the end.  A lane's
// operands are 16 bytes of a row as they lie in memory (the order of the contraction is free).
// FUSED: the workgroup quantises the tokens itself, into LDS, while its first weights are on their way.
template <int NT, int KW, bool FUSED>
__global__ __launch_bounds__(64 * KW) void i8_few_kernel(FewArgs a)
{
    constexpr int AHEAD = NT > 2 ? 2 : 4;   // blocks of a wave whose loads are on their way together
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16, nb = a.pitch / 128, lp = a.pitch + 16;
    const char *w = a.W + (int64_t)min(n0 + m, a.d_out - 1) * a.pitch + g * 32;
    uint4 wa[AHEAD][2];
    auto load_w = [&](int b0) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const char *p = w + min(b0 + u * KW, nb - 1) * 128;
            wa[u][0] = *reinterpret_cast<const uint4 *>(p);
            wa[u][1] = *reinterpret_cast<const uint4 *>(p + 16);
        }
    };
    load_w(wave);
    float *lds_s = reinterpret_cast<float *>(smem + (FUSED ? a.T * lp : 0));   // [16 NT] the tokens' scales
    if constexpr (FUSED) {
        const int n8 = a.d_in / 8;
        for (int t = wave; t < a.T; t += KW) {
            const char *x = a.x + (int64_t)t * a.d_in * 2;
            uint32_t amax = 0;
            for (int c = lane; c < n8; c += 64) amax = max(amax, bf16x8_amax(*reinterpret_cast<const uint4 *>(x + c * 16)));
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, d));
            const float s = i8_scale_of(amax), inv = 1.f / s;
            if (lane == 0) lds_s[t] = s;
            for (int c = lane; c < a.pitch / 8; c += 64)
                *reinterpret_cast<uint2 *>(smem + t * lp + c * 8) = c < n8 ? i8_codes(*reinterpret_cast<const uint4 *>(x + c * 16), s, inv) : make_uint2(0, 0);
        }
    } else {
        for (int t = threadIdx.x; t < 16 * NT; t += 64 * KW) lds_s[t] = a.xs[min(t, a.T - 1)];
    }
    lds_barrier();
    i32x4_t acc[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) acc[nt] = i32x4_t{0, 0, 0, 0};
    const char *x[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int t = min(nt * 16 + m, a.T - 1);
        x[nt] = FUSED ? smem + t * lp + g * 32 : a.xq + (int64_t)t * a.pitch + g * 32;
    }
    for (int b0 = wave; b0 < nb; b0 += KW * AHEAD) {
        i32x4_t av[AHEAD][2];
        uint4 xb[AHEAD][NT][2];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const bool in = b0 + u * KW < nb;
            const int at = min(b0 + u * KW, nb - 1) * 128;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int z = 0; z < 2; ++z) xb[u][nt][z] = *reinterpret_cast<const uint4 *>(x[nt] + at + z * 16);
#pragma unroll
            for (int z = 0; z < 2; ++z) av[u][z] = __builtin_bit_cast(i32x4_t, in ? wa[u][z] : make_uint4(0, 0, 0, 0));
        }
        if (b0 + KW * AHEAD < nb) load_w(b0 + KW * AHEAD);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    acc[nt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(av[u][z], __builtin_bit_cast(i32x4_t, xb[u][nt][z]), acc[nt], 0, 0, 0);
    }
    // the waves' sums, through LDS behind the scales
    i32x4_t *sums = reinterpret_cast<i32x4_t *>(lds_s + 16 * NT);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) sums[(wave * NT + nt) * 64 + lane] = acc[nt];
    lds_barrier();
    for (int i = threadIdx.x; i < NT * 64; i += 64 * KW) {
        i32x4_t v = sums[i];
#pragma unroll
        for (int k = 1; k < KW; ++k) v += sums[k * NT * 64 + i];
        const int t = (i >> 6) * 16 + (i & 15), o = n0 + ((i & 63) >> 4) * 4;
        if (t >= a.T || o >= a.d_out) continue;
        const float st = lds_s[t];
        const f32x4_t so = *reinterpret_cast<const f32x4_t *>(a.ws + o);
        float r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = (float)v[e] * (st * so[e]);
        const int64_t at = (int64_t)t * a.d_out + o;
        if (a.y_f32) *reinterpret_cast<float4 *>(a.y + at * 4) = make_float4(r[0], r[1], r[2], r[3]);
        else *reinterpret_cast<uint2 *>(a.y + at * 2) = make_uint2(pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]));
    }
}

constexpr int FUSED_BYTES = 32768;   // of the tokens' codes that a workgroup keeps in LDS

template <int NT, int KW, bool FUSED>
hipError_t few(const FewArgs &a, hipStream_t stream)
{
    const size_t lds = (FUSED ? (size_t)a.T * (a.pitch + 16) : 0) + 16 * NT * 4 + (size_t)KW * NT * 1024;
    hipLaunchKernelGGL((i8_few_kernel<NT, KW, FUSED>), dim3((unsigned)((a.d_out + 15) / 16)), dim3(64 * KW), lds, stream, a);
    return hipGetLastError();
}
template <int KW>
hipError_t few_tokens(const FewArgs &a, bool fused, hipStream_t stream)
{
    if (fused) return few<1, KW, true>(a, stream);
    return a.T <= 16 ? few<1, KW, false>(a, stream) : a.T <= 32 ? few<2, KW, false>(a, stream) : few<4, KW, false>(a, stream);
}

}  // namespace

hipError_t launch_i8_quantize(const void *src, int64_t rows, int cols, void *codes, float *scales, hipStream_t stream)
{
    if (rows <= 0) return hipSuccess;
    if (rows >= 4 * compute_units())
        hipLaunchKernelGGL(i8_quantize_kernel<1>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, static_cast<const char *>(src), rows, cols,
                           i8_pitch(cols), static_cast<char *>(codes), scales);
    else
        hipLaunchKernelGGL(i8_quantize_kernel<4>, dim3((unsigned)rows), dim3(256), 0, stream, static_cast<const char *>(src), rows, cols,
                           i8_pitch(cols), static_cast<char *>(codes), scales);
    return hipGetLastError();
}

bool i8_few_quantises(int64_t T, int d_in) { return T <= 16 && T * i8_pitch(d_in) <= FUSED_BYTES; }

hipError_t launch_i8_few(const void *x, const void *xq, const float *xs, const void *Wq, const float *ws, int T, int d_in, int d_out, void *y,
                         int y_f32, hipStream_t stream)
{
    const FewArgs a{static_cast<const char *>(x), static_cast<const char *>(xq), xs, static_cast<const char *>(Wq), ws, static_cast<char *>(y),
                    T, d_in, i8_pitch(d_in), d_out, y_f32};
    const bool fused = i8_few_quantises(T, d_in);
    const int tiles = (d_out + 15) / 16;
    return tiles * 2 < 3 * compute_units() ? few_tokens<8>(a, fused, stream) : few_tokens<4>(a, fused, stream);
}

}  // namespace moin

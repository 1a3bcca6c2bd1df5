// Matrix product in 8-bit integers: rows of x [T, d_in] and of the weight [d_out, d_in] have a scale each,
//     s = max(amax / 127 in fp32, 2^-126),   code = x / s to the nearest, ties to even,   y = s_t s_o sum_c xq_c wq_c,
// sums in int32, exact; one rounding to fp32, two for the scales (i8_scale.h).  A row with an infinity or a NaN has a scale of NaN and codes of 0.
// (s rounded to fp32 belongs to the definition, so that codes are the same wherever they are made.)
// This file: the quantiser, and the product of up to 128 tokens, bound by the weight's bytes.  Larger ones run on the
// streams of tiles of mx.hip.
#include <algorithm>

#include "gemm_core.h"
#include "i8_scale.h"
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
// x / s to the nearest, eight values.  The product with the reciprocal may land on the wrong side of a midpoint; what it leaves, x - q s, is exact
// in fp32 (x has 8 bits, s 24, q 7, and x's last bit lies above s's) and shows it: where none of eight leaves half a step or more, all are right.
// (Magnitudes above 127 do not come: s is the largest value's 127th part, rounded.)
__device__ __forceinline__ uint2 i8_codes(const uint4 &v, float s, float inv)
{
    if (!(s == s)) return make_uint2(0, 0);   // (the scale alone says so)
    float q[8], most = 0.f;
    auto x = [&](int i) { return bits_f32(i & 1 ? word(v, i >> 1) & 0xFFFF0000u : word(v, i >> 1) << 16); };
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        q[i] = rintf(x(i) * inv);
        most = fmaxf(most, fabsf(fmaf(-q[i], s, x(i))));
    }
    if (2.f * most >= s) {   // (twice what is left, not half of s: the smallest scales have no half in fp32)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float left = fmaf(-q[i], s, x(i)), twice = 2.f * fabsf(left);
            if (twice > s || (twice == s && ((int)q[i] & 1))) q[i] += copysignf(1.f, left);
        }
    }
    uint32_t c[2] = {0, 0};   // (of q + 128, whose high bit is then turned)
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i / 4] = __builtin_amdgcn_cvt_pk_u8_f32(q[i] + 128.f, i % 4, c[i / 4]);
    return make_uint2(c[0] ^ 0x80808080u, c[1] ^ 0x80808080u);
}

// A row to WAVES waves (1: four rows a workgroup; 4 or 16: one): its largest magnitude, then its codes, zeros up to the pitch.  Rows of up to
// KEEP chunks of 8 a lane stay in registers between the two.
template <int WAVES>
__global__ __launch_bounds__(WAVES == 16 ? 1024 : 256) void i8_quantize_kernel(const char *__restrict__ src, int64_t rows, int cols, int pitch, char *__restrict__ codes,
                                                          float *__restrict__ scales)
{
    constexpr int N = WAVES * 64, KEEP = WAVES == 16 ? 1 : 4;
    __shared__ uint32_t lds_amax[WAVES];
    const int wave = uniform(threadIdx.x >> 6), tid = threadIdx.x % N;
    const int64_t row = WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
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
    if constexpr (WAVES > 1) {
        if ((tid & 63) == 0) lds_amax[wave] = amax;
        lds_barrier();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) amax = max(amax, lds_amax[w]);
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

// A workgroup quantises the tokens itself up to this many pieces of 512 columns.  (2048 -> 2048, six tokens, 24 pieces: 5.9 us, 7.9 in a launch of its own;
// 2048 -> 5632, eight tokens, 32 pieces: 10.3 and 8.6.)
constexpr int FUSED_ITEMS = 24;
int fused_items(int64_t T, int d_in) { return T > 16 ? FUSED_ITEMS + 1 : (int)T * ((i8_pitch(d_in) + 511) / 512); }

struct FewArgs {
    const char *x, *xq;    // bf16 tokens (FUSED) or their codes
    const float *xs;
    const char *W;
    const float *ws;
    char *y;
    int T, d_in, pitch, d_out, y_f32;
};

// 16 RT outputs a workgroup, all tokens; its KW waves take a range of the contraction's 128-byte blocks each and add their sums at the end.  A lane's
// operands are 16 bytes of a row as they lie in memory (the order of the contraction is free).
// FUSED: the workgroup quantises the tokens itself, into LDS, while its first weights are on their way: a launch less (one token 2048 -> 5632 10.7 us when
// one wave did it, 5.6 with pieces dealt to sixteen).
// One token 8192 -> 28672 44 us, 5.4 TB/s of weights (a long read: 6.8), 41 where the last-level cache has part of the 235 MB from the call before; 24 tokens 48, 4.8 TB/s,
// where the tokens come out of L2 for every 64 outputs.  In turn instead of in
// ranges the waves' blocks take 55 and 65 (of 32 outputs); 24 tokens and 16 / 32 / 64 outputs a workgroup 77 / 64 / 54, 64 tokens 134 / 97 / 73.  Past the
// caches: 61 for the 24.
template <int RT, int NT, int KW, bool FUSED>
__global__ __launch_bounds__(64 * KW) void i8_few_kernel(FewArgs a)
{
    constexpr int AHEAD = NT > 1 ? 1 : 2;                    // blocks of a wave whose loads are on their way together
    constexpr int KEEP = (FUSED_ITEMS + KW - 1) / KW;        // pieces of 512 columns of the tokens that a wave quantises
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16 * RT, nb = a.pitch / 128, lp = a.pitch + 16;
    if (blockIdx.y) {   // a group of 128 tokens behind the first
        const int t0 = blockIdx.y * 128;
        a.xq += (int64_t)t0 * a.pitch;
        a.xs += t0;
        a.y += (int64_t)t0 * a.d_out * (a.y_f32 ? 4 : 2);
        a.T -= t0;
    }
    a.T = min(a.T, 128);
    const int per = (nb + KW - 1) / KW, first = wave * per, end = min(nb, first + per);
    const char *w[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) w[rt] = a.W + (int64_t)min(n0 + rt * 16 + m, a.d_out - 1) * a.pitch + g * 32;
    uint4 wa[AHEAD][RT][2];
    auto load_w = [&](int b0) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (b0 + u < end)   // (uniform)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const char *p = w[rt] + (b0 + u) * 128;
                    wa[u][rt][0] = *reinterpret_cast<const uint4 *>(p);
                    wa[u][rt][1] = *reinterpret_cast<const uint4 *>(p + 16);
                }
    };
    float *lds_s = reinterpret_cast<float *>(smem + (FUSED ? a.T * lp : 0));   // [16 NT] the tokens' scales
    if constexpr (FUSED) {
        // pieces of 512 columns, dealt to the waves: all of them read at once, the largest magnitudes meet in LDS
        uint32_t *amax = reinterpret_cast<uint32_t *>(lds_s);
        const int n8 = a.d_in / 8, p8 = a.pitch / 8, segs = (p8 + 63) >> 6, items = a.T * segs;
        uint4 x[KEEP];
#pragma unroll
        for (int u = 0; u < KEEP; ++u) {
            const int i = wave + u * KW, t = i / segs, c = (i - t * segs) * 64 + lane;
            x[u] = i < items && c < n8 ? *reinterpret_cast<const uint4 *>(a.x + ((int64_t)t * n8 + c) * 16) : make_uint4(0, 0, 0, 0);
        }
        if (threadIdx.x < 16) amax[threadIdx.x] = 0;
        load_w(first);
        lds_barrier();
#pragma unroll
        for (int u = 0; u < KEEP; ++u) {
            const int i = wave + u * KW;
            if (i >= items) break;
            uint32_t top = bf16x8_amax(x[u]);
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
            if (lane == 0) atomicMax(&amax[i / segs], top);
        }
        lds_barrier();
        float s_t = 0.f;
        if (threadIdx.x < 16) s_t = i8_scale_of(amax[threadIdx.x]);
#pragma unroll
        for (int u = 0; u < KEEP; ++u) {
            const int i = wave + u * KW, t = i / segs, c = (i - t * segs) * 64 + lane;
            if (i >= items) break;
            const float s = i8_scale_of(amax[t]);
            if (c < p8) *reinterpret_cast<uint2 *>(smem + t * lp + c * 8) = i8_codes(x[u], s, 1.f / s);   // (zeros beyond the columns)
        }
        lds_barrier();
        if (threadIdx.x < 16) lds_s[threadIdx.x] = s_t;
    } else {
        load_w(first);
        for (int t = threadIdx.x; t < 16 * NT; t += 64 * KW) lds_s[t] = a.xs[min(t, a.T - 1)];
    }
    i32x4_t acc[RT][NT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[rt][nt] = i32x4_t{0, 0, 0, 0};
    const char *x[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int t = min(nt * 16 + m, a.T - 1);
        x[nt] = FUSED ? smem + t * lp + g * 32 : a.xq + (int64_t)t * a.pitch + g * 32;
    }
    for (int b0 = first; b0 < end; b0 += AHEAD) {
        i32x4_t av[AHEAD][RT][2], xb[AHEAD][NT][2];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int at = min(b0 + u, nb - 1) * 128;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int z = 0; z < 2; ++z) xb[u][nt][z] = *reinterpret_cast<const i32x4_t *>(x[nt] + at + z * 16);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int z = 0; z < 2; ++z) av[u][rt][z] = __builtin_bit_cast(i32x4_t, wa[u][rt][z]);
        }
        load_w(b0 + AHEAD);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (b0 + u < end)
#pragma unroll
                for (int z = 0; z < 2; ++z)
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            acc[rt][nt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(av[u][rt][z], xb[u][nt][z], acc[rt][nt], 0, 0, 0);
    }
    // the waves' sums, through LDS behind the scales
    i32x4_t *sums = reinterpret_cast<i32x4_t *>(lds_s + 16 * NT);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sums[((wave * RT + rt) * NT + nt) * 64 + lane] = acc[rt][nt];
    lds_barrier();
    for (int i = threadIdx.x; i < RT * NT * 64; i += 64 * KW) {
        i32x4_t v = sums[i];
#pragma unroll
        for (int k = 1; k < KW; ++k) v += sums[k * RT * NT * 64 + i];
        const int t = (i >> 6) % NT * 16 + (i & 15), o = n0 + (i >> 6) / NT * 16 + ((i & 63) >> 4) * 4;
        if (t >= a.T || o >= a.d_out) continue;
        const I8Token st(lds_s[t]);
        const f32x4_t so = *reinterpret_cast<const f32x4_t *>(a.ws + o);
        float r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = st(v[e], so[e]);
        const int64_t at = (int64_t)t * a.d_out + o;
        if (a.y_f32) *reinterpret_cast<float4 *>(a.y + at * 4) = make_float4(r[0], r[1], r[2], r[3]);
        else *reinterpret_cast<uint2 *>(a.y + at * 2) = make_uint2(pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]));
    }
}

// A thread takes four outputs of a token.
__global__ __launch_bounds__(256) void i8_join_kernel(const i32x4_t *__restrict__ parts, int n, const float *__restrict__ xs, const float *__restrict__ ws,
                                                      int64_t quads, int per_row, char *__restrict__ y, int y_f32)
{
    const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (q >= quads) return;
    i32x4_t v = parts[q];
    for (int u = 1; u < n; ++u) v += parts[u * quads + q];
    const int64_t t = q / per_row;
    const I8Token st(xs[t]);
    const f32x4_t so = reinterpret_cast<const f32x4_t *>(ws)[q - t * per_row];
    float r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = st(v[e], so[e]);
    if (y_f32) *reinterpret_cast<float4 *>(y + q * 16) = make_float4(r[0], r[1], r[2], r[3]);
    else *reinterpret_cast<uint2 *>(y + q * 8) = make_uint2(pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]));
}

constexpr int few_lds(int RT, int NT, int KW) { return 16 * NT * 4 + KW * RT * NT * 1024; }   // scales, the waves' sums
template <int RT, int NT, int KW, bool FUSED>
hipError_t few(const FewArgs &a, hipStream_t stream)
{
    const size_t lds = (FUSED ? (size_t)a.T * (a.pitch + 16) : 0) + few_lds(RT, NT, KW);
    hipLaunchKernelGGL((i8_few_kernel<RT, NT, KW, FUSED>), dim3((unsigned)((a.d_out + 16 * RT - 1) / (16 * RT)), (unsigned)((a.T + 127) / 128)),
                       dim3(64 * KW), lds, stream, a);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_i8_quantize(const void *src, int64_t rows, int cols, void *codes, float *scales, hipStream_t stream)
{
    if (rows <= 0) return hipSuccess;
    constexpr int64_t AT_ONCE = 1 << 23;   // rows of a launch, whose threads number less than 2^32
    for (; rows > AT_ONCE; rows -= AT_ONCE) {
        const hipError_t e = launch_i8_quantize(src, AT_ONCE, cols, codes, scales, stream);
        if (e != hipSuccess) return e;
        src = static_cast<const char *>(src) + AT_ONCE * cols * 2;
        codes = static_cast<char *>(codes) + AT_ONCE * i8_pitch(cols);
        scales += AT_ONCE;
    }
    auto go = [&](auto kernel, int64_t wgs, int threads) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(threads), 0, stream, static_cast<const char *>(src), rows, cols, i8_pitch(cols),
                           static_cast<char *>(codes), scales);
    };
    // Many rows: a wave each, as long as it keeps them (2048 columns; 8192 x 8192 70 us like that, 41 with four waves to a row).  Few: as many lanes as there
    // are chunks (24 x 8192 5.2 us with four waves to a row, 4.6 with 16).
    if (rows >= 4 * compute_units() && cols <= 2048) go(&i8_quantize_kernel<1>, (rows + 3) / 4, 256);
    else if (rows < compute_units() && cols > 2048) go(&i8_quantize_kernel<16>, rows, 1024);
    else go(&i8_quantize_kernel<4>, rows, 256);
    return hipGetLastError();
}

// Each group of 128 tokens reads the weight for itself, a workgroup all of its tokens' codes: what a token costs grows with d_in, what the tiles of
// 128 x 128 cost does so over the parts of their contraction.  Us, few / tiles, weights out of memory: 64 tokens 2048 -> 2048 10.9 / 13.1, 4096 -> 4096
// 15.8 / 16.9, 5632 -> 2048 18.9 / 17.0; 128 2048 -> 5632 16.9 / 18.6, 2048 -> 256 14.0 / 12.9, 4096 -> 4096 23 / 20; 32 8192 -> 28672 55 / 59, 8192 -> 1024 17.0 / 17.9; 24
// 32768 -> 2048 48 / 43, 16 of it 39 / 43.  Large weights of many outputs: 32 tokens 4096 -> 14336 22.6 / 21.1, 64 29 / 23; 96 2048 -> 32000 34 / 23.  More than one group
// only while each workgroup has a compute unit of its own: 1000 tokens 1024 -> 256 11.4 / 13.7, 256 2048 -> 2048 14.3 / 16.0, but 1000 1024 -> 2048 27 / 22.
bool i8_few_pays(int64_t T, int d_in, int d_out)
{
    const int64_t tiles = (d_out + 15) / 16;
    if (T <= 24) return true;
    if (T > 32 && d_out >= 32 * compute_units() && (int64_t)d_in * d_out >= 1 << 25) return false;
    return std::min<int64_t>(T, 128) * d_in <= 1 << 18 && (T <= 128 || (T + 127) / 128 * tiles <= compute_units());
}

bool i8_few_quantises(int64_t T, int d_in) { return fused_items(T, d_in) <= FUSED_ITEMS; }

hipError_t launch_i8_few(const void *x, const void *xq, const float *xs, const void *Wq, const float *ws, int T, int d_in, int d_out, void *y,
                         int y_f32, hipStream_t stream)
{
    const FewArgs a{static_cast<const char *>(x), static_cast<const char *>(xq), xs, static_cast<const char *>(Wq), ws, static_cast<char *>(y),
                    T, d_in, i8_pitch(d_in), d_out, y_f32};
    // Outputs a workgroup and waves by the weight's rows: 64 or 32 outputs where that leaves a workgroup for every unit, as the tokens come from L2 once for
    // each; else as many waves as hide the trips.  Us: 32 tokens 2048 -> 5632 with 16 / 32 outputs 10.9 / 9.1, 64 tokens 14.7 / 11.1, but 2048 -> 2048 7.9 /
    // 9.0 and 9.6 / 11.0; one token 2048 -> 2048 with 8 / 16 waves 5.5 / 5.2, six 7.2 / 5.9.
    const int tiles = (d_out + 15) / 16, n_cus = compute_units();
    const bool wide = tiles >= 4 * n_cus, broad = tiles * 4 >= 5 * n_cus;
    if (i8_few_quantises(T, d_in)) return wide ? few<2, 1, 4, true>(a, stream) : tiles * 2 >= 3 * n_cus ? few<1, 1, 8, true>(a, stream) : few<1, 1, 16, true>(a, stream);
    if (T <= 16) return wide ? few<2, 1, 4, false>(a, stream) : few<1, 1, 8, false>(a, stream);
    if (T <= 32) return wide ? few<4, 2, 4, false>(a, stream) : broad ? few<2, 2, 4, false>(a, stream) : few<1, 2, 8, false>(a, stream);
    if (T <= 64) return wide ? few<4, 4, 4, false>(a, stream) : broad ? few<2, 4, 8, false>(a, stream) : few<1, 4, 8, false>(a, stream);
    return wide ? few<4, 8, 4, false>(a, stream) : broad ? few<2, 8, 4, false>(a, stream) : few<1, 8, 8, false>(a, stream);
}

hipError_t launch_i8_join(const void *parts, int n, const float *xs, const float *ws, int64_t T, int d_out, void *y, int y_f32, hipStream_t stream)
{
    const int64_t quads = T * (d_out / 4);
    hipLaunchKernelGGL(i8_join_kernel, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, stream, static_cast<const i32x4_t *>(parts), n, xs, ws, quads,
                       d_out / 4, static_cast<char *>(y), y_f32);
    return hipGetLastError();
}

hipError_t prepare_i8_kernels()
{
    auto allow = [](auto kernel, int bytes) {
        return hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    };
    hipError_t e = allow(&i8_few_kernel<4, 8, 4, false>, few_lds(4, 8, 4));
    if (e == hipSuccess) e = allow(&i8_few_kernel<2, 8, 4, false>, few_lds(2, 8, 4));
    if (e == hipSuccess) e = allow(&i8_few_kernel<1, 8, 8, false>, few_lds(1, 8, 8));
    if (e == hipSuccess) e = allow(&i8_few_kernel<2, 4, 8, false>, few_lds(2, 4, 8));
    if (e == hipSuccess) e = allow(&i8_few_kernel<4, 4, 4, false>, few_lds(4, 4, 4));
    return e;
}

}  // namespace moin

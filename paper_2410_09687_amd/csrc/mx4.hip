// Base weights in MXFP4 ("Future Works", an aggressively quantised base whose loss the experts recover) and the
// matrix-vector products of a few tokens with them:  y = x dq(W)^T.
//
// Layout: records of 16 rows x 512 columns, 4352 bytes, [row tile][column tile]: column 128 j + 32 g + c of row m at byte
// [j][g][m][c / 2] (the even column in the low nibble), then the scale bytes at [g][m][j].  That is the order in which the
// kernel's lanes take them: lane (m, g) holds 32 columns of row m, 16 bytes, and the scale bytes of four such blocks are a word; a wave's load is
// 1 KB of consecutive memory.  Rows and columns beyond the weight's are zeros.
//
// Product: y^T = W x^T on v_mfma_f32_16x16x32_bf16, 16 rows of W by 16 tokens.  The codes become bf16 exactly (two a
// conversion, the scale in the same instruction), x is bf16: the fp32 sums are the only rounding.
// The contraction order is free: a block's 32 columns are four steps of eight, which are 16 consecutive bytes of x.
#include "kernels.h"
#include "mxfp4.h"

namespace moin {

constexpr int MX4_REC = 4352, MX4_COLS = 512;

// A thread takes eight columns of a row, four neighbours a block of 32.  Padding is written too.
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const char *__restrict__ src, char *__restrict__ dst, int rows, int cols,
                                                           int col_tiles, int64_t units)
{
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (u >= units) return;
    const int per_row = col_tiles * (MX4_COLS / 8);
    const int64_t row = u / per_row;
    const int c8 = (int)(u - row * per_row), col = c8 * 8;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (row < rows && col < cols) x = *reinterpret_cast<const uint4 *>(src + (row * cols + col) * 2);   // cols % 8 == 0
    uint32_t amax = bf16x8_amax(x);
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
    const uint32_t E = mx4_scale_byte(amax);
    const int m = (int)(row & 15), ct = c8 >> 6, j = (c8 >> 4) & 3, g = (c8 >> 2) & 3;
    char *rec = dst + ((row >> 4) * col_tiles + ct) * MX4_REC;
    *reinterpret_cast<uint32_t *>(rec + j * 1024 + g * 256 + m * 16 + (c8 & 3) * 4) = mx4_encode(x, bits_f32(E << 23));
    if ((c8 & 3) == 0) rec[4096 + g * 64 + m * 4 + j] = (char)E;
}

__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const char *__restrict__ src, char *__restrict__ dst, int cols, int col_tiles,
                                                             int64_t units)
{
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (u >= units) return;
    const int per_row = cols / 8;
    const int64_t row = u / per_row;
    const int c8 = (int)(u - row * per_row), m = (int)(row & 15), ct = c8 >> 6, j = (c8 >> 4) & 3, g = (c8 >> 2) & 3;
    const char *rec = src + ((row >> 4) * col_tiles + ct) * MX4_REC;
    const uint32_t codes = *reinterpret_cast<const uint32_t *>(rec + j * 1024 + g * 256 + m * 16 + (c8 & 3) * 4);
    const uint32_t scales = *reinterpret_cast<const uint32_t *>(rec + 4096 + g * 64 + m * 4);
    *reinterpret_cast<uint4 *>(dst + (row * cols + c8 * 8) * 2) = mx4_decode(codes, bits_f32((scales >> (8 * j) & 255u) << 23));
}

// A workgroup has 16 rows of W and 16 NT tokens; its four waves take the column blocks of 128 in turn and add up
// through LDS.
template <int NT, bool Y32>
__global__ __launch_bounds__(256) void mx4_linear_kernel(const char *__restrict__ x, const char *__restrict__ W, void *__restrict__ y, int64_t T,
                                                         int d_in, int d_out, int col_tiles)
{
    __shared__ float lds[4][NT][16][20];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
    const int rt = blockIdx.x;
    const int64_t t0 = (int64_t)blockIdx.y * (16 * NT);
    const char *w = W + (int64_t)rt * col_tiles * MX4_REC;
    f32x4_t acc[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) acc[nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int blocks = (d_in + 127) / 128;
    for (int b = wave; b < blocks; b += 4) {
        const char *rec = w + (int64_t)(b >> 2) * MX4_REC;
        const uint4 codes = *reinterpret_cast<const uint4 *>(rec + (b & 3) * 1024 + lane * 16);
        const uint32_t scales = *reinterpret_cast<const uint32_t *>(rec + 4096 + lane * 4);
        const float scale = bits_f32((scales >> (8 * (b & 3)) & 255u) << 23);
        const uint32_t c[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bf16x8_t a = __builtin_bit_cast(bf16x8_t, mx4_decode(c[j], scale));
            const int col = b * 128 + g * 32 + j * 8;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int64_t t = t0 + nt * 16 + n;
                uint4 v = make_uint4(0, 0, 0, 0);
                if (t < T && col < d_in) v = *reinterpret_cast<const uint4 *>(x + (t * d_in + col) * 2);
                acc[nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8_t, v), acc[nt], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
        *reinterpret_cast<f32x4_t *>(&lds[wave][nt][n][g * 4]) = acc[nt];
    __syncthreads();
    for (int i = tid; i < NT * 64; i += 256) {   // (token, four rows)
        const int nt = i >> 6, tok = (i >> 2) & 15, r = (i & 3) * 4;
        f32x4_t s = *reinterpret_cast<const f32x4_t *>(&lds[0][nt][tok][r]);
#pragma unroll
        for (int u = 1; u < 4; ++u) s += *reinterpret_cast<const f32x4_t *>(&lds[u][nt][tok][r]);
        const int64_t t = t0 + nt * 16 + tok;
        const int row = rt * 16 + r;
        if (t >= T || row >= d_out) continue;   // d_out % 8 == 0: the four rows are in or out together
        if constexpr (Y32) *reinterpret_cast<f32x4_t *>(static_cast<float *>(y) + t * d_out + row) = s;
        else *reinterpret_cast<uint2 *>(static_cast<char *>(y) + (t * d_out + row) * 2) = make_uint2(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]));
    }
}

int64_t mx4_bytes(int64_t rows, int64_t cols) { return (rows + 15) / 16 * ((cols + MX4_COLS - 1) / MX4_COLS) * MX4_REC; }

hipError_t launch_mx4_quantize(const void *src, int64_t rows, int64_t cols, void *dst, hipStream_t stream)
{
    const int ct = (int)((cols + MX4_COLS - 1) / MX4_COLS);
    const int64_t units = (rows + 15) / 16 * 16 * ct * (MX4_COLS / 8);
    hipLaunchKernelGGL(mx4_quantize_kernel, dim3((unsigned)((units + 255) / 256)), dim3(256), 0, stream, static_cast<const char *>(src),
                       static_cast<char *>(dst), (int)rows, (int)cols, ct, units);
    return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const void *src, int64_t rows, int64_t cols, void *dst, hipStream_t stream)
{
    const int ct = (int)((cols + MX4_COLS - 1) / MX4_COLS);
    const int64_t units = rows * (cols / 8);
    hipLaunchKernelGGL(mx4_dequantize_kernel, dim3((unsigned)((units + 255) / 256)), dim3(256), 0, stream, static_cast<const char *>(src),
                       static_cast<char *>(dst), (int)cols, ct, units);
    return hipGetLastError();
}

template <int NT>
static void launch_nt(const void *x, const void *W, void *y, int y_f32, int64_t T, int d_in, int d_out, hipStream_t stream)
{
    const dim3 grid((unsigned)((d_out + 15) / 16), (unsigned)((T + 16 * NT - 1) / (16 * NT)));
    const int ct = (d_in + MX4_COLS - 1) / MX4_COLS;
    if (y_f32)
        hipLaunchKernelGGL((mx4_linear_kernel<NT, true>), grid, dim3(256), 0, stream, static_cast<const char *>(x), static_cast<const char *>(W), y, T,
                           d_in, d_out, ct);
    else
        hipLaunchKernelGGL((mx4_linear_kernel<NT, false>), grid, dim3(256), 0, stream, static_cast<const char *>(x), static_cast<const char *>(W), y, T,
                           d_in, d_out, ct);
}

bool mx4_direct_pays(int64_t T, int d_in, int d_out) { return T <= MX4_DIRECT_MAX_T; }

hipError_t launch_mx4_linear(const void *x, const void *W, void *y, int y_f32, int64_t T, int d_in, int d_out, hipStream_t stream)
{
    if (T <= 16) launch_nt<1>(x, W, y, y_f32, T, d_in, d_out, stream);
    else if (T <= 32) launch_nt<2>(x, W, y, y_f32, T, d_in, d_out, stream);
    else launch_nt<4>(x, W, y, y_f32, T, d_in, d_out, stream);
    return hipGetLastError();
}

}  // namespace moin

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

// Sixteen bytes of zeros: what the last block's columns of x beyond d_in are taken from.
static __device__ __align__(16) const uint32_t mx4_zeros[4] = {0, 0, 0, 0};

// A workgroup has 16 RT rows of W and 16 NT tokens; its KW waves take the column blocks of 128 in turn and add up through
// LDS.  Codes and x of a wave's next block are on their way while it multiplies the present one.
template <int RT, int NT, int KW, bool Y32>
__global__ __launch_bounds__(64 * KW) void mx4_linear_kernel(const char *__restrict__ x, const char *__restrict__ W, void *__restrict__ y, int64_t T,
                                                             int d_in, int d_out, int col_tiles)
{
    __shared__ float lds[KW][RT * NT][16][20];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
    const int row_tiles = (d_out + 15) >> 4, rt0 = blockIdx.x * RT;
    const int64_t t0 = (int64_t)blockIdx.y * (16 * NT);
    const char *w[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) w[r] = W + (int64_t)min(rt0 + r, row_tiles - 1) * col_tiles * MX4_REC;
    // rows of x beyond T are its last (their results are not written)
    const char *xr[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) xr[nt] = x + min(t0 + nt * 16 + n, T - 1) * d_in * 2;
    struct Block {
        uint4 codes[RT], v[NT][4];
        uint32_t scales[RT];
    };
    auto load = [&](Block &k, int b) {
        const int at = (b >> 2) * MX4_REC;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            k.codes[r] = *reinterpret_cast<const uint4 *>(w[r] + at + (b & 3) * 1024 + lane * 16);
            k.scales[r] = *reinterpret_cast<const uint8_t *>(w[r] + at + 4096 + lane * 4 + (b & 3));
        }
        const int c0 = b * 128 + g * 32;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                k.v[nt][j] = *reinterpret_cast<const uint4 *>(c0 + j * 8 < d_in ? xr[nt] + (c0 + j * 8) * 2 : reinterpret_cast<const char *>(mx4_zeros));
    };
    f32x4_t acc[RT][NT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[r][nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](const Block &k) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const float scale = bits_f32(k.scales[r] << 23);
            const uint32_t c[4] = {k.codes[r].x, k.codes[r].y, k.codes[r].z, k.codes[r].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x8_t a = __builtin_bit_cast(bf16x8_t, mx4_decode(c[j], scale));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    acc[r][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8_t, k.v[nt][j]), acc[r][nt], 0, 0, 0);
            }
        }
    };
    const int blocks = (d_in + 127) / 128;
    if (wave < blocks) {
        Block k0, k1;
        load(k0, wave);
        for (int b = wave; b < blocks; b += 2 * KW) {
            if (b + KW < blocks) load(k1, b + KW);
            multiply(k0);
            if (b + KW >= blocks) break;
            if (b + 2 * KW < blocks) load(k0, b + 2 * KW);
            multiply(k1);
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) *reinterpret_cast<f32x4_t *>(&lds[wave][r * NT + nt][n][g * 4]) = acc[r][nt];
    __syncthreads();
    for (int i = tid; i < RT * NT * 64; i += 64 * KW) {   // (tile, token, four rows)
        const int tile = i >> 6, tok = (i >> 2) & 15, q = (i & 3) * 4;
        f32x4_t s = *reinterpret_cast<const f32x4_t *>(&lds[0][tile][tok][q]);
#pragma unroll
        for (int u = 1; u < KW; ++u) s += *reinterpret_cast<const f32x4_t *>(&lds[u][tile][tok][q]);
        const int64_t t = t0 + (tile % NT) * 16 + tok;
        const int row = (rt0 + tile / NT) * 16 + q;
        if (t >= T || row >= d_out) continue;   // d_out % 8 == 0: the four rows are in or out together
        if constexpr (Y32) *reinterpret_cast<f32x4_t *>(static_cast<float *>(y) + t * d_out + row) = s;
        else *reinterpret_cast<uint2 *>(static_cast<char *>(y) + (t * d_out + row) * 2) = make_uint2(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]));
    }
}

// The last NS - 1 rounds, of which nothing follows.
template <int NS, int LOADS, int U = 1, class Codes, class Multiply>
__device__ __forceinline__ void drain(const Codes *ring, Multiply &multiply)
{
    if constexpr (U < NS) {
        wait_vm_then_barrier<(NS - 1 - U) * LOADS>();
        multiply(ring[U], U);
        drain<NS, LOADS, U + 1>(ring, multiply);
    }
}

// A workgroup: KW groups of RW waves; a wave has 16 RT rows of W and all of the workgroup's 16 NT tokens, the groups take the column
// blocks of 128 in turn and add up in LDS at the end.  NS - 1 blocks are on their way: x, which the waves of a group share, straight
// to LDS, its 16-byte pieces at [piece ^ token] (the 16 tokens of an operand then lie in 16 different places of the LDS's
// width); every wave's own codes and scales to registers.
template <int RT, int NT, int RW, int KW, int NS, bool Y32>
__global__ __launch_bounds__(64 * RW * KW) void mx4_tile_kernel(const char *__restrict__ x, const char *__restrict__ W, void *__restrict__ y, int64_t T,
                                                                int d_in, int d_out, int col_tiles)
{
    constexpr int XI = NT * 4 / RW > 0 ? NT * 4 / RW : 1;    // wave loads of x per block: 1 KB, four tokens each
    static_assert(NT * 4 % RW == 0, "x loads");
    constexpr int X_BYTES = NT * 4096, STAGE_BYTES = KW * X_BYTES;
    constexpr int LOADS = XI + 2 * RT;                        // of a wave per block
    static_assert((NS - 1) * LOADS < 64, "vmcnt field");
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4, wave = uniform(tid >> 6);
    const int kw = wave / RW, rw = wave % RW;
    const int row_tiles = (d_out + 15) >> 4, rt0 = (blockIdx.x * RW + rw) * RT;
    const int64_t t0 = (int64_t)blockIdx.y * (16 * NT);
    const char *w[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) w[r] = W + (int64_t)min(rt0 + r, row_tiles - 1) * col_tiles * MX4_REC;
    // x: load i of the wave fills tokens 4 (rw XI + i) .. + 3; lane l its place l % 16 of token l / 16
    const char *xp[XI];
    int xc[XI];
#pragma unroll
    for (int i = 0; i < XI; ++i) {
        const int row = (rw * XI + i) * 4 + (lane >> 4);
        xp[i] = x + min(t0 + row, T - 1) * d_in * 2;
        xc[i] = ((lane ^ row) & 15) * 8;
    }
    char *const mine = lds + kw * X_BYTES;
    const int blocks = (d_in + 127) / 128, rounds = ((blocks + KW - 1) / KW + NS - 1) / NS * NS;
    struct Codes {
        uint4 c[RT];
        uint32_t s[RT];
    };
    Codes ring[NS];
    auto issue = [&](Codes &k, int i, int place) {
        const int whole = kw + i * KW, b = min(whole, blocks - 1), at = (b >> 2) * MX4_REC;
#pragma unroll
        for (int u = 0; u < XI; ++u) {
            const int col = whole * 128 + xc[u];
            const char *from = col < d_in ? xp[u] + col * 2 : reinterpret_cast<const char *>(mx4_zeros);
            __builtin_amdgcn_global_load_lds(MOIN_GPTR(from), MOIN_LPTR(mine + place * STAGE_BYTES + (rw * XI + u) * 1024), 16, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            k.c[r] = *reinterpret_cast<const uint4 *>(w[r] + at + (b & 3) * 1024 + lane * 16);
            k.s[r] = *reinterpret_cast<const uint8_t *>(w[r] + at + 4096 + lane * 4 + (b & 3));
        }
        asm volatile("" ::: "memory");   // a round's loads stay together, in the rounds' order: the waits count them
    };
    f32x4_t acc[RT][NT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[r][nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](const Codes &k, int place) {
        const char *xs = mine + place * STAGE_BYTES + n * 256;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bf16x8_t v[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                v[nt] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4 *>(xs + nt * 4096 + (((g * 4 + j) ^ n) & 15) * 16));
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const bf16x8_t a = __builtin_bit_cast(
                    bf16x8_t, mx4_decode(j == 0 ? k.c[r].x : j == 1 ? k.c[r].y : j == 2 ? k.c[r].z : k.c[r].w, bits_f32(k.s[r] << 23)));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) acc[r][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, v[nt], acc[r][nt], 0, 0, 0);
            }
        }
    };
    // All waves make the same rounds, a multiple of NS: beyond its last block a group has codes of the last one and an x of zeros.  No
    // branch decides what is on its way, so the counts below hold and the compiler's own waits for the codes are as exact.  At a round's
    // wait it has landed while the newer ones, which issued LOADS each, may be on their way, and every wave is done with
    // the round before, whose place is filled next.
#pragma unroll
    for (int i = 0; i < NS - 1; ++i) issue(ring[i], i, i);
    for (int i = 0; i + NS < rounds; i += NS) {
#pragma unroll
        for (int u = 0; u < NS; ++u) {
            wait_vm_then_barrier<(NS - 2) * LOADS>();
            issue(ring[(u + NS - 1) % NS], i + u + NS - 1, (u + NS - 1) % NS);
            multiply(ring[u], u);
        }
    }
    wait_vm_then_barrier<(NS - 2) * LOADS>();
    issue(ring[NS - 1], rounds - 1, NS - 1);
    multiply(ring[0], 0);
    drain<NS, LOADS>(ring, multiply);
    if constexpr (KW > 1) {
        wait_vm_then_barrier<0>();   // nothing is on its way into LDS any more, and all of it has been read
        f32x4_t *red = reinterpret_cast<f32x4_t *>(lds);
        if (kw > 0) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) red[((((kw - 1) * RW + rw) * RT + r) * NT + nt) * 64 + lane] = acc[r][nt];
        }
        lds_barrier();
        if (kw > 0) return;
#pragma unroll
        for (int u = 1; u < KW; ++u)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) acc[r][nt] += red[((((u - 1) * RW + rw) * RT + r) * NT + nt) * 64 + lane];
    } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load into LDS outlives the workgroup
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int64_t t = t0 + nt * 16 + n;
            const int row = (rt0 + r) * 16 + g * 4;
            const f32x4_t s = acc[r][nt];
            if (t >= T || row >= d_out) continue;
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

template <int RT, int NT, int KW>
static hipError_t launch_as(const void *x, const void *W, void *y, int y_f32, int64_t T, int d_in, int d_out, hipStream_t stream)
{
    const dim3 grid((unsigned)(((d_out + 15) / 16 + RT - 1) / RT), (unsigned)((T + 16 * NT - 1) / (16 * NT)));
    const int ct = (d_in + MX4_COLS - 1) / MX4_COLS;
    if (y_f32)
        hipLaunchKernelGGL((mx4_linear_kernel<RT, NT, KW, true>), grid, dim3(64 * KW), 0, stream, static_cast<const char *>(x),
                           static_cast<const char *>(W), y, T, d_in, d_out, ct);
    else
        hipLaunchKernelGGL((mx4_linear_kernel<RT, NT, KW, false>), grid, dim3(64 * KW), 0, stream, static_cast<const char *>(x),
                           static_cast<const char *>(W), y, T, d_in, d_out, ct);
    return hipGetLastError();
}

template <int RT, int NT, int RW, int KW, int NS>
constexpr int tile_lds_bytes()
{
    constexpr int stages = NS * KW * NT * 4096, sums = (KW - 1) * RW * RT * NT * 1024;
    return stages > sums ? stages : sums;
}

template <int RT, int NT, int RW, int KW, int NS>
static hipError_t launch_tile(const void *x, const void *W, void *y, int y_f32, int64_t T, int d_in, int d_out, hipStream_t stream)
{
    const dim3 grid((unsigned)(((d_out + 15) / 16 + RT * RW - 1) / (RT * RW)), (unsigned)((T + 16 * NT - 1) / (16 * NT)));
    const int ct = (d_in + MX4_COLS - 1) / MX4_COLS;
    constexpr int lds = tile_lds_bytes<RT, NT, RW, KW, NS>();
    if (y_f32)
        hipLaunchKernelGGL((mx4_tile_kernel<RT, NT, RW, KW, NS, true>), grid, dim3(64 * RW * KW), lds, stream, static_cast<const char *>(x),
                           static_cast<const char *>(W), y, T, d_in, d_out, ct);
    else
        hipLaunchKernelGGL((mx4_tile_kernel<RT, NT, RW, KW, NS, false>), grid, dim3(64 * RW * KW), lds, stream, static_cast<const char *>(x),
                           static_cast<const char *>(W), y, T, d_in, d_out, ct);
    return hipGetLastError();
}

// One token to four: lanes of the columns without a token load nothing new, so x costs little and the loop without LDS wins.  Rows of a
// workgroup go by how many there are for the chip.  Us of a call of one token, 16 / 32 / 64 rows of W in a workgroup of eight waves
// / the tiles below: 2048 -> 2048 3.2 / 3.4 / 4.3 / 3.4, 5632 -> 2048 4.3 / 5.2 / 7.4 / 6.3, 2048 -> 5632 4.2 / 3.6 / 4.4 / 3.9, 8192 -> 8192
// 12.3 / 8.7 / 12.2 / 10.8, 8192 -> 28672 35 / 29.3 / 28.1 / 29.6 (28.1: 4.5 TB/s of codes).  Five tokens 8192 -> 28672 29.1 / 29.6,
// 16: 8192 -> 8192 13.0 / 11.1, 8192 -> 28672 35.4 / 30.7.
constexpr int MX4_VECTOR_MAX_T = 4;

// More tokens, 16, 32 or 64 to a workgroup, whose shape goes by the tiles of 16 rows (by 64 tokens) that there are.  Few: its waves share the
// contraction, so that its chain of blocks is short; many: they share x.  Beyond 32 tokens the lines lie where the first two shapes have a
// workgroup for every compute unit, of which each takes one (128 KB of LDS).  Us of a call with the shapes of each rule in turn:
//  5 to 16 tokens: 2048 -> 2048 3.5 / 3.7 / 8.4, 2048 -> 5632 4.5 / 4.0 / 8.5, 8192 -> 8192 12.7 / 11.1 / 23.8, 8192 -> 28672 49 / 36 / 30.7
//  17 to 32: 2048 -> 2048 4.3 / 4.7 / 7.9, 2048 -> 5632 8.3 / 5.0 / 8.4, 8192 -> 8192 22.4 / 15.5 / 28.6, 8192 -> 28672 81 / 60 / 35
//  64: 2048 -> 2048 6.9 / 11.0 / 17, 5632 -> 2048 16.2 / 27 / 47, 8192 -> 28672 69 / 43.6 / 73
//  256: 2048 -> 2048 7.9 / 11.5 / 17, 2048 -> 5632 21 / 13.3 / 20, 8192 -> 8192 65 / 45 / 69, 8192 -> 28672 - / 150 / 108 (1.1 PFLOP/s)
//  (8192 -> 28672 at 17 to 32 tokens is 224 workgroups, one a compute unit: 32 units have none, and the codes come at 3.6 TB/s)
//  1024: 2048 -> 2048 22 / 14.6 / 20.5, 2048 -> 5632 - / 38 / 32, 8192 -> 8192 - / 160 / 108, 8192 -> 28672 - / - / 390 (1.23 PFLOP/s)
hipError_t launch_mx4_linear(const void *x, const void *W, void *y, int y_f32, int64_t T, int d_in, int d_out, hipStream_t stream)
{
    const int64_t tiles = (d_out + 15) / 16;
    if (T <= MX4_VECTOR_MAX_T) {
        if (tiles <= 256) return launch_as<1, 1, 8>(x, W, y, y_f32, T, d_in, d_out, stream);
        if (tiles <= 1024) return launch_as<2, 1, 8>(x, W, y, y_f32, T, d_in, d_out, stream);
        return launch_as<4, 1, 8>(x, W, y, y_f32, T, d_in, d_out, stream);
    }
    if (T <= 16) {
        if (tiles <= 256) return launch_tile<1, 1, 1, 8, 2>(x, W, y, y_f32, T, d_in, d_out, stream);
        if (tiles <= 1024) return launch_tile<1, 1, 2, 4, 4>(x, W, y, y_f32, T, d_in, d_out, stream);
        return launch_tile<2, 1, 4, 2, 6>(x, W, y, y_f32, T, d_in, d_out, stream);
    }
    if (T <= 32) {
        if (tiles <= 256) return launch_tile<1, 2, 1, 8, 2>(x, W, y, y_f32, T, d_in, d_out, stream);
        if (tiles <= 1024) return launch_tile<1, 2, 2, 4, 4>(x, W, y, y_f32, T, d_in, d_out, stream);
        return launch_tile<2, 2, 4, 2, 4>(x, W, y, y_f32, T, d_in, d_out, stream);
    }
    const int64_t work = tiles * ((T + 63) / 64);
    if (work <= 512) return launch_tile<1, 4, 2, 4, 2>(x, W, y, y_f32, T, d_in, d_out, stream);
    if (work <= 2048) return launch_tile<2, 4, 4, 2, 4>(x, W, y, y_f32, T, d_in, d_out, stream);
    return launch_tile<2, 4, 8, 1, 4>(x, W, y, y_f32, T, d_in, d_out, stream);
}

template <int RT, int NT, int RW, int KW, int NS>
static hipError_t allow_lds()
{
    constexpr int lds = tile_lds_bytes<RT, NT, RW, KW, NS>();
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&mx4_tile_kernel<RT, NT, RW, KW, NS, true>),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    return hipFuncSetAttribute(reinterpret_cast<const void *>(&mx4_tile_kernel<RT, NT, RW, KW, NS, false>),
                               hipFuncAttributeMaxDynamicSharedMemorySize, lds);
}

hipError_t prepare_mx4_kernels()
{
    hipError_t e;
    if ((e = allow_lds<1, 1, 1, 8, 2>()) != hipSuccess) return e;
    if ((e = allow_lds<1, 1, 2, 4, 4>()) != hipSuccess) return e;
    if ((e = allow_lds<2, 1, 4, 2, 6>()) != hipSuccess) return e;
    if ((e = allow_lds<1, 2, 1, 8, 2>()) != hipSuccess) return e;
    if ((e = allow_lds<1, 2, 2, 4, 4>()) != hipSuccess) return e;
    if ((e = allow_lds<2, 2, 4, 2, 4>()) != hipSuccess) return e;
    if ((e = allow_lds<1, 4, 2, 4, 2>()) != hipSuccess) return e;
    if ((e = allow_lds<2, 4, 4, 2, 4>()) != hipSuccess) return e;
    return allow_lds<2, 4, 8, 1, 4>();
}

}  // namespace moin

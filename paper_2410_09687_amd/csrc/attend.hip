// Attention of a step's tokens over the paged MXFP4 cache.  For a token at position p of its request, query head h of the
// group that shares a kv head, and the keys j <= p (and > p - window):
//     s_j = scale q . k_j,   y = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),   m = max_j s_j,   lse = m + log sum,
// in one pass over the keys with the running maximum and sum; a row that sees no key gives zeros and lse = -inf.
//
// Both products are taken transposed, S^T = K Q^T and O^T = V^T P^T: the codes are the A operand and a row of queries is a
// COLUMN of the accumulators.  A lane then holds 16 scores of one query row per record of 64 tokens, the softmax's
// statistics are its own, the scores turn into the second product's B operand
// where they are (the contraction order over the keys is free: the keys of a lane's accumulators are taken as its slots), and the
// rescaling of O^T is a product with the lane's own factor.  Scores and weights never leave the registers.
//   K: lane (m, g) (m = lane % 16, g = lane / 16) takes row m of a tile of 16 keys, channels [D/4 g, D/4 g + D/4);
//   V: word m of each key (8 channels), for the 4 keys 4 g .. 4 g + 3 of a tile: one 16-byte load, whose eight channels are rows m
//      of eight accumulators.  (D = 64: words m % 8, the nibbles of half m / 8.)
// Codes become bf16 exactly, two a conversion, the block's scale in the same instruction; V's pairs of channels are then regrouped into pairs
// of keys, one v_perm a pair.  Scores, statistics and sums are fp32; the weights exp(s - m) are rounded to bf16 for the second product, for
// fp32 results as the sum of three bf16; their sum is taken before.  For bf16 results one it is: beside the result's own rounding it shows
// little, and two cost more than they give (error against 64 bits and us, one / two: 256 requests 1.644e-3 and 35.0 / 1.609e-3 and 36.6, 8 tokens at
// 128 channels 1.756e-3 and 40.9 / 1.732e-3 and 46.2, prompts 1.729e-3 and 196 / 1.626e-3 and 258).
//
// Up to 32 rows of queries to a request and kv head (a token or a few): the workgroup's waves take the records in turn, each decodes its own,
// and the work is cut along the keys until the chip is full.  Bound by memory: 68 D bytes a record and kv head against 4 D flops a row and key.
// 256 requests of up to 4096 keys, 32 heads on 4 of 64 channels, 35 us: 4.3 TB/s; two of 100000 and more, 64 heads on 8 of 128, 61 us: 4.3 TB/s;
// a thousand keys 7.6 us: half a dozen trips to memory.  (An even cut over a grid that stays: 47 - 52 us for the first, a piece's beginning and
// end cost 4 to 6.)  A few tokens a request: 64 requests of 2000 keys and 4 tokens, 32 heads on 4 of 64, 18.2 us (floor 7.4), 8 tokens, 32 on 8 of 128,
// 40.8 (29.5), where a wave's two columns leave a SIMD one wave.
// More rows (prompts, chunks of them): tiles of 128, every wave has 32 rows and walks all records, a quarter of which it decodes into
// LDS for the others.  Bound by the vector unit (eight prompts of 2048, 32 heads on 4 of 64 channels, 196 us, 0.70 PFLOP/s: busy 76 % of the
// cycles in which a compute unit has work, the matrix cores 32 %).  265 vector instructions a wave and record by the counters: 32 of the matrix cores, 181 of the
// others where every row sees the record and the reference stays (the softmax's fma, exp and sum of 32 scores a lane 104, packs 18, decoding 49), and some 50
// for the rest: a tile's first record, whose weights are computed twice, its last one's masks, its beginning and end with
// their divisions.  Long prompts 0.91 PFLOP/s (64 channels), 1.05 (128); fp32 results 339 us; heads of 256 channels 241 for the same products.  A record's keys multiplied ahead, beside the weights of the one before: 272 us, the registers then hold two waves of a
// SIMD instead of three.
#include "attend_core.h"
#include "mxfp4.h"

namespace moin {

namespace {

__device__ __forceinline__ uint32_t pair_of(uint32_t codes, float scale, int u)   // u: a constant once unrolled
{
    return u == 0 ? mx4_pair<0>(codes, scale) : u == 1 ? mx4_pair<1>(codes, scale) : u == 2 ? mx4_pair<2>(codes, scale) : mx4_pair<3>(codes, scale);
}

// V^T operands of two channels, byte u of the lane's words shifted down by `shift`: the 4 keys of its group in two tiles of 16 (words c0 and
// c1, whose scales are bytes i and i + 1 of vs).
__device__ __forceinline__ void value_operands(const uint4 &c0, const uint4 &c1, const uint4 &vs, int i, int shift, int u, bf16x8_t &even, bf16x8_t &odd)
{
    uint32_t x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        x[e] = pair_of(word(e < 4 ? c0 : c1, e & 3) >> shift, mx4_scale(word(vs, e & 3), i + e / 4), u);
    }
    even = operand(lows(x[0], x[1]), lows(x[2], x[3]), lows(x[4], x[5]), lows(x[6], x[7]));
    odd = operand(highs(x[0], x[1]), highs(x[2], x[3]), highs(x[4], x[5]), highs(x[6], x[7]));
}

template <int D_>
struct Mx4 {
    static constexpr int D = D_, NJ = D / 16;
    static constexpr int KD = D / 32;            // words of K codes per tile and lane (8 channels each)
    static constexpr int SB = D == 256 ? 2 : 1;  // blocks of 32 channels per lane

    using Source = const char *;
    __device__ __forceinline__ static int record_bytes(int d) { return kv_record_bytes(d); }
    __device__ __forceinline__ static int64_t page_bytes(const KvPages &p) { return p.page_bytes(); }
    __device__ __forceinline__ static const char *tail(const KvPages &, int) { return nullptr; }   // (the scales are in the records)
    __device__ __forceinline__ static Source source(const char *rec, const char *, int) { return rec; }

    // Waves per SIMD that the registers are to leave room for.  (D = 64: four spill, 43 -> 55 us for 256 requests; D = 128: three spill,
    // 65 -> 80 us for two long ones.)
    template <int NT>
    static constexpr int min_waves()
    {
        return NT > 1 ? (D == 64 ? 2 : 1) : D == 64 ? 3 : D == 128 ? 2 : 1;
    }

    // What a wave holds of a record: codes and scale words.
    struct Record {
        uint32_t k[4][KD];
        uint32_t ks[SB];
        uint4 v[4][SB];
        uint4 vs[SB];
    };

    // Where in a record a lane's pieces lie.
    struct Places {
        uint32_t k, v, ks, vs;
        __device__ __forceinline__ explicit Places(int lane)
        {
            const uint32_t m = lane & 15, g = lane >> 4;
            k = D == 64 ? (g >> 1) * 256 + m * 16 + (g & 1) * 8 : g * 256 + m * 16;
            ks = 64 * D + (D == 64 ? g >> 1 : g) * 64 + m * 4;
            v = 32 * D + (D == 64 ? m & 7 : m) * 64 + g * 16;
            vs = 66 * D + (D == 64 ? (m & 7) >> 2 : m >> 2) * 64 + g * 16;
        }
    };

    __device__ __forceinline__ static void load(Record &r, Source rec, const Places &at)
    {
#pragma unroll
        for (int b = 0; b < SB; ++b) {
            r.ks[b] = *reinterpret_cast<const uint32_t *>(rec + (at.ks + b * 256));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (D == 64) {
                    const uint2 x = *reinterpret_cast<const uint2 *>(rec + (at.k + i * 8 * D));
                    r.k[i][0] = x.x;
                    r.k[i][1] = x.y;
                } else {
                    const uint4 x = *reinterpret_cast<const uint4 *>(rec + (at.k + i * 8 * D + b * 1024));
                    r.k[i][4 * b] = x.x;
                    r.k[i][4 * b + 1] = x.y;
                    r.k[i][4 * b + 2] = x.z;
                    r.k[i][4 * b + 3] = x.w;
                }
            }
            r.vs[b] = *reinterpret_cast<const uint4 *>(rec + (at.vs + b * 256));
#pragma unroll
            for (int i = 0; i < 4; ++i) r.v[i][b] = *reinterpret_cast<const uint4 *>(rec + (at.v + i * 8 * D + b * 1024));
        }
    }

    __device__ __forceinline__ static int k_channel(int j, int g)
    {
        return D == 64 ? g * 16 + j * 8 : (j >> 2) * 128 + g * 32 + (j & 3) * 8;
    }
    __device__ __forceinline__ static int o_channel(int m)   // of accumulator 0; the others follow (D = 256: 8 further on by 128)
    {
        return D == 64 ? (m & 7) * 8 + (m >> 3) * 4 : m * 8;
    }
    __device__ __forceinline__ static int o_channel(int m, int j) { return o_channel(m) + (D == 256 ? (j >> 3) * 128 + (j & 7) : j); }

    __device__ __forceinline__ static bf16x8_t k_operand(const Record &r, int i, int j)
    {
        return __builtin_bit_cast(bf16x8_t, mx4_decode(r.k[i][j], mx4_scale(r.ks[j / 4], i)));
    }
    __device__ __forceinline__ static void v_operands(const Record &r, int h, int u, int lane, bf16x8_t &even, bf16x8_t &odd)
    {
        constexpr int PAIRS = D == 64 ? 2 : 4;   // pairs of channels of a word
        const int b = u / PAIRS;
        value_operands(r.v[2 * h][b], r.v[2 * h + 1][b], r.vs[b], 2 * h, D == 64 ? (lane & 8) * 2 : 0, u % PAIRS, even, odd);
    }

    template <int NT>
    __device__ __forceinline__ static void mask(Record &r, f32x4_t (&o)[NT][NJ], int n_cols, int tok, const int *lo, const int *hi, int end, int lane)
    {
        mask_values<NT>(r.vs, o, n_cols, tok, lo, hi, end, lane);
    }
    // The values of a record that not every row sees: what lies beyond the request's keys may hold anything and a block may
    // stand for NaN, and 0 times that is not 0 in the product.  Their scales become 2^-127; a row that does see a block of NaNs gets
    // its channels' NaN here, from a product of what is seen with what is NaN.
    template <int NT>
    __device__ __forceinline__ static void mask_values(uint4 (&vs)[SB], f32x4_t (&o)[NT][NJ], int n_cols, int tok, const int *lo, const int *hi, int end, int lane)
    {
        const int g = lane >> 4;
        uint32_t full = 0;   // bit 7 of a byte: it is 255
#pragma unroll
        for (int b = 0; b < SB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) full |= word(vs[b], e) & ((word(vs[b], e) & 0x7F7F7F7Fu) + 0x01010101u);
        if (tok + 64 <= end && __ballot((full & 0x80808080u) != 0) == 0) return;   // (a prompt's own triangle, as a rule)
#pragma unroll
        for (int b = 0; b < SB; ++b) {
            uint32_t nan[4], any = 0;   // [key e]: byte i is 255 where the block stands for NaN and the request has the key
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t w = word(vs[b], e), bad = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t byte = 255u << (8 * i);
                    const bool has = tok + i * 16 + g * 4 + e < end;
                    if (has && (w & byte) == byte) bad |= byte;
                    if (!has || (w & byte) == byte) w &= ~byte;
                }
                nan[e] = bad;
                any |= bad;
                if (e == 0) vs[b].x = w;
                else if (e == 1) vs[b].y = w;
                else if (e == 2) vs[b].z = w;
                else vs[b].w = w;
            }
            if (__ballot(any != 0) == 0) continue;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (nt > 0 && nt >= n_cols) continue;
                f32x4_t count{0.f, 0.f, 0.f, 0.f};   // row m: of the channels whose scales lane (m, .) holds
#pragma unroll
                for (int a = 0; a < 2; ++a) {
                    uint32_t is[4], sees[4];
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const int i = 2 * a + h / 2, e = (h & 1) * 2, key = tok + i * 16 + g * 4 + e;
                        is[h] = (nan[e] >> (8 * i) & 1 ? 0x3F80u : 0u) | (nan[e + 1] >> (8 * i) & 1 ? 0x3F800000u : 0u);
                        sees[h] = (key >= lo[nt] && key < hi[nt] ? 0x3F80u : 0u) | (key + 1 >= lo[nt] && key + 1 < hi[nt] ? 0x3F800000u : 0u);
                    }
                    count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(is[0], is[1], is[2], is[3]),
                                                                    operand(sees[0], sees[1], sees[2], sees[3]), count, 0, 0, 0);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (count[e] > 0.f)
#pragma unroll
                        for (int j = b * 8; j < (SB == 1 ? NJ : b * 8 + 8); ++j) o[nt][j][e] = bits_f32(0x7FC00000u);
            }
        }
    }

    struct Operands {
        uint4 k[4][KD][64], v[2][NJ][64];
    };
    // Keys 16 wave .. + 15; of the values those of half wave / 2, MINE pairs of accumulators from u0 on.
    struct Share {
        static constexpr int MINE = NJ / 4;   // pairs of accumulators of each half whose V operands a wave decodes
        const Places at;
        const int lane, wave, half, u0;
        uint32_t kc[KD], ks[SB];
        uint4 vc[2], vs[SB];
        __device__ __forceinline__ Share(int lane, int wave) : at(lane), lane(lane), wave(wave), half(wave >> 1), u0((wave & 1) * MINE) {}
        __device__ __forceinline__ void load(Source rec)
        {
#pragma unroll
            for (int b = 0; b < SB; ++b) {
                ks[b] = *reinterpret_cast<const uint32_t *>(rec + (at.ks + b * 256));
                vs[b] = *reinterpret_cast<const uint4 *>(rec + (at.vs + b * 256));
                if constexpr (D == 64) {
                    const uint2 x = *reinterpret_cast<const uint2 *>(rec + (at.k + wave * 8 * D));
                    kc[0] = x.x;
                    kc[1] = x.y;
                } else {
                    const uint4 x = *reinterpret_cast<const uint4 *>(rec + (at.k + wave * 8 * D + b * 1024));
                    kc[4 * b] = x.x;
                    kc[4 * b + 1] = x.y;
                    kc[4 * b + 2] = x.z;
                    kc[4 * b + 3] = x.w;
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
                vc[i] = *reinterpret_cast<const uint4 *>(rec + (at.v + (2 * half + i) * 8 * D + (D == 256 ? wave & 1 : 0) * 1024));
        }
        template <int NT>
        __device__ __forceinline__ void mask(f32x4_t (&o)[NT][NJ], int n_cols, int tok, const int *lo, const int *hi, int end)
        {
            mask_values<NT>(vs, o, n_cols, tok, lo, hi, end, lane);
        }
        __device__ __forceinline__ void decode(Operands &o) const
        {
#pragma unroll
            for (int j = 0; j < KD; ++j) o.k[wave][j][lane] = mx4_decode(kc[j], mx4_scale(ks[j / 4] >> (8 * wave), 0));
            uint4 scales = SB == 2 && (wave & 1) ? vs[SB - 1] : vs[0];
            scales = make_uint4(scales.x >> (16 * half), scales.y >> (16 * half), scales.z >> (16 * half), scales.w >> (16 * half));
#pragma unroll
            for (int u = 0; u < MINE; ++u) {
                bf16x8_t even, odd;
                value_operands(vc[0], vc[1], scales, 0, (D == 64 ? (lane & 8) * 2 : 0) + (D == 256 ? 0 : 8 * u0), u, even, odd);
                o.v[half][2 * (u0 + u)][lane] = __builtin_bit_cast(uint4, even);
                o.v[half][2 * (u0 + u) + 1][lane] = __builtin_bit_cast(uint4, odd);
            }
        }
    };

    __device__ __forceinline__ static void store(const AttendArgs &a, int64_t y, const f32x4_t (&o)[NJ], float inv, int g)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (int b = 0; b < SB; ++b) {
                constexpr int N = D == 64 ? 4 : 8;
                float x[N];
#pragma unroll
                for (int j = 0; j < N; ++j) x[j] = o[b * 8 + j][e] * inv;
                store_y(a, y, D, o_channel(g * 4 + e) + b * 128, x);
            }
        }
    }
};

}  // namespace

int64_t attend_partial_floats(const KvPlanView &v, int pslots, int D)
{
    return (int64_t)pslots * v.n_kv * KV_FEW_ROWS * (D + 2);
}

hipError_t launch_attend(const KvPlanView &v, const AttendArgs &a, hipStream_t stream)
{
    switch (a.pages.D) {
    case 64: return a.y_f32 ? launch_d<Mx4<64>, true>(v, a, stream) : launch_d<Mx4<64>, false>(v, a, stream);
    case 128: return a.y_f32 ? launch_d<Mx4<128>, true>(v, a, stream) : launch_d<Mx4<128>, false>(v, a, stream);
    case 256: return a.y_f32 ? launch_d<Mx4<256>, true>(v, a, stream) : launch_d<Mx4<256>, false>(v, a, stream);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace moin

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
#include "kv.h"
#include "mxfp4.h"

namespace moin {

namespace {

constexpr float NEG_INF = -__builtin_huge_valf();

// What a wave holds of a record: codes and scale words.
template <int D>
struct Record {
    static constexpr int KD = D / 32;            // words of K codes per tile and lane (8 channels each)
    static constexpr int SB = D == 256 ? 2 : 1;  // blocks of 32 channels per lane
    uint32_t k[4][KD];
    uint32_t ks[SB];
    uint4 v[4][SB];
    uint4 vs[SB];
};

// Where in a record a lane's pieces lie.
template <int D>
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

template <int D>
__device__ __forceinline__ void load_record(Record<D> &r, const char *rec, const Places<D> &at)
{
#pragma unroll
    for (int b = 0; b < Record<D>::SB; ++b) {
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

// Channel of a query that element e of K operand j holds for lanes of group g; the same for the rows of O^T: channel of
// accumulator j, row m.
template <int D>
__device__ __forceinline__ int k_channel(int j, int g)
{
    return D == 64 ? g * 16 + j * 8 : (j >> 2) * 128 + g * 32 + (j & 3) * 8;
}
template <int D>
__device__ __forceinline__ int o_channel(int m)   // of accumulator 0; the others follow (D = 256: 8 further on by 128)
{
    return D == 64 ? (m & 7) * 8 + (m >> 3) * 4 : m * 8;
}

__device__ __forceinline__ uint32_t lows(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t highs(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ bf16x8_t operand(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_bit_cast(bf16x8_t, make_uint4(a, b, c, d));
}
__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Maximum and sum over the four lanes of a column.
__device__ __forceinline__ float max4(float v)
{
    auto a = __builtin_amdgcn_permlane32_swap(f32_bits(v), f32_bits(v), false, false);
    v = fmaxf(bits_f32(a[0]), bits_f32(a[1]));
    a = __builtin_amdgcn_permlane16_swap(f32_bits(v), f32_bits(v), false, false);
    return fmaxf(bits_f32(a[0]), bits_f32(a[1]));
}
__device__ __forceinline__ float sum4(float v)
{
    auto a = __builtin_amdgcn_permlane32_swap(f32_bits(v), f32_bits(v), false, false);
    v = bits_f32(a[0]) + bits_f32(a[1]);
    a = __builtin_amdgcn_permlane16_swap(f32_bits(v), f32_bits(v), false, false);
    return bits_f32(a[0]) + bits_f32(a[1]);
}

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

struct AttendK {
    KvPlanView v;
    AttendArgs a;
    int list;              // 0: the tiles of few rows, 1: the others
};

// A workgroup's work: rows [t.row0, row_end) of a request's tile, one kv head, records [b0, b1).
struct Work {
    KvTile t;
    int h, row_end;
    int pos0, first, last;   // positions of the request's first new token, and of the rows' first and last
    int window, b0, b1;

    // False: nothing to do.  `height`: rows of a tile.
    __device__ __forceinline__ bool find(const AttendK &p, int height)
    {
        const KvPlanView &v = p.v;
        const int rec_id = blockIdx.x / v.n_kv;
        h = blockIdx.x - rec_id * v.n_kv;
        const int4 *line = reinterpret_cast<const int4 *>((p.list ? v.tile : v.few) + rec_id);
        const int4 ta = line[0], tb = line[1];   // (beside the list's length, not after it)
        if (rec_id >= v.head[p.list]) return false;
        t = KvTile{uniform(ta.x), uniform(ta.y), uniform(ta.z), uniform(ta.w), uniform(tb.x), uniform(tb.y), uniform(tb.z), uniform(tb.w)};
        const int rows = t.n_tok * v.group;
        row_end = min(rows, t.row0 + height);
        pos0 = t.kv_len - t.n_tok;
        first = pos0 + t.row0 / v.group;
        last = pos0 + (row_end - 1) / v.group;
        window = min(p.a.window > 0 ? p.a.window : 0x7fffffff, t.kv_len + 1);   // (no further: no position minus it overflows)
        const int lo_all = max(0, first - window + 1), hi_all = max(0, last + 1);
        const int b_lo = lo_all >> 6, n_blocks = hi_all > lo_all ? ((hi_all + 63) >> 6) - b_lo : 0;
        b0 = b_lo + (int)((int64_t)n_blocks * t.part / t.n_parts);
        b1 = b_lo + (int)((int64_t)n_blocks * (t.part + 1) / t.n_parts);
        return true;
    }
    // Every row sees all of record b.
    __device__ __forceinline__ bool whole(int b) const { return b * 64 >= last - window + 1 && b * 64 + 63 <= first; }
};

// A wave's columns (16 NT rows of queries) over the records that it walks.
template <int D, int NT, bool Y32>
struct Columns {
    static constexpr int KD = Record<D>::KD, SB = Record<D>::SB, NJ = D / 16;
    bf16x8_t q[NT][KD];
    f32x4_t o[NT][NJ];
    float m[NT], l[NT];    // reference of the weights, in units of log2 e / scale: the largest score so far or near it; this lane's share of the sum

    // The rows row0 .. of the workgroup's: their queries, and the keys [lo, hi) that each sees.
    __device__ __forceinline__ void begin(const AttendArgs &a, const Work &k, int row0, int group, int n_kv, int *lo, int *hi, int lane)
    {
        const int n = lane & 15, g = lane >> 4;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = row0 + nt * 16 + n;
            const bool real = row < k.row_end;
            const int i = real ? row / group : 0, pos = k.pos0 + i;
            lo[nt] = real ? max(0, pos - k.window + 1) : 0;
            hi[nt] = real ? max(0, pos + 1) : 0;
            m[nt] = real ? NEG_INF : 0.f;   // (a row that is none never asks for a maximum)
            l[nt] = 0.f;
#pragma unroll
            for (int j = 0; j < NJ; ++j) o[nt][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            const char *x = static_cast<const char *>(a.q) +
                            ((k.t.tok0 + i) * a.q_stride + (int64_t)(k.h * group + (real ? row - i * group : 0)) * D) * 2;
#pragma unroll
            for (int j = 0; j < KD; ++j) {
                const uint4 u = *reinterpret_cast<const uint4 *>(x + k_channel<D>(j, g) * 2);
                q[nt][j] = __builtin_bit_cast(bf16x8_t, real ? u : make_uint4(0, 0, 0, 0));
            }
        }
    }

    static constexpr int NP = Y32 ? 3 : 1;
    using Scores = f32x4_t[NT][4];          // [.][tile of 16 keys]: this lane's row, its group's four keys
    using Weights = uint32_t[NP][NT][4][2]; // as a sum of NP bf16, keys 0 1 and 2 3 of a tile's four

    // Scores of tile i, whose K operands are k.
    __device__ __forceinline__ void score(const bf16x8_t (&k)[KD], Scores &s, int i, int n_cols) const
    {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (nt > 0 && nt >= n_cols) continue;
            s[nt][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < KD; ++j) s[nt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[j], q[nt][j], s[nt][i], 0, 0, 0);
        }
    }
    // The softmax of a record: scores to weights.  masked: row nt of this lane sees keys [lo[nt], hi[nt]) alone; tok: the record's first token.
    __device__ __forceinline__ void weigh(Scores &s, Weights &p, int n_cols, float c, int tok, bool masked, const int *lo, const int *hi, int lane)
    {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (nt > 0 && nt >= n_cols) continue;
            if (masked) {
                int key = tok + (lane >> 4) * 4;
                asm volatile("" : "+v"(key));   // (or the sixteen sums move up, in front of the condition)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[nt][i][e] = key + i * 16 + e >= lo[nt] && key + i * 16 + e < hi[nt] ? s[nt][i][e] : NEG_INF;
            }
            auto fill = [&]() {
                const float base = m[nt] == NEG_INF ? 0.f : m[nt] * c;
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w[e] = __builtin_amdgcn_exp2f(fmaf(s[nt][i][e], c, -base));
                        sum += w[e];
                    }
#pragma unroll
                    for (int u = 0; u < NP; ++u) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t hi2 = pack_bf16x2(w[2 * h], w[2 * h + 1]);
                            p[u][nt][i][h] = hi2;
                            w[2 * h] -= bits_f32(hi2 << 16);
                            w[2 * h + 1] -= bits_f32(hi2 & 0xFFFF0000u);
                        }
                    }
                }
                return sum;
            };
            // Any reference near the maximum does: it moves only where the weights would pass 2^8, which their sum shows, so that the maximum
            // itself is rarely taken.  (Taken in every record it is new for one of 16 rows in most records of a prompt.)
            float sum = fill();
            if (__ballot(!(sum <= 256.f) || m[nt] == NEG_INF)) {
                float top = m[nt];
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(fmaxf(top, fmaxf(s[nt][i][0], s[nt][i][1])), fmaxf(s[nt][i][2], s[nt][i][3]));
                top = max4(top);
                const float shrink = m[nt] == top ? 1.f : __builtin_amdgcn_exp2f((m[nt] - top) * c);   // exp2(-inf) = 0 for the first keys
                l[nt] *= shrink;
#pragma unroll
                for (int j = 0; j < NJ; ++j) o[nt][j] *= shrink;
                m[nt] = top;
                sum = fill();
            }
            l[nt] += sum;
        }
    }
    // Values of tiles 2 h and 2 h + 1 into accumulators 2 u and 2 u + 1, whose V^T operands are even and odd.
    __device__ __forceinline__ void add(const Weights &p, int h, int u, bf16x8_t even, bf16x8_t odd, int n_cols)
    {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (nt > 0 && nt >= n_cols) continue;
#pragma unroll
            for (int z = 0; z < NP; ++z) {
                const bf16x8_t pz = operand(p[z][nt][2 * h][0], p[z][nt][2 * h][1], p[z][nt][2 * h + 1][0], p[z][nt][2 * h + 1][1]);
                o[nt][2 * u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, pz, o[nt][2 * u], 0, 0, 0);
                o[nt][2 * u + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, pz, o[nt][2 * u + 1], 0, 0, 0);
            }
        }
    }

    // A record in this wave's own registers.  masked: not every row sees all of it; end: keys that the request has.
    __device__ __forceinline__ void step(Record<D> &r, int n_cols, float c, int tok, bool masked, const int *lo, const int *hi, int end, int lane)
    {
        if (masked) mask_values(r.vs, n_cols, tok, lo, hi, end, lane);
        Scores s;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bf16x8_t k[KD];
#pragma unroll
            for (int j = 0; j < KD; ++j) k[j] = __builtin_bit_cast(bf16x8_t, mx4_decode(r.k[i][j], mx4_scale(r.ks[j / 4], i)));
            score(k, s, i, n_cols);
        }
        Weights p;
        weigh(s, p, n_cols, c, tok, masked, lo, hi, lane);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int u = 0; u < NJ / 2; ++u) {
                constexpr int PAIRS = D == 64 ? 2 : 4;   // pairs of channels of a word
                const int b = u / PAIRS;
                bf16x8_t even, odd;
                value_operands(r.v[2 * h][b], r.v[2 * h + 1][b], r.vs[b], 2 * h, D == 64 ? (lane & 8) * 2 : 0, u % PAIRS, even, odd);
                add(p, h, u, even, odd, n_cols);
            }
    }

    // The values of a record that not every row sees: what lies beyond the request's keys may hold anything and a block may
    // stand for NaN, and 0 times that is not 0 in the product.  Their scales become 2^-127; a row that does see a block of NaNs gets
    // its channels' NaN here, from a product of what is seen with what is NaN.
    __device__ __forceinline__ void mask_values(uint4 (&vs)[SB], int n_cols, int tok, const int *lo, const int *hi, int end, int lane)
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
};

// Output row of the request's tokens: group rows of a token are query heads of the kv head.
__device__ __forceinline__ int64_t y_row(const KvTile &t, int row, int group, int n_kv, int h)
{
    const int i = row / group;
    return ((int64_t)t.tok0 + i) * (n_kv * group) + h * group + (row - i * group);
}

// Partial results cross from one XCD's L2 to another's: device-scope accesses, two floats each (p 8-byte aligned).
__device__ __forceinline__ void put_agent(float *p, float a, float b)
{
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), (uint64_t)f32_bits(b) << 32 | f32_bits(a), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get_agent(const float *p)
{
    const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(bits_f32((uint32_t)v), bits_f32((uint32_t)(v >> 32)));
}

template <int N>
__device__ __forceinline__ void store_y(const AttendArgs &a, int64_t row, int D, int ch, const float (&x)[N])
{
    if (a.y_f32) {
        float *y = static_cast<float *>(a.y) + row * D + ch;
#pragma unroll
        for (int i = 0; i < N; i += 4) *reinterpret_cast<float4 *>(y + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    } else {
        char *y = static_cast<char *>(a.y) + (row * D + ch) * 2;
#pragma unroll
        for (int i = 0; i < N; i += 4)
            *reinterpret_cast<uint2 *>(y + i * 2) = make_uint2(pack_bf16x2(x[i], x[i + 1]), pack_bf16x2(x[i + 2], x[i + 3]));
    }
}

constexpr float LN2 = 0.69314718055994530942f, LOG2E = 1.44269504088896340736f;

// (a row that saw nothing has a sum of zero; NaN stays)
__device__ __forceinline__ float inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float log_sum(float m, float l, float c) { return l == 0.f ? NEG_INF : (m * c + __builtin_amdgcn_logf(l)) * LN2; }

// Waves per SIMD that the registers are to leave room for.  (D = 64: four spill, 43 -> 55 us for 256 requests; D = 128: three spill,
// 65 -> 80 us for two long ones.)
template <int D, int NT>
constexpr int min_waves()
{
    return NT > 1 ? (D == 64 ? 2 : 1) : D == 64 ? 3 : D == 128 ? 2 : 1;
}

// The end of a workgroup whose tile has several parts, its own left in `partial`: whether it is the last of the tile's to report, which then joins
// the parts, in their order.  What the parts leave are device-scope stores: a workgroup waits for its own before it reports, and nobody's L2
// has to be written back.
// `place`: which of the tile's tickets (it has as many as parts); `expected`: how many report there.
__device__ __forceinline__ bool last_of(const KvPlanView &v, const Work &k, int place, int expected, int *flag)
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int *ticket = v.tickets + (int64_t)(k.t.pslot + place) * v.n_kv + k.h;
    if (threadIdx.x == 0) {
        *flag = atomicAdd(ticket, 1) == expected - 1;
        if (*flag) *ticket = 0;   // clean for the next call
    }
    __syncthreads();
    return *flag;
}

// The groups in which a tile's parts are joined: one workgroup reads them at a microsecond or more each, so beyond eight they are joined in
// groups first, whose last ones to report join the groups.  (A prompt of 64 behind 30000 keys, 32 parts, 62 us; one after the other 104.)
struct Groups {
    int size, first, last;   // parts of a whole group; the first of this part's, and behind its last
    __device__ __forceinline__ explicit Groups(const KvTile &t)
    {
        size = t.n_parts;
        if (t.n_parts > 8)
            for (size = 3; size * size < t.n_parts;) ++size;
        first = t.part - t.part % size;
        last = min(first + size, t.n_parts);
    }
};

// Joins parts from, from + step ... below `to` of a tile of few rows, a part's rows one after the other, {m, l, channels} each: to part `from`, or to y.
// 256 threads, 16 to a row, everything of four parts on its way at once and of two rows a thread: a trip to memory for 32 rows.
template <int D, int ROWS>
__device__ __forceinline__ void join_rows(const AttendK &p, const Work &k, float c, int from, int to, int step, bool final)
{
    constexpr int CH = D / 16, AHEAD = 4, G = ROWS > 16 ? 2 : 1;   // CH: channels of a row per thread
    const KvPlanView &v = p.v;
    const KvTile &t = k.t;
    const int row = threadIdx.x >> 4, ch = (threadIdx.x & 15) * CH, n_rows = k.row_end - t.row0;
    const int64_t part_step = (int64_t)v.n_kv * KV_FEW_ROWS * (D + 2);
    float *tile = p.a.partial + ((int64_t)t.pslot * v.n_kv + k.h) * KV_FEW_ROWS * (D + 2);
    for (int r0 = 0; r0 < n_rows; r0 += 16 * G) {
        float m[G], l[G], x[G][CH];
#pragma unroll
        for (int z = 0; z < G; ++z) {
            m[z] = NEG_INF;
            l[z] = 0.f;
#pragma unroll
            for (int i = 0; i < CH; ++i) x[z][i] = 0.f;
        }
        for (int u0 = from; u0 < to; u0 += AHEAD * step) {
            float2 ml[G][AHEAD], a[G][AHEAD][CH / 2];
#pragma unroll
            for (int z = 0; z < G; ++z) {
                const float *o = tile + min(r0 + 16 * z + row, n_rows - 1) * (D + 2);
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const float *part = o + (u0 + u * step < to ? u0 + u * step : from) * part_step;
                    ml[z][u] = get_agent(part);
#pragma unroll
                    for (int i = 0; i < CH / 2; ++i) a[z][u][i] = get_agent(part + 2 + ch + 2 * i);
                }
            }
#pragma unroll
            for (int z = 0; z < G; ++z) {
                float top = m[z];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) top = fmaxf(top, ml[z][u].x);   // (one part more than once: no harm to a maximum)
                const float base = top == NEG_INF ? 0.f : top * c;
                const float shrink = __builtin_amdgcn_exp2f(fmaf(m[z], c, -base));
                m[z] = top;
                l[z] *= shrink;
#pragma unroll
                for (int i = 0; i < CH; ++i) x[z][i] *= shrink;
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    if (u0 + u * step >= to) break;
                    const float f = __builtin_amdgcn_exp2f(fmaf(ml[z][u].x, c, -base));
                    l[z] = fmaf(ml[z][u].y, f, l[z]);
#pragma unroll
                    for (int i = 0; i < CH / 2; ++i) {
                        x[z][2 * i] = fmaf(a[z][u][i].x, f, x[z][2 * i]);
                        x[z][2 * i + 1] = fmaf(a[z][u][i].y, f, x[z][2 * i + 1]);
                    }
                }
            }
        }
#pragma unroll
        for (int z = 0; z < G; ++z) {
            const int local = r0 + 16 * z + row;
            if (local >= n_rows) continue;
            if (final) {
                const float inv = inverse(l[z]);
#pragma unroll
                for (int i = 0; i < CH; ++i) x[z][i] *= inv;
                const int64_t at = y_row(t, t.row0 + local, v.group, v.n_kv, k.h);
                store_y(p.a, at, D, ch, x[z]);
                if (p.a.lse && ch == 0) p.a.lse[at] = log_sum(m[z], l[z], c);
            } else {
                float *o = tile + from * part_step + local * (D + 2);   // (nobody but the row's own threads reads it here, all of them before)
#pragma unroll
                for (int i = 0; i < CH; i += 2) put_agent(o + 2 + ch + i, x[z][i], x[z][i + 1]);
                if (ch == 0) put_agent(o, m[z], l[z]);
            }
        }
    }
}

// Where the records of a request's kv head lie.
struct Records {
    const int *table;
    const char *head;
    int64_t page_bytes;
    int log_blocks, n_pages, record;

    __device__ __forceinline__ Records(const AttendArgs &a, const Work &k)
        : table(a.block_table + (int64_t)k.t.req * a.max_pages),
          head(a.pages.data + (((int64_t)k.h * kv_record_bytes(a.pages.D)) << a.pages.log_blocks)),
          page_bytes(a.pages.page_bytes()), log_blocks(a.pages.log_blocks), n_pages(a.pages.n_pages), record(kv_record_bytes(a.pages.D))
    {
    }
    // Record b; `ok`: its page exists (else one of page 0).
    __device__ __forceinline__ const char *at(int b, int page, bool &ok) const
    {
        ok = page >= 0 && page < n_pages;
        return head + (int64_t)(ok ? page : 0) * page_bytes + (b & ((1 << log_blocks) - 1)) * record;
    }
};

// Tiles of few rows: CW groups of KW waves; a group has 16 NT rows of the tile, its waves take the records in turn and decode them in
// their registers.
template <int D, int NT, int CW, int KW, bool Y32>
__global__ __launch_bounds__(64 * CW * KW, (min_waves<D, NT>())) void attend_few_kernel(AttendK p)
{
    constexpr int ROWS = 16 * NT * CW, CH = D / 16;   // CH: channels of a row per thread in the joins
    constexpr int LDO = D + 4;
    static_assert(CW * KW == 4, "the join's threads: 16 rows of 16");
    __shared__ float lds_o[KW][16][LDO];
    __shared__ float lds_ml[KW][16][2];
    __shared__ int lds_last;
    const KvPlanView &v = p.v;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), kw = wave % KW, cw = wave / KW, n = lane & 15, g = lane >> 4;
    Work k;
    if (!k.find(p, ROWS)) return;
    const KvTile &t = k.t;
    const int wrow0 = t.row0 + cw * 16 * NT;
    const int n_cols = max(0, min(NT, (k.row_end - wrow0 + 15) >> 4));
    Columns<D, NT, Y32> w;
    int lo[NT], hi[NT];
    w.begin(p.a, k, wrow0, v.group, v.n_kv, lo, hi, lane);
    const float c = p.a.scale * LOG2E;
    const Records recs(p.a, k);
    const int b1 = k.b1, first_b = k.b0 + kw;
    if (first_b < b1 && n_cols > 0) {
        Record<D> r0, r1;
        const Places<D> at(lane);
        bool bad = false;
        // 64 records of the wave at a time, whose pages lie one to a lane: a read of the table among the loads below would have to wait for
        // every load that is on its way ahead of it.
        for (int c0 = first_b; c0 < b1; c0 += 64 * KW) {
            const int pages = recs.table[min(c0 + lane * KW, b1 - 1) >> recs.log_blocks];
            // Starts the loads of record b, the i-th of the 64; whether its page exists.
            auto start = [&](Record<D> &r, int i, int b) {
                bool ok;
                load_record<D>(r, recs.at(min(b, b1 - 1), __builtin_amdgcn_readlane(pages, i), ok), at);
                bad |= !ok;
                return ok;
            };
            auto take = [&](Record<D> &r, int b, bool ok) {
                if (ok) w.step(r, n_cols, c, b * 64, !k.whole(b), lo, hi, t.kv_len, lane);
            };
            const int count = min(64, (b1 - c0 + KW - 1) / KW);
            bool ok0 = start(r0, 0, c0), ok1;
            for (int i = 0, b = c0;;) {
                ok1 = start(r1, min(i + 1, count - 1), b + KW);
                take(r0, b, ok0);
                b += KW;
                if (++i >= count) break;
                ok0 = start(r0, min(i + 1, count - 1), b + KW);
                take(r1, b, ok1);
                b += KW;
                if (++i >= count) break;
            }
        }
        if (bad && lane == 0) atomicOr(p.a.err_word, ERR_BAD_PAGE);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) w.l[nt] = sum4(w.l[nt]);

    float *part_o = p.a.partial + (((int64_t)(t.pslot + t.part) * v.n_kv + k.h) * KV_FEW_ROWS) * (D + 2);
    const bool alone = t.n_parts == 1;
    const int row = tid >> 4, ch = (tid & 15) * CH;
    for (int ct = 0; ct < CW * NT; ++ct) {
        if (ct * 16 >= k.row_end - t.row0) break;
        if (ct) __syncthreads();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
            if (cw * NT + nt == ct) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int j = 0; j < D / 16; ++j)
                        lds_o[kw][n][o_channel<D>(g * 4 + e) + (D == 256 ? (j >> 3) * 128 + (j & 7) : j)] = w.o[nt][j][e];
                if (g == 0) {
                    lds_ml[kw][n][0] = w.m[nt];
                    lds_ml[kw][n][1] = w.l[nt];
                }
            }
        __syncthreads();
        float m = NEG_INF, l = 0.f, x[CH];
#pragma unroll
        for (int u = 0; u < KW; ++u) m = fmaxf(m, lds_ml[u][row][0]);
#pragma unroll
        for (int i = 0; i < CH; ++i) x[i] = 0.f;
        const float base = m == NEG_INF ? 0.f : m * c;
#pragma unroll
        for (int u = 0; u < KW; ++u) {
            const float f = __builtin_amdgcn_exp2f(fmaf(lds_ml[u][row][0], c, -base));
            l = fmaf(lds_ml[u][row][1], f, l);
#pragma unroll
            for (int i = 0; i < CH; ++i) x[i] = fmaf(lds_o[u][row][ch + i], f, x[i]);
        }
        const int r = t.row0 + ct * 16 + row;
        if (r >= k.row_end) continue;
        if (alone) {
            const float inv = inverse(l);
#pragma unroll
            for (int i = 0; i < CH; ++i) x[i] *= inv;
            const int64_t y = y_row(t, r, v.group, v.n_kv, k.h);
            store_y(p.a, y, D, ch, x);
            if (p.a.lse && ch == 0) p.a.lse[y] = log_sum(m, l, c);
        } else {
            float *o = part_o + (ct * 16 + row) * (D + 2);
#pragma unroll
            for (int i = 0; i < CH; i += 2) put_agent(o + 2 + ch + i, x[i], x[i + 1]);
            if (ch == 0) put_agent(o, m, l);
        }
    }
    if (alone) return;
    const Groups of(t);
    if (!last_of(v, k, 1 + of.first / of.size, of.last - of.first, &lds_last)) return;
    join_rows<D, ROWS>(p, k, c, of.first, of.last, 1, of.size == t.n_parts);
    if (of.size < t.n_parts && last_of(v, k, 0, (t.n_parts + of.size - 1) / of.size, &lds_last))
        join_rows<D, ROWS>(p, k, c, 0, t.n_parts, of.size, true);
}

// Tiles of many rows: every one of the four waves has 32 rows and walks all of the records, a quarter of which it decodes into LDS for
// all, one record ahead.
template <int D, bool Y32>
__global__ __launch_bounds__(256, (D == 256 ? 1 : 2)) void attend_tile_kernel(AttendK p)
{
    using Wave = Columns<D, 2, Y32>;
    constexpr int KD = Wave::KD, SB = Wave::SB, NJ = Wave::NJ, FRAGS = 4 * KD + 2 * NJ;
    constexpr int MINE = NJ / 4;   // pairs of accumulators of each half whose V operands a wave decodes
    struct Operands {
        uint4 k[4][KD][64], v[2][NJ][64];
    };
    static_assert(sizeof(Operands) == FRAGS * 1024, "");
    __shared__ Operands ops[2];
    __shared__ int lds_last;
    const KvPlanView &v = p.v;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), n = lane & 15, g = lane >> 4;
    Work k;
    if (!k.find(p, KV_TILE_ROWS)) return;
    const KvTile &t = k.t;
    const int wrow0 = t.row0 + wave * 32;
    Wave w;
    int lo[2], hi[2];
    w.begin(p.a, k, wrow0, v.group, v.n_kv, lo, hi, lane);
    const float c = p.a.scale * LOG2E;
    const Records recs(p.a, k);
    const int b1 = k.b1;
    if (k.b0 < b1) {
        const Places<D> at(lane);
        // This wave's share of a record: keys 16 wave .. + 15; of the values those of half wave / 2, MINE pairs of accumulators from u0 on.
        const int half = wave >> 1, u0 = (wave & 1) * MINE;
        uint32_t kc[KD], ks[SB];
        uint4 vc[2], vs[SB];
        auto start = [&](const char *rec) {
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
        };
        auto decode = [&](Operands &o, int b, bool ok) {   // ok: else it is some other record, of which nothing is used
            if (ok && !k.whole(b)) w.mask_values(vs, 2, b * 64, lo, hi, t.kv_len, lane);
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
        };
        bool bad = false;
        for (int c0 = k.b0; c0 < b1; c0 += 64) {   // (64 pages at a time, one to a lane, as above)
            const int pages = recs.table[min(c0 + lane, b1 - 1) >> recs.log_blocks];
            const int count = min(64, b1 - c0);
            bool ok, next_ok = false;
            start(recs.at(c0, __builtin_amdgcn_readlane(pages, 0), ok));
            decode(ops[0], c0, ok);
            for (int i = 0; i < count; ++i) {
                const int b = c0 + i;
                const bool more = i + 1 < count;
                // (without a condition: loads under one are waited for where it ends)
                start(recs.at(more ? b + 1 : b, __builtin_amdgcn_readlane(pages, more ? i + 1 : i), next_ok));
                // Record b is whole in LDS; nobody reads the other half any more.
                lds_barrier();
                const Operands &o = ops[i & 1];
                if (ok) {
                    const bool masked = !k.whole(b);
                    typename Wave::Scores s;
#pragma unroll
                    for (int tile = 0; tile < 4; ++tile) {
                        bf16x8_t x[KD];
#pragma unroll
                        for (int j = 0; j < KD; ++j) x[j] = __builtin_bit_cast(bf16x8_t, o.k[tile][j][lane]);
                        w.score(x, s, tile, 2);
                    }
                    typename Wave::Weights x;
                    w.weigh(s, x, 2, c, b * 64, masked, lo, hi, lane);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int u = 0; u < NJ / 2; ++u)
                            w.add(x, h, u, __builtin_bit_cast(bf16x8_t, o.v[h][2 * u][lane]), __builtin_bit_cast(bf16x8_t, o.v[h][2 * u + 1][lane]), 2);
                }
                bad |= !ok;
                if (more) decode(ops[(i + 1) & 1], b + 1, next_ok);
                ok = next_ok;
            }
        }
        if (bad && tid == 0) atomicOr(p.a.err_word, ERR_BAD_PAGE);
    }
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) w.l[nt] = sum4(w.l[nt]);
    if (t.n_parts > 1) {
        // A part's results lie as the lanes have them: whole lines, and the join needs no order of rows.
        const int64_t part_step = (int64_t)v.n_kv * KV_TILE_ROWS * (D + 2);
        float *first_part = p.a.partial + ((int64_t)t.pslot * v.n_kv * KV_FEW_ROWS + k.h * KV_TILE_ROWS) * (D + 2);
        const int ml_at = KV_TILE_ROWS * D + (wave * 32 + n) * 2, o_at = (wave * 4 * NJ * 64 + lane) * 2;
        auto leave = [&](int part) {
            float *mine = first_part + part * part_step;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
                if (g == 0) put_agent(mine + ml_at + nt * 32, w.m[nt], w.l[nt]);
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        put_agent(mine + o_at + ((nt * NJ + j) * 2 + e) * 128, w.o[nt][j][2 * e], w.o[nt][j][2 * e + 1]);
            }
        };
        auto join = [&](int from, int to, int step) {
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
                w.m[nt] = NEG_INF;
                w.l[nt] = 0.f;
#pragma unroll
                for (int j = 0; j < NJ; ++j) w.o[nt][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
            for (int u = from; u < to; u += step) {
                const float *part = first_part + u * part_step;
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) {
                    const float2 ml = get_agent(part + ml_at + nt * 32);
                    float2 x[NJ][2];
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e) x[j][e] = get_agent(part + o_at + ((nt * NJ + j) * 2 + e) * 128);
                    const float top = fmaxf(w.m[nt], ml.x), base = top == NEG_INF ? 0.f : top * c;
                    const float f0 = __builtin_amdgcn_exp2f(fmaf(w.m[nt], c, -base)), f1 = __builtin_amdgcn_exp2f(fmaf(ml.x, c, -base));
                    w.m[nt] = top;
                    w.l[nt] = fmaf(ml.y, f1, w.l[nt] * f0);
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            w.o[nt][j][2 * e] = fmaf(x[j][e].x, f1, w.o[nt][j][2 * e] * f0);
                            w.o[nt][j][2 * e + 1] = fmaf(x[j][e].y, f1, w.o[nt][j][2 * e + 1] * f0);
                        }
                }
            }
        };
        const Groups of(t);
        leave(t.part);
        if (!last_of(v, k, 1 + of.first / of.size, of.last - of.first, &lds_last)) return;
        join(of.first, of.last, 1);
        if (of.size < t.n_parts) {
            leave(of.first);
            if (!last_of(v, k, 0, (t.n_parts + of.size - 1) / of.size, &lds_last)) return;
            join(0, t.n_parts, of.size);
        }
    }
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
        const int r = wrow0 + nt * 16 + n;
        if (r >= k.row_end) continue;
        const float inv = inverse(w.l[nt]);
        const int64_t y = y_row(t, r, v.group, v.n_kv, k.h);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (int b = 0; b < SB; ++b) {
                constexpr int N = D == 64 ? 4 : 8;
                float x[N];
#pragma unroll
                for (int j = 0; j < N; ++j) x[j] = w.o[nt][b * 8 + j][e] * inv;
                store_y(p.a, y, D, o_channel<D>(g * 4 + e) + b * 128, x);
            }
        }
        if (g == 0 && p.a.lse) p.a.lse[y] = log_sum(w.m[nt], w.l[nt], c);
    }
}

template <int D, int NT, int CW, int KW, bool Y32>
void launch_few(const AttendK &p, hipStream_t stream)
{
    hipLaunchKernelGGL((attend_few_kernel<D, NT, CW, KW, Y32>), dim3((unsigned)p.v.max_few * p.v.n_kv), dim3(256), 0, stream, p);
}

template <int D, bool Y32>
hipError_t launch_d(const KvPlanView &v, const AttendArgs &a, hipStream_t stream)
{
    constexpr bool WIDE = D == 256;   // two columns of accumulators would leave no registers for the rest
    AttendK p{v, a, 0};
    if (v.has_few) {
        if (std::min(v.max_new * (int64_t)v.group, (int64_t)KV_FEW_ROWS) <= 16) launch_few<D, 1, 1, 4, Y32>(p, stream);
        else launch_few<D, WIDE ? 1 : 2, WIDE ? 2 : 1, WIDE ? 2 : 4, Y32>(p, stream);
    }
    if (v.has_tile) {
        p.list = 1;
        hipLaunchKernelGGL((attend_tile_kernel<D, Y32>), dim3((unsigned)v.max_tile * v.n_kv), dim3(256), 0, stream, p);
    }
    return hipGetLastError();
}

}  // namespace

int64_t attend_partial_floats(const KvPlanView &v, int pslots, int D)
{
    return (int64_t)pslots * v.n_kv * KV_FEW_ROWS * (D + 2);
}

hipError_t launch_attend(const KvPlanView &v, const AttendArgs &a, hipStream_t stream)
{
    switch (a.pages.D) {
    case 64: return a.y_f32 ? launch_d<64, true>(v, a, stream) : launch_d<64, false>(v, a, stream);
    case 128: return a.y_f32 ? launch_d<128, true>(v, a, stream) : launch_d<128, false>(v, a, stream);
    case 256: return a.y_f32 ? launch_d<256, true>(v, a, stream) : launch_d<256, false>(v, a, stream);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace moin

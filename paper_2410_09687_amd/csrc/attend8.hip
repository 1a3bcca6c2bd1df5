// Attention of a step's tokens over the paged E4M3 cache: the kernels of attend_core.h on records whose keys and values have one
// power of two each for 64 tokens of a head (kv8.h).
//
// Both products are taken transposed, as on the 4-bit cache.  The records are laid out so that what a lane loads is what
// it feeds the matrix cores, one conversion for two values and nothing else:
//   K: lane (m, g) takes key m of a tile of 16, channels 64 l + 16 g .. + 15: 16 bytes, two operands of eight channels;
//   V: channel 16 j + m of the 16 keys 16 w + 4 g + e (w, e < 4): 16 bytes, of which eight are the lane's half of an
//      operand of 32 keys, in the order in which the scores' accumulators hold their keys.
// E4M3 becomes bf16 exactly, the block's scale in the same instruction.  (E4M3 rather than integers: channels of keys are of uneven strength, and a
// scale for 64 tokens and all channels leaves an integer's small channels few steps; and the card converts two of them an instruction.)
//
// Tiles of few rows are bound by memory, 128 D bytes a record and kv head: 256 requests of up to 4096 keys, 32 heads on 4 of 64 channels, 50 us, 5.4 TB/s (a
// long contiguous read reaches 6.8, a copy 5.0 there and back); two of 100000 and more, 64 heads on 8 of 128, 104 us, 4.6 TB/s: beginning, last records and joins take
// a time that does not go with the keys (64 requests of 32 heads on 4 of 64: 8 us for one token, 12 for four, and 6.2 TB/s beside them); four times as many keys take 3.3 times as long.  A thousand keys: 7.4 us, half a dozen trips to memory.  Registers for four waves of a SIMD instead of three
// (64 channels) spill: 96 us for the first.
// Tiles of many rows are bound by the vector unit, as on the 4-bit cache: eight prompts of 2048, 32 heads on 4 of 64 channels, 177 - 185 us, 0.74 - 0.78 PFLOP/s; 198
// vector instructions beside 32 of the matrix cores a wave and record by the counters, some 160 of them on the steady path (the softmax of 32 scores 104, packs 18, decoding
// 18), the unit busy 73 % of the cycles in which a compute unit has work, the matrix cores 35 %.  Four waves of a SIMD instead of three change
// nothing (204, 212 us), nor does a higher priority for the decoding or the products (191 - 196).
#include "attend_core.h"
#include "kv8.h"

namespace moin {

namespace {

// Four E4M3 to two words of bf16.
__device__ __forceinline__ uint32_t e4m3_low(uint32_t w, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
}
__device__ __forceinline__ uint32_t e4m3_high(uint32_t w, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
}
__device__ __forceinline__ bf16x8_t e4m3_operand(uint32_t a, uint32_t b, float scale)
{
    return operand(e4m3_low(a, scale), e4m3_high(a, scale), e4m3_low(b, scale), e4m3_high(b, scale));
}

// Records of tiles of few rows are read once: past the caches.  (256 requests of up to 4096 keys 53.9 us, 50.6 like this; two of 100000 and more 112, 104.)
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_once(const char *p)
{
    return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p)));
}

template <int D_>
struct E4M3 {
    static constexpr int D = D_, NJ = D / 16, KD = D / 32, KL = D / 64;

    struct Source {
        const char *rec, *scales;
    };
    __device__ __forceinline__ static int record_bytes(int d) { return kv8_record_bytes(d); }
    __device__ __forceinline__ static int64_t page_bytes(const KvPages &p) { return kv8_page_bytes(p); }
    __device__ __forceinline__ static const char *tail(const KvPages &p, int h) { return p.data + kv8_scales_at(p, h, 0); }
    __device__ __forceinline__ static Source source(const char *rec, const char *tail, int blk) { return Source{rec, tail + blk * 2}; }

    // Waves per SIMD that the registers are to leave room for.
    template <int NT>
    static constexpr int min_waves()
    {
        return NT > 1 ? (D == 64 ? 2 : 1) : D == 64 ? 3 : D == 128 ? 2 : 1;
    }

    struct Record {
        uint4 k[4][KL], v[NJ];
        uint32_t scales;   // the keys' byte, the values'
    };
    struct Places {
        uint32_t k, v;
        __device__ __forceinline__ explicit Places(int lane) : k((lane & 15) * 64 + (lane >> 4) * 16), v(64 * D + k) {}
    };
    __device__ __forceinline__ static void load(Record &r, const Source &s, const Places &at)
    {
        r.scales = *reinterpret_cast<const uint16_t *>(s.scales);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int l = 0; l < KL; ++l) r.k[i][l] = load_once(s.rec + (at.k + (i * KL + l) * 1024));
#pragma unroll
        for (int j = 0; j < NJ; ++j) r.v[j] = load_once(s.rec + (at.v + j * 1024));
    }

    __device__ __forceinline__ static int k_channel(int j, int g) { return (j >> 1) * 64 + g * 16 + (j & 1) * 8; }
    __device__ __forceinline__ static int o_channel(int m, int j) { return j * 16 + m; }
    __device__ __forceinline__ static float k_scale(uint32_t scales) { return bits_f32((scales & 255u) << 23); }
    __device__ __forceinline__ static float v_scale(uint32_t scales) { return bits_f32((scales >> 8 & 255u) << 23); }

    __device__ __forceinline__ static bf16x8_t k_operand(const uint4 &k, int u, float scale)
    {
        return u ? e4m3_operand(k.z, k.w, scale) : e4m3_operand(k.x, k.y, scale);
    }
    __device__ __forceinline__ static bf16x8_t k_operand(const Record &r, int i, int j) { return k_operand(r.k[i][j >> 1], j & 1, k_scale(r.scales)); }
    __device__ __forceinline__ static void v_operands(const Record &r, int h, int u, int, bf16x8_t &even, bf16x8_t &odd)
    {
        even = k_operand(r.v[2 * u], h, v_scale(r.scales));
        odd = k_operand(r.v[2 * u + 1], h, v_scale(r.scales));
    }

    // What lies beyond the request's keys may hold anything, NaN among it, and 0 times that is not 0 in the product: it becomes 0.  A block whose
    // scale stands for NaN gives NaN in every channel to the rows that see a key of it, and nothing to the others.
    template <int NT, int N>
    __device__ __forceinline__ static void mask_values(uint4 (&v)[N], uint32_t scales, f32x4_t (&o)[NT][NJ], int n_cols, int tok, const int *lo,
                                                       const int *hi, int end, int lane)
    {
        const bool nan = uniform((int)(scales >> 8 & 255u)) == 255;
        if (tok + 64 <= end && !nan) return;
        uint32_t keep[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int left = end - tok - 16 * w - 4 * (lane >> 4);   // keys from this word's first on
            keep[w] = nan || left <= 0 ? 0u : left >= 4 ? ~0u : (1u << 8 * left) - 1;
        }
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = make_uint4(v[j].x & keep[0], v[j].y & keep[1], v[j].z & keep[2], v[j].w & keep[3]);
        if (!nan) return;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (nt > 0 && nt >= n_cols) continue;
            if (max(lo[nt], tok) < min(hi[nt], min(tok + 64, end)))
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[nt][j][e] = bits_f32(0x7FC00000u);
        }
    }
    // (a zero times a scale that stands for NaN)
    __device__ __forceinline__ static uint32_t finite_values(uint32_t scales) { return scales >> 8 == 255u ? scales & 0x7FFFu : scales; }
    template <int NT>
    __device__ __forceinline__ static void mask(Record &r, f32x4_t (&o)[NT][NJ], int n_cols, int tok, const int *lo, const int *hi, int end, int lane)
    {
        mask_values<NT>(r.v, r.scales, o, n_cols, tok, lo, hi, end, lane);
        r.scales = finite_values(r.scales);
    }

    struct Operands {
        uint4 k[4][KD][64], v[2][NJ][64];
    };
    // Keys 16 wave .. + 15, and the channels of a quarter of the accumulators.
    struct Share {
        static constexpr int MINE = NJ / 4;
        const Places at;
        const int lane, wave;
        uint4 kc[KL], vc[MINE];
        uint32_t scales;
        __device__ __forceinline__ Share(int lane, int wave) : at(lane), lane(lane), wave(wave) {}
        __device__ __forceinline__ void load(const Source &s)
        {
            scales = *reinterpret_cast<const uint16_t *>(s.scales);
#pragma unroll
            for (int l = 0; l < KL; ++l) kc[l] = *reinterpret_cast<const uint4 *>(s.rec + (at.k + (wave * KL + l) * 1024));
#pragma unroll
            for (int j = 0; j < MINE; ++j) vc[j] = *reinterpret_cast<const uint4 *>(s.rec + (at.v + (wave * MINE + j) * 1024));
        }
        template <int NT>
        __device__ __forceinline__ void mask(f32x4_t (&o)[NT][NJ], int n_cols, int tok, const int *lo, const int *hi, int end)
        {
            mask_values<NT>(vc, scales, o, n_cols, tok, lo, hi, end, lane);
            scales = finite_values(scales);
        }
        __device__ __forceinline__ void decode(Operands &o) const
        {
#pragma unroll
            for (int j = 0; j < KD; ++j) o.k[wave][j][lane] = __builtin_bit_cast(uint4, k_operand(kc[j >> 1], j & 1, k_scale(scales)));
#pragma unroll
            for (int j = 0; j < MINE; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) o.v[h][wave * MINE + j][lane] = __builtin_bit_cast(uint4, k_operand(vc[j], h, v_scale(scales)));
        }
    };

    __device__ __forceinline__ static void store(const AttendArgs &a, int64_t y, const f32x4_t (&o)[NJ], float inv, int g)
    {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const float x[4] = {o[j][0] * inv, o[j][1] * inv, o[j][2] * inv, o[j][3] * inv};
            store_y(a, y, D, j * 16 + g * 4, x);
        }
    }
};

}  // namespace

hipError_t launch_attend8(const KvPlanView &v, const AttendArgs &a, hipStream_t stream)
{
    switch (a.pages.D) {
    case 64: return a.y_f32 ? launch_d<E4M3<64>, true>(v, a, stream) : launch_d<E4M3<64>, false>(v, a, stream);
    case 128: return a.y_f32 ? launch_d<E4M3<128>, true>(v, a, stream) : launch_d<E4M3<128>, false>(v, a, stream);
    case 256: return a.y_f32 ? launch_d<E4M3<256>, true>(v, a, stream) : launch_d<E4M3<256>, false>(v, a, stream);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace moin

// Tokens into the paged E4M3 cache, and back.  A block of 64 tokens of a head has one power of two 2^(E - 127) for its keys and one for its
// values: the smallest in whose units its largest magnitude is below 464, which rounds to E4M3's largest value, 448.  A step's tokens find
// blocks that earlier ones have begun: E is then the larger one of the block's and what the new tokens ask for, and where
// it grows, what the block holds is rounded again -- a shift of the exponent, exact but for values that become subnormal.
//
// So the block, not the token, is what a workgroup takes: it alone reads and writes its codes of one head's keys or values.  Bound by memory: 65536 tokens of
// eight heads of 128 97 us, 4.2 TB/s, and back 81 - 96, 4.2 - 5.0 TB/s (a copy of 1 GiB 5.0); 256 single tokens of four heads of 64 6.2 us, a chain of
// four trips to memory; where each of them makes the scales of its block of 41 grow, 8.2 us, and of eight heads of 128 20.9 instead of 11.7: a trip more, and the block's codes
// there and back.  (65536 tokens behind 40 of each of 32 requests: 97 instead of 94.)
#include <algorithm>
#include <type_traits>

#include "gemm_core.h"
#include "kv8.h"

namespace moin {

namespace {

__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// The bf16 side of a copy passes through once: past L2, which holds the lines of the cache until they are whole.
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_once(const char *p)
{
    return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p)));
}
__device__ __forceinline__ void store_once(char *p, const uint4 &v)
{
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), reinterpret_cast<u32x4_t *>(p));
}

constexpr uint32_t KV8_MIN_E = 10, KV8_MAX_E = 246, KV8_NAN = 255;

// E of values whose largest magnitude has these fp32 bits.  At least 10: the smallest code, 2^-9 units, is then a normal number of bf16.  At
// most 246: so is the largest, 448 units (what is beyond them, 2.98e38, becomes 448 units).  255, which stands for NaN,
// where a value is infinite or NaN.
__device__ __forceinline__ uint32_t kv8_scale_byte(uint32_t amax)
{
    const int e = (int)((amax + 0x180000u) >> 23) - 8;
    return amax >= 0x7F800000u ? KV8_NAN : (uint32_t)min(max(e, (int)KV8_MIN_E), (int)KV8_MAX_E);
}
__device__ __forceinline__ uint32_t bf16x8_amax(const uint4 &v)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = word(v, i);
        m = max(m, max((w << 16) & 0x7FFF0000u, w & 0x7FFF0000u));
    }
    return m;
}
__device__ __forceinline__ float in_range(float x) { return fminf(fmaxf(x, -448.f), 448.f); }
// Four values of units to codes, the first in the lowest byte; nearest, ties to even.
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(in_range(a), in_range(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(in_range(c), in_range(d), w, true);
}
// Four codes in units `shrink` times as large.
__device__ __forceinline__ uint32_t recode(uint32_t w, float shrink)
{
    const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return encode4(lo[0] * shrink, lo[1] * shrink, hi[0] * shrink, hi[1] * shrink);
}

// Which of a request's blocks a workgroup serves.  Places 0 to S - 1 are the first blocks of the requests, without a search: all there is of a
// step of single tokens.  Behind them request s owns the places R(s) to R(s + 1), R(s) = seq_offsets[s] / 64 + s, at least as many
// as the further blocks that its tokens can touch; all lanes of the wave look for theirs, 64 ways at a time.
__device__ __forceinline__ int request_at(const int *seq_offsets, int S, int id)
{
    int lo = 0, hi = S;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) >> 6, s = lo + (int)(threadIdx.x & 63) * step;
        const bool before = s < hi && (seq_offsets[min(s, S)] >> 6) + s <= id;
        const int count = max(1, (int)__popcll(__ballot(before)));   // (1: offsets that run backwards)
        lo += (count - 1) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

// NT threads take a block's keys (of an even place) or values of one head.  Registers hold the new tokens between the search for their largest magnitude and
// the conversion.
template <int D, int NT>
__global__ __launch_bounds__(NT) void kv8_append_kernel(unsigned place0, KvPages p, const char *__restrict__ k, const char *__restrict__ v, int64_t k_stride,
                                                        int64_t v_stride, int T, const int *__restrict__ seq_offsets, int S,
                                                        const int *__restrict__ slots, int *err_word)
{
    __shared__ uint32_t lds_amax[NT / 64];
    const int tid = threadIdx.x, lane = tid & 63;
    const unsigned place = place0 + blockIdx.x;
    const bool is_v = place & 1;
    const int h = (int)((place >> 1) % (unsigned)p.n_kv), id = (int)((place >> 1) / (unsigned)p.n_kv);
    const int s = id < S ? id : uniform(request_at(seq_offsets, S, id - S));
    const int tok0 = uniform(seq_offsets[s]), n_all = uniform(seq_offsets[s + 1]) - tok0, r = id < S ? 0 : id - S - ((tok0 >> 6) + s) + 1;
    if (tok0 < 0 || n_all < 0 || n_all > T - tok0) {
        if (tid == 0) atomicOr(err_word, ERR_BAD_LENGTHS);
        return;
    }
    if (n_all == 0 || r < 0 || (id >= S && r == 0)) return;
    // (a request's first block: its slots and the first of them in one trip to memory)
    const int log_page = p.log_blocks + 6, ahead = slots[tok0 + (id < S ? min(lane, n_all - 1) : 0)], slot0 = uniform(ahead);
    if (slot0 < 0 || (slot0 >> log_page) >= p.n_pages) {   // a request that got no pages, or one that is given others' than there are
        if (slot0 != -1 && tid == 0) atomicOr(err_word, ERR_BAD_PAGE);
        return;
    }
    const int first = max(0, 64 * r - (slot0 & 63)), n = min(n_all, 64 * (r + 1) - (slot0 & 63)) - first;   // its tokens in this block
    if (n <= 0) return;
    const int slot = id < S ? __shfl(ahead, min(lane, n - 1)) : slots[tok0 + first + min(lane, n - 1)], start = uniform(slot);
    const bool wrong = start < 0 || (start >> log_page) >= p.n_pages || (start & 63) + n > 64;
    if (wrong || __ballot(slot != start + min(lane, n - 1))) {   // a page that there is not, or tokens that do not follow each other
        if (tid == 0) atomicOr(err_word, ERR_BAD_PAGE);
        return;
    }
    const int p0 = start & 63, p1 = p0 + n, in_page = start & ((1 << log_page) - 1);
    char *page = p.data + (int64_t)(start >> log_page) * kv8_page_bytes(p);
    char *rec = page + ((int64_t)((h << p.log_blocks) + (in_page >> 6))) * kv8_record_bytes(D);
    uint8_t *scale = reinterpret_cast<uint8_t *>(page + kv8_scales_at(p, h, in_page >> 6) + (is_v ? 1 : 0));
    const uint32_t E0 = p0 > 0 ? *scale : 0u;   // (a block that begins here: whatever its place held before does not count)
    // row of the block's token 0: 64 tokens at most before the batch's first, of which nothing is read
    const char *rows = (is_v ? v : k) + (int64_t)h * D * 2 + (int64_t)(tok0 + first - p0) * (is_v ? v_stride : k_stride) * 2;
    const int64_t stride = (is_v ? v_stride : k_stride) * 2;

    constexpr int KC = 64 * D / 8 / NT, VC = (16 * D / 8 + NT - 1) / NT;   // chunks of a thread: a token's 8 channels; 4 tokens' 8 channels
    // chunks of values: a wave's lanes are 8 quads of tokens x 8 groups of channels, 128 bytes of a row and half a channel's run
    auto quad_of = [](int chunk) { return (chunk & 7) + (chunk >> 6 & 1) * 8; };
    auto group_of = [](int chunk) { return (chunk >> 3 & 7) + (chunk >> 7) * 8; };
    uint4 x[KC > 4 * VC ? KC : 4 * VC];
    uint32_t amax = 0;
    if (is_v) {
#pragma unroll
        for (int u = 0; u < VC; ++u) {
            const int chunk = u * NT + tid, t4 = quad_of(chunk) * 4, c = group_of(chunk) * 8;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool is = c < D && t4 + e >= p0 && t4 + e < p1;
                x[4 * u + e] = is ? load_once(rows + (t4 + e) * stride + c * 2) : make_uint4(0, 0, 0, 0);
                amax = max(amax, bf16x8_amax(x[4 * u + e]));
            }
        }
    } else {
#pragma unroll
        for (int u = 0; u < KC; ++u) {
            const int chunk = u * NT + tid, t = chunk / (D / 8), c = chunk % (D / 8) * 8;
            x[u] = t >= p0 && t < p1 ? load_once(rows + t * stride + c * 2) : make_uint4(0, 0, 0, 0);
            amax = max(amax, bf16x8_amax(x[u]));
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, d));
    if constexpr (NT > 64) {
        if (lane == 0) lds_amax[tid >> 6] = amax;
        __syncthreads();   // (every wave has read E0, too, before it changes)
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) amax = max(amax, lds_amax[w]);
    }
    const uint32_t E1 = kv8_scale_byte(amax), E = max(E0, E1);
    const bool grows = E0 != 0 && E > E0;
    const float inv = bits_f32(E <= KV8_MAX_E ? (254u - E) << 23 : 0x3F800000u);
    const float shrink = grows && E - E0 < 127u ? bits_f32((127u - (E - E0)) << 23) : 0.f;
    if (tid == 0 && E != E0) *scale = (uint8_t)E;
    auto at = [&](const uint4 &q, int i) { return bits_f32(i & 1 ? word(q, i >> 1) & 0xFFFF0000u : word(q, i >> 1) << 16) * inv; };
    if (is_v) {
#pragma unroll
        for (int u = 0; u < VC; ++u) {
            const int chunk = u * NT + tid, quad = quad_of(chunk), t4 = quad * 4, c = group_of(chunk) * 8;
            if (c >= D || t4 >= p1 || (t4 + 4 <= p0 && !grows)) continue;
            uint32_t is_new = 0, is_old = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (t4 + e >= p0 && t4 + e < p1) is_new |= 255u << 8 * e;
                if (t4 + e < p0) is_old |= 255u << 8 * e;
            }
            char *dst = rec + 64 * D + (c >> 4) * 1024 + (c & 8) * 64 + (quad & 3) * 16 + (quad >> 2) * 4;
            uint32_t codes[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) codes[i] = encode4(at(x[4 * u], i), at(x[4 * u + 1], i), at(x[4 * u + 2], i), at(x[4 * u + 3], i));
            if (is_new == ~0u) {
#pragma unroll
                for (int i = 0; i < 8; ++i) *reinterpret_cast<uint32_t *>(dst + i * 64) = codes[i];
            } else if (grows && is_old) {
                uint32_t was[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) was[i] = *reinterpret_cast<const uint32_t *>(dst + i * 64);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    *reinterpret_cast<uint32_t *>(dst + i * 64) = (codes[i] & is_new) | (recode(was[i], shrink) & is_old) | (was[i] & ~(is_new | is_old));
            } else {   // what lies beside the new tokens in their words stays: bytes, no trip to memory for the words
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (is_new >> 8 * e & 255)
#pragma unroll
                        for (int i = 0; i < 8; ++i) dst[i * 64 + e] = (char)(codes[i] >> 8 * e);
            }
        }
    } else {
#pragma unroll
        for (int u = 0; u < KC; ++u) {
            const int chunk = u * NT + tid, t = chunk / (D / 8), c = chunk % (D / 8) * 8;
            if (t >= p1 || (t < p0 && !grows)) continue;
            uint2 *dst = reinterpret_cast<uint2 *>(rec + (t >> 4) * 16 * D + (c >> 6) * 1024 + (t & 15) * 64 + (c & 63));
            if (t < p0) {
                const uint2 w = *dst;
                *dst = make_uint2(recode(w.x, shrink), recode(w.y, shrink));
            } else {
                *dst = make_uint2(encode4(at(x[u], 0), at(x[u], 1), at(x[u], 2), at(x[u], 3)), encode4(at(x[u], 4), at(x[u], 5), at(x[u], 6), at(x[u], 7)));
            }
        }
    }
}

// 64 tokens of the batch, one head's keys (blockIdx.x even) or values.  (Values a byte at a time, lanes as tokens: 219 us instead of 101 for 65536 tokens; each quad reading its slots itself: a trip
// to memory more, 101 and 9.2 instead of 96 and 7.6 for the begun blocks of 256 requests.)
template <int D>
__global__ __launch_bounds__(256) void kv8_gather_kernel(KvPages p, char *__restrict__ k, char *__restrict__ v, int64_t T,
                                                         const int *__restrict__ slots, int *err_word)
{
    const int tid = threadIdx.x, log_page = p.log_blocks + 6;
    const bool is_v = blockIdx.x & 1;
    const int h = (int)((blockIdx.x >> 1) % (unsigned)p.n_kv);
    const int64_t t0 = (int64_t)((blockIdx.x >> 1) / (unsigned)p.n_kv) * 64;
    auto place = [&](int slot, const char *&rec, int &tok, float &unit) {   // false: zeros
        const bool in = slot >= 0 && (slot >> log_page) < p.n_pages;
        if (!in && slot != -1) atomicOr(err_word, ERR_BAD_PAGE);
        const int at = in ? slot & ((1 << log_page) - 1) : 0;
        const char *page = p.data + (int64_t)(in ? slot >> log_page : 0) * kv8_page_bytes(p);
        rec = page + ((int64_t)((h << p.log_blocks) + (at >> 6))) * kv8_record_bytes(D);
        tok = at & 63;
        unit = bits_f32((uint32_t) * reinterpret_cast<const uint8_t *>(page + kv8_scales_at(p, h, at >> 6) + (is_v ? 1 : 0)) << 23);
        return in;
    };
    auto pair = [](uint32_t w, float unit, auto high) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, unit, decltype(high)::value));
    };
    using Low = std::integral_constant<bool, false>;
    using High = std::integral_constant<bool, true>;
    char *out = (is_v ? v : k) + (int64_t)h * D * 2;
    const int64_t row = (int64_t)p.n_kv * D * 2;
    if (is_v) {
        // Four tokens that lie in one word of every channel, eight channels: eight words, turned into the tokens' rows with v_perm.  The batch's tokens
        // need not begin where the cache's words do: the first and last quads are then cut off, and one more is needed.
        // A wave takes 8 quads x 8 groups of channels: 32 bytes of a channel's run, 128 of a token's row.
        const int lane = tid & 63, own = t0 + lane < T ? slots[t0 + lane] : -1;   // (the batch's 64 slots in one trip to memory)
        const int shift = max(uniform(own), 0) & 3;
        for (int b = tid >> 6; b < 3 * (D / 64); b += 4) {
            const int quad = b / (D / 64) * 8 + (lane & 7), c = (b % (D / 64) * 8 + (lane >> 3)) * 8;
            const int64_t first = t0 - shift + quad * 4;
            int slot[4];
            bool in[4];
            int from = -1, any = -1;
            bool one = true;   // the quad's tokens are neighbours in the cache, as a request's are
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t t = first + e;
                in[e] = t >= t0 && t < min(t0 + 64, T);
                slot[e] = __shfl(own, (quad * 4 - shift + e) & 63);
                if (in[e]) {
                    any = slot[e];
                    if (from < 0) from = slot[e] - e;
                    one &= slot[e] == from + e && slot[e] >= 0 && (slot[e] >> log_page) < p.n_pages;
                }
            }
            if (!(in[0] | in[1] | in[2] | in[3])) continue;
            uint4 y[4];
            if (one && (from & 3) == 0) {
                const char *rec;
                int tok;
                float unit;
                place(any, rec, tok, unit);   // (whichever: they share their words)
                const char *src = rec + 64 * D + ((tok >> 2) & 3) * 16 + (tok >> 4) * 4 + c * 64;
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const uint32_t *>(src + i * 64);
                auto rows4 = [&](const uint32_t *q, uint32_t (&o)[4]) {   // bytes [channel][token] to [token][channel]
                    const uint32_t a = __builtin_amdgcn_perm(q[1], q[0], 0x05010400u), b = __builtin_amdgcn_perm(q[3], q[2], 0x05010400u);
                    const uint32_t d = __builtin_amdgcn_perm(q[1], q[0], 0x07030602u), f = __builtin_amdgcn_perm(q[3], q[2], 0x07030602u);
                    o[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
                    o[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
                    o[2] = __builtin_amdgcn_perm(f, d, 0x05040100u);
                    o[3] = __builtin_amdgcn_perm(f, d, 0x07060302u);
                };
                uint32_t lo[4], hi[4];
                rows4(w, lo);
                rows4(w + 4, hi);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    y[e] = make_uint4(pair(lo[e], unit, Low{}), pair(lo[e], unit, High{}), pair(hi[e], unit, Low{}), pair(hi[e], unit, High{}));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[e] = make_uint4(0, 0, 0, 0);
                    const char *rec;
                    int tok;
                    float unit;
                    if (!in[e] || !place(slot[e], rec, tok, unit)) continue;
                    const uint8_t *src = reinterpret_cast<const uint8_t *>(rec) + 64 * D + ((tok >> 2) & 3) * 16 + (tok >> 4) * 4 + (tok & 3) + c * 64;
                    uint32_t b[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) b[i] = src[i * 64];
                    const uint32_t w0 = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24, w1 = b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24;
                    y[e] = make_uint4(pair(w0, unit, Low{}), pair(w0, unit, High{}), pair(w1, unit, Low{}), pair(w1, unit, High{}));
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (in[e]) store_once(out + (first + e) * row + c * 2, y[e]);
        }
    } else {
        constexpr int PER = D / 8;   // threads of a token
#pragma unroll
        for (int u = 0; u < 64 * PER / 256; ++u) {
            const int64_t t = t0 + (u * 256 + tid) / PER;
            if (t >= T) break;
            const int c = tid % PER * 8;
            const char *rec;
            int tok;
            float unit;
            const bool in = place(slots[t], rec, tok, unit);
            const uint2 w = *reinterpret_cast<const uint2 *>(rec + (tok >> 4) * 16 * D + (c >> 6) * 1024 + (tok & 15) * 64 + (c & 63));
            const uint4 y = make_uint4(pair(w.x, unit, Low{}), pair(w.x, unit, High{}), pair(w.y, unit, Low{}), pair(w.y, unit, High{}));
            store_once(out + t * row + c * 2, in ? y : make_uint4(0, 0, 0, 0));
        }
    }
}

constexpr int64_t AT_ONCE = 1 << 23;   // workgroups of a launch, whose threads number less than 2^32

template <int D>
hipError_t launch_append(const KvPages &p, const void *k, const void *v, int64_t k_stride, int64_t v_stride, int64_t T, const int *seq_offsets,
                         int S, const int *slots, int *err_word, hipStream_t stream)
{
    const int64_t places = T / 64 + 2 * (int64_t)S;
    auto go = [&](auto nt) {
        constexpr int NT = decltype(nt)::value;
        const int64_t all = places * 2 * p.n_kv;
        for (int64_t at = 0; at < all; at += AT_ONCE)
            hipLaunchKernelGGL((kv8_append_kernel<D, NT>), dim3((unsigned)std::min(all - at, AT_ONCE)), dim3(NT), 0, stream, (unsigned)at, p,
                               static_cast<const char *>(k), static_cast<const char *>(v), k_stride, v_stride, (int)T, seq_offsets, S, slots, err_word);
    };
    // (a token or a few to a request: a wave has room for them, and four would wait for each other)
    if (T <= 4 * (int64_t)S) go(std::integral_constant<int, 64>{});
    else go(std::integral_constant<int, 256>{});
    return hipGetLastError();
}

template <int D>
hipError_t launch_gather(const KvPages &p, void *k, void *v, int64_t T, const int *slots, int *err_word, hipStream_t stream)
{
    const int64_t row = (int64_t)p.n_kv * D * 2, most = std::max<int64_t>(1, AT_ONCE / (2 * p.n_kv)) * 64;
    for (int64_t t = 0; t < T; t += most)
        hipLaunchKernelGGL(kv8_gather_kernel<D>, dim3((unsigned)((std::min(T - t, most) + 63) / 64 * 2 * p.n_kv)), dim3(256), 0, stream, p,
                           static_cast<char *>(k) + t * row, static_cast<char *>(v) + t * row, std::min(T - t, most), slots + t, err_word);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv8_append(const KvPages &p, const void *k, const void *v, int64_t k_stride, int64_t v_stride, int64_t T,
                             const int *seq_offsets, int S, const int *slots, int *err_word, hipStream_t stream)
{
    auto go = [&](auto d) { return launch_append<decltype(d)::value>(p, k, v, k_stride, v_stride, T, seq_offsets, S, slots, err_word, stream); };
    return p.D == 64 ? go(std::integral_constant<int, 64>{}) : p.D == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 256>{});
}

hipError_t launch_kv8_gather(const KvPages &p, void *k, void *v, int64_t T, const int *slots, int *err_word, hipStream_t stream)
{
    auto go = [&](auto d) { return launch_gather<decltype(d)::value>(p, k, v, T, slots, err_word, stream); };
    return p.D == 64 ? go(std::integral_constant<int, 64>{}) : p.D == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 256>{});
}

}  // namespace moin

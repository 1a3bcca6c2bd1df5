// Attention over a paged cache, whatever the format of its records: the work of a workgroup, the softmax in one pass, the joins of
// parts, the two kernels.  attend.hip (MXFP4) and attend8.hip (E4M3) give the formats and say what bounds them.
//
// A format F<D> has
//   Record, Places      what a wave holds of a record of 64 tokens, and where a lane's pieces lie in it;
//   Source, source()    where a record is in memory; load();
//   k_channel(j, g)     the channel of a query that element 0 of K operand j holds for lanes of group g (eight follow);
//   o_channel(m, j)     the channel that is row m of accumulator j;
//   k_operand(), v_operands()   the operands of a record in registers;
//   mask()              values of a record that not every row sees;
//   Share               a wave's share of a record that four waves decode for each other;
//   store()             a row's results from the accumulators.
#pragma once
#include "gemm_core.h"
#include "kv.h"

namespace moin {

namespace {

constexpr float NEG_INF = -__builtin_huge_valf();

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
template <class F, int NT, bool Y32>
struct Columns {
    static constexpr int D = F::D, KD = D / 32, NJ = D / 16;
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
                const uint4 u = *reinterpret_cast<const uint4 *>(x + F::k_channel(j, g) * 2);
                q[nt][j] = __builtin_bit_cast(bf16x8_t, real ? u : make_uint4(0, 0, 0, 0));
            }
        }
    }

    // The weights enter the second product as bf16: their sum is taken in fp32 before, each rounding is at most 2^-9 of a weight, on its own, and the result
    // is rounded by as much (prompts of 2048: error of 0.00182 of the results' norm, 0.00172 with three parts, of which 0.0017 are the result's own
    // rounding).  fp32 results take three parts, 24 bits: eight such prompts 314 us over the 8-bit cache, 180 with one.
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
    __device__ __forceinline__ void step(typename F::Record &r, int n_cols, float c, int tok, bool masked, const int *lo, const int *hi, int end, int lane)
    {
        if (masked) F::template mask<NT>(r, o, n_cols, tok, lo, hi, end, lane);
        Scores s;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bf16x8_t k[KD];
#pragma unroll
            for (int j = 0; j < KD; ++j) k[j] = F::k_operand(r, i, j);
            score(k, s, i, n_cols);
        }
        Weights p;
        weigh(s, p, n_cols, c, tok, masked, lo, hi, lane);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int u = 0; u < NJ / 2; ++u) {
                bf16x8_t even, odd;
                F::v_operands(r, h, u, lane, even, odd);
                add(p, h, u, even, odd, n_cols);
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
template <class F>
struct Records {
    const int *table;
    const char *head, *tail;   // of page 0
    int64_t page_bytes;
    int log_blocks, n_pages, record;

    __device__ __forceinline__ Records(const AttendArgs &a, const Work &k)
        : table(a.block_table + (int64_t)k.t.req * a.max_pages),
          head(a.pages.data + (((int64_t)k.h * F::record_bytes(a.pages.D)) << a.pages.log_blocks)), tail(F::tail(a.pages, k.h)),
          page_bytes(F::page_bytes(a.pages)), log_blocks(a.pages.log_blocks), n_pages(a.pages.n_pages), record(F::record_bytes(a.pages.D))
    {
    }
    // Record b; `ok`: its page exists (else one of page 0).
    __device__ __forceinline__ typename F::Source at(int b, int page, bool &ok) const
    {
        ok = page >= 0 && page < n_pages;
        const int64_t at_page = (int64_t)(ok ? page : 0) * page_bytes;
        const int blk = b & ((1 << log_blocks) - 1);
        return F::source(head + at_page + blk * record, tail + at_page, blk);
    }
};

// Tiles of few rows: CW groups of KW waves; a group has 16 NT rows of the tile, its waves take the records in turn and decode them in
// their registers.
template <class F, int NT, int CW, int KW, bool Y32>
__global__ __launch_bounds__(64 * CW * KW, (F::template min_waves<NT>())) void attend_few_kernel(AttendK p)
{
    constexpr int D = F::D, ROWS = 16 * NT * CW, CH = D / 16;   // CH: channels of a row per thread in the joins
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
    Columns<F, NT, Y32> w;
    int lo[NT], hi[NT];
    w.begin(p.a, k, wrow0, v.group, v.n_kv, lo, hi, lane);
    const float c = p.a.scale * LOG2E;
    const Records<F> recs(p.a, k);
    const int b1 = k.b1, first_b = k.b0 + kw;
    if (first_b < b1 && n_cols > 0) {
        typename F::Record r0, r1;
        const typename F::Places at(lane);
        bool bad = false;
        // 64 records of the wave at a time, whose pages lie one to a lane: a read of the table among the loads below would have to wait for
        // every load that is on its way ahead of it.
        for (int c0 = first_b; c0 < b1; c0 += 64 * KW) {
            const int pages = recs.table[min(c0 + lane * KW, b1 - 1) >> recs.log_blocks];
            // Starts the loads of record b, the i-th of the 64; whether its page exists.
            auto start = [&](typename F::Record &r, int i, int b) {
                bool ok;
                F::load(r, recs.at(min(b, b1 - 1), __builtin_amdgcn_readlane(pages, i), ok), at);
                bad |= !ok;
                return ok;
            };
            auto take = [&](typename F::Record &r, int b, bool ok) {
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
                        lds_o[kw][n][F::o_channel(g * 4 + e, j)] = w.o[nt][j][e];
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
template <class F, bool Y32>
__global__ __launch_bounds__(256, (F::D == 256 ? 1 : 2)) void attend_tile_kernel(AttendK p)
{
    using Wave = Columns<F, 2, Y32>;
    constexpr int D = F::D, KD = Wave::KD, NJ = Wave::NJ, FRAGS = 4 * KD + 2 * NJ;
    using Operands = typename F::Operands;   // [tile][j][lane] of the keys, [half][j][lane] of the values
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
    const Records<F> recs(p.a, k);
    const int b1 = k.b1;
    if (k.b0 < b1) {
        typename F::Share mine(lane, wave);   // of a record, which the four waves decode for each other
        auto decode = [&](Operands &o, int b, bool ok) {   // ok: else it is some other record, of which nothing is used
            if (ok && !k.whole(b)) mine.template mask<2>(w.o, 2, b * 64, lo, hi, t.kv_len);
            mine.decode(o);
        };
        bool bad = false;
        for (int c0 = k.b0; c0 < b1; c0 += 64) {   // (64 pages at a time, one to a lane, as above)
            const int pages = recs.table[min(c0 + lane, b1 - 1) >> recs.log_blocks];
            const int count = min(64, b1 - c0);
            bool ok, next_ok = false;
            mine.load(recs.at(c0, __builtin_amdgcn_readlane(pages, 0), ok));
            decode(ops[0], c0, ok);
            for (int i = 0; i < count; ++i) {
                const int b = c0 + i;
                const bool more = i + 1 < count;
                // (without a condition: loads under one are waited for where it ends)
                mine.load(recs.at(more ? b + 1 : b, __builtin_amdgcn_readlane(pages, more ? i + 1 : i), next_ok));
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
        F::store(p.a, y, w.o[nt], inv, g);
        if (g == 0 && p.a.lse) p.a.lse[y] = log_sum(w.m[nt], w.l[nt], c);
    }
}

template <class F, int NT, int CW, int KW, bool Y32>
void launch_few(const AttendK &p, hipStream_t stream)
{
    hipLaunchKernelGGL((attend_few_kernel<F, NT, CW, KW, Y32>), dim3((unsigned)p.v.max_few * p.v.n_kv), dim3(256), 0, stream, p);
}

template <class F, bool Y32>
hipError_t launch_d(const KvPlanView &v, const AttendArgs &a, hipStream_t stream)
{
    constexpr bool WIDE = F::D == 256;   // two columns of accumulators would leave no registers for the rest
    AttendK p{v, a, 0};
    if (v.has_few) {
        if (std::min(v.max_new * (int64_t)v.group, (int64_t)KV_FEW_ROWS) <= 16) launch_few<F, 1, 1, 4, Y32>(p, stream);
        else launch_few<F, WIDE ? 1 : 2, WIDE ? 2 : 1, WIDE ? 2 : 4, Y32>(p, stream);
    }
    if (v.has_tile) {
        p.list = 1;
        hipLaunchKernelGGL((attend_tile_kernel<F, Y32>), dim3((unsigned)v.max_tile * v.n_kv), dim3(256), 0, stream, p);
    }
    return hipGetLastError();
}

}  // namespace

}  // namespace moin

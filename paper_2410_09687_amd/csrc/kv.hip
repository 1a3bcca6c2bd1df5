// The paged MXFP4 cache's bookkeeping and its writes: block tables and slot maps from the requests' lengths, pages given
// back, tokens appended, tokens read back.
#include "kv.h"
#include "mxfp4.h"

namespace moin {

constexpr int KV_RELEASE_THREADS = 1024;
constexpr int KV_SLOT_CHUNK = 2048;   // tokens of a request per workgroup of the second launch

// Inclusive scans over the workgroup, two quantities at once; `total` gets the workgroup's sums.
struct Scan2 {
    long long a;
    int b;
};
template <int PT>
__device__ __forceinline__ Scan2 block_scan(Scan2 v, Scan2 *lds, Scan2 &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const long long a = __shfl_up(v.a, d);
        const int b = __shfl_up(v.b, d);
        if (lane >= d) {
            v.a += a;
            v.b += b;
        }
    }
    lds_barrier();   // (what an earlier scan left has been read)
    if (lane == 63) lds[wave] = v;
    lds_barrier();
    Scan2 before{0, 0};
    total = Scan2{0, 0};
#pragma unroll
    for (int w = 0; w < PT / 64; ++w) {
        const Scan2 x = lds[w];
        if (w < wave) {
            before.a += x.a;
            before.b += x.b;
        }
        total.a += x.a;
        total.b += x.b;
    }
    v.a += before.a;
    v.b += before.b;
    return v;
}

__device__ __forceinline__ int ceil_shift(int v, int s) { return (v >> s) + ((v & ((1 << s) - 1)) != 0); }

// Slot of a request's token at position `pos`; `dealt` >= 0: the first of its new pages among those the step deals.
__device__ __forceinline__ int kv_slot(const KvPlanArgs &a, int s, int pos, int log_page, int have, int dealt, int n_free)
{
    const int pi = pos >> log_page;
    const int page = pi >= have ? a.free_pages[n_free - 1 - (dealt + pi - have)] : a.block_table[(int64_t)s * a.max_pages + pi];
    if (page < 0 || page >= a.n_pages) {
        atomicOr(a.err_word, ERR_BAD_PAGE);
        return -1;
    }
    return (page << log_page) + (pos & ((1 << log_page) - 1));
}

__device__ __forceinline__ void kv_write_tile(KvTile *dst, int tok0, int n_tok, int L, int s, int row0, int part, int n_parts, int pslot)
{
    int4 *d = reinterpret_cast<int4 *>(dst);
    d[0] = make_int4(tok0, n_tok, L, s);
    d[1] = make_int4(row0, part, n_parts, pslot);
}

// Whether a request's rows are tiles of many: also few rows where the launch for those is left out.
__device__ __forceinline__ bool kv_tiled(const KvPlanView &v, int64_t rows) { return rows > (v.has_few ? KV_FEW_ROWS : 0); }

// Height of the stack of free pages, of at most its room.
__device__ __forceinline__ int free_pages_there(int n_free, int free_cap, int &err)
{
    if (n_free < 0 || n_free > free_cap) err |= ERR_NO_PAGES;
    return max(0, min(n_free, free_cap));
}

// A step without requests.
__global__ __launch_bounds__(64) void kv_plan_empty_kernel(const int *n_free, int free_cap, int *n_free_out, int *seq_offsets, int *err_word)
{
    if (threadIdx.x) return;
    int err = 0;
    *n_free_out = free_pages_there(*n_free, free_cap, err);
    *seq_offsets = 0;
    if (err) atomicOr(err_word, err);
}

// One workgroup walks the requests, PT at a time, twice.  First: offsets (a sum over the new tokens), pages to deal (a sum over
// the pages that each request lacks), which requests are served.  Then, with the keys of all requests known, the
// size of the parts that fill the chip and everybody's place in the lists.  Up to KV_FEW_TOKENS new tokens a
// request (decode), it writes slots and table entries itself; else a second launch does, a workgroup for 2048 tokens of a request.
// Bound by latency: a chain of a dozen trips to memory and barriers.
template <int PT>
__global__ __launch_bounds__(PT) void kv_plan_kernel(KvPlanView v, KvPlanArgs a, int log_page, int few_tokens)
{
    __shared__ Scan2 lds[PT / 64];
    __shared__ int lds_err;
    const int tid = threadIdx.x;
    if (tid == 0) lds_err = 0;
    for (int i = tid; i < v.max_pslots * v.n_kv; i += PT) v.tickets[i] = 0;
    int err = 0;
    const int n_free = free_pages_there(*a.n_free, a.free_cap, err);
    const long long row_max = (long long)a.max_pages << log_page;
    long long tok_base = 0;
    int page_base = 0, taken = 0;
    long long few_blocks = 0, tile_blocks = 0;   // records that the tiles of either kind walk, one kv head
    int tiles = 0;
    for (int s0 = 0; s0 < v.S; s0 += PT) {
        const int s = s0 + tid;
        const bool in = s < v.S;
        const int kv = in ? a.kv_lens[s] : 0, n0 = in ? a.new_lens[s] : 0;
        const bool sane = kv >= 0 && n0 >= 0 && n0 <= v.max_new && (long long)max(kv, 0) + n0 <= row_max;
        const int have = ceil_shift(max(kv, 0), log_page);
        const int need = sane ? ceil_shift(kv + n0, log_page) - have : 0;
        Scan2 total;
        const Scan2 up = block_scan<PT>(Scan2{max(n0, 0), need}, lds, total);
        const long long end = tok_base + up.a, begin = end - max(n0, 0);
        const int dealt = page_base + up.b - need;
        const bool whole = end <= v.T;
        const bool served = sane && whole && (need == 0 || dealt + need <= n_free);
        if (in) {
            if (!sane || !whole) err |= ERR_BAD_LENGTHS;
            else if (!served) err |= ERR_NO_PAGES;
            const int tok0 = (int)min(begin, (long long)v.T), n = (int)(min(end, (long long)v.T) - tok0);
            a.seq_offsets[s] = tok0;
            if (s == v.S - 1) {
                a.seq_offsets[v.S] = tok0 + n;
                if (end != v.T) err |= ERR_BAD_LENGTHS;
                for (int64_t t = end; t < v.T; ++t) a.slots[t] = -1;   // tokens of no request
            }
            a.kv_lens_out[s] = served ? kv + n0 : max(kv, 0);
            v.req[s] = make_int4(max(kv, 0), served ? dealt : -1, need, n);
            // (a request that is not served has no keys: its rows come out as zeros)
            const int64_t rows = (int64_t)n * v.group;
            const int blocks = served ? ceil_shift(kv + n0, 6) : 0;
            if (kv_tiled(v, rows)) {
                const int own = (int)min((rows + KV_TILE_ROWS - 1) / KV_TILE_ROWS, (int64_t)KV_TILE_TARGET);   // (as many fill the chip alone)
                tiles += own;
                tile_blocks += (long long)own * blocks;
            } else if (rows > 0) {
                few_blocks += blocks;
            }
            if (served && need > 0) taken = dealt + need;
            if (few_tokens || n > v.max_new) {   // (more than the second launch covers: not served)
                for (int i = 0; i < n; ++i)
                    a.slots[tok0 + i] = served ? kv_slot(a, s, kv + i, log_page, have, dealt, n_free) : -1;
            }
            if (few_tokens && served) {
                for (int j = 0; j < need; ++j)
                    a.block_table[(int64_t)s * a.max_pages + have + j] = a.free_pages[n_free - 1 - (dealt + j)];
            }
        }
        tok_base += total.a;
        page_base += total.b;
    }
    // sums over the workgroup (served requests are a prefix of those that want pages: the last one's end is what is taken)
    Scan2 sums, t2;
    block_scan<PT>(Scan2{few_blocks, 0}, lds, sums);
    const long long few_all = sums.a;
    block_scan<PT>(Scan2{tile_blocks, tiles}, lds, sums);
    const long long tile_all = sums.a;
    const int tiles_all = sums.b;
    lds_barrier();
    __shared__ int lds_taken;
    if (tid == 0) lds_taken = 0;
    lds_barrier();
    if (taken) atomicMax(&lds_taken, taken);
    if (err) atomicOr(&lds_err, err);
    lds_barrier();
    if (tid == 0) {
        *a.n_free_out = n_free - lds_taken;
        v.head[2] = n_free;
        if (lds_err) atomicOr(a.err_word, lds_err);
    }
    // parts: so large that the launch has about its target of workgroups, over all kv heads
    const int few_goal = max(1, KV_FEW_TARGET / v.n_kv), tile_goal = max(1, KV_TILE_TARGET / v.n_kv);
    const int few_chunk = (int)max((long long)KV_FEW_MIN, (few_all + few_goal - 1) / few_goal);
    int tile_chunk = (int)max((long long)KV_TILE_MIN, (tile_all + tile_goal - 1) / tile_goal);
    // Tiles of many rows run long, and a few that begin when the others end cost as much as all of those: chunks of 400 - 500 tokens of four
    // requests 161 us in 640 workgroups, 127 in 448; 16 prefixes of 4000 113 us whole, 86 halved.  So a few sizes of parts, from the
    // smallest on, are weighed by when the last part would end: beside the others if all have room, else when the work before it is done.
    constexpr int SIZES = 8, COST = 4;   // COST: of a workgroup's beginning and end, in records
    __shared__ int count[SIZES], longest[SIZES];
    __shared__ int2 work[PT];
    if (tiles_all > 0 && tiles_all < 4 * tile_goal) {
        // (a thread to a size and every PT / 8-th request; through LDS, and sums by shuffles: atomics of all requests on eight words took 36 us
        // for 64 of them)
        const int i = tid % SIZES;
        const int eighths = (int)(0x2014100E0C0A0908uLL >> 8 * i & 255);   // of the smallest: 8, 9, 10, 12, 14, 16, 20, 32
        const int size = (int)min(0x3fffffffLL, max((long long)KV_TILE_MIN, (tile_all * eighths / 8 + tile_goal - 1) / tile_goal));
        int parts_all = 0, top = 0;
        if (tid < SIZES) count[tid] = longest[tid] = 0;
        for (int s0 = 0; s0 < v.S; s0 += PT) {
            const int s = s0 + tid;
            int2 own = make_int2(0, 0);
            if (s < v.S) {
                const int4 q = v.req[s];   // (what this thread wrote in the first walk)
                const int64_t rows = (int64_t)q.w * v.group;
                if (kv_tiled(v, rows))
                    own = make_int2((int)min((rows + KV_TILE_ROWS - 1) / KV_TILE_ROWS, (int64_t)KV_TILE_TARGET), q.y >= 0 ? ceil_shift(q.x + q.w, 6) : 0);
            }
            work[tid] = own;
            lds_barrier();
            for (int r = tid / SIZES; r < min(PT, v.S - s0); r += PT / SIZES) {
                const int2 w = work[r];
                if (w.x == 0) continue;
                const int parts = min(KV_MAX_PARTS, max(1, (w.y + size - 1) / size));
                parts_all += w.x * parts;
                top = max(top, (w.y + parts - 1) / parts);
            }
            lds_barrier();
        }
#pragma unroll
        for (int d = SIZES; d < 64; d <<= 1) {
            parts_all += __shfl_xor(parts_all, d);
            top = max(top, __shfl_xor(top, d));
        }
        if ((tid & 63) < SIZES) {
            atomicAdd(&count[i], parts_all);
            atomicMax(&longest[i], top);
        }
        lds_barrier();
        // (the eight in neighbouring lanes; of equals the smaller size)
        long long best = ((count[i] <= tile_goal ? 0 : (tile_all + (long long)COST * count[i]) / tile_goal) + longest[i] + COST) * SIZES + i;
#pragma unroll
        for (int d = 1; d < SIZES; d <<= 1) best = min(best, (long long)__shfl_xor(best, d));
        tile_chunk = __shfl(size, (int)(best % SIZES));
    }
    // Tiles of few rows are listed by the length of their parts, longest first (in 64 steps; who is first in a step is left to chance and
    // shows in no result): the last workgroups to begin are then short ones.
    __shared__ int place[64];
    if (tid < 64) place[tid] = 0;
    lds_barrier();
    auto work_of = [&](int s, int &tok0, int &n, int &L) {   // (what this thread wrote in the first walk)
        const int4 q = v.req[s];
        tok0 = a.seq_offsets[s];
        n = q.w;
        L = q.y >= 0 ? q.x + n : 0;
    };
    auto parts_of = [&](int L, int size) { return min(KV_MAX_PARTS, max(1, (ceil_shift(L, 6) + size - 1) / size)); };
    auto step_of = [&](int L, int parts) { return 63 - min(63, (ceil_shift(L, 6) + parts - 1) / parts * 63 / few_chunk); };
    auto is_few = [&](int n) { return n > 0 && !kv_tiled(v, (int64_t)n * v.group); };
    if (v.has_few) {
        for (int s = tid; s < v.S; s += PT) {
            int tok0, n, L;
            work_of(s, tok0, n, L);
            if (!is_few(n)) continue;
            const int parts = parts_of(L, few_chunk);
            atomicAdd(&place[step_of(L, parts)], parts);
        }
        lds_barrier();
        if (tid < 64) {
            const int own = place[tid];
            int up = own;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int x = __shfl_up(up, d);
                if (tid >= d) up += x;
            }
            place[tid] = up - own;
            if (tid == 63) v.head[0] = min(up, v.max_few);
        }
        lds_barrier();
    } else if (tid == 0) {
        v.head[0] = 0;
    }
    int tile_base = 0, ps_base = 0;
    for (int s0 = 0; s0 < v.S; s0 += PT) {
        const int s = s0 + tid;
        const bool in = s < v.S;
        int tok0 = 0, n = 0, L = 0;
        if (in) work_of(s, tok0, n, L);
        const int64_t rows = (int64_t)n * v.group;
        const bool few = is_few(n) && v.has_few, tiled = kv_tiled(v, rows) && v.has_tile;
        const int n_tiles = tiled ? (int)((rows + KV_TILE_ROWS - 1) / KV_TILE_ROWS) : few ? 1 : 0;
        const int parts = parts_of(L, tiled ? tile_chunk : few_chunk);
        const int recs = n_tiles * parts, ps = parts > 1 ? recs * (tiled ? KV_TILE_PLACES : 1) : 0;
        const Scan2 up = block_scan<PT>(Scan2{tiled ? recs : 0, ps}, lds, t2);
        const int tile_at = tile_base + (int)up.a - (tiled ? recs : 0), ps_at = ps_base + up.b - ps;
        if (few) {
            const int at = atomicAdd(&place[step_of(L, parts)], parts);
            if (at + parts <= v.max_few && ps_at + ps <= v.max_pslots)
                for (int p = 0; p < parts; ++p) kv_write_tile(v.few + at + p, tok0, n, L, s, 0, p, parts, ps_at);
        }
        if (in) {
            v.req[s].w = tiled ? tile_at : -1;
            v.req_tiles[s] = make_int2(parts, ps_at);
        }
        if (few_tokens && tiled && tile_at + recs <= v.max_tile && ps_at + ps <= v.max_pslots)
            for (int t = 0; t < n_tiles; ++t)   // the last rows see the most keys: their tiles first
                for (int p = 0; p < parts; ++p)
                    kv_write_tile(v.tile + tile_at + t * parts + p, tok0, n, L, s, (n_tiles - 1 - t) * KV_TILE_ROWS, p, parts,
                                  ps_at + (parts > 1 ? t * parts * KV_TILE_PLACES : 0));
        tile_base += (int)t2.a;
        ps_base += t2.b;
    }
    if (tid == 0) v.head[1] = min(tile_base, v.max_tile);
}

// Slots, table entries and tiles of requests with many new tokens: workgroup (request, chunk of 2048 tokens).
__global__ __launch_bounds__(256) void kv_slots_kernel(KvPlanView v, KvPlanArgs a, int log_page)
{
    const int s = blockIdx.x, c = blockIdx.y, nc = gridDim.y, tid = threadIdx.x;
    const int tok0 = a.seq_offsets[s], n = a.seq_offsets[s + 1] - tok0;
    const int4 q = v.req[s];
    const int n_free = v.head[2], kv = q.x, dealt = q.y, have = ceil_shift(kv, log_page);
    const bool served = dealt >= 0;
    const int end = min(n, (c + 1) * KV_SLOT_CHUNK);
    for (int i = c * KV_SLOT_CHUNK + tid; i < end; i += 256)
        a.slots[tok0 + i] = served ? kv_slot(a, s, kv + i, log_page, have, dealt, n_free) : -1;
    if (served) {
        for (int j = c * 256 + tid; j < q.z; j += nc * 256)
            a.block_table[(int64_t)s * a.max_pages + have + j] = a.free_pages[n_free - 1 - (dealt + j)];
    }
    if (q.w < 0 || !v.has_tile) return;
    const int L = served ? kv + n : 0;
    const int2 t2 = v.req_tiles[s];
    const int parts = t2.x, n_tiles = (int)(((int64_t)n * v.group + KV_TILE_ROWS - 1) / KV_TILE_ROWS), recs = n_tiles * parts;
    if (q.w + recs > v.max_tile || (parts > 1 && t2.y + recs * KV_TILE_PLACES > v.max_pslots)) return;
    for (int r = c * 256 + tid; r < recs; r += nc * 256) {
        const int t = r / parts, p = r - t * parts;
        kv_write_tile(v.tile + q.w + r, tok0, n, L, s, (n_tiles - 1 - t) * KV_TILE_ROWS, p, parts, t2.y + (parts > 1 ? t * parts * KV_TILE_PLACES : 0));
    }
}

static int log2_of(int v)
{
    int s = 0;
    while ((1 << s) < v) ++s;
    return s;
}

hipError_t launch_kv_plan_empty(const int *n_free, int free_cap, int *n_free_out, int *seq_offsets, int *err_word, hipStream_t stream)
{
    hipLaunchKernelGGL(kv_plan_empty_kernel, dim3(1), dim3(64), 0, stream, n_free, free_cap, n_free_out, seq_offsets, err_word);
    return hipGetLastError();
}

hipError_t launch_kv_plan(const KvPlanView &v, const KvPlanArgs &a, hipStream_t stream)
{
    const int few_tokens = v.max_new <= KV_FEW_TOKENS, log_page = log2_of(a.page_tokens);
    // (a barrier costs fewer waves less: 64 requests in 13.2 us with 1024 threads, 8.1 with 256; 1000 prompts in 22.3 with 1024, 17.2 with 512)
    if (v.S <= 256) hipLaunchKernelGGL(kv_plan_kernel<256>, dim3(1), dim3(256), 0, stream, v, a, log_page, few_tokens);
    else hipLaunchKernelGGL(kv_plan_kernel<512>, dim3(1), dim3(512), 0, stream, v, a, log_page, few_tokens);
    if (!few_tokens)
        hipLaunchKernelGGL(kv_slots_kernel, dim3((unsigned)v.S, (unsigned)((v.max_new + KV_SLOT_CHUNK - 1) / KV_SLOT_CHUNK)), dim3(256), 0,
                           stream, v, a, log_page);
    return hipGetLastError();
}

// Pages of finished requests go back on the stack, in the requests' order; their rows of the table become -1, their lengths 0.  Every page is
// written where it belongs if all of them exist and fit (1000 requests of 32 pages 40 us; counted first and written then, 46 to 63).  Where one does not, the
// places of those that do not exist are closed up afterwards, and entries that found no room have what that leaves.
__global__ __launch_bounds__(KV_RELEASE_THREADS) void kv_release_kernel(const int *finished, int S, int *kv_lens, int *block_table, int max_pages,
                                                                     int log_page, int *free_pages, int *n_free, int free_cap, int n_pages,
                                                                     int *err_word)
{
    __shared__ Scan2 lds[KV_RELEASE_THREADS / 64];
    __shared__ int2 range[KV_RELEASE_THREADS];   // of a request: where its pages go, how many they are
    __shared__ int lds_gaps, lds_top;
    const int tid = threadIdx.x, lane = tid & 63;
    int base = *n_free;
    const int before = base;
    bool bad = base < 0 || base > free_cap;
    base = max(0, min(base, free_cap));
    for (int s0 = 0; s0 < S; s0 += KV_RELEASE_THREADS) {
        const int s = s0 + tid, in_pass = min(KV_RELEASE_THREADS, S - s0);
        const bool done = s < S && finished[s] != 0;
        const int kv = done ? kv_lens[s] : 0;
        const int pages = done ? min(ceil_shift(max(kv, 0), log_page), max_pages) : 0;
        if (done && (kv < 0 || ceil_shift(max(kv, 0), log_page) > max_pages)) bad = true;
        Scan2 total;
        const Scan2 up = block_scan<KV_RELEASE_THREADS>(Scan2{0, pages}, lds, total);
        range[tid] = make_int2(base + up.b - pages, pages);
        if (tid == 0) lds_gaps = 0;
        if (done) kv_lens[s] = 0;
        lds_barrier();
        bool gaps = false;
        for (int w = tid >> 6; w < in_pass; w += KV_RELEASE_THREADS / 64) {   // a wave per request
            const int2 r = range[w];
            for (int j = lane; j < r.y; j += 64) {
                int *entry = block_table + (int64_t)(s0 + w) * max_pages + j;
                const int page = *entry, to = r.x + j;
                const bool exists = page >= 0 && page < n_pages;
                if (to < free_cap) {
                    free_pages[to] = exists ? page : -1;
                    *entry = -1;
                }
                gaps |= !exists || to >= free_cap;
                bad |= !exists;
            }
        }
        if (gaps) lds_gaps = 1;
        __syncthreads();
        int top = min(base + total.b, free_cap);
        if (lds_gaps) {
            if (tid < 64) {
                int at = base;
                for (int p0 = base; p0 < top; p0 += 64) {   // (what is written lies behind what is yet to be read)
                    const int page = p0 + lane < top ? free_pages[p0 + lane] : -1;
                    const uint64_t there = __ballot(page >= 0);
                    if (page >= 0) free_pages[at + __popcll(there & ((1ull << lane) - 1))] = page;
                    at += __popcll(there);
                }
                for (int w = 0; w < in_pass; ++w) {
                    const int2 r = range[w];
                    for (int j0 = max(0, free_cap - r.x); j0 < r.y; j0 += 64) {
                        const bool in = j0 + lane < r.y;
                        int *entry = block_table + (int64_t)(s0 + w) * max_pages + j0 + lane;
                        const int page = in ? *entry : -1;
                        const bool exists = page >= 0 && page < n_pages;
                        const uint64_t there = __ballot(exists);
                        const int to = at + __popcll(there & ((1ull << lane) - 1));
                        if (exists && to < free_cap) free_pages[to] = page;
                        bad |= exists && to >= free_cap;
                        if (in) *entry = -1;
                        at = min(at + __popcll(there), free_cap);
                    }
                }
                if (lane == 0) lds_top = at;
            }
            __syncthreads();
            top = lds_top;
        }
        base = top;
    }
    __syncthreads();
    if (tid == 0 && base != before) *n_free = base;
    if (bad) atomicOr(err_word, ERR_BAD_PAGE);
}

hipError_t launch_kv_release(const int *finished, int S, int *kv_lens, int *block_table, int max_pages, int page_tokens, int *free_pages,
                             int *n_free, int free_cap, int n_pages, int *err_word, hipStream_t stream)
{
    hipLaunchKernelGGL(kv_release_kernel, dim3(1), dim3(KV_RELEASE_THREADS), 0, stream, finished, S, kv_lens, block_table, max_pages,
                       log2_of(page_tokens), free_pages, n_free, free_cap, n_pages, err_word);
    return hipGetLastError();
}

// The bf16 side of a copy passes through once: past L2, which holds the lines of the cache until they are whole (169 -> 150 us for 65536 tokens
// there and back).
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_once(const char *p)
{
    return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p)));
}
__device__ __forceinline__ void store_once(char *p, const uint4 &v)
{
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), reinterpret_cast<u32x4_t *>(p));
}

// A wave takes one block of 32 channels of the keys or values of 64 tokens: four at a time of its lanes a token's block, 16 bytes of bf16 and
// four bytes of codes each.  Tokens of a request follow each other in its pages, so that the codes of 16 are a run of 256 bytes in the
// cache (in the order of a token's channels alone they are pieces of four: 131 us for 65536 tokens of eight heads of 128, 80 like
// this, 4.3 TB/s; back 117 and 69, 4.9 TB/s); a workgroup's four waves take neighbouring blocks, whose halves of lines meet in L2.
template <bool APPEND>
__global__ __launch_bounds__(256) void kv_copy_kernel(KvPages p, char *k, char *v, int64_t k_stride, int64_t v_stride, int64_t T, int groups,
                                                      const int *__restrict__ slots, int *err_word)
{
    const int lane = threadIdx.x & 63, c = lane & 3, DB = p.D / 32, half = p.n_kv * DB;
    const int64_t chunk = blockIdx.x / groups;
    int blk = (int)(blockIdx.x - chunk * groups) * 4 + (threadIdx.x >> 6);
    const bool is_v = blk >= half;
    if (is_v) blk -= half;
    const int h = blk / DB, b = blk - h * DB, log_page = p.log_blocks + 6;
    const int64_t t0 = chunk * 64 + (lane >> 2), stride = (is_v ? v_stride : k_stride) * 2;
    char *row = (is_v ? v : k) + blk * 64 + c * 16;
    int slot[4];
    uint4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t t = min(t0 + i * 16, T - 1);
        slot[i] = slots[t];
        if constexpr (APPEND) x[i] = load_once(row + t * stride);
    }
    char *rec[4], *scale[4];
    int at[4];
    bool bad = false, there[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool in = slot[i] >= 0 && (slot[i] >> log_page) < p.n_pages;
        there[i] = in && t0 + i * 16 < T;
        bad |= !in && slot[i] != -1;
        const int s = in ? slot[i] : 0, in_page = s & ((1 << log_page) - 1), tile = (in_page >> 4) & 3, m = in_page & 15;
        rec[i] = p.data + (int64_t)(s >> log_page) * p.page_bytes() + ((int64_t)((h << p.log_blocks) + (in_page >> 6))) * kv_record_bytes(p.D);
        at[i] = is_v ? 32 * p.D + (tile * p.D / 8 + b * 4 + c) * 64 + m * 4 : (tile * DB + b) * 256 + m * 16 + c * 4;
        scale[i] = rec[i] + (is_v ? 66 : 64) * p.D + b * 64 + m * 4 + tile;
    }
    if (bad) atomicOr(err_word, ERR_BAD_PAGE);
    if constexpr (APPEND) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t amax = bf16x8_amax(x[i]);
            amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
            amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
            const uint32_t E = mx4_scale_byte(amax);
            if (!there[i]) continue;
            *reinterpret_cast<uint32_t *>(rec[i] + at[i]) = mx4_encode(x[i], bits_f32(E << 23));
            if (c == 0) *scale[i] = (char)E;
        }
    } else {
        uint32_t codes[4], E[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // (a slot that names nothing reads the first token's, and drops it)
            codes[i] = *reinterpret_cast<const uint32_t *>(rec[i] + at[i]);
            E[i] = *reinterpret_cast<const uint8_t *>(scale[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (t0 + i * 16 >= T) continue;
            store_once(row + (t0 + i * 16) * stride, there[i] ? mx4_decode(codes[i], bits_f32(E[i] << 23)) : make_uint4(0, 0, 0, 0));
        }
    }
}

template <bool APPEND>
static hipError_t launch_copy(const KvPages &p, void *k, void *v, int64_t k_stride, int64_t v_stride, int64_t T, const int *slots, int *err_word,
                              hipStream_t stream)
{
    const int groups = 2 * p.n_kv * p.D / 32 / 4;   // (four blocks a workgroup: D is 64 or more)
    hipLaunchKernelGGL(kv_copy_kernel<APPEND>, dim3((unsigned)((T + 63) / 64 * groups)), dim3(256), 0, stream, p, static_cast<char *>(k),
                       static_cast<char *>(v), k_stride, v_stride, T, groups, slots, err_word);
    return hipGetLastError();
}

hipError_t launch_kv_append(const KvPages &p, const void *k, const void *v, int64_t k_stride, int64_t v_stride, int64_t T,
                            const int *slots, int *err_word, hipStream_t stream)
{
    return launch_copy<true>(p, const_cast<void *>(k), const_cast<void *>(v), k_stride, v_stride, T, slots, err_word, stream);
}

hipError_t launch_kv_gather(const KvPages &p, void *k, void *v, int64_t T, const int *slots, int *err_word, hipStream_t stream)
{
    return launch_copy<false>(p, k, v, (int64_t)p.n_kv * p.D, (int64_t)p.n_kv * p.D, T, slots, err_word, stream);
}

}  // namespace moin

// The paged cache of keys and values in MXFP4, and the plan of a step: what kv.hip, attend.hip and the C ABI share.
//
// A page holds `page_tokens` tokens (64, 128 or 256) of every kv head: [kv heads][page_tokens / 64] records of 64 tokens x D
// channels, 68 D bytes each.  Token 16 i + m of a record (i < 4, m < 16) has its
//   keys    at [i][D / 32][m][16 bytes],
//   values  at [i][D / 8][m][4 bytes]     (from byte 32 D on),
//   scales  at [D / 32][m][i]             (keys' from byte 64 D on, values' from byte 66 D on),
// which is the order in which the attention kernel's lanes take them: a 16-token operand tile of either is one run of memory, and a
// lane's scale bytes for the four tiles of a record are words.
#pragma once
#include <algorithm>
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace moin {

constexpr int KV_BLOCK = 64;                                             // tokens of a record
__host__ __device__ constexpr int kv_record_bytes(int D) { return 68 * D; }
constexpr bool kv_head_dim_ok(int D) { return D == 64 || D == 128 || D == 256; }

struct KvPages {
    char *data;
    int n_pages, n_kv, D;
    int log_blocks;        // log2 of the records a page holds of one head
    __host__ __device__ int64_t page_bytes() const { return ((int64_t)n_kv * kv_record_bytes(D)) << log_blocks; }
};

// Query rows of a request (its tokens times the query heads of a kv head) are cut into tiles.  Requests of up to KV_FEW_ROWS
// rows are one tile, whose workgroup's waves take the records in turn; larger ones have tiles of KV_TILE_ROWS rows, KV_TILE_ROWS / 4 to
// a wave, and every wave walks all the keys.  A tile's keys are cut into parts where there are too few tiles to fill the
// chip; the workgroup of a tile that ends last joins its parts.
// (Rows 32: 64 requests of 2000 keys and 4 tokens, 32 heads on 4 of 64 channels, 19.5 us as one tile of few rows, 36 as tiles of 128; 32 heads on 8 of
// 128, 8 tokens 41 and 76.)
constexpr int KV_FEW_ROWS = 32, KV_TILE_ROWS = 128;
// Partial results are counted in places of KV_FEW_ROWS rows: a part of a tile of few rows takes one, of the others as many as here.
constexpr int KV_TILE_PLACES = KV_TILE_ROWS / KV_FEW_ROWS;
// Up to here (new tokens of a request) the plan is one launch: 64 requests of 4 tokens 7.0 us, 9.4 in two; of 32 tokens 16.0 and 11.5.
constexpr int KV_FEW_TOKENS = 8;
// Workgroups aimed at per launch where the keys allow, two for every compute unit.  Us with 384 / 512 / 768 / 1024: two requests of 100000 keys and
// more 67 / 61 / 71 / 70, 256 of up to 4096 34.7 / 34.8 / 37 / 39, 64 of 2000 13.7 / 13.8 / 14.8 / 18.5.  Tiles of 128 with 512 / 768: 8 prompts of 128
// behind 2000 keys 55 / 68.
constexpr int KV_FEW_TARGET = 512, KV_TILE_TARGET = 512;
// The fewest records of a part, of all the keys that a request has: a window is the attention's own, which divides what it leaves among the same
// parts, so that short windows of long requests have parts of fewer records or of none.  Us with 4 / 8 / 16: one request of 1000 keys 7.0 / 7.6 / 7.3, of 4000 9.1 / 8.6 / 9.3, four of 8000 and 4 tokens 19.5 / 13.8 /
// 14.7, 16 of 2000 and 3 tokens 14.0 / 11.2 / 13.4; a prompt of 128 behind 3000 28 / 20 / 24, of 64 behind 500 12.5 / 14.2 / 15.8.
constexpr int KV_FEW_MIN = 8, KV_TILE_MIN = 8;
constexpr int KV_MAX_PARTS = 128;  // of a tile

struct KvTile {            // one workgroup's work, per kv head
    int tok0, n_tok;       // the request's tokens in the batch
    int kv_len;            // keys the request has, its new tokens included
    int req;
    int row0;              // first row of the tile, of the request's n_tok * group
    int part, n_parts;
    int pslot;             // n_parts > 1: place of the tile's first part among the partial results
};

struct KvPlanView {
    int *head;             // [4]: records of either list; free pages before the step; tiles of many rows, also those that the list has no room for
    int4 *req;             // [S] {keys before, first of its pages among those the step deals or -1, pages dealt, first record in `tile`}
    int2 *req_tiles;       // [S] {parts of each of its tiles, first place of their partial results}
    KvTile *few, *tile;
    int *tickets;          // [max_pslots * n_kv], zero between calls
    int S, n_kv, group, max_new, max_pages, page_tokens;
    int64_t T;
    int max_few, max_tile, max_pslots;
    int room_pslots;       // the most of any step of up to these requests and tokens
    bool has_few, has_tile;
};

// The list of tiles of many rows of up to this many requests goes by the keys that a tile sees, the most first (kv_slots_kernel).
constexpr int KV_ORDERED_REQUESTS = 64;
__host__ __device__ inline int kv_tiles_of(int n, int group) { return (int)(((int64_t)n * group + KV_TILE_ROWS - 1) / KV_TILE_ROWS); }
// A request as that order has it: keys before its new tokens, those, its tiles and their parts; zeros: not in the list.  One that is not served has
// no keys, whatever length it came with: keys and new tokens together stay below 2^31, and no position or difference of two wraps.
struct alignas(16) KvListed {
    int kv, n, tiles, parts;
};
__host__ __device__ inline KvListed kv_listed(const int4 &req, int n, int parts, int group)
{
    return req.w >= 0 ? KvListed{req.y >= 0 ? req.x : 0, n, kv_tiles_of(n, group), parts} : KvListed{0, 0, 0, 0};
}
// Position of the last row of its tile t: the first one ends with the last token, the others with row 128 k - 1.
__host__ __device__ inline int kv_tile_sees(const KvListed &r, int t, int group)
{
    return r.kv + (t ? ((r.tiles - t) * KV_TILE_ROWS - 1) / group : r.n - 1);
}
// Records of request o in front of a tile of another that sees so much; `wins`: of equals o's come first.
__host__ __device__ inline int kv_records_before(const KvListed &o, int sees, bool wins, int group)
{
    const int y = sees - o.kv + (wins ? 0 : 1);   // o's tokens from this one on see more, or as much and come first
    // (tokens times group stay below 2^31 - 128)
    return o.parts * (y <= 0 ? o.tiles : y >= o.n ? 0 : 1 + o.tiles - (y * group + KV_TILE_ROWS) / KV_TILE_ROWS);
}

struct KvPlanArgs {
    const int *kv_lens, *new_lens;
    int *block_table;
    int max_pages;
    const int *free_pages, *n_free;
    int free_cap, n_pages, page_tokens;
    int *n_free_out, *kv_lens_out, *seq_offsets, *slots;
    int *err_word;
};
hipError_t launch_kv_plan(const KvPlanView &v, const KvPlanArgs &a, hipStream_t stream);
hipError_t launch_kv_plan_empty(const int *n_free, int free_cap, int *n_free_out, int *seq_offsets, int *err_word, hipStream_t stream);
hipError_t launch_kv_release(const int *finished, int S, int *kv_lens, int *block_table, int max_pages, int page_tokens, int *free_pages,
                             int *n_free, int free_cap, int n_pages, int *err_word, hipStream_t stream);
// k / v: [T, n_kv, D] bf16, rows of tokens k_stride / v_stride elements apart
hipError_t launch_kv_append(const KvPages &p, const void *k, const void *v, int64_t k_stride, int64_t v_stride, int64_t T,
                            const int *slots, int *err_word, hipStream_t stream);
hipError_t launch_kv_gather(const KvPages &p, void *k, void *v, int64_t T, const int *slots, int *err_word, hipStream_t stream);

struct AttendArgs {
    KvPages pages;
    const void *q;
    int64_t q_stride;      // elements between the rows of tokens
    const int *block_table;
    int max_pages, window;
    float scale;
    void *y;
    int y_f32;
    float *lse;            // or null
    float *partial;        // attend_partial_floats()
    int *err_word;
};
// fp32 words of that many places of partial results.
int64_t attend_partial_floats(const KvPlanView &v, int pslots, int D);
hipError_t launch_attend(const KvPlanView &v, const AttendArgs &a, hipStream_t stream);

constexpr int ERR_BAD_LENGTHS = 16;   // lengths that are negative, beyond the table's rows, or do not add up to the tokens
constexpr int ERR_NO_PAGES = 32;      // requests that the free pages do not serve
constexpr int ERR_BAD_PAGE = 64;      // a page or slot that the cache does not have

}  // namespace moin

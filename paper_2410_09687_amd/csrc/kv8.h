// The paged cache of keys and values in E4M3 with one power of two 2^(E - 127) for the keys and one for the values of each 64
// tokens and head: what kv8.hip, attend8.hip and the C ABI share.
//
// A page holds `page_tokens` tokens (64, 128 or 256) of every kv head: [kv heads][page_tokens / 64] records of 64 tokens x D channels,
// 128 D bytes each,
//   keys    channel 64 l + c of token 16 i + m (i, l: tiles of 16 tokens, 64 channels) at [i][l][m][c],
//   values  channel 16 j + m of token 16 w + 4 g + e (w, g, e < 4) at [j][m][g][w][e], from byte 64 D on,
// so that the 16 bytes of a lane of the attention kernels are operands as they are, 64 lanes a run of memory, and a token's keys
// are runs of 64 bytes, a channel's values one.  Behind the records, the bytes E [kv heads][page_tokens / 64][2], keys' and values', up to
// a multiple of 128 bytes.
#pragma once
#include "kv.h"

namespace moin {

__host__ __device__ constexpr int kv8_record_bytes(int D) { return 128 * D; }
// Byte of a page where the two scales of a head's block lie.
__host__ __device__ inline int64_t kv8_scales_at(const KvPages &p, int h, int blk)
{
    return (((int64_t)p.n_kv * kv8_record_bytes(p.D)) << p.log_blocks) + 2 * (((int64_t)h << p.log_blocks) + blk);
}
__host__ __device__ inline int64_t kv8_page_bytes(const KvPages &p) { return (kv8_scales_at(p, p.n_kv, 0) + 127) & ~(int64_t)127; }

// k / v: [T, n_kv, D] bf16, rows of tokens k_stride / v_stride elements apart; a request's tokens are those of seq_offsets[s] to [s + 1].
hipError_t launch_kv8_append(const KvPages &p, const void *k, const void *v, int64_t k_stride, int64_t v_stride, int64_t T,
                             const int *seq_offsets, int S, const int *slots, int *err_word, hipStream_t stream);
hipError_t launch_kv8_gather(const KvPages &p, void *k, void *v, int64_t T, const int *slots, int *err_word, hipStream_t stream);
hipError_t launch_attend8(const KvPlanView &v, const AttendArgs &a, hipStream_t stream);

}  // namespace moin

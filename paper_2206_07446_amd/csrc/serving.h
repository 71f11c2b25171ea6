// Declarations shared by the host side and the kernels of the serving operators.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "nnv.h"

namespace nnv {

size_t linear_transformed_bytes(const nnv_linear_desc &d);
size_t linear_workspace_bytes(const nnv_linear_desc &d, int m);
hipError_t launch_linear_pack(const nnv_linear_desc &d, const void *raw, void *tx, hipStream_t st);
hipError_t launch_linear(const nnv_linear_desc &d, int m, const void *x, int64_t ldx, const void *tx, const float *bias, void *y, int64_t ldy,
                         void *ws, hipStream_t st);

// A block of the cache holds, for one key/value head after the other, its tokens as the attention kernel's wavefronts read them
// (D = head_dim, T = block_tokens; c = 0 .. 15 stands for values c D/16 .. + D/16 - 1 of a head):
//   keys          [T][D/2]            codes of a token, the even value of a pair in the low half of its byte
//   values        [T/4][16 c][4][D/32] codes of four tokens side by side
//   key scales    [T][D/32]
//   value scales  [T/4][D/32][4]
struct KvLayout {
    int dim, tokens;
    __host__ __device__ int head_bytes() const { return tokens * (dim + dim / 16); }
    __host__ __device__ int value_at() const { return tokens * dim / 2; }
    __host__ __device__ int key_scale_at() const { return tokens * dim; }
    __host__ __device__ int value_scale_at() const { return tokens * (dim + dim / 32); }
};

struct PlanArgs {
    const int32_t *held, *fresh, *free_blocks, *free_count;
    int32_t *table, *starts, *lengths, *positions, *left;
    int64_t *slots;
    int requests, rows, block_log, blocks, width;
};
hipError_t launch_kv_plan(const PlanArgs &a, hipStream_t st);

struct RopeArgs {
    const void *q, *k, *v;
    int64_t ldq, ldk, ldv;
    const float *q_weight, *k_weight, *rope;
    const int32_t *positions;
    const int64_t *slots;
    void *q_out, *k_out;
    char *cache;
    int rows, q_heads, kv_heads, rotary, interleaved, max_position, block_log;
    int64_t total_slots;
    float eps;
};
hipError_t launch_qk_norm_rope(const RopeArgs &a, int dim, int dtype, hipStream_t st);
hipError_t launch_kv_read(int n, const int64_t *slots, const char *cache, void *k, void *v, int kv_heads, int dim, int block_log, int64_t total_slots,
                          int dtype, hipStream_t st);

struct AttendArgs {
    const void *q;
    const int32_t *table, *starts, *lengths, *positions;
    const char *cache;
    void *out;
    float *parts;
    int requests, rows, q_heads, kv_heads, group, block_log, blocks, width, window, sinks;
    int tiles, splits, many, many_tiles;       // many: requests of many rows go to a kernel of their own
    int ordered;                               // whether that takes the tiles of the longest requests first
    uint32_t group_inverse;                    // 2^21 / group, rounded up
    float scale;        // magnitude of the factor of the scores, times log2(e); never 0, so that a score of -infinity stays one
    int flip;           // sign bits of a pair of 16-bit values where the factor is negative
    const int32_t *groups, *shared, *selected;
    int n_groups, keep;
    // nnv_kv_attention_shared: partial results of a row and query head, the most splits of a prefix (their results come first), workgroups that prefixes are cut into (of a
    // key head) and the fewest steps of one, launched workgroups of prefixes and of requests of many rows
    int tail;                                  // workgroups of a key head that the chip holds: tiles that do not fill it once more are split (0: none are)
    int slots, prefix_splits, prefix_units, prefix_least, prefix_short, prefix_groups, own_many;
};
int64_t kv_attention_groups(const nnv_attention_desc &d, int requests, int rows);     // tiles of rows times key/value heads
size_t kv_attention_workspace_bytes(const nnv_attention_desc &d, int requests, int rows);
hipError_t launch_kv_attention(const nnv_attention_desc &d, const AttendArgs &a, void *ws, hipStream_t st);
int64_t kv_attention_shared_groups(const nnv_attention_desc &d, int requests, int rows, int groups);
size_t kv_attention_shared_workspace_bytes(const nnv_attention_desc &d, int requests, int rows, int groups);
hipError_t launch_kv_attention_shared(const nnv_attention_desc &d, const AttendArgs &a, void *ws, hipStream_t st);
int64_t kv_attention_blocks_groups(const nnv_attention_desc &d, int rows);
size_t kv_attention_blocks_workspace_bytes(const nnv_attention_desc &d, int rows, int keep);
hipError_t launch_kv_attention_blocks(const nnv_attention_desc &d, const AttendArgs &a, void *ws, hipStream_t st);

struct BoundsArgs {
    const int32_t *table, *starts, *lengths;
    const char *cache;
    __bf16 *bounds;
    int requests, rows, kv_heads, block_log, blocks, width, units;
};
hipError_t launch_kv_bounds(const BoundsArgs &a, int dim, hipStream_t st);

struct SelectArgs {
    const void *q;
    const int32_t *table, *starts, *lengths, *positions;
    const __bf16 *bounds;
    int32_t *selected;
    uint64_t *scores;
    int requests, row0, rows, q_heads, kv_heads, group, block_log, blocks, width, keep, first, last;
    int tile_rows, tiles, chunks, chunk_blocks, flip;
};
constexpr int kMostSelectBlocks = 32768;       // columns of the table: kv_pick holds the scores of all in registers
size_t kv_select_workspace_bytes(const nnv_attention_desc &d, int rows);
hipError_t launch_kv_select(const nnv_attention_desc &d, const SelectArgs &a, hipStream_t st);

struct ResidualArgs {
    const void *x, *y, *gate;
    const float *post, *pre;
    const int32_t *index;
    void *x_out, *h;
    int64_t ldx, ldy, ldg, ldo, ldh;
    int m, n, gates, h_dtype, threads;         // threads: of a row
    float scale, eps;
};
hipError_t launch_residual_norm(const nnv_residual_desc &d, const ResidualArgs &a, hipStream_t st);

}  // namespace nnv

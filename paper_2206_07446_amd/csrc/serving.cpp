// Host side of the serving operators declared in nnv.h: descriptors, sizes, argument checks, dispatch.
#include <algorithm>
#include <cmath>
#include "nnv_internal.h"
#include "serving.h"

using namespace nnv;

namespace {

inline bool off16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
inline bool off8(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 7) != 0; }
inline bool off4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) != 0; }

inline int finish(hipError_t e) { return e == hipSuccess ? NNV_OK : record_hip_error(e); }

// Sizes that the kernels' grids can hold.
constexpr int kMostLinearN = 1 << 22, kMostLinearK = 1 << 20, kMostLinearRows = 65535 * 16;
constexpr int kMostRows = 1 << 24, kMostRequests = 1 << 20;
constexpr int64_t kMostGroups = (1 << 24) - 1;        // workgroups of 256: a launch has fewer than 2^32 threads

int check_linear(const nnv_linear_desc *d) {
    if (!d) return NNV_E_NULL;
    if (d->n <= 0 || d->k <= 0 || d->n > kMostLinearN || d->k > kMostLinearK) return NNV_E_BAD_DESC;
    for (int t : {d->x_dtype, d->y_dtype, d->raw_dtype})
        if (t != NNV_F32 && t != NNV_F16 && t != NNV_BF16) return NNV_E_BAD_DESC;
    return NNV_OK;
}

// A buffer of a call, as bytes.
struct Bytes {
    uintptr_t at;
    size_t count;
    Bytes(const void *p, size_t n) : at(reinterpret_cast<uintptr_t>(p)), count(p ? n : 0) {}
    bool meets(const Bytes &o) const { return count && o.count && at < o.at + o.count && o.at < at + count; }
};

// Whether rows of two matrices meet, each given by its first row and the bytes from a row to the next (no fewer than a row has).  Columns of one buffer
// may lie between each other, so where the whole of both overlaps, the rows are gone through in the order that they lie in.
bool rows_meet(int m, Bytes a, int64_t a_stride, Bytes b, int64_t b_stride) {
    typedef unsigned __int128 Wide;
    const Wide a_end = a.at + (Wide)(m - 1) * a_stride + a.count, b_end = b.at + (Wide)(m - 1) * b_stride + b.count;
    if (a.at >= b_end || b.at >= a_end) return false;
    for (int i = 0, j = 0; i < m && j < m;) {
        const Wide x = a.at + (Wide)i * a_stride, y = b.at + (Wide)j * b_stride;
        if (x < y + b.count && y < x + a.count) return true;
        if (x < y) ++i; else ++j;
    }
    return false;
}

int element_bytes(int dtype) { return dtype == NNV_F32 ? 4 : 2; }

int log2_of(int v) { int l = 0; while ((1 << l) < v) ++l; return l; }

int check_attention(const nnv_attention_desc *d) {
    if (!d) return NNV_E_NULL;
    if (d->q_heads <= 0 || d->kv_heads <= 0 || d->head_dim <= 0 || d->block_tokens <= 0 || d->blocks <= 0 || d->table_blocks <= 0) return NNV_E_BAD_DESC;
    if (d->blocks > 1 << 30) return NNV_E_BAD_DESC;
    if (d->q_heads > 1024 || d->q_heads % d->kv_heads) return NNV_E_BAD_DESC;
    if (d->rotary_dim < 0 || d->rotary_dim % 2 || d->rotary_dim > d->head_dim || (d->rotary_dim > 0 && d->positions <= 0)) return NNV_E_BAD_DESC;
    if (d->rotary_interleaved != 0 && d->rotary_interleaved != 1) return NNV_E_BAD_DESC;
    if (d->window < 0 || d->sinks < 0) return NNV_E_BAD_DESC;
    if (!std::isfinite(d->scale) || !std::isfinite(d->eps) || d->eps < 0) return NNV_E_BAD_DESC;
    if (d->dtype != NNV_F16 && d->dtype != NNV_BF16 && d->dtype != NNV_F32) return NNV_E_BAD_DESC;
    // a request's tokens are counted in 32 bits
    if ((int64_t)d->table_blocks * d->block_tokens > INT32_MAX / 2) return NNV_E_BAD_DESC;
    if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256) return NNV_E_UNSUPPORTED;
    if (d->block_tokens < 16 || d->block_tokens > 256 || (d->block_tokens & (d->block_tokens - 1))) return NNV_E_UNSUPPORTED;
    if (d->dtype == NNV_F32) return NNV_E_UNSUPPORTED;
    return NNV_OK;
}

int check_counts(int n_requests, int n_rows) {
    return n_requests < 0 || n_rows < 0 || n_requests > kMostRequests || n_rows > kMostRows ? NNV_E_ARG : NNV_OK;
}

}  // namespace

extern "C" {

size_t nnv_linear_transformed_bytes(const nnv_linear_desc *desc) { return check_linear(desc) ? 0 : linear_transformed_bytes(*desc); }

size_t nnv_linear_workspace_bytes(const nnv_linear_desc *desc, int m) {
    return check_linear(desc) || m <= 0 || m > kMostLinearRows ? 0 : linear_workspace_bytes(*desc, m);
}

int nnv_linear_transform_weights(const nnv_linear_desc *desc, const void *w_raw, void *w_tx, void *hip_stream) {
    if (const int rc = check_linear(desc)) return rc;
    if (!w_raw || !w_tx) return NNV_E_NULL;
    if (off16(w_raw) || off16(w_tx)) return NNV_E_ALIGN;
    return finish(launch_linear_pack(*desc, w_raw, w_tx, static_cast<hipStream_t>(hip_stream)));
}

int nnv_linear_forward(const nnv_linear_desc *desc, int m, const void *x, int64_t ldx, const void *w_tx, const float *bias, void *y,
                       int64_t ldy, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (const int rc = check_linear(desc)) return rc;
    if (m < 0 || m > kMostLinearRows) return NNV_E_ARG;
    if (m == 0) return NNV_OK;
    if (m > 1 && (ldx < desc->k || ldy < desc->n)) return NNV_E_ARG;
    if (!x || !w_tx || !y) return NNV_E_NULL;
    const size_t need = linear_workspace_bytes(*desc, m);
    if (need && !workspace) return NNV_E_NULL;
    if (workspace_bytes < need) return NNV_E_WORKSPACE;
    if (off16(x) || off16(w_tx) || off16(y) || (need && off16(workspace)) || (bias && off4(bias))) return NNV_E_ALIGN;
    const int xb = element_bytes(desc->x_dtype), yb = element_bytes(desc->y_dtype);
    // (workgroups of other outputs still read x)
    if (rows_meet(m, {x, (size_t)desc->k * xb}, m > 1 ? ldx * xb : 0, {y, (size_t)desc->n * yb}, m > 1 ? ldy * yb : 0)) return NNV_E_ARG;
    return finish(launch_linear(*desc, m, x, ldx, w_tx, bias, y, ldy, workspace, static_cast<hipStream_t>(hip_stream)));
}

size_t nnv_kv_cache_bytes(const nnv_attention_desc *desc) {
    if (check_attention(desc)) return 0;
    return (size_t)desc->blocks * desc->kv_heads * KvLayout{desc->head_dim, desc->block_tokens}.head_bytes();
}

int nnv_kv_plan(const nnv_attention_desc *desc, int n_requests, int n_rows, const int32_t *held, const int32_t *fresh,
                const int32_t *free_blocks, const int32_t *free_count, int32_t *block_table, int32_t *starts, int32_t *lengths,
                int32_t *positions, int64_t *slots, int32_t *free_left, void *hip_stream) {
    if (const int rc = check_attention(desc)) return rc;
    if (const int rc = check_counts(n_requests, n_rows)) return rc;
    if (!free_blocks || !free_count || !starts || !free_left) return NNV_E_NULL;
    if (n_requests && (!held || !fresh || !block_table || !lengths)) return NNV_E_NULL;
    if (n_rows && (!positions || !slots)) return NNV_E_NULL;
    if (off4(held) || off4(fresh) || off4(free_blocks) || off4(free_count) || off4(block_table) || off4(starts) || off4(lengths) ||
        off4(positions) || off8(slots) || off4(free_left))
        return NNV_E_ALIGN;
    // A workgroup reads all requests while others write: no output may lie in an input or in another output.  (How much of the free list is
    // read is known on the device: here its first entry.)
    const size_t n = n_requests, r = n_rows;
    const Bytes buffers[] = {{held, 4 * n}, {fresh, 4 * n}, {free_blocks, 4}, {free_count, 4}, {block_table, 4 * n * desc->table_blocks}, {starts, 4 * (n + 1)},
                             {lengths, 4 * n}, {positions, 4 * r}, {slots, 8 * r}, {free_left, 4}};
    for (int out = 4; out < 10; ++out)
        for (int other = 0; other < out; ++other)
            if (buffers[out].meets(buffers[other])) return NNV_E_ARG;
    PlanArgs a{held, fresh, free_blocks, free_count, block_table, starts, lengths, positions, free_left, slots, n_requests, n_rows,
               log2_of(desc->block_tokens), desc->blocks, desc->table_blocks};
    return finish(launch_kv_plan(a, static_cast<hipStream_t>(hip_stream)));
}

int nnv_qk_norm_rope(const nnv_attention_desc *desc, int n_rows, const void *q, int64_t ldq, const void *k, int64_t ldk, const void *v, int64_t ldv,
                     const float *q_weight, const float *k_weight, const float *rope, const int32_t *positions, const int64_t *slots, void *q_out,
                     void *k_out, void *cache, void *hip_stream) {
    if (const int rc = check_attention(desc)) return rc;
    if (const int rc = check_counts(0, n_rows)) return rc;
    if (n_rows == 0 || (!q && !k)) return NNV_OK;
    const int64_t dq = (int64_t)desc->q_heads * desc->head_dim, dk = (int64_t)desc->kv_heads * desc->head_dim;
    if (n_rows * (dq + 2 * dk) / 8 > INT32_MAX) return NNV_E_ARG;      // (threads are numbered in 32 bits)
    if (n_rows > 1 && ((q && ldq < dq) || (k && ldk < dk) || (k && cache && ldv < dk))) return NNV_E_ARG;
    if (!positions || (q && !q_out) || (desc->rotary_dim && !rope) || (k && !cache && !k_out) || (k && cache && (!v || !slots))) return NNV_E_NULL;
    if (off16(q) || off16(k) || off16(v) || off16(q_weight) || off16(k_weight) || off16(rope) || off4(positions) || off8(slots) || off16(q_out) ||
        off16(k_out) || off16(cache))
        return NNV_E_ALIGN;
    RopeArgs a{q, k, v, ldq, ldk, ldv, q_weight, k_weight, rope, positions, slots, q_out, k_out, static_cast<char *>(k ? cache : nullptr), n_rows,
               desc->q_heads, desc->kv_heads, desc->rotary_dim, desc->rotary_interleaved, desc->positions, log2_of(desc->block_tokens),
               (int64_t)desc->blocks * desc->block_tokens, desc->eps};
    return finish(launch_qk_norm_rope(a, desc->head_dim, desc->dtype, static_cast<hipStream_t>(hip_stream)));
}

int nnv_kv_read(const nnv_attention_desc *desc, int n, const int64_t *slots, const void *cache, void *k, void *v, void *hip_stream) {
    if (const int rc = check_attention(desc)) return rc;
    if (n < 0 || (int64_t)n * desc->kv_heads * (desc->head_dim / 8) * 2 > kMostGroups * 256) return NNV_E_ARG;
    if (n == 0 || (!k && !v)) return NNV_OK;
    if (!slots || !cache) return NNV_E_NULL;
    if (off8(slots) || off16(cache) || off16(k) || off16(v)) return NNV_E_ALIGN;
    return finish(launch_kv_read(n, slots, static_cast<const char *>(cache), k, v, desc->kv_heads, desc->head_dim, log2_of(desc->block_tokens),
                                 (int64_t)desc->blocks * desc->block_tokens, desc->dtype, static_cast<hipStream_t>(hip_stream)));
}

size_t nnv_kv_attention_workspace_bytes(const nnv_attention_desc *desc, int n_requests, int n_rows) {
    if (check_attention(desc) || check_counts(n_requests, n_rows) || n_rows == 0 ||
        kv_attention_groups(*desc, n_requests, n_rows) > kMostGroups)
        return 0;
    return kv_attention_workspace_bytes(*desc, n_requests, n_rows);
}

int nnv_kv_attention(const nnv_attention_desc *desc, int n_requests, int n_rows, const void *q, const int32_t *block_table, const int32_t *starts,
                     const int32_t *lengths, const int32_t *positions, const void *cache, void *out, void *workspace, size_t workspace_bytes,
                     void *hip_stream) {
    if (const int rc = check_attention(desc)) return rc;
    if (const int rc = check_counts(n_requests, n_rows)) return rc;
    if (n_rows == 0) return NNV_OK;
    if (kv_attention_groups(*desc, n_requests, n_rows) > kMostGroups) return NNV_E_ARG;
    if (!q || !starts || !positions || !cache || !out || (n_requests && (!block_table || !lengths))) return NNV_E_NULL;
    const size_t need = kv_attention_workspace_bytes(*desc, n_requests, n_rows);
    if (need && !workspace) return NNV_E_NULL;
    if (workspace_bytes < need) return NNV_E_WORKSPACE;
    if (off16(q) || off4(block_table) || off4(starts) || off4(lengths) || off4(positions) || off16(cache) || off16(out) || (need && off16(workspace)))
        return NNV_E_ALIGN;
    AttendArgs a{};
    a.q = q; a.table = block_table; a.starts = starts; a.lengths = lengths; a.positions = positions;
    a.cache = static_cast<const char *>(cache); a.out = out;
    a.requests = n_requests; a.rows = n_rows; a.q_heads = desc->q_heads; a.kv_heads = desc->kv_heads; a.group = desc->q_heads / desc->kv_heads;
    a.block_log = log2_of(desc->block_tokens); a.blocks = desc->blocks; a.width = desc->table_blocks; a.window = desc->window;
    a.sinks = (int)std::min((int64_t)desc->sinks, (int64_t)desc->table_blocks * desc->block_tokens);     // (no more than there can be: sums of it stay within 32 bits)
    a.scale = std::fmax(std::fabs(desc->scale) * 1.4426950408889634f, 1e-30f);
    a.flip = desc->scale < 0 ? (int)0x80008000u : 0;
    return finish(launch_kv_attention(*desc, a, workspace, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"

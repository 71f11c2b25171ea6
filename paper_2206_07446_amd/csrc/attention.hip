// Attention over a cache of keys and values held in 4 bits, in blocks.
//
// A tile is 16 rows of the matrix products: consecutive (row, query head of the group) pairs of one request and one key/value head, so that
// the heads of a group read the cache once.  Scores are K Q^T (16 tokens x 16 rows a 16x16x32 instruction: lane l holds the four tokens 4 (l / 16) ..
// of row l % 16), outputs V^T P^T, with the weights of a lane's own tokens as its part of the second operand: token
// 4 g + j of the first 16 and of the second 16 of a step of 32 are entries j and 4 + j of lane group g.  The products sum over tokens in any
// order as long as both operands keep to the same one, so the weights never leave their lanes.
//
// Tokens go to the products by conversion instructions that apply the scale, two values each.  Keys come out in pairs along
// a head, as scores need them; values in pairs along a head too, and two permutes make pairs along the tokens of two of them.
#include "nnv_internal.h"
#include "serving.h"
#include "lowbits.h"

namespace nnv {

constexpr int kStep = 32;          // tokens of a wavefront's step
constexpr int kTileRows = 16;
constexpr int kAttendWaves = 4;

template <int DT> struct Mfma;
template <> struct Mfma<NNV_F16> {
    typedef ElemVec<NNV_F16, 8> V8;
    static __device__ f32x4_t dot(i32x4_t a, i32x4_t b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
    }
    template <int SEL> static __device__ int pair(uint32_t w, float scale) { return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, SEL)); }
};
template <> struct Mfma<NNV_BF16> {
    typedef ElemVec<NNV_BF16, 8> V8;
    static __device__ f32x4_t dot(i32x4_t a, i32x4_t b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
    }
    template <int SEL> static __device__ int pair(uint32_t w, float scale) { return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL)); }
};

template <int DT> __device__ static inline int round_pair(float a, float b) {
    ElemVec<DT, 2> v = {(typename Elem<DT>::type)a, (typename Elem<DT>::type)b};
    return __builtin_bit_cast(int, v);
}

// Eight codes of a word as an operand.
template <int DT> __device__ static inline i32x4_t octet(uint32_t w, float scale) {
    return i32x4_t{Mfma<DT>::template pair<0>(w, scale), Mfma<DT>::template pair<1>(w, scale), Mfma<DT>::template pair<2>(w, scale),
                   Mfma<DT>::template pair<3>(w, scale)};
}

template <int DT> __device__ static inline float clamped_scale(uint32_t byte) { return scale_of_byte(min(byte, kMostE2m1Byte<DT>)); }

// A tile of a request: which rows, and which steps of tokens they see: [0, sink_steps) and [first_step, first_step + steps - sink_steps).
struct Tile {
    int request, row0, pair0, pairs;     // first row of the request, first (row, head) pair of the tile, pairs in it
    int length, steps, sink_steps, first_step;
    __device__ int step_at(int i) const { return i < sink_steps ? i : first_step + i - sink_steps; }
};

// Finds tile u.  Tiles of request i start at floor(starts[i] * group / 16) + i: enough for its pairs, with gaps; request `requests` stands for the
// rows that belong to none.  All threads of the workgroup take part (scratch: 3 ints).  pairs = 0 for a gap.
__device__ static inline Tile find_tile(const AttendArgs &a, int u, int *scratch) {
    Tile t;
    const int tid = threadIdx.x, n = blockDim.x;
    if (tid == 0) { scratch[0] = 0; scratch[1] = -1; scratch[2] = 0x7fffffff; }
    __syncthreads();
    // starts are clamped, but may still descend where they are no plan's: the count below is in range whatever they hold
    int mine = 0;
    for (int i = tid; i <= a.requests; i += n) {
        const int64_t start = min(max(a.starts[i], 0), a.rows);
        mine += start * a.group / kTileRows + i <= u ? 1 : 0;
    }
    for (int s = 1; s < 64; s *= 2) mine += __shfl_xor(mine, s);
    if ((tid & 63) == 0) atomicAdd(&scratch[0], mine);
    __syncthreads();
    t.request = max(scratch[0] - 1, 0);
    const int start = min(max(a.starts[t.request], 0), a.rows);
    const int end = t.request < a.requests ? min(max(a.starts[t.request + 1], 0), a.rows) : a.rows;
    const int local = u - ((int)((int64_t)start * a.group / kTileRows) + t.request);
    t.row0 = start;
    t.pair0 = local * kTileRows;
    const int64_t left = (int64_t)(end - start) * a.group - (int64_t)local * kTileRows;
    t.pairs = (int)min(max(left, (int64_t)0), (int64_t)kTileRows);
    if (local < 0) t.pairs = 0;
    const int64_t capacity = (int64_t)a.width << a.block_log;
    t.length = t.request < a.requests ? (int)min((int64_t)max(a.lengths[t.request], 0), capacity) : 0;
    // positions of the tile's rows: the last token any of them sees, and the first behind the sinks
    if (tid < t.pairs) {
        const int p = a.positions[t.row0 + (t.pair0 + tid) / a.group];
        if (p >= 0) {
            atomicMax(&scratch[1], p);
            atomicMin(&scratch[2], a.window ? max(0, p - a.window + 1) : 0);
        }
    }
    __syncthreads();
    const int end_token = min(scratch[1], t.length - 1) + 1, from = scratch[1] < 0 ? 0 : scratch[2];
    t.sink_steps = a.window ? min((a.sinks + kStep - 1) / kStep, (end_token + kStep - 1) / kStep) : 0;
    t.first_step = max(from / kStep, t.sink_steps);
    t.steps = end_token > 0 ? t.sink_steps + max(0, (end_token + kStep - 1) / kStep - t.first_step) : 0;
    return t;
}

// Steps of a split: whole rounds of the wavefronts.
__device__ static inline int steps_each(int steps, int splits) {
    const int rounds = (steps + kAttendWaves - 1) / kAttendWaves;
    return (rounds + splits - 1) / splits * kAttendWaves;
}

// What a wavefront loads of a step, as it lies in the cache.
template <int DIM> struct Held {
    uint32_t key[2][DIM / 32];        // of two tokens, DIM / 4 values each from d = DIM/4 * (lane / 16)
    uint32_t key_scale[2];            // a byte per 32 values of these (DIM = 256: two)
    uint32_t value[2][DIM / 32];      // of two fours of tokens, DIM / 16 values each from d = DIM/16 * (lane % 16)
    uint32_t value_scale[2];          // a byte per token
};

template <int N> __device__ static inline void load_words(const char *p, uint32_t (&w)[N]) {
    if constexpr (N == 2) {
        const i32x2_t v = *reinterpret_cast<const i32x2_t *>(p);
        w[0] = v[0]; w[1] = v[1];
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const i32x4_t v = *reinterpret_cast<const i32x4_t *>(p + 4 * i);
            w[i] = v[0]; w[i + 1] = v[1]; w[i + 2] = v[2]; w[i + 3] = v[3];
        }
    }
}

template <int DIM> __device__ static inline void load_step(const AttendArgs &a, const int32_t *table, int head, int step, int length, Held<DIM> &h, int (&ok)[2]) {
    const int lane = threadIdx.x & 63, col = lane % 16, g = lane / 16, block = 1 << a.block_log;
    const KvLayout at{DIM, block};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int token0 = step * kStep + i * 16;        // 16 tokens lie in one block
        const int b = token0 >> a.block_log;
        const int id = token0 < length ? table[b] : -1;
        ok[i] = id >= 0 && id < a.blocks;
        if (!ok[i]) {
#pragma unroll
            for (int j = 0; j < DIM / 32; ++j) h.key[i][j] = h.value[i][j] = 0;
            h.key_scale[i] = h.value_scale[i] = 0;
            continue;
        }
        const char *p = a.cache + ((int64_t)id * a.kv_heads + head) * at.head_bytes();
        const int token = token0 & (block - 1);
        load_words(p + (token + col) * (DIM / 2) + g * (DIM / 8), h.key[i]);
        const char *ks = p + at.key_scale_at() + (token + col) * (DIM / 32);
        if constexpr (DIM == 256) h.key_scale[i] = *reinterpret_cast<const uint16_t *>(ks + 2 * g);
        else h.key_scale[i] = *reinterpret_cast<const uint8_t *>(ks + (DIM == 128 ? g : g / 2));
        const int four = token / 4 + g;
        load_words(p + at.value_at() + (four * 16 + col) * (DIM / 8), h.value[i]);
        h.value_scale[i] = *reinterpret_cast<const uint32_t *>(p + at.value_scale_at() + (four * (DIM / 32) + col * (DIM / 16) / 32) * 4);
    }
}

// One (tile, key/value head, split): its wavefronts take steps in turn, each with a running maximum and sum of its own, and are joined in the LDS.
template <int DT, int DIM>
__global__ __launch_bounds__(64 * kAttendWaves) void kv_attend(AttendArgs a) {
    typedef typename Elem<DT>::type T;
    constexpr int kQ = DIM / 32, kJ = DIM / 16;          // instructions of a score, of an output
    __shared__ int scratch[3];
    __shared__ float join[kAttendWaves][kTileRows][DIM + 4];
    __shared__ float join_max[kAttendWaves][kTileRows], join_sum[kAttendWaves][kTileRows];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane % 16, g = lane / 16;
    const int u = blockIdx.x % a.tiles, rest = blockIdx.x / a.tiles, head = rest % a.kv_heads, split = rest / a.kv_heads;
    const Tile t = find_tile(a, u, scratch);
    if (t.pairs == 0) return;
    const int each = steps_each(t.steps, a.splits), begin = split * each, end = min(t.steps, begin + each);
    if (split > 0 && begin >= end) return;
    const bool whole = each >= t.steps;                  // no other split has any steps

    const int pair = t.pair0 + col;
    const bool there = col < t.pairs;
    const int row = t.row0 + pair / a.group, qh = head * a.group + pair % a.group;
    const int own = there ? a.positions[row] : -1, position = min(own, t.length - 1);
    i32x4_t q[kQ];
#pragma unroll
    for (int s = 0; s < kQ; ++s)
        q[s] = there ? *reinterpret_cast<const i32x4_t *>(static_cast<const T *>(a.q) + ((int64_t)row * a.q_heads + qh) * DIM + g * (DIM / 4) + s * 8)
                     : i32x4_t{0, 0, 0, 0};
    f32x4_t o[kJ];
#pragma unroll
    for (int j = 0; j < kJ; ++j) o[j] = f32x4_t{0, 0, 0, 0};
    float most = -INFINITY, sum = 0;
    const int32_t *table = a.table + (int64_t)t.request * a.width;
    const int last_seen = a.window ? own - a.window : -1;            // tokens up to this one are seen as sinks only

    for (int i = begin + wave; i < end; i += kAttendWaves) {
        const int step = t.step_at(i);
        Held<DIM> h;
        int ok[2];
        load_step<DIM>(a, table, head, step, t.length, h, ok);
        float p[8];
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            f32x4_t s = {0, 0, 0, 0};
#pragma unroll
            for (int d = 0; d < kQ; ++d) {
                const uint32_t byte = DIM == 256 && d >= kQ / 2 ? h.key_scale[k] >> 8 : h.key_scale[k] & 255;
                s = Mfma<DT>::dot(octet<DT>(h.key[k][d], clamped_scale<DT>(byte)), q[d], s);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int token = step * kStep + k * 16 + g * 4 + r;
                const bool seen = ok[k] && token <= position && (token > last_seen || token < a.sinks);
                p[k * 4 + r] = seen ? s[r] * a.scale : -INFINITY;
                top = fmaxf(top, p[k * 4 + r]);
            }
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = fmaxf(most, top);
        const float base = now == -INFINITY ? 0.f : now;             // a row that has seen nothing yet: exp2(-inf) below, not of a NaN
        const float keep = exp2f(most - base);
        most = now;
        float part = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            p[e] = exp2f(p[e] - base);
            part += p[e];
        }
        sum = sum * keep + part;
        const i32x4_t weights = {round_pair<DT>(p[0], p[1]), round_pair<DT>(p[2], p[3]), round_pair<DT>(p[4], p[5]), round_pair<DT>(p[6], p[7])};
        // values: words of eight codes, kJ codes to a token
        float scale[2][4];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) scale[k][r] = clamped_scale<DT>((h.value_scale[k] >> (8 * r)) & 255);
        auto pairs_of = [&](int k, int r, int jj) {       // codes 2 jj, 2 jj + 1 of token r of four k
            const int code = r * kJ + 2 * jj;
            const uint32_t w = h.value[k][code / 8];
            const int sel = code % 8 / 2;
            return sel == 0 ? Mfma<DT>::template pair<0>(w, scale[k][r]) : sel == 1 ? Mfma<DT>::template pair<1>(w, scale[k][r])
                 : sel == 2 ? Mfma<DT>::template pair<2>(w, scale[k][r]) : Mfma<DT>::template pair<3>(w, scale[k][r]);
        };
#pragma unroll
        for (int jj = 0; jj < kJ / 2; ++jj) {
            i32x4_t even, odd;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int r = 0; r < 4; r += 2) {
                    const uint32_t x = pairs_of(k, r, jj), y = pairs_of(k, r + 1, jj);
                    even[k * 2 + r / 2] = (int)__builtin_amdgcn_perm(y, x, 0x05040100);
                    odd[k * 2 + r / 2] = (int)__builtin_amdgcn_perm(y, x, 0x07060302);
                }
            o[2 * jj] = Mfma<DT>::dot(even, weights, o[2 * jj] * keep);
            o[2 * jj + 1] = Mfma<DT>::dot(odd, weights, o[2 * jj + 1] * keep);
        }
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);

    // lane: row col, values (4 g + r) * kJ + j
    if (g == 0) { join_max[wave][col] = most; join_sum[wave][col] = sum; }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < kJ; ++j) join[wave][col][(4 * g + r) * kJ + j] = o[j][r];
    __syncthreads();
    // a thread joins values of a row in the order of the wavefronts
    for (int e = threadIdx.x; e < t.pairs * DIM; e += 64 * kAttendWaves) {
        const int c = e / DIM, d = e % DIM;
        float m = -INFINITY, l = 0, v = 0;
#pragma unroll
        for (int w = 0; w < kAttendWaves; ++w) m = fmaxf(m, join_max[w][c]);
        const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int w = 0; w < kAttendWaves; ++w) {
            const float f = exp2f(join_max[w][c] - base);
            l += join_sum[w][c] * f;
            v += join[w][c][d] * f;
        }
        const int pr = t.pair0 + c;
        const int64_t out_row = (int64_t)(t.row0 + pr / a.group) * a.q_heads + head * a.group + pr % a.group;
        if (whole) {
            static_cast<T *>(a.out)[out_row * DIM + d] = (T)(l > 0 ? v / l : 0.f);
        } else {
            float *p = a.parts + (out_row * a.splits + split) * (DIM + 2);
            p[d] = v;
            if (d == 0) { p[DIM] = m; p[DIM + 1] = l; }
        }
    }
}

// Joins the splits of a tile in their order.
template <int DT, int DIM>
__global__ __launch_bounds__(256) void kv_attend_join(AttendArgs a) {
    typedef typename Elem<DT>::type T;
    __shared__ int scratch[3];
    const int u = blockIdx.x % a.tiles, head = blockIdx.x / a.tiles;
    const Tile t = find_tile(a, u, scratch);
    const int each = steps_each(t.steps, a.splits);
    if (t.pairs == 0 || each >= t.steps) return;
    const int splits = (t.steps + each - 1) / each;
    for (int e = threadIdx.x; e < t.pairs * DIM; e += 256) {
        const int pr = t.pair0 + e / DIM, d = e % DIM;
        const int64_t out_row = (int64_t)(t.row0 + pr / a.group) * a.q_heads + head * a.group + pr % a.group;
        const float *p = a.parts + out_row * a.splits * (DIM + 2);
        float m = -INFINITY, l = 0, v = 0;
        for (int s = 0; s < splits; ++s) m = fmaxf(m, p[s * (DIM + 2) + DIM]);
        const float base = m == -INFINITY ? 0.f : m;
        for (int s = 0; s < splits; ++s) {
            const float f = exp2f(p[s * (DIM + 2) + DIM] - base);
            l += p[s * (DIM + 2) + DIM + 1] * f;
            v += p[s * (DIM + 2) + d] * f;
        }
        static_cast<T *>(a.out)[out_row * DIM + d] = (T)(l > 0 ? v / l : 0.f);
    }
}

static int attend_tiles(int requests, int rows, int group) { return (int)(((int64_t)rows * group) / kTileRows) + requests + 1; }

int64_t kv_attention_groups(const nnv_attention_desc &d, int requests, int rows) {
    return ((int64_t)rows * (d.q_heads / d.kv_heads) / kTileRows + requests + 1) * d.kv_heads;
}

// Splits of a tile's tokens, from what the host knows: enough that the tiles fill the chip, and that no split is longer than 2048 tokens
// where a request may be, within 256 MB of partial sums.
static int attend_splits(const nnv_attention_desc &d, int requests, int rows) {
    const int64_t capacity = (int64_t)d.table_blocks * d.block_tokens;
    const int64_t groups = kv_attention_groups(d, requests, rows);
    int64_t s = (1024 + groups - 1) / groups;
    if (s < (capacity + 2047) / 2048) s = (capacity + 2047) / 2048;
    if (s > (capacity + 255) / 256) s = (capacity + 255) / 256;
    const int64_t per = (int64_t)rows * d.q_heads * (d.head_dim + 2) * 4;
    while (s > 1 && (s * per > (int64_t)256 << 20 || s * groups > (int64_t)1 << 30)) s = s / 2;
    return (int)(s < 1 ? 1 : s);
}

size_t kv_attention_workspace_bytes(const nnv_attention_desc &d, int requests, int rows) {
    const int s = attend_splits(d, requests, rows);
    return s == 1 ? 0 : (size_t)rows * d.q_heads * s * (d.head_dim + 2) * 4;
}

template <int DT, int DIM> static hipError_t launch_attend_dim(const AttendArgs &a, hipStream_t st) {
    kv_attend<DT, DIM><<<(unsigned)(a.tiles * a.kv_heads * a.splits), 64 * kAttendWaves, 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    kv_attend_join<DT, DIM><<<(unsigned)(a.tiles * a.kv_heads), 256, 0, st>>>(a);
    return hipGetLastError();
}
template <int DT> static hipError_t launch_attend_type(const AttendArgs &a, int dim, hipStream_t st) {
    return dim == 64 ? launch_attend_dim<DT, 64>(a, st) : dim == 128 ? launch_attend_dim<DT, 128>(a, st) : launch_attend_dim<DT, 256>(a, st);
}

hipError_t launch_kv_attention(const nnv_attention_desc &d, const AttendArgs &args, void *ws, hipStream_t st) {
    AttendArgs a = args;
    a.tiles = attend_tiles(a.requests, a.rows, a.group);
    a.splits = attend_splits(d, a.requests, a.rows);
    a.parts = static_cast<float *>(ws);
    return d.dtype == NNV_F16 ? launch_attend_type<NNV_F16>(a, d.head_dim, st) : launch_attend_type<NNV_BF16>(a, d.head_dim, st);
}

}  // namespace nnv

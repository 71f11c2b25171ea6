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

// Over the 16 lanes of a row, everywhere.
__device__ static inline int row_max(int v) {
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0xb1, 0xf, 0xf, false));      // lanes xor 1
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x4e, 0xf, 0xf, false));      // xor 2
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x141, 0xf, 0xf, false));     // mirrored halves of a row
    return max(v, __builtin_amdgcn_update_dpp(v, v, 0x140, 0xf, 0xf, false));  // mirrored row
}
__device__ static inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A tile of a request: which rows, and which steps of tokens they see: [0, sink_steps) and [first_step, first_step + steps - sink_steps).
struct Tile {
    int request, row0, pair0, pairs;     // first row of the request, first (row, head) pair of the tile, pairs in it
    int position;                        // of the row of column lane % 16; -1 of a column that is no pair
    int lowest, highest;                 // of the tile's positions; lowest -1 where a row sees nothing
    int length, steps, sink_steps, first_step;
    __device__ int step_at(int i) const { return i < sink_steps ? i : first_step + i - sink_steps; }
};

// Finds tile u.  Tiles of request i start at floor(starts[i] * group / 16) + i: enough for its pairs, with gaps; request `requests` stands for the
// rows that belong to none.  Every wavefront does so by itself: 64 starts at a time are compared with u, so that 4096 requests
// take two loads one after the other.  pairs = 0 for a gap.  Whatever starts, lengths and positions hold, the tile stays within a.rows rows.
__device__ static inline Tile find_tile(const AttendArgs &a, int u) {
    Tile t;
    const int lane = threadIdx.x & 63;
    int lo = 0, span = a.requests + 1;
    while (span > 1) {
        const int each = (span + 63) / 64, i = lo + lane * each;
        const bool reached = lane * each < span && (int64_t)min(max(a.starts[i], 0), a.rows) * a.group / kTileRows + i <= u;
        const int n = max(__builtin_popcountll(__ballot(reached)), 1);
        lo += (n - 1) * each;
        span = min(each, span - (n - 1) * each);
    }
    t.request = uniform(lo);
    const int start = min(max(a.starts[t.request], 0), a.rows);
    const int end = t.request < a.requests ? min(max(a.starts[t.request + 1], 0), a.rows) : a.rows;
    const int local = u - ((int)((int64_t)start * a.group / kTileRows) + t.request);
    const int64_t left = (int64_t)(end - start) * a.group - (int64_t)local * kTileRows;
    t.row0 = start;
    t.pair0 = local * kTileRows;
    t.pairs = local < 0 ? 0 : (int)min(max(left, (int64_t)0), (int64_t)kTileRows);
    t.length = t.request < a.requests ? (int)min((int64_t)max(a.lengths[t.request], 0), (int64_t)a.width << a.block_log) : 0;
    const int col = lane % 16;
    t.position = col < t.pairs ? a.positions[t.row0 + (t.pair0 + col) / a.group] : -1;
    t.highest = uniform(row_max(t.position));
    t.lowest = -uniform(row_max(col < t.pairs ? -max(t.position, -1) : -0x7fffffff));
    // the lowest of the rows that see anything
    const int seeing = t.lowest >= 0 ? t.lowest : -uniform(row_max(t.position >= 0 ? -t.position : -0x7fffffff));
    const int end_token = min(t.highest, t.length - 1) + 1, end_step = (end_token + kStep - 1) / kStep;
    t.sink_steps = a.window ? min((a.sinks + kStep - 1) / kStep, end_step) : 0;
    t.first_step = max(a.window ? max(seeing - a.window + 1, 0) / kStep : 0, t.sink_steps);
    t.steps = end_token > 0 ? t.sink_steps + max(0, end_step - t.first_step) : 0;
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

// Blocks of the two sixteens of a step (a sixteen lies in one block); -1: none, or behind the request's tokens.
struct StepBlocks { int id[2]; };
__device__ static inline StepBlocks blocks_of(const AttendArgs &a, const int32_t *table, int step, int length) {
    StepBlocks s;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int token0 = step * kStep + i * 16;
        const int id = token0 < length ? table[token0 >> a.block_log] : -1;
        s.id[i] = id >= 0 && id < a.blocks ? id : -1;
    }
    return s;
}

// Of a block that is none, block 0 is read in its place; its tokens are not seen.
template <int DIM> __device__ static inline void load_step(const AttendArgs &a, int head, int step, StepBlocks blocks, Held<DIM> &h) {
    const int lane = threadIdx.x & 63, col = lane % 16, g = lane / 16;
    const KvLayout at{DIM, 1 << a.block_log};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int token = (step * kStep + i * 16) & (at.tokens - 1), id = max(blocks.id[i], 0);
        const char *p = a.cache + ((int64_t)id * a.kv_heads + head) * at.head_bytes();
        load_words(p + token * (DIM / 2) + (col * (DIM / 2) + g * (DIM / 8)), h.key[i]);
        load_words(p + (at.value_at() + token * (DIM / 2)) + (g * 16 + col) * (DIM / 8), h.value[i]);
        const char *ks = p + (at.key_scale_at() + token * (DIM / 32)) + col * (DIM / 32);
        if constexpr (DIM == 256) h.key_scale[i] = *reinterpret_cast<const uint16_t *>(ks + 2 * g);
        else h.key_scale[i] = *reinterpret_cast<const uint8_t *>(ks + (DIM == 128 ? g : g / 2));
        h.value_scale[i] = *reinterpret_cast<const uint32_t *>(p + (at.value_scale_at() + token * (DIM / 32)) + (g * (DIM / 32) + col * (DIM / 16) / 32) * 4);
    }
}

constexpr int kPartExtra = 4;      // floats of a partial result behind its values: base, sum, number of splits

// One (tile, key/value head, split): its wavefronts take steps in turn, each with a softmax of its own, and are joined in the LDS.  The next
// step's loads are in flight while one is computed, the block numbers of the one after that too.
//
// A column's scores are taken relative to a base that all its lanes share.  It need not be the maximum: it is raised,
// and what was summed is scaled down, only when a score of the wavefront lies 2^8 above it, which past the
// first steps is hardly ever; weights up to 2^8 cost the sums in float32 and the rounding to 16 bits nothing.
template <int DT, int DIM>
__global__ __launch_bounds__(64 * kAttendWaves, DIM == 256 ? 2 : 4) void kv_attend(AttendArgs a) {
    typedef typename Elem<DT>::type T;
    constexpr int kQ = DIM / 32, kJ = DIM / 16;          // instructions of a score, of an output
    __shared__ float join[kAttendWaves][kTileRows][DIM / 2 + 4];
    __shared__ float join_base[kAttendWaves][kTileRows], join_sum[kAttendWaves][kTileRows];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane % 16, g = lane / 16;
    const int u = blockIdx.x % a.tiles, rest = blockIdx.x / a.tiles, head = rest % a.kv_heads, split = rest / a.kv_heads;
    const Tile t = find_tile(a, u);
    if (t.pairs == 0) return;
    const int each = steps_each(t.steps, a.splits), begin = split * each, end = min(t.steps, begin + each);
    if (split > 0 && begin >= end) return;
    const bool whole = each >= t.steps;                  // no other split has any steps

    const int32_t *table = a.table + (int64_t)t.request * a.width;
    Held<DIM> held;
    StepBlocks blocks = {{-1, -1}}, next_blocks = {{-1, -1}};
    if (begin + wave < end) {
        blocks = blocks_of(a, table, t.step_at(begin + wave), t.length);
        load_step<DIM>(a, head, t.step_at(begin + wave), blocks, held);
        if (begin + wave + kAttendWaves < end) next_blocks = blocks_of(a, table, t.step_at(begin + wave + kAttendWaves), t.length);
    }
    const int pair = t.pair0 + col;
    const bool there = col < t.pairs;
    const int row = t.row0 + pair / a.group, qh = head * a.group + pair % a.group;
    const int position = min(t.position, t.length - 1), last_sink = a.window ? t.position - a.window : -1;    // tokens up to this one are seen as sinks only
    i32x4_t q[kQ];
#pragma unroll
    for (int s = 0; s < kQ; ++s)
        q[s] = there ? *reinterpret_cast<const i32x4_t *>(static_cast<const T *>(a.q) + ((int64_t)row * a.q_heads + qh) * DIM + g * (DIM / 4) + s * 8)
                     : i32x4_t{0, 0, 0, 0};
    f32x4_t o[kJ];
#pragma unroll
    for (int j = 0; j < kJ; ++j) o[j] = f32x4_t{0, 0, 0, 0};
    float base = -3.4028234663852886e38f, sum = 0;
    const int full_to = min(t.lowest, t.length - 1);                       // steps that end here or before are seen by all rows,
    const int full_from = a.window ? t.highest - a.window + 1 : 0;        // if they begin here or behind

    for (int i = begin + wave; i < end; i += kAttendWaves) {
        const int step = t.step_at(i);
        Held<DIM> next;
        StepBlocks later = {{-1, -1}};
        if (i + kAttendWaves < end) {
            load_step<DIM>(a, head, t.step_at(i + kAttendWaves), next_blocks, next);
            if (i + 2 * kAttendWaves < end) later = blocks_of(a, table, t.step_at(i + 2 * kAttendWaves), t.length);
        }
        f32x4_t s[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            s[k] = f32x4_t{0, 0, 0, 0};
#pragma unroll
            for (int d = 0; d < kQ; ++d) {
                const uint32_t byte = DIM != 256 ? held.key_scale[k] : d >= kQ / 2 ? held.key_scale[k] >> 8 : held.key_scale[k] & 255;
                s[k] = Mfma<DT>::dot(octet<DT>(held.key[k][d], scale_of_byte(byte)), q[d], s[k]);
            }
        }
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = s[e / 4][e % 4] * a.scale;
        const int token0 = step * kStep;
        if (token0 + kStep - 1 > full_to || (token0 < full_from && token0 + kStep > a.sinks) || blocks.id[0] < 0 || blocks.id[1] < 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int token = token0 + e / 4 * 16 + g * 4 + e % 4;
                const bool seen = blocks.id[e / 4] >= 0 && token <= position && (token > last_sink || token < a.sinks);
                p[e] = seen ? p[e] : -INFINITY;
            }
            // codes and scales of what is not held may be anything: a weight of 0 needs a finite value beside it
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const bool is = blocks.id[k] >= 0 && token0 + k * 16 + g * 4 + r < t.length;
                    held.value_scale[k] &= is ? 0xffffffffu : ~(0xffu << (8 * r));
                }
        }
        float top = fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7])));
        if (__any(top > base + 8.f)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float now = fmaxf(base, top), keep = __builtin_amdgcn_exp2f(base - now);
            base = now;
            sum *= keep;
#pragma unroll
            for (int j = 0; j < kJ; ++j) o[j] *= keep;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(p[e] - base);
        sum += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
        const i32x4_t weights = {round_pair<DT>(p[0], p[1]), round_pair<DT>(p[2], p[3]), round_pair<DT>(p[4], p[5]), round_pair<DT>(p[6], p[7])};
        // values: words of eight codes, kJ codes to a token
        float scale[2][4];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) scale[k][r] = scale_of_byte((held.value_scale[k] >> (8 * r)) & 255);
        auto pairs_of = [&](int k, int r, int jj) {       // codes 2 jj, 2 jj + 1 of token r of four k
            const int code = r * kJ + 2 * jj;
            const uint32_t w = held.value[k][code / 8];
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
            o[2 * jj] = Mfma<DT>::dot(even, weights, o[2 * jj]);
            o[2 * jj + 1] = Mfma<DT>::dot(odd, weights, o[2 * jj + 1]);
        }
        held = next;
        blocks = next_blocks;
        next_blocks = later;
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);

    // lane: column col, values (4 g + r) * kJ + j; joined in the order of the wavefronts, half of the values at a time
    if (g == 0) { join_base[wave][col] = base; join_sum[wave][col] = sum; }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if (half) __syncthreads();
        if (g / 2 == half)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int j = 0; j < kJ; ++j) join[wave][col][(4 * (g & 1) + r) * kJ + j] = o[j][r];
        __syncthreads();
        for (int e = threadIdx.x; e < t.pairs * (DIM / 2); e += 64 * kAttendWaves) {
            const int c = e / (DIM / 2), d = e % (DIM / 2);
            float m = join_base[0][c], l = 0, v = 0;
#pragma unroll
            for (int w = 1; w < kAttendWaves; ++w) m = fmaxf(m, join_base[w][c]);
#pragma unroll
            for (int w = 0; w < kAttendWaves; ++w) {
                const float f = __builtin_amdgcn_exp2f(join_base[w][c] - m);
                l += join_sum[w][c] * f;
                v += join[w][c][d] * f;
            }
            const int pr = t.pair0 + c;
            const int64_t out_row = (int64_t)(t.row0 + pr / a.group) * a.q_heads + head * a.group + pr % a.group;
            float *part = a.parts + (out_row * a.splits + split) * (DIM + kPartExtra);
            if (whole) static_cast<T *>(a.out)[out_row * DIM + half * (DIM / 2) + d] = (T)(l > 0 ? v / l : 0.f);
            else part[half * (DIM / 2) + d] = v;
            if (half == 0 && d == 0 && a.splits > 1) {
                part[DIM] = m;
                part[DIM + 1] = l;
                part[DIM + 2] = __builtin_bit_cast(float, whole ? 1 : (t.steps + each - 1) / each);
            }
        }
    }
}

constexpr int kMostSplits = 128;

// Joins the splits of a row and query head in their order, a workgroup each: the splits' factors first, then 1024 / DIM groups of lanes take splits in
// turn, four values a lane, and add up in the LDS.
template <int DT, int DIM>
__global__ __launch_bounds__(256) void kv_attend_join(AttendArgs a) {
    typedef typename Elem<DT>::type T;
    constexpr int kLanes = DIM / 4, kGroups = 256 / kLanes;
    __shared__ float factor[kMostSplits], bases[4], sums[4];
    __shared__ f32x4_t part[kGroups][kLanes];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float *p = a.parts + (int64_t)blockIdx.x * a.splits * (DIM + kPartExtra);
    const int splits = __builtin_bit_cast(int, p[DIM + 2]);
    if (splits <= 1) return;
    const bool mine = tid < splits;
    const float base = mine ? p[tid * (DIM + kPartExtra) + DIM] : -3.4028234663852886e38f;
    float m = base;
    for (int s = 1; s < 64; s *= 2) m = fmaxf(m, __shfl_xor(m, s));
    if (lane == 0) bases[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(bases[0], bases[1]), fmaxf(bases[2], bases[3]));
    const float f = mine ? __builtin_amdgcn_exp2f(base - m) : 0.f;
    float l = mine ? p[tid * (DIM + kPartExtra) + DIM + 1] * f : 0.f;
    for (int s = 1; s < 64; s *= 2) l += __shfl_xor(l, s);
    if (lane == 0) sums[wave] = l;
    if (mine) factor[tid] = f;
    __syncthreads();
    l = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    const int group = tid / kLanes, at = tid % kLanes;
    f32x4_t v = {0, 0, 0, 0};
#pragma unroll 4
    for (int s = group; s < splits; s += kGroups) v += *reinterpret_cast<const f32x4_t *>(p + s * (DIM + kPartExtra) + 4 * at) * factor[s];
    part[group][at] = v;
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int i = 1; i < kGroups; ++i) v += part[i][at];
    ElemVec<DT, 4> y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (T)(l > 0 ? v[i] / l : 0.f);
    *reinterpret_cast<ElemVec<DT, 4> *>(static_cast<T *>(a.out) + (int64_t)blockIdx.x * DIM + 4 * at) = y;
}

static int attend_tiles(int requests, int rows, int group) { return (int)(((int64_t)rows * group) / kTileRows) + requests + 1; }

int64_t kv_attention_groups(const nnv_attention_desc &d, int requests, int rows) {
    return ((int64_t)rows * (d.q_heads / d.kv_heads) / kTileRows + requests + 1) * d.kv_heads;
}

// Splits of a tile's tokens, from what the host knows: 1024 workgroups where there are that few (four to a compute unit; with 512 to 4096 one
// request of 32768 tokens and 8 heads takes the same 20 us), of at least 512 tokens (with 256 it takes 24 us, more partial
// results to join), at most 2048 of them, or 8192 where there are tiles enough, within 256 MB of partial results.
static int attend_splits(const nnv_attention_desc &d, int requests, int rows) {
    const int64_t capacity = (int64_t)d.table_blocks * d.block_tokens;
    const int64_t reach = d.window && (int64_t)d.window + d.sinks < capacity ? (int64_t)d.window + d.sinks : capacity;
    const int64_t pairs = (int64_t)rows * (d.q_heads / d.kv_heads), least = requests < rows ? requests : rows;
    const int64_t tiles = pairs / kTileRows > least ? pairs / kTileRows : least;
    const int64_t groups = (tiles > 0 ? tiles : 1) * d.kv_heads;
    int64_t s = (1024 + groups - 1) / groups;
    const int64_t longest = groups >= 2048 ? 8192 : 2048;
    if (s < (reach + longest - 1) / longest) s = (reach + longest - 1) / longest;
    if (s > (reach + 511) / 512) s = (reach + 511) / 512;
    if (s > kMostSplits) s = kMostSplits;
    const int64_t per = (int64_t)rows * d.q_heads * (d.head_dim + kPartExtra) * 4;
    while (s > 1 && (s * per > (int64_t)256 << 20 || s * kv_attention_groups(d, requests, rows) > (int64_t)1 << 30)) s = s / 2;
    return (int)(s < 1 ? 1 : s);
}

size_t kv_attention_workspace_bytes(const nnv_attention_desc &d, int requests, int rows) {
    const int s = attend_splits(d, requests, rows);
    return s == 1 ? 0 : (size_t)rows * d.q_heads * s * (d.head_dim + kPartExtra) * 4;
}

template <int DT, int DIM> static hipError_t launch_attend_dim(const AttendArgs &a, hipStream_t st) {
    kv_attend<DT, DIM><<<(unsigned)(a.tiles * a.kv_heads * a.splits), 64 * kAttendWaves, 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    kv_attend_join<DT, DIM><<<(unsigned)(a.rows * a.q_heads), 256, 0, st>>>(a);
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

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
constexpr int kManyPairs = 32;     // pairs of a request from which on kv_attend_many takes it, where both kernels run

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

// Weights as they are rounded for the products, in powers of two: what the largest is given when a column's base is raised, and the most that one may be before
// it is raised again.  bfloat16 has float32's exponents.  float16's numbers end at 2^16, and those below 2^-14 have fewer bits: with the largest at 2^10
// or more, a weight keeps all its bits down to 2^-24 of the largest, and is off by 2^-35 of that at most below; thousands of tokens beside one that lies far above
// them then count for what they are.
template <int DT> struct WeightRange { static constexpr float kTop = 0, kMost = 8; };
template <> struct WeightRange<NNV_F16> { static constexpr float kTop = 10, kMost = 15; };

// The base that a largest score asks for; where float32 has no number kTop below it, none that gives a weight of more than kMost.
template <int DT> __device__ static inline float raised(float base, float top) {
    const float now = fmaxf(base, top - WeightRange<DT>::kTop);
    return top - now > WeightRange<DT>::kMost ? top : now;
}
// Scores in powers of two have their product with the factor rounded before the base is taken off, so that the largest is its base's own however large it is: in
// one instruction with that, which sees the product unrounded, the two are apart by half a step of float32 at that size, more than a weight can stand from 2^24 or so.
__device__ static inline float in_twos(float score, float scale) {
#pragma clang fp contract(off)
    return score * scale;
}
// kv_attend_many, where vector instructions count (4 prompts of 1024 rows 134 -> 155 us with heads of 64, 213 -> 222 with 128), does that only for bases beyond 2^12
// (but not for that of a column that has seen nothing): up to there the two are 2^-13 apart, and no rounding to 16 bits sees it.
__device__ static inline bool far_out(float base) { return __any(fabsf(base) > 0x1p12f && base > -3e38f); }

// Over the 16 lanes of a row, everywhere.
__device__ static inline int row_max(int v) {
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0xb1, 0xf, 0xf, false));      // lanes xor 1
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x4e, 0xf, 0xf, false));      // xor 2
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x141, 0xf, 0xf, false));     // mirrored halves of a row
    return max(v, __builtin_amdgcn_update_dpp(v, v, 0x140, 0xf, 0xf, false));  // mirrored row
}
__device__ static inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ static inline int wave_max(int v) {
    v = row_max(v);
    v = max(v, __shfl_xor(v, 16));
    return uniform(max(v, __shfl_xor(v, 32)));
}

// x / group for x below 2 x 1024: rounded up 2^21 / group times x is off by less than x * group <= 2^21 parts of 2^21.
__device__ static inline int by_group(const AttendArgs &a, int x) { return (int)((uint32_t)x * a.group_inverse >> 21); }

// A tile of a request: R consecutive pairs of a row and a query head of the group.
struct Tile {
    int request, row0, pair0, pairs;     // first row of the request, first pair of the tile, pairs in it
    int request_pairs, length;
};

// Whatever starts and lengths hold, a tile stays within a.rows rows.
__device__ static inline int clamped_start(const AttendArgs &a, int v) { return min(max(v, 0), a.rows); }

// Tile `local` of a request, from what starts and lengths hold for it.
template <int R> __device__ static inline Tile tile_of(const AttendArgs &a, int request, int start, int end, int length, int64_t local) {
    Tile t;
    const int64_t all = max((int64_t)(end - start) * a.group, (int64_t)0);
    t.request = request;
    t.row0 = start;
    t.pair0 = (int)(local * R);
    t.pairs = local < 0 ? 0 : (int)min(max(all - local * R, (int64_t)0), (int64_t)R);
    t.request_pairs = (int)min(all, (int64_t)0x7fffffff);
    t.length = (int)min((int64_t)max(length, 0), (int64_t)a.width << a.block_log);
    return t;
}

// Finds tile u.  Tiles of request i start at floor(starts[i] * group / R) + i: enough for its pairs, with gaps (pairs = 0); request `requests`
// stands for the rows that belong to none.  Every wavefront does so by itself: 64 starts at a time are compared with u, and in the last round,
// the only one of up to 63 requests, come with the starts after them and the lengths, so that a chain of loads is one link long.
template <int R> __device__ static inline Tile find_tile(const AttendArgs &a, int u) {
    const int lane = threadIdx.x & 63;
    int lo = 0, span = a.requests + 1;
    for (;;) {
        const int each = (span + 63) / 64, i = lo + lane * each;
        const bool mine = lane * each < span, request = mine && i < a.requests;
        const int start = mine ? clamped_start(a, a.starts[i]) : a.rows;
        const int end = each == 1 && request ? clamped_start(a, a.starts[i + 1]) : a.rows, length = each == 1 && request ? a.lengths[i] : 0;
        const int n = max(__builtin_popcountll(__ballot(mine && (int64_t)start * a.group / R + i <= u)), 1);
        lo = uniform(lo + (n - 1) * each);
        span = uniform(min(each, span - (n - 1) * each));
        if (each == 1) {
            const int at = uniform(n - 1), from = __builtin_amdgcn_readlane(start, at);
            return tile_of<R>(a, lo, from, __builtin_amdgcn_readlane(end, at), __builtin_amdgcn_readlane(length, at), u - ((int64_t)from * a.group / R + lo));
        }
    }
}

// Tile u of up to 63 requests with those of the longest requests first, and of each the last: every lane adds up the tiles of the
// requests before its own.  The tiles that take longest then begin first, and the end of a launch is not theirs (4 prompts of 1024 rows over 876 to
// 6000 tokens: see kv_attend_many).
template <int R> __device__ static inline Tile find_longest(const AttendArgs &a, int u) {
    const int lane = threadIdx.x & 63;
    const bool mine = lane <= a.requests, request = lane < a.requests;
    const int start = mine ? clamped_start(a, a.starts[lane]) : a.rows, end = request ? clamped_start(a, a.starts[lane + 1]) : a.rows;
    const int length = request ? a.lengths[lane] : mine ? 0 : -1;
    const int tiles = (int)((max((int64_t)(end - start) * a.group, (int64_t)0) + R - 1) / R);
    int before = 0;
    for (int j = 0; j <= a.requests; ++j) {
        const int other = __builtin_amdgcn_readlane(length, j);
        if (other > length || (other == length && j < lane)) before += __builtin_amdgcn_readlane(tiles, j);
    }
    const uint64_t found = __ballot(mine && before <= u && u < before + tiles);
    if (!found) {
        Tile none{};
        return none;
    }
    const int at = __builtin_ctzll(found);
    return tile_of<R>(a, at, __builtin_amdgcn_readlane(start, at), __builtin_amdgcn_readlane(end, at), __builtin_amdgcn_readlane(length, at),
                      __builtin_amdgcn_readlane(before + tiles, at) - 1 - u);
}

// Which steps of S tokens rows at positions `lowest` (of those that see anything) to `highest` see: [0, sinks) and [first, first + count - sinks).
struct Steps {
    int count, sinks, first;
    __device__ int at(int i) const { return i < sinks ? i : first + i - sinks; }
};
template <int S> __device__ static inline Steps steps_of(const AttendArgs &a, int lowest, int highest, int length) {
    const int end_token = min(highest, length - 1) + 1, end = (end_token + S - 1) / S;
    Steps s;
    s.sinks = a.window ? min((a.sinks + S - 1) / S, end) : 0;
    s.first = max(a.window ? max(lowest - a.window + 1, 0) / S : 0, s.sinks);
    s.count = end_token > 0 ? s.sinks + max(0, end - s.first) : 0;
    return s;
}

// Steps of a split: whole rounds of the wavefronts.
__device__ static inline int steps_each(int steps, int splits) {
    const int rounds = (steps + kAttendWaves - 1) / kAttendWaves;
    return (rounds + splits - 1) / splits * kAttendWaves;
}

// Eight values of a query; their signs turned where the factor of the scores is negative, so that the kernels' own is not.
__device__ static inline i32x4_t query_words(const void *p, int flip) {
    const i32x4_t v = *static_cast<const i32x4_t *>(p);
    return i32x4_t{v[0] ^ flip, v[1] ^ flip, v[2] ^ flip, v[3] ^ flip};
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

// A request's row of the block table, in the address space of constants: nothing here writes it, and its entries are read by the scalar unit.
typedef const __attribute__((address_space(4))) int32_t *TableRow;
__device__ static inline TableRow table_row(const AttendArgs &a, int request) {
    return reinterpret_cast<TableRow>(reinterpret_cast<uintptr_t>(a.table + (int64_t)request * a.width));
}

// Blocks of the two sixteens of a step (a sixteen lies in one block); -1: none, or behind the request's tokens.
struct StepBlocks { int id[2]; };
__device__ static inline StepBlocks blocks_of(const AttendArgs &a, TableRow table, int step, int length) {
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
    const uint32_t lane = threadIdx.x & 63, col = lane % 16, g = lane / 16;
    const KvLayout at{DIM, 1 << a.block_log};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int token = (step * kStep + i * 16) & (at.tokens - 1), id = max(blocks.id[i], 0);
        const char *p = a.cache + ((int64_t)id * a.kv_heads + head) * at.head_bytes();
        const char *keys = p + token * (DIM / 2), *values = p + at.value_at() + token * (DIM / 2);
        const char *key_scales = p + at.key_scale_at() + token * (DIM / 32), *value_scales = p + at.value_scale_at() + token * (DIM / 32);
        load_words(keys + (col * (DIM / 2) + g * (DIM / 8)), h.key[i]);
        if constexpr (DIM == 256) h.key_scale[i] = *reinterpret_cast<const uint16_t *>(key_scales + (col * (DIM / 32) + 2 * g));
        else h.key_scale[i] = *reinterpret_cast<const uint8_t *>(key_scales + (col * (DIM / 32) + (DIM == 128 ? g : g / 2)));
        load_words(values + (g * 16 + col) * (DIM / 8), h.value[i]);
        h.value_scale[i] = *reinterpret_cast<const uint32_t *>(value_scales + (g * (DIM / 32) + col * (DIM / 16) / 32) * 4);
    }
}

constexpr int kPartExtra = 4;      // floats of a partial result behind its values: base, sum, number of splits

// Where there is much to read (64 rows over up to 8192 tokens, 287 MB: 71 us, 4.0 TB/s; a copy moves 5.2 TB/s here, half of it reads) vector instructions take 51 % of a
// compute unit's busy time and its wavefronts wait for 46 % of theirs, so that neither is shown to bound alone; where there is little, the chain of starts, table
// and codes does (one row over 32768 tokens, 36 MB: 16 us).
// One (tile, key/value head, split): its wavefronts take steps in turn, each with a softmax of its own, and are joined in the LDS.  The next
// step's loads are in flight while one is computed, the block numbers of the one after that too.
//
// A column's scores are taken relative to a base that all its lanes share.  It need not be the maximum: it is raised,
// and what was summed is scaled down, only when a weight of the wavefront would pass the most of WeightRange, which past the
// first steps is hardly ever.
template <int DT, int DIM>
__global__ __launch_bounds__(64 * kAttendWaves, DIM == 256 ? 2 : 4) void kv_attend(AttendArgs a) {
    typedef typename Elem<DT>::type T;
    constexpr int kQ = DIM / 32, kJ = DIM / 16;          // instructions of a score, of an output
    __shared__ float join[kAttendWaves][kTileRows][DIM / 2 + 4];
    __shared__ float join_base[kAttendWaves][kTileRows], join_sum[kAttendWaves][kTileRows];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane % 16, g = lane / 16;
    const int u = blockIdx.x % a.tiles, rest = blockIdx.x / a.tiles, head = rest % a.kv_heads, split = rest / a.kv_heads;
    // beside kv_attend_many, requests of fewer than 32 pairs: two tiles each
    static_assert(kManyPairs <= 2 * kTileRows, "two tiles hold them");
    const Tile t = a.many ? tile_of<kTileRows>(a, u / 2, clamped_start(a, a.starts[u / 2]), clamped_start(a, a.starts[u / 2 + 1]), a.lengths[u / 2], u % 2)
                          : find_tile<kTileRows>(a, u);
    if (t.pairs == 0 || (a.many && t.request_pairs >= kManyPairs)) return;
    const bool there = col < t.pairs;
    const int pair = t.pair0 + col, row = t.row0 + pair / a.group, qh = head * a.group + pair % a.group, own = there ? a.positions[row] : -1;
    i32x4_t q[kQ];
#pragma unroll
    for (int s = 0; s < kQ; ++s)
        q[s] = there ? query_words(static_cast<const T *>(a.q) + ((int64_t)row * a.q_heads + qh) * DIM + g * (DIM / 4) + s * 8, a.flip) : i32x4_t{0, 0, 0, 0};
    // Without a window the steps are those of the request's length, so that the first codes need not wait for the positions; the
    // last of them may be masked whole.
    Steps steps = {t.length > 0 ? (t.length + kStep - 1) / kStep : 0, 0, 0};
    if (a.window) {
        const int seeing = -uniform(row_max(own >= 0 ? -own : -0x7fffffff));
        steps = steps_of<kStep>(a, seeing, uniform(row_max(own)), t.length);
    }
    const int each = steps_each(steps.count, a.splits), begin = split * each, end = min(steps.count, begin + each);
    if (split > 0 && begin >= end) return;
    const bool whole = each >= steps.count;              // no other split has any steps

    const TableRow table = table_row(a, t.request);
    // the last step of this wavefront is loaded again where there is no next one: a load that some rounds leave out would
    // make every round wait for all that are on their way
    Held<DIM> held_a, held_b;
    StepBlocks blocks = {{-1, -1}}, next_blocks = {{-1, -1}};
    const int first = begin + wave, last = first + (end - 1 - first) / kAttendWaves * kAttendWaves;
    if (first < end) {
        blocks = blocks_of(a, table, steps.at(first), t.length);
        next_blocks = blocks_of(a, table, steps.at(min(first + kAttendWaves, last)), t.length);
        load_step<DIM>(a, head, steps.at(first), blocks, held_a);
    }
    const int highest = uniform(row_max(own)), lowest = -uniform(row_max(there ? -max(own, -1) : -0x7fffffff));
    const int position = min(own, t.length - 1), last_sink = a.window ? own - a.window : -1;    // tokens up to this one are seen as sinks only
    f32x4_t o[kJ];
#pragma unroll
    for (int j = 0; j < kJ; ++j) o[j] = f32x4_t{0, 0, 0, 0};
    float base = -3.4028234663852886e38f, sum = 0;
    const int full_to = min(lowest, t.length - 1);                       // steps that end here or before are seen by all rows,
    const int full_from = a.window ? highest - a.window + 1 : 0;        // if they begin here or behind

    __builtin_amdgcn_s_waitcnt(0xf70);                    // vmcnt 0: the queries are here before the rounds begin
    auto round = [&](int i, Held<DIM> &held, Held<DIM> &next) {
        const int step = steps.at(i);
        load_step<DIM>(a, head, steps.at(min(i + kAttendWaves, last)), next_blocks, next);
        const StepBlocks later = blocks_of(a, table, steps.at(min(i + 2 * kAttendWaves, last)), t.length);
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
        for (int e = 0; e < 8; ++e) p[e] = in_twos(s[e / 4][e % 4], a.scale);
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
        if (__any(top - base > WeightRange<DT>::kMost)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float now = raised<DT>(base, top), keep = __builtin_amdgcn_exp2f(base - now);
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
        blocks = next_blocks;
        next_blocks = later;
    };
    // two rounds at a time, so that codes stay in the registers that they were loaded into
    for (int i = first; i < end;) {
        round(i, held_a, held_b);
        i += kAttendWaves;
        if (i >= end) break;
        round(i, held_b, held_a);
        i += kAttendWaves;
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
            if (whole) static_cast<T *>(a.out)[out_row * DIM + half * (DIM / 2) + d] = (T)(l == 0 ? 0.f : v / l);
            else part[half * (DIM / 2) + d] = v;
            if (half == 0 && d == 0 && a.splits > 1) {
                part[DIM] = m;
                part[DIM + 1] = l;
                part[DIM + 2] = __builtin_bit_cast(float, whole ? 1 : (steps.count + each - 1) / each);
            }
        }
    }
}

// Requests of many rows: a workgroup holds 128 pairs, 32 to a wavefront, and goes over the tokens 64 at a time.  Each wavefront turns the codes of 16
// of them into operands in the LDS, once for all 128 pairs, where kv_attend would do so for every 16; the codes of the tokens after
// that are on their way meanwhile.  Keys lie there as [32 tokens][16 values][8 of them][token], values as [32 values][16 tokens][8 of them][value],
// every 16 bytes a lane's part of an operand.  The four lanes' worth of a token's values that a lane has in hand go to rows that lie 8 apart;
// the row is xor-ed with its sixteen, so that they meet different banks, and reading does so as well.
// The conversions run beside the scores' products, the exponentials beside the outputs'.  4 prompts of 1024 rows over 876 to 6000 tokens, 32 heads of
// 128 and 8 of keys: 203-213 us, 0.93-0.97 PFLOP/s of what the rows see; vector instructions take 60 % of a compute unit's busy time, matrix ones 47 %,
// and two workgroups that do not wait for one another are what lets them overlap (one of eight wavefronts for 256 pairs, with half the
// conversions: 327 us).
constexpr int kManyStep = 64, kManyRows = 128;

template <int DT> struct Mfma32;
template <> struct Mfma32<NNV_F16> {
    static __device__ f32x16_t dot(i32x4_t a, i32x4_t b, f32x16_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(Mfma<NNV_F16>::V8, a), __builtin_bit_cast(Mfma<NNV_F16>::V8, b), c, 0, 0, 0);
    }
};
template <> struct Mfma32<NNV_BF16> {
    static __device__ f32x16_t dot(i32x4_t a, i32x4_t b, f32x16_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Mfma<NNV_BF16>::V8, a), __builtin_bit_cast(Mfma<NNV_BF16>::V8, b), c, 0, 0, 0);
    }
};

// What a wavefront loads of its 16 tokens: of a lane's token and quarter of a head the key's codes, of two fours of tokens the values'.
template <int DIM> struct HeldMany { uint32_t key[DIM / 32], key_scale, value[2][DIM / 32], value_scale[2]; };

// Where a lane finds these in a head's part of a block, but for the token: the rest of an address is the same for all lanes.
template <int DIM> struct ManyPlaces {
    uint32_t key, key_scale, key_shift, value, value_scale;      // (key_scale: of the word that the scale's byte lies in, key_shift: bits before it)
    __device__ ManyPlaces(const KvLayout &at, uint32_t lane) {
        const uint32_t col = lane % 16, g = lane / 16, four = g % 2;
        key = col * (DIM / 2) + g * (DIM / 8);
        const uint32_t byte = col * (DIM / 32) + (DIM == 256 ? 2 * g : DIM == 128 ? g : g / 2);
        key_scale = at.key_scale_at() + byte / 4 * 4;
        key_shift = byte % 4 * 8;
        value = at.value_at() + (four * 16 + col) * (DIM / 8);
        value_scale = at.value_scale_at() + (four * (DIM / 32) + col * (DIM / 16) / 32) * 4;
    }
};
template <int DIM> __device__ static inline void load_many(const char *block, uint32_t token, const ManyPlaces<DIM> &at, HeldMany<DIM> &h) {
    const uint32_t codes = token * (DIM / 2), scales = token * (DIM / 32);
    load_words(block + (at.key + codes), h.key);
    h.key_scale = *reinterpret_cast<const uint32_t *>(block + (at.key_scale + scales));
#pragma unroll
    for (int k = 0; k < 2; ++k) {                        // fours 0 or 1, then 2 or 3 of the sixteen
        load_words(block + (at.value + codes) + k * 32 * (DIM / 8), h.value[k]);
        h.value_scale[k] = *reinterpret_cast<const uint32_t *>(block + (at.value_scale + scales) + k * 2 * (DIM / 32) * 4);
    }
}

template <int DT, int DIM>
__global__ __launch_bounds__(256, DIM == 256 ? 1 : DIM == 128 ? 2 : 3) void kv_attend_many(AttendArgs a) {
    typedef typename Elem<DT>::type T;
    constexpr int kQ = DIM / 16, kJ = DIM / 16, kD = DIM / 32;
    // Which part of a step goes before other wavefronts' work (4 prompts of 1024 rows, 4096 pairs each: heads of 64 scores 241 us, weights and outputs 262,
    // neither 256; of 128 210, 205, 208; of 256 362 all).
    constexpr bool kScoresFirst = DIM == 64;
    __shared__ i32x4_t keys[2][2][kQ][2][32], values[2][kD][4][2][32];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane % 32, half = lane / 32;
    const int head = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads, u = rest % a.many_tiles, split = rest / a.many_tiles;
    const Tile t = a.ordered ? find_longest<kManyRows>(a, u) : find_tile<kManyRows>(a, u);
    if (t.pairs == 0 || (t.request < a.requests && t.request_pairs < kManyPairs)) return;
    // positions: of the tile for the steps, of the wavefront for its masks
    const int row0 = t.row0 + t.pair0 / a.group, rest0 = t.pair0 % a.group;       // row and head of the tile's first pair
    auto position_of = [&](int i) { return i < t.pairs ? a.positions[row0 + by_group(a, rest0 + i)] : -1; };
    const int p0 = position_of(lane), p1 = position_of(lane + 64);
    // the wavefront's queries
    const int i0 = wave * 32 + col;
    const bool there = i0 < t.pairs, idle = wave * 32 >= t.pairs;
    const int row = row0 + by_group(a, rest0 + i0), qh = head * a.group + (rest0 + i0) - by_group(a, rest0 + i0) * a.group;
    i32x4_t q[kQ];
#pragma unroll
    for (int s = 0; s < kQ; ++s)
        q[s] = there ? query_words(static_cast<const T *>(a.q) + ((int64_t)row * a.q_heads + qh) * DIM + s * 16 + half * 8, a.flip) : i32x4_t{0, 0, 0, 0};

    // The blocks of a step: lane l loads the entry of sixteen l % 4, through the vector unit, whose loads end in order (a scalar load on
    // its way would make every wait for the LDS one for all).  It is asked for three steps ahead, the codes two.
    const int32_t *table = a.table + (int64_t)t.request * a.width;
    auto token_of = [&](int step) { return step * kManyStep + lane % 4 * 16; };
    auto entry_at = [&](int step) { const int token = token_of(step); return table[token < t.length ? token >> a.block_log : 0]; };
    struct Blocks { int own, here; };                     // of the wavefront's sixteen, -1: none; a bit for each sixteen that has one
    auto blocks_at = [&](int step, int entry) {
        const bool is = token_of(step) < t.length && (uint32_t)entry < (uint32_t)a.blocks;
        return Blocks{__builtin_amdgcn_readlane(is ? entry : -1, wave), (int)__ballot(is) & 15};
    };
    const KvLayout layout{DIM, 1 << a.block_log};
    const ManyPlaces<DIM> places(layout, lane);
    const char *head_part = a.cache + (int64_t)head * layout.head_bytes();
    const uint32_t block_bytes = (uint32_t)a.kv_heads * layout.head_bytes();
    HeldMany<DIM> held;
    auto load = [&](int step, int id) {
        load_many<DIM>(head_part + (uint64_t)(uint32_t)max(id, 0) * block_bytes, (step * kManyStep + wave * 16) & (layout.tokens - 1), places, held);
    };
    // Without a window and splits the first steps are known before the positions are, and with them the first codes: the chain of loads
    // that a tile begins with is then one link shorter.
    const bool early = !a.window && a.splits == 1;
    const int held_steps = (t.length + kManyStep - 1) / kManyStep;
    int step = 0, step_1 = 0, step_2 = 0, entry = 0;      // this step and those after it
    Blocks these = {-1, 0}, next = {-1, 0};               // of this step and the next
    auto begin_at = [&](int s0, int s1, int s2) {
        step = s0;
        step_1 = s1;
        step_2 = s2;
        const int first = entry_at(step), second = entry_at(step_1);
        entry = entry_at(step_2);
        these = blocks_at(step, first);
        next = blocks_at(step_1, second);
        load(step, these.own);
    };
    if (early && held_steps > 0) begin_at(0, min(1, held_steps - 1), min(2, held_steps - 1));
    const int highest = wave_max(max(p0, p1));
    const int seeing = -wave_max(max(p0 >= 0 ? -p0 : -0x7fffffff, p1 >= 0 ? -p1 : -0x7fffffff));
    const Steps steps = steps_of<kManyStep>(a, seeing, highest, t.length);
    const int each = (steps.count + a.splits - 1) / a.splits, begin = split * each, end = min(steps.count, begin + each);
    if (split > 0 && begin >= end) return;
    const bool whole = each >= steps.count;
    auto clamped = [&](int i) { return steps.at(min(i, end - 1)); };       // behind the last step, that one again (see kv_attend)
    if (!early && begin < end) begin_at(steps.at(begin), clamped(begin + 1), clamped(begin + 2));
    const int own = __shfl(wave < 2 ? p0 : p1, wave % 2 * 32 + col);
    const int position = min(own, t.length - 1), last_sink = a.window ? own - a.window : -1;
    const int wave_lowest = -wave_max(there ? -max(own, -1) : -0x7fffffff), wave_highest = wave_max(own);
    const int full_to = min(wave_lowest, t.length - 1), full_from = a.window ? wave_highest - a.window + 1 : 0;
    f32x16_t o[kD];
#pragma unroll
    for (int d = 0; d < kD; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = 0;
    float base = -3.4028234663852886e38f, sum = 0;
    bool far = false;                                     // far_out(base)

    // what is not held may be anything: its values are to be finite, its scores are masked
    auto blank = [&](int step, int id) {
        const int g = lane / 16, h = g % 2, token0 = step * kManyStep + wave * 16;
        if (id >= 0 && token0 + 16 <= t.length) return;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool is = id >= 0 && token0 + (h + 2 * k) * 4 + r < t.length;
                held.value_scale[k] &= is ? 0xffffffffu : ~(0xffu << (8 * r));
            }
    };
    // The wavefront's sixteen tokens of a step into a buffer, in kQ pieces: eight values of a lane's key each, then halves of two values of eight tokens.
    const int c = lane % 16, g = lane / 16, upper = g / 2;
    i32x4_t even, odd;
    auto spread = [&](int buffer, int piece) {
        if (piece < kQ / 2) {
            const uint32_t byte = (held.key_scale >> (places.key_shift + (DIM == 256 && piece >= DIM / 64 ? 8 : 0))) & 255;
            const int octet_at = g * (DIM / 32) + piece;
            keys[buffer][wave / 2][octet_at / 2][octet_at % 2][wave % 2 * 16 + c] = octet<DT>(held.key[piece], scale_of_byte(byte));
            return;
        }
        const int jj = (piece - kQ / 2) / 2, k = piece % 2, d = c * kJ + upper * (kJ / 2) + 2 * jj;
        auto pair_at = [&](int r) {
            const float scale = scale_of_byte((held.value_scale[k] >> (8 * r)) & 255);
            uint32_t w;
            if constexpr (DIM == 256) w = upper ? held.value[k][2 * r + 1] : held.value[k][2 * r];
            else if constexpr (DIM == 128) w = held.value[k][r] >> (16 * upper);
            else w = held.value[k][r / 2] >> (16 * (r % 2) + 8 * upper);
            return (uint32_t)(jj == 0 ? Mfma<DT>::template pair<0>(w, scale) : jj == 1 ? Mfma<DT>::template pair<1>(w, scale)
                            : jj == 2 ? Mfma<DT>::template pair<2>(w, scale) : Mfma<DT>::template pair<3>(w, scale));
        };
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
            const uint32_t x = pair_at(r), y = pair_at(r + 1);
            even[k * 2 + r / 2] = (int)__builtin_amdgcn_perm(y, x, 0x05040100);
            odd[k * 2 + r / 2] = (int)__builtin_amdgcn_perm(y, x, 0x07060302);
        }
        if (k) {
            values[buffer][d / 32][wave][g % 2][(d % 32) ^ (d / 16)] = even;
            values[buffer][d / 32][wave][g % 2][((d + 1) % 32) ^ (d / 16)] = odd;
        }
    };
    if (begin < end) {
        blank(step, these.own);
#pragma unroll
        for (int d = 0; d < kQ; ++d) spread(0, d);
        load(step_1, next.own);
    }
    __builtin_amdgcn_s_waitcnt(0xf70);                    // vmcnt 0: the queries are here before the rounds begin
    __syncthreads();
    for (int i = begin; i < end; ++i) {
        const int buffer = (i - begin) & 1, token0 = step * kManyStep;
        blank(step_1, next.own);
        // scores, and in the shadow of their products the next step's codes into the other buffer
        f32x16_t s[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[b][r] = 0;
        if (kScoresFirst) __builtin_amdgcn_s_setprio(1);
        i32x4_t k[2][2] = {{keys[buffer][0][0][half][col], keys[buffer][1][0][half][col]}, {}};
#pragma unroll
        for (int d = 0; d < kQ; ++d) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if (d + 1 < kQ) k[(d + 1) & 1][b] = keys[buffer][b][d + 1][half][col];
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) s[b] = Mfma32<DT>::dot(k[d & 1][b], q[d], s[b]);
            spread(buffer ^ 1, d);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (kScoresFirst) __builtin_amdgcn_s_setprio(0);
        const Blocks later = blocks_at(step_2, entry);
        const int step_3 = clamped(i + 3);
        entry = entry_at(step_3);
        load(step_2, later.own);
        if (!idle && token0 <= min(wave_highest, t.length - 1)) {
            if (token0 + kManyStep - 1 > full_to || (token0 < full_from && token0 + kManyStep > a.sinks) || these.here != 15) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int token = token0 + b * 32 + 8 * (r / 4) + 4 * half + r % 4;
                        const bool seen = (these.here >> (2 * b + r / 8) & 1) && token <= position && (token > last_sink || token < a.sinks);
                        s[b][r] = seen ? s[b][r] : -INFINITY;
                    }
            }
            if (!kScoresFirst) __builtin_amdgcn_s_setprio(1);
            float top = -INFINITY;
#pragma unroll
            for (int e = 0; e < 32; ++e) top = fmaxf(top, s[e / 16][e % 16]);
            top *= a.scale;
            if (__any(top - base > WeightRange<DT>::kMost)) {
                top = fmaxf(top, __shfl_xor(top, 32));
                const float now = raised<DT>(base, top), keep = __builtin_amdgcn_exp2f(base - now);
                base = now;
                far = far_out(base);
                sum *= keep;
#pragma unroll
                for (int d = 0; d < kD; ++d) o[d] *= keep;
            }
            const float factor = far ? 1.f : a.scale, less = far ? 0.f : base;
            if (far)
#pragma unroll
                for (int e = 0; e < 32; ++e) s[e / 16][e % 16] = in_twos(s[e / 16][e % 16], a.scale) - base;
            float part[4] = {0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                s[e / 16][e % 16] = __builtin_amdgcn_exp2f(fmaf(s[e / 16][e % 16], factor, -less));
                part[e % 4] += s[e / 16][e % 16];
            }
            sum += (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const f32x16_t &p = s[k / 2];
                const int r = k % 2 * 8;
                const i32x4_t weights = {round_pair<DT>(p[r], p[r + 1]), round_pair<DT>(p[r + 2], p[r + 3]), round_pair<DT>(p[r + 4], p[r + 5]),
                                         round_pair<DT>(p[r + 6], p[r + 7])};
#pragma unroll
                for (int d = 0; d < kD; ++d) o[d] = Mfma32<DT>::dot(values[buffer][d][k][half][col ^ (2 * d + col / 16)], weights, o[d]);
            }
        }
        if (!kScoresFirst) __builtin_amdgcn_s_setprio(0);
        these = next;
        next = later;
        step = step_1;
        step_1 = step_2;
        step_2 = step_3;
        __syncthreads();
    }
    sum += __shfl_xor(sum, 32);
    if (!there) return;
    // lane: pair col, values 32 d + 8 (r / 4) + 4 half + r % 4
    const int64_t out_row = (int64_t)row * a.q_heads + qh;
    float *parts = a.parts + (out_row * a.splits + split) * (DIM + kPartExtra);
    const float inverse = sum == 0 ? 0.f : 1.f / sum;
#pragma unroll
    for (int d = 0; d < kD; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int at = 32 * d + 2 * r + 4 * half;
            if (whole) {
                ElemVec<DT, 4> y;
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = (T)(o[d][r + j] * inverse);
                *reinterpret_cast<ElemVec<DT, 4> *>(static_cast<T *>(a.out) + out_row * DIM + at) = y;
            } else {
                *reinterpret_cast<f32x4_t *>(parts + at) = f32x4_t{o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]};
            }
        }
    if (a.splits > 1 && half == 0) {
        parts[DIM] = base;
        parts[DIM + 1] = sum;
        parts[DIM + 2] = __builtin_bit_cast(float, whole ? 1 : (steps.count + each - 1) / each);
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
    // (what is read of splits that there are not is not used)
    const bool slot = tid < a.splits;
    const float own_base = slot ? p[tid * (DIM + kPartExtra) + DIM] : 0.f, own_sum = slot ? p[tid * (DIM + kPartExtra) + DIM + 1] : 0.f;
    // (a row that starts leave out has no partial results: what the workspace holds there may be any number)
    const int splits = min(__builtin_bit_cast(int, p[DIM + 2]), a.splits);
    if (splits <= 1) return;
    const bool mine = tid < splits;
    const float base = mine ? own_base : -3.4028234663852886e38f;
    float m = base;
    for (int s = 1; s < 64; s *= 2) m = fmaxf(m, __shfl_xor(m, s));
    if (lane == 0) bases[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(bases[0], bases[1]), fmaxf(bases[2], bases[3]));
    const float f = mine ? __builtin_amdgcn_exp2f(base - m) : 0.f;
    float l = mine ? own_sum * f : 0.f;
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
    for (int i = 0; i < 4; ++i) y[i] = (T)(l == 0 ? 0.f : v[i] / l);
    *reinterpret_cast<ElemVec<DT, 4> *>(static_cast<T *>(a.out) + (int64_t)blockIdx.x * DIM + 4 * at) = y;
}

static int attend_tiles(int requests, int rows, int group, int tile) { return (int)(((int64_t)rows * group) / tile) + requests + 1; }

int64_t kv_attention_groups(const nnv_attention_desc &d, int requests, int rows) {
    return ((int64_t)rows * (d.q_heads / d.kv_heads) / kTileRows + 2 * (int64_t)requests + 1) * d.kv_heads;
}

// Whether a request of many rows is to be expected: then both kernels run, each on the requests it is for.  (16 requests of 4 rows, group 4:
// 18 us by kv_attend, 21 with a launch beside it that finds nothing; 4 requests of 1024 rows: 412 us by kv_attend alone, 203 by both; 80 requests
// of 15 rows, group 4: 218 and 212.)
static bool attend_many(const nnv_attention_desc &d, int requests, int rows) { return (int64_t)(rows - requests) * (d.q_heads / d.kv_heads) >= 512; }

// Splits of a tile's tokens, from what the host knows: 1024 workgroups where there are that few (four to a compute unit), or 512 of up to 8 tiles of rows,
// which end together or have the chip to themselves (with 1024: 4 requests of up to 16000 tokens and 8 heads 22.5 us, 18.5 so; 8 of up to 12000 and 4 heads of 256
// 28.7, 23.1 so; but 16 requests of 8 rows, up to 4096 tokens and 8 heads 32 us with 1024, 36 with 512); of at least 512 tokens of as long a request as the
// table has room for (with 256 one request of 32768 tokens and 8 heads takes 26 us, more partial results to join, against 20; a shorter request beside it is cut into as
// many, down to a round of the wavefronts each), at most 2048 of them, or 8192 where there are tiles enough, within 256 MB of partial results.
static int attend_splits(const nnv_attention_desc &d, int requests, int rows) {
    // (One number for both kernels: running requests beside a prompt get the prompt's.)
    const int64_t capacity = (int64_t)d.table_blocks * d.block_tokens;
    const int64_t reach = d.window && (int64_t)d.window + d.sinks < capacity ? (int64_t)d.window + d.sinks : capacity;
    const bool many = attend_many(d, requests, rows);
    const int64_t pairs = (int64_t)rows * (d.q_heads / d.kv_heads), least = requests < rows ? requests : rows;
    const int64_t full = pairs / (many ? kManyRows : kTileRows), tiles = full > least ? full : least;
    const int64_t groups = (tiles > 0 ? tiles : 1) * d.kv_heads, fill = many || tiles <= 8 ? 512 : 1024;
    int64_t s = (fill + groups - 1) / groups;
    const int64_t longest = groups >= 2048 || many ? 8192 : 2048;
    if (s < (reach + longest - 1) / longest) s = (reach + longest - 1) / longest;
    if (s > (reach + 511) / 512) s = (reach + 511) / 512;
    if (s > kMostSplits) s = kMostSplits;
    const int64_t per = (int64_t)rows * d.q_heads * (d.head_dim + kPartExtra) * 4;
    while (s > 1 && (s * per > (int64_t)256 << 20 || s * kv_attention_groups(d, requests, rows) >= 1 << 24)) s = s / 2;
    return (int)(s < 1 ? 1 : s);
}

size_t kv_attention_workspace_bytes(const nnv_attention_desc &d, int requests, int rows) {
    const int s = attend_splits(d, requests, rows);
    return s == 1 ? 0 : (size_t)rows * d.q_heads * s * (d.head_dim + kPartExtra) * 4;
}

template <int DT, int DIM> static hipError_t launch_attend_dim(const AttendArgs &a, hipStream_t st) {
    if (a.many) {
        kv_attend_many<DT, DIM><<<(unsigned)(a.many_tiles * a.kv_heads * a.splits), 256, 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.tiles) kv_attend<DT, DIM><<<(unsigned)(a.tiles * a.kv_heads * a.splits), 64 * kAttendWaves, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    kv_attend_join<DT, DIM><<<(unsigned)(a.rows * a.q_heads), 256, 0, st>>>(a);
    return hipGetLastError();
}
template <int DT> static hipError_t launch_attend_type(const AttendArgs &a, int dim, hipStream_t st) {
    return dim == 64 ? launch_attend_dim<DT, 64>(a, st) : dim == 128 ? launch_attend_dim<DT, 128>(a, st) : launch_attend_dim<DT, 256>(a, st);
}

hipError_t launch_kv_attention(const nnv_attention_desc &d, const AttendArgs &args, void *ws, hipStream_t st) {
    AttendArgs a = args;
    a.many = attend_many(d, a.requests, a.rows);
    a.tiles = a.many ? 2 * a.requests : attend_tiles(a.requests, a.rows, a.group, kTileRows);
    a.many_tiles = attend_tiles(a.requests, a.rows, a.group, kManyRows);
    a.splits = attend_splits(d, a.requests, a.rows);
    a.parts = static_cast<float *>(ws);
    a.group_inverse = ((1u << 21) + a.group - 1) / a.group;
    // the order costs a loop over the requests, and is for tiles that take many steps
    a.ordered = a.requests < 64 && (int64_t)d.table_blocks * d.block_tokens > 1024;
    return d.dtype == NNV_F16 ? launch_attend_type<NNV_F16>(a, d.head_dim, st) : launch_attend_type<NNV_BF16>(a, d.head_dim, st);
}

}  // namespace nnv

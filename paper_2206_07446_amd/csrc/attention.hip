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

// Which tokens the rows of a launch see: all of their request's; of a group of requests those that they have in common; of a request those behind the ones that it
// has in common with others; both of these; or those of the blocks that a row and key head's list names.
enum Seen { kAll, kPrefix, kOwn, kListed, kBoth };

// A tile of a request: R consecutive pairs of a row and a query head of the group.
struct Tile {
    int request, row0, pair0, pairs;     // first row of the request, first pair of the tile, pairs in it
    int request_pairs, length;
};

// Whatever starts and lengths hold, a tile stays within a.rows rows.
__device__ static inline int clamped_start(const AttendArgs &a, int v) { return min(max(v, 0), a.rows); }

__device__ static inline int capacity_of(const AttendArgs &a) { return (int)min((int64_t)a.width << a.block_log, (int64_t)0x7fffffff); }

// Whatever groups and shared hold: the first request of group i (or of none), and how many tokens the group has in common.
__device__ static inline int leader_of(const AttendArgs &a, int i) { return min(max(a.groups[i], 0), a.requests); }
__device__ static inline int prefix_of(const AttendArgs &a, int i) {
    const int leader = leader_of(a, i), held = leader < a.requests ? a.lengths[leader] : 0;
    return max(min(min(a.shared[i], held), capacity_of(a)), 0);
}
// Of a request; no tokens where no group has it.
struct Prefix { int tokens, leader; };
__device__ static inline Prefix request_prefix(const AttendArgs &a, int request) {
    const int lane = threadIdx.x & 63;
    int lo = 0, span = a.n_groups;
    while (span > 0) {
        const int each = (span + 63) / 64, i = lo + lane * each;
        const bool mine = lane * each < span;
        const bool before = mine && leader_of(a, mine ? i : lo) <= request;
        const int held = before && each == 1 && request < leader_of(a, i + 1) ? prefix_of(a, i) : 0, leader = before && each == 1 ? leader_of(a, i) : 0;
        const int n = __builtin_popcountll(__ballot(before));
        if (n == 0) break;
        if (each == 1) return {__builtin_amdgcn_readlane(held, n - 1), __builtin_amdgcn_readlane(leader, n - 1)};
        lo = uniform(lo + (n - 1) * each);
        span = uniform(min(each, span - (n - 1) * each));
    }
    return {0, 0};
}

// What a launch's rows are divided by: requests, or groups of them.
template <int SEEN> __device__ static inline int units_of(const AttendArgs &a) { return SEEN == kPrefix ? a.n_groups : a.requests; }
template <int SEEN> __device__ static inline int start_of(const AttendArgs &a, int i) {
    if constexpr (SEEN == kPrefix) return clamped_start(a, a.starts[leader_of(a, i)]);
    return clamped_start(a, a.starts[i]);
}
template <int SEEN> __device__ static inline int length_of(const AttendArgs &a, int i) {
    if constexpr (SEEN == kPrefix) return prefix_of(a, i);
    return a.lengths[i];
}

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
template <int R, int SEEN> __device__ static inline Tile find_tile(const AttendArgs &a, int u, Prefix *prefix) {
    constexpr bool kBehind = SEEN == kOwn || SEEN == kBoth;
    const int lane = threadIdx.x & 63, units = units_of<SEEN>(a);
    auto place = [&](int start, int i) { return (int64_t)start * a.group / R + i; };
    auto rest = [&](int start) { return tile_of<R>(a, units, start, a.rows, 0, u - place(start, units)); };
    if (kBehind) *prefix = Prefix{0, 0};
    if (units == 0) return rest(start_of<SEEN>(a, 0));
    // (of up to 64 groups what they have in common comes with the requests' starts)
    const bool grouped = kBehind && units <= 64 && a.n_groups <= 64, one = grouped && lane < a.n_groups;
    const int first = one ? leader_of(a, lane) : 0x7fffffff, next = one ? leader_of(a, lane + 1) : 0, shared = one ? a.shared[lane] : 0;
    int lo = 0, span = units;
    for (;;) {
        const int each = (span + 63) / 64, i = lo + lane * each;
        const bool mine = lane * each < span;
        const int start = mine ? start_of<SEEN>(a, i) : a.rows;
        const int end = each == 1 && mine ? start_of<SEEN>(a, i + 1) : a.rows, length = each == 1 && mine ? length_of<SEEN>(a, i) : 0;
        const int n = max(__builtin_popcountll(__ballot(mine && place(start, i) <= u)), 1);
        lo = uniform(lo + (n - 1) * each);
        span = uniform(min(each, span - (n - 1) * each));
        if (each > 1) continue;
        const int at = uniform(n - 1), from = __builtin_amdgcn_readlane(start, at), to = __builtin_amdgcn_readlane(end, at);
        if (lo == units - 1 && u >= place(to, units)) return rest(to);
        if (grouped) {
            const int g = __builtin_popcountll(__ballot(first <= lo)) - 1;
            if (g >= 0 && lo < __builtin_amdgcn_readlane(next, g)) {
                const int leader = __builtin_amdgcn_readlane(first, g), held = __builtin_amdgcn_readlane(length, leader);
                *prefix = Prefix{max(min(min(__builtin_amdgcn_readlane(shared, g), held), capacity_of(a)), 0), leader};
            }
        } else if (kBehind) {
            *prefix = request_prefix(a, lo);
        }
        return tile_of<R>(a, lo, from, to, __builtin_amdgcn_readlane(length, at), u - place(from, lo));
    }
}

// A part of a group's tile over its prefix: of `splits` parts the one of number `split`.
struct Part { Tile tile; int split, splits; };

// Part u of a key head.  Groups differ in rows and in prefixes: their tiles are cut so that parts have as many steps of S tokens each (a.prefix_units of them in all
// and one more of each tile at most), which every wavefront works out by itself, a lane to a group.  More than 64 groups have tiles enough, cut alike (200 requests behind 4000 tokens: 64
// groups 64.6 us, 65 64.7; behind 900 37.3, 38.0).
template <int R, int S> __device__ static inline Part find_part(const AttendArgs &a, int u) {
    if (a.n_groups > 64) return {find_tile<R, kPrefix>(a, u / a.prefix_splits, nullptr), u % a.prefix_splits, a.prefix_splits};
    const int lane = threadIdx.x & 63;
    const bool mine = lane < a.n_groups;
    const int start = mine ? start_of<kPrefix>(a, lane) : 0, end = mine ? start_of<kPrefix>(a, lane + 1) : 0, tokens = mine ? prefix_of(a, lane) : 0;
    const int tiles = (int)((max((int64_t)(end - start) * a.group, (int64_t)0) + R - 1) / R), steps = (tokens + S - 1) / S;
    float total = (float)tiles * (float)steps, whole = (float)tiles;
    for (int s = 1; s < 64; s *= 2) {
        total += __shfl_xor(total, s);
        whole += __shfl_xor(whole, s);
    }
    // (each tile's last part counts as one more; rounded up by more than the sum is off: no more parts than there are workgroups)
    const float units = fmaxf(a.prefix_units - whole, 0.5f * a.prefix_units);
    int each = max(a.prefix_least, (int)fminf(ceilf(total * 1.001f / units), 1e9f));
    // (where that would be less than prefix_short, two thirds of the parts: what a part costs beside its steps is then most of it.  192 requests behind 2400 tokens 47.6 us, with
    // all parts 51.1; 64 behind 4800 30.7, 32.1; 16 behind 9600 21.5, 22.7; of 18 such sizes the others alike)
    auto shortest_of = [&](float length) { return length < a.prefix_short ? min(max((int)ceilf(length * 1.5f), a.prefix_least), a.prefix_short) : (int)fminf(ceilf(length), 1e9f); };
    if (a.n_groups <= 16) {
        // of 64 lengths from the shortest that could do, a lane each, the first that gives no more parts than that.  (128 requests, 8000 tokens: 16 groups 65.9 us, with
        // the bound above 67.9, 5 groups 51.5, 50.3; 24 groups 75.0 so, 78.0, but behind 1000 tokens 29.7, 27.6, and 64 groups 95.8, 91.9: the loop over the groups)
        const int shortest = max(a.prefix_least, shortest_of(total / a.prefix_units)), tried = shortest + lane * ((shortest + 63) / 64);
        float parts = 0;
        for (int g = 0; g < a.n_groups; ++g)
            parts += (float)__builtin_amdgcn_readlane(tiles, g) * (float)min((__builtin_amdgcn_readlane(steps, g) + tried - 1) / tried, a.prefix_splits);
        const uint64_t fits = __ballot(parts <= a.prefix_units);
        if (fits) each = __builtin_amdgcn_readlane(tried, __builtin_ctzll(fits));
    }
    const int splits = min((steps + each - 1) / each, a.prefix_splits), parts = tiles * splits;
    int before = 0, sum = parts;
    for (int s = 1; s < 64; s *= 2) {
        const int other = __shfl_up(sum, s);
        sum += lane >= s ? other : 0;
    }
    before = sum - parts;
    const uint64_t found = __ballot(before <= u && u < sum);
    if (!found) return {};
    const int at = __builtin_ctzll(found), local = u - __builtin_amdgcn_readlane(before, at), of = __builtin_amdgcn_readlane(splits, at);
    return {tile_of<R>(a, at, __builtin_amdgcn_readlane(start, at), __builtin_amdgcn_readlane(end, at), __builtin_amdgcn_readlane(tokens, at), local / of), local % of, of};
}

// Tile u of up to 63 requests with those of the longest requests first, and of each the last: every lane adds up the tiles of the
// requests before its own.  The tiles that take longest then begin first, and the end of a launch is not theirs (4 prompts of 1024 rows over 876 to
// 6000 tokens: see kv_attend_many).
//
// With a.tail the last tiles, those that would leave part of the chip idle, are cut into as many splits as fill it: u counts splits there.
template <int R, bool TAIL> __device__ static inline Tile find_longest(const AttendArgs &a, int u, int *split, int *splits) {
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
    if (TAIL && a.tail) {
        int all = tiles;
        for (int s = 1; s < 64; s *= 2) all += __shfl_xor(all, s);
        const int last = uniform(all) % a.tail, whole = uniform(all) - last;
        *splits = 1;
        if (u >= whole) {
            *splits = last ? min(max(a.tail / last, 1), a.splits) : 1;
            *split = (u - whole) % *splits;
            u = whole + (u - whole) / *splits;
        }
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

// A row's tile of R query heads of a group, and the request that it belongs to.
template <int R> __device__ static inline Tile find_row(const AttendArgs &a, int row, int first_head) {
    const int lane = threadIdx.x & 63;
    Tile t{};
    int lo = 0, span = a.requests;
    t.request = a.requests;
    while (span > 0) {
        const int each = (span + 63) / 64, i = lo + lane * each;
        const bool mine = lane * each < span;
        const int n = __builtin_popcountll(__ballot(mine && clamped_start(a, a.starts[mine ? i : lo]) <= row));
        if (n == 0) break;
        lo = uniform(lo + (n - 1) * each);
        span = uniform(min(each, span - (n - 1) * each));
        if (each > 1) continue;
        if (row < clamped_start(a, a.starts[lo + 1])) t.request = lo;
        break;
    }
    t.row0 = row;
    t.pair0 = first_head;
    t.pairs = min(R, a.group - first_head);
    t.length = t.request < a.requests ? min(max(a.lengths[t.request], 0), capacity_of(a)) : 0;
    return t;
}

// Which steps of S tokens rows at positions `lowest` (of those that see anything) to `highest` see of the tokens from `from` on: [low, low + sinks) and
// [first, first + count - sinks).
struct Steps {
    int count, sinks, first, low;
    __device__ int at(int i) const { return i < sinks ? low + i : first + i - sinks; }
};
template <int S> __device__ static inline Steps steps_of(const AttendArgs &a, int lowest, int highest, int length, int from) {
    const int end_token = min(highest, length - 1) + 1, end = (end_token + S - 1) / S;
    Steps s;
    s.low = from / S;
    s.sinks = a.window ? max(min((a.sinks + S - 1) / S, end) - s.low, 0) : 0;
    s.first = max(a.window ? max(lowest - a.window + 1, 0) / S : 0, s.low + s.sinks);
    s.count = end_token > from ? s.sinks + max(0, end - s.first) : 0;
    return s;
}

// The steps that a workgroup goes through.  BOTH: first those of the prefix, then those behind it; one that the two share inside is gone through twice, and a bit says
// for which of them.
constexpr int kOwnStep = 1 << 30;
template <bool BOTH> struct Walk {
    Steps common, own;
    int count;
    __device__ int at(int i) const {
        if constexpr (!BOTH) return own.at(i);
        return i < common.count ? common.at(i) : own.at(i - common.count) | kOwnStep;
    }
    __device__ void sum() { count = BOTH ? common.count + own.count : own.count; }
};
// Of a step of a tile whose first `from` tokens are common: its number, and the tokens that are looked at.
template <int SEEN> __device__ static inline int number_of(int step) { return SEEN == kBoth ? step & (kOwnStep - 1) : step; }
template <int SEEN> __device__ static inline int least_of(int step, int from) { return SEEN == kOwn ? from : SEEN == kBoth && step & kOwnStep ? from : 0; }
template <int SEEN> __device__ static inline int end_of(int step, int from, int length) { return SEEN == kBoth && !(step & kOwnStep) ? from : length; }

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

// Blocks of the two sixteens of a step (a sixteen lies in one block); -1: none, or behind the request's tokens.  token: the first of each, where a list says which.
struct StepBlocks { int id[2], token[2]; };
__device__ static inline StepBlocks blocks_of(const AttendArgs &a, TableRow table, int step, int length) {
    StepBlocks s = {};
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

constexpr int kPartExtra = 4;      // floats of a partial result behind its values: base, sum, number of splits, whether there are any of a prefix
constexpr int kFewestListed = 128; // of a split of a list: a round of the wavefronts (one row over 4096 tokens: 512 11.4 us, 256 10.8, 128 9.9)
constexpr int kFewest = 512;       // tokens of a split at least, where the host knows no bound near their number

// Where there is much to read (64 rows over up to 8192 tokens, 287 MB: 71 us, 4.0 TB/s; a copy moves 5.2 TB/s here, half of it reads) vector instructions take 51 % of a
// compute unit's busy time and its wavefronts wait for 46 % of theirs, so that neither is shown to bound alone; where there is little, the chain of starts, table
// and codes does (one row over 32768 tokens, 36 MB: 16 us).
// One (tile, key/value head, split): its wavefronts take steps in turn, each with a softmax of its own, and are joined in the LDS.  The next
// step's loads are in flight while one is computed, the block numbers of the one after that too.
//
// A column's scores are taken relative to a base that all its lanes share.  It need not be the maximum: it is raised,
// and what was summed is scaled down, only when a weight of the wavefront would pass the most of WeightRange, which past the
// first steps is hardly ever.
template <int DIM> using FewJoin = float[kAttendWaves][kTileRows][DIM / 2 + 4];
using FewSums = float[kAttendWaves][kTileRows];

// DEPTH: steps of a wavefront that are on their way while it computes one.
template <int DT, int DIM, int SEEN, int DEPTH> __device__ static inline void attend_few(const AttendArgs &a, int group, FewJoin<DIM> &join, FewSums &join_base, FewSums &join_sum) {
    typedef typename Elem<DT>::type T;
    constexpr int kQ = DIM / 32, kJ = DIM / 16;          // instructions of a score, of an output
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane % 16, g = lane / 16;
    int head, split, splits;
    Tile t;
    Prefix prefix = {0, 0};
    // beside kv_attend_many, requests of fewer than 32 pairs: two tiles each
    static_assert(kManyPairs <= 2 * kTileRows, "two tiles hold them");
    if constexpr (SEEN == kPrefix) {
        const Part part = find_part<kTileRows, kStep>(a, group / a.kv_heads);
        t = part.tile;
        split = part.split;
        splits = part.splits;
        head = group % a.kv_heads;
    } else {
        const int u = group % a.tiles, rest = group / a.tiles;
        head = rest % a.kv_heads;
        split = rest / a.kv_heads;
        splits = a.splits;
        if constexpr (SEEN == kListed) {
            const int each = (a.group + kTileRows - 1) / kTileRows;
            t = find_row<kTileRows>(a, u / each, u % each * kTileRows);
        } else if (a.many) {
            t = tile_of<kTileRows>(a, u / 2, clamped_start(a, a.starts[u / 2]), clamped_start(a, a.starts[u / 2 + 1]), a.lengths[u / 2], u % 2);
            if (t.pairs == 0 || t.request_pairs >= kManyPairs) return;
            if (SEEN == kOwn || SEEN == kBoth) prefix = request_prefix(a, u / 2);
        } else {
            t = find_tile<kTileRows, SEEN>(a, u, &prefix);
        }
    }
    if (t.pairs == 0 || (a.many && t.request_pairs >= kManyPairs)) return;
    if (SEEN == kPrefix && (t.request >= a.n_groups || t.length == 0)) return;
    constexpr bool kBehind = SEEN == kOwn || SEEN == kBoth;
    const int from = kBehind ? prefix.tokens : 0;        // the request's own tokens begin here
    const bool there = col < t.pairs;
    const int pair = t.pair0 + col, row = t.row0 + pair / a.group, qh = head * a.group + pair % a.group, own = there ? a.positions[row] : -1;
    i32x4_t q[kQ];
#pragma unroll
    for (int s = 0; s < kQ; ++s)
        q[s] = there ? query_words(static_cast<const T *>(a.q) + ((int64_t)row * a.q_heads + qh) * DIM + g * (DIM / 4) + s * 8, a.flip) : i32x4_t{0, 0, 0, 0};
    // Without a window the steps are those of the request's length, so that the first codes need not wait for the positions; the
    // last of them may be masked whole.
    Walk<SEEN == kBoth> steps{{(from + kStep - 1) / kStep, 0, 0, 0}, {t.length > from ? (t.length + kStep - 1) / kStep - from / kStep : 0, 0, from / kStep, 0}, 0};
    const int32_t *list = nullptr;                       // of this row and key head
    int listed = 0, visible = 0;                         // places of it up to the last that is looked at; tokens that the row sees
    if constexpr (SEEN == kListed) {
        list = a.selected + ((int64_t)t.row0 * a.kv_heads + head) * a.keep;
        visible = min(uniform(row_max(own)), t.length - 1) + 1;
        for (int i = lane; i < a.keep && visible > 0; i += 64) {
            const int block = list[i];
            if (block >= 0 && (int64_t)block << a.block_log < visible) listed = i + 1;
        }
        listed = wave_max(listed);
        steps.own.count = (int)((((int64_t)listed << a.block_log) + kStep - 1) / kStep);
    } else if (a.window) {
        const int seeing = -uniform(row_max(own >= 0 ? -own : -0x7fffffff));
        steps.own = steps_of<kStep>(a, seeing, uniform(row_max(own)), t.length, from);
        if (SEEN == kBoth) steps.common = steps_of<kStep>(a, seeing, uniform(row_max(own)), from, 0);
    }
    steps.sum();
    const int each = max(steps_each(steps.count, splits), SEEN == kOwn ? kFewest / kStep : SEEN == kListed ? kFewestListed / kStep : 0), begin = split * each, end = min(steps.count, begin + each);
    if (split > 0 && begin >= end) return;
    const bool whole = each >= steps.count && SEEN != kPrefix && (SEEN != kOwn || from == 0);      // no other split, or launch, has any steps

    const TableRow table = table_row(a, SEEN == kPrefix ? leader_of(a, t.request) : t.request);
    // the last step of this wavefront is loaded again where there is no next one: a load that some rounds leave out would
    // make every round wait for all that are on their way
    Held<DIM> held_steps[DEPTH + 1];
    StepBlocks blocks = {{-1, -1}, {}}, next_blocks[DEPTH];        // of the step that is computed, of those after it
    const int first = begin + wave, last = first + (end - 1 - first) / kAttendWaves * kAttendWaves;
    // Of a list, the blocks of 32 rounds at a time are looked up, two lanes a round: list and table are a chain that no round should wait for.
    int entry_id = -1, entry_token = 0, entries_from = -1;
    auto step_blocks = [&](int i) {
        if constexpr (SEEN == kBoth) {
            const int step = steps.at(i);
            return blocks_of(a, step & kOwnStep ? table : table_row(a, prefix.leader), number_of<SEEN>(step), end_of<SEEN>(step, from, t.length));
        } else if constexpr (SEEN != kListed) {
            return blocks_of(a, table, steps.at(i), t.length);
        }
        const int r = (i - first) / kAttendWaves;         // round of this wavefront
        if ((r & ~31) != entries_from) {
            entries_from = r & ~31;
            const int token = (first + (entries_from + lane / 2) * kAttendWaves) * kStep + lane % 2 * 16, place = token >> a.block_log;
            const int block = place < listed ? list[place] : -1;
            const bool seen = block >= 0 && (int64_t)block << a.block_log < visible;
            const int id = seen ? a.table[(int64_t)t.request * a.width + block] : -1;
            entry_id = id < a.blocks ? id : -1;
            entry_token = seen ? (block << a.block_log) + (token & ((1 << a.block_log) - 1)) : 0;
        }
        const int at = r % 32 * 2;
        return StepBlocks{{max(__builtin_amdgcn_readlane(entry_id, at), -1), max(__builtin_amdgcn_readlane(entry_id, at + 1), -1)},
                          {__builtin_amdgcn_readlane(entry_token, at), __builtin_amdgcn_readlane(entry_token, at + 1)}};
    };
    if (first < end) {
        blocks = step_blocks(first);
#pragma unroll
        for (int k = 0; k < DEPTH; ++k) next_blocks[k] = step_blocks(min(first + (k + 1) * kAttendWaves, last));
        load_step<DIM>(a, head, number_of<SEEN>(steps.at(first)), blocks, held_steps[0]);
#pragma unroll
        for (int k = 1; k < DEPTH; ++k) load_step<DIM>(a, head, number_of<SEEN>(steps.at(min(first + k * kAttendWaves, last))), next_blocks[k - 1], held_steps[k]);
    }
    const int highest = uniform(row_max(own)), lowest = -uniform(row_max(there ? -max(own, -1) : -0x7fffffff));
    const int tokens = SEEN == kBoth ? max(t.length, from) : t.length;
    const int position = min(own, tokens - 1), last_sink = a.window ? own - a.window : -1;    // tokens up to this one are seen as sinks only
    f32x4_t o[kJ];
#pragma unroll
    for (int j = 0; j < kJ; ++j) o[j] = f32x4_t{0, 0, 0, 0};
    float base = -3.4028234663852886e38f, sum = 0;
    const int full_to = min(lowest, tokens - 1);                         // steps that end here or before are seen by all rows,
    const int full_from = a.window ? highest - a.window + 1 : 0;        // if they begin here or behind

    __builtin_amdgcn_s_waitcnt(0xf70);                    // vmcnt 0: the queries are here before the rounds begin
    auto round = [&](int i, Held<DIM> &held, Held<DIM> &next) {
        const int step = steps.at(i);
        load_step<DIM>(a, head, number_of<SEEN>(steps.at(min(i + DEPTH * kAttendWaves, last))), next_blocks[DEPTH - 1], next);
        const StepBlocks later = step_blocks(min(i + (DEPTH + 1) * kAttendWaves, last));
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
        const int token0 = number_of<SEEN>(step) * kStep, least = least_of<SEEN>(step, from), limit = end_of<SEEN>(step, from, t.length);
        const int sixteen[2] = {SEEN == kListed ? blocks.token[0] : token0, SEEN == kListed ? blocks.token[1] : token0 + 16};
        if (max(sixteen[0], sixteen[1]) + 15 > full_to || (token0 < full_from && token0 + kStep > a.sinks) ||
            (kBehind && (token0 < least || token0 + kStep > limit)) || blocks.id[0] < 0 || blocks.id[1] < 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int token = sixteen[e / 4] + g * 4 + e % 4;
                const bool seen = blocks.id[e / 4] >= 0 && token <= position && (token > last_sink || token < a.sinks) &&
                                  (!kBehind || (token >= least && token < limit));
                p[e] = seen ? p[e] : -INFINITY;
            }
            // codes and scales of what is not held may be anything: a weight of 0 needs a finite value beside it
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int token = sixteen[k] + g * 4 + r;
                    const bool is = blocks.id[k] >= 0 && token < limit && (!kBehind || token >= least);
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
        blocks = next_blocks[0];
#pragma unroll
        for (int k = 1; k < DEPTH; ++k) next_blocks[k - 1] = next_blocks[k];
        next_blocks[DEPTH - 1] = later;
    };
    // as many rounds at a time as there are steps in registers, so that codes stay in those that they were loaded into
    for (int i = first; i < end;) {
        round(i, held_steps[0], held_steps[DEPTH]);
        i += kAttendWaves;
        if (i >= end) break;
        round(i, held_steps[1], held_steps[0]);
        i += kAttendWaves;
        if constexpr (DEPTH == 2) {
            if (i >= end) break;
            round(i, held_steps[2], held_steps[1]);
            i += kAttendWaves;
        }
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
            float *part = a.parts + (SEEN == kPrefix ? out_row * a.slots + split : SEEN == kOwn ? out_row * a.slots + a.prefix_splits + split : out_row * a.splits + split) * (DIM + kPartExtra);
            if (whole) static_cast<T *>(a.out)[out_row * DIM + half * (DIM / 2) + d] = (T)(l == 0 ? 0.f : v / l);
            else part[half * (DIM / 2) + d] = v;
            if (half == 0 && d == 0 && (splits > 1 || SEEN == kPrefix || SEEN == kOwn)) {
                part[DIM] = m;
                part[DIM + 1] = l;
                part[DIM + 2] = __builtin_bit_cast(float, whole || steps.count == 0 ? 1 : (steps.count + each - 1) / each);
                part[DIM + 3] = __builtin_bit_cast(float, (int)(from > 0));
            }
        }
    }
}

template <int DT, int DIM, int SEEN>
__global__ __launch_bounds__(64 * kAttendWaves, DIM == 256 ? 2 : 4) void kv_attend(AttendArgs a) {
    __shared__ FewJoin<DIM> join;
    __shared__ FewSums join_base, join_sum;
    attend_few<DT, DIM, SEEN, 1>(a, blockIdx.x, join, join_base, join_sum);
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

template <int DIM> using ManyKeys = i32x4_t[2][2][DIM / 16][2][32];
template <int DIM> using ManyValues = i32x4_t[2][DIM / 32][4][2][32];

template <int DT, int DIM, int SEEN> __device__ static inline void attend_many_rows(const AttendArgs &a, int group, ManyKeys<DIM> &keys, ManyValues<DIM> &values) {
    typedef typename Elem<DT>::type T;
    constexpr int kQ = DIM / 16, kJ = DIM / 16, kD = DIM / 32;
    // Which part of a step goes before other wavefronts' work (4 prompts of 1024 rows, 4096 pairs each: heads of 64 scores 241 us, weights and outputs 262,
    // neither 256; of 128 210, 205, 208; of 256 362 all).
    constexpr bool kScoresFirst = DIM == 64;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane % 32, half = lane / 32;
    const int head = group % a.kv_heads, rest = group / a.kv_heads;
    int split, splits;
    Tile t;
    Prefix prefix = {0, 0};
    if constexpr (SEEN == kPrefix) {
        const Part part = find_part<kManyRows, kManyStep>(a, rest);
        t = part.tile;
        split = part.split;
        splits = part.splits;
    } else {
        const bool tail = SEEN == kBoth && a.tail;
        const int u = tail ? rest : rest % a.many_tiles;
        split = tail ? 0 : rest / a.many_tiles;
        splits = a.splits;
        if (a.ordered) {
            t = find_longest<kManyRows, SEEN == kBoth>(a, u, &split, &splits);
            if ((SEEN == kOwn || SEEN == kBoth) && t.pairs > 0 && t.request < a.requests) {
                if (t.request_pairs < kManyPairs) return;
                prefix = request_prefix(a, t.request);
            }
        } else {
            t = find_tile<kManyRows, SEEN>(a, u, &prefix);
        }
    }
    if (t.pairs == 0 || (SEEN != kPrefix && t.request < a.requests && t.request_pairs < kManyPairs)) return;
    if (SEEN == kPrefix && (t.request >= a.n_groups || t.length == 0)) return;
    constexpr bool kBehind = SEEN == kOwn || SEEN == kBoth;
    const int from = kBehind ? prefix.tokens : 0;        // the request's own tokens begin here
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
    const int32_t *table = a.table + (int64_t)(SEEN == kPrefix ? leader_of(a, t.request) : t.request) * a.width;
    const int32_t *common_table = a.table + (int64_t)prefix.leader * a.width;
    auto token_of = [&](int step) { return number_of<SEEN>(step) * kManyStep + lane % 4 * 16; };
    auto entry_at = [&](int step) {
        const int token = token_of(step);
        return (SEEN == kBoth && !(step & kOwnStep) ? common_table : table)[token < end_of<SEEN>(step, from, t.length) ? token >> a.block_log : 0];
    };
    struct Blocks { int own, here; };                     // of the wavefront's sixteen, -1: none; a bit for each sixteen that has one
    auto blocks_at = [&](int step, int entry) {
        const bool is = token_of(step) < end_of<SEEN>(step, from, t.length) && (uint32_t)entry < (uint32_t)a.blocks;
        return Blocks{__builtin_amdgcn_readlane(is ? entry : -1, wave), (int)__ballot(is) & 15};
    };
    const KvLayout layout{DIM, 1 << a.block_log};
    const ManyPlaces<DIM> places(layout, lane);
    const char *head_part = a.cache + (int64_t)head * layout.head_bytes();
    const uint32_t block_bytes = (uint32_t)a.kv_heads * layout.head_bytes();
    HeldMany<DIM> held;
    auto load = [&](int step, int id) {
        load_many<DIM>(head_part + (uint64_t)(uint32_t)max(id, 0) * block_bytes, (number_of<SEEN>(step) * kManyStep + wave * 16) & (layout.tokens - 1), places, held);
    };
    // Without a window and splits the first steps are known before the positions are, and with them the first codes: the chain of loads
    // that a tile begins with is then one link shorter.
    const bool early = !a.window && splits == 1;
    Walk<SEEN == kBoth> steps{{(from + kManyStep - 1) / kManyStep, 0, 0, 0},
                              {t.length > from ? (t.length + kManyStep - 1) / kManyStep - from / kManyStep : 0, 0, from / kManyStep, 0}, 0};
    steps.sum();
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
    if (early && steps.count > 0) begin_at(steps.at(0), steps.at(min(1, steps.count - 1)), steps.at(min(2, steps.count - 1)));
    const int highest = wave_max(max(p0, p1));
    const int seeing = -wave_max(max(p0 >= 0 ? -p0 : -0x7fffffff, p1 >= 0 ? -p1 : -0x7fffffff));
    steps.own = steps_of<kManyStep>(a, seeing, highest, t.length, from);
    if (SEEN == kBoth) steps.common = steps_of<kManyStep>(a, seeing, highest, from, 0);
    steps.sum();
    const int each = max((steps.count + splits - 1) / splits, SEEN == kOwn ? kFewest / kManyStep : 0), begin = split * each, end = min(steps.count, begin + each);
    if (split > 0 && begin >= end) return;
    const bool whole = each >= steps.count && SEEN != kPrefix && (SEEN != kOwn || from == 0);
    auto clamped = [&](int i) { return steps.at(min(i, end - 1)); };       // behind the last step, that one again (see kv_attend)
    if (!early && begin < end) begin_at(steps.at(begin), clamped(begin + 1), clamped(begin + 2));
    const int own = __shfl(wave < 2 ? p0 : p1, wave % 2 * 32 + col);
    const int tokens = SEEN == kBoth ? max(t.length, from) : t.length;
    const int position = min(own, tokens - 1), last_sink = a.window ? own - a.window : -1;
    const int wave_lowest = -wave_max(there ? -max(own, -1) : -0x7fffffff), wave_highest = wave_max(own);
    const int full_to = min(wave_lowest, tokens - 1), full_from = a.window ? wave_highest - a.window + 1 : 0;
    f32x16_t o[kD];
#pragma unroll
    for (int d = 0; d < kD; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = 0;
    float base = -3.4028234663852886e38f, sum = 0;
    bool far = false;                                     // far_out(base)

    // what is not held may be anything: its values are to be finite, its scores are masked
    auto blank = [&](int step, int id) {
        const int g = lane / 16, h = g % 2, token0 = number_of<SEEN>(step) * kManyStep + wave * 16, least = least_of<SEEN>(step, from), limit = end_of<SEEN>(step, from, t.length);
        if (id >= 0 && token0 + 16 <= limit && (!kBehind || token0 >= least)) return;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int token = token0 + (h + 2 * k) * 4 + r;
                const bool is = id >= 0 && token < limit && (!kBehind || token >= least);
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
        const int buffer = (i - begin) & 1, token0 = number_of<SEEN>(step) * kManyStep, least = least_of<SEEN>(step, from), limit = end_of<SEEN>(step, from, t.length);
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
        if (!idle && token0 <= min(wave_highest, limit - 1)) {
            if (token0 + kManyStep - 1 > full_to || (token0 < full_from && token0 + kManyStep > a.sinks) ||
                (kBehind && (token0 < least || token0 + kManyStep > limit)) || these.here != 15) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int token = token0 + b * 32 + 8 * (r / 4) + 4 * half + r % 4;
                        const bool seen = (these.here >> (2 * b + r / 8) & 1) && token <= position && (token > last_sink || token < a.sinks) &&
                                          (!kBehind || (token >= least && token < limit));
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
    float *parts = a.parts + (SEEN == kPrefix ? out_row * a.slots + split : SEEN == kOwn ? out_row * a.slots + a.prefix_splits + split : out_row * a.splits + split) * (DIM + kPartExtra);
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
    if ((a.splits > 1 || SEEN == kPrefix || SEEN == kOwn) && half == 0) {
        parts[DIM] = base;
        parts[DIM + 1] = sum;
        parts[DIM + 2] = __builtin_bit_cast(float, whole || steps.count == 0 ? 1 : (steps.count + each - 1) / each);
        parts[DIM + 3] = __builtin_bit_cast(float, (int)(from > 0));
    }
}

template <int DT, int DIM, int SEEN>
__global__ __launch_bounds__(256, DIM == 256 ? 1 : DIM == 128 ? 2 : 3) void kv_attend_many(AttendArgs a) {
    __shared__ ManyKeys<DIM> keys;
    __shared__ ManyValues<DIM> values;
    attend_many_rows<DT, DIM, SEEN>(a, blockIdx.x, keys, values);
}

// Prefixes and what requests have behind them in one launch: the workgroups of prefixes first, which take longest; while they keep the matrix cores busy, the
// others read.  softmax over the tokens of both is that of two softmaxes with bases and sums of their own, which the join brings to one base.  MANY: prefixes by 128 pairs.
// (64 requests of up to 1024 tokens behind 8192, 32 heads of 128: the call 41-42 us, with a launch each 48; traced 37 and the join 6, prefixes by themselves 23, the others 17.5.
// 96 requests of 15 pairs behind five prefixes: the call 115 us, with a launch each 140; traced 121 and the join 9, vector instructions 49 % of a compute unit's busy time, matrix ones 34 %: of 128
// pairs of a tile 104 are there on average.  7 requests of 4 pairs: the call 11.7 us, traced 8.4 and 3.1, a chain of loads.)  With the longest of the others first, or all of
// them before the prefixes, the first of these calls takes as long or longer (43, 43 us).
template <int DT, int DIM, bool MANY>
__global__ __launch_bounds__(256, MANY ? (DIM == 256 ? 1 : DIM == 128 ? 2 : 3) : DIM == 256 ? 2 : 4) void kv_attend_shared(AttendArgs a) {
    __shared__ union Lds {
        __device__ Lds() {}
        struct { FewJoin<DIM> join; FewSums base, sum; } few;
        struct { ManyKeys<MANY ? DIM : 32> keys; ManyValues<MANY ? DIM : 32> values; } many;
    } lds;
    const int group = blockIdx.x;
    if constexpr (MANY) {
        if (group < a.prefix_groups) attend_many_rows<DT, DIM, kPrefix>(a, group, lds.many.keys, lds.many.values);
        else if (group < a.prefix_groups + a.own_many) attend_many_rows<DT, DIM, kOwn>(a, group - a.prefix_groups, lds.many.keys, lds.many.values);
        else attend_few<DT, DIM, kOwn, 2>(a, group - a.prefix_groups - a.own_many, lds.few.join, lds.few.base, lds.few.sum);
    } else {
        if (group < a.prefix_groups) attend_few<DT, DIM, kPrefix, 1>(a, group, lds.few.join, lds.few.base, lds.few.sum);
        else attend_few<DT, DIM, kOwn, 1>(a, group - a.prefix_groups, lds.few.join, lds.few.base, lds.few.sum);
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

// Joins what the prefix's splits (the first a.prefix_splits slots of a row and query head) and its own (those behind) gave, as kv_attend_join.
template <int DT, int DIM>
__global__ __launch_bounds__(256) void kv_attend_join_shared(AttendArgs a) {
    typedef typename Elem<DT>::type T;
    constexpr int kLanes = DIM / 4, kGroups = 256 / kLanes;
    __shared__ float factor[256], bases[4], sums[4];
    __shared__ f32x4_t part[kGroups][kLanes];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float *p = a.parts + (int64_t)blockIdx.x * a.slots * (DIM + kPartExtra), *own = p + a.prefix_splits * (DIM + kPartExtra);
    const bool slot = tid < a.slots;
    const float own_base = slot ? p[tid * (DIM + kPartExtra) + DIM] : 0.f, own_sum = slot ? p[tid * (DIM + kPartExtra) + DIM + 1] : 0.f;
    // (what is read of results that there are not is not used: a row that starts leave out may have any numbers)
    const int own_count = max(min(__builtin_bit_cast(int, own[DIM + 2]), a.splits), 0);
    const int count = __builtin_bit_cast(int, own[DIM + 3]) != 0 ? max(min(__builtin_bit_cast(int, p[DIM + 2]), a.prefix_splits), 0) : 0;
    if (count + own_count <= 1 && count == 0) return;
    const bool mine = tid < count || (tid >= a.prefix_splits && tid - a.prefix_splits < own_count);
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
    factor[tid] = f;
    __syncthreads();
    l = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    const int group = tid / kLanes, at = tid % kLanes;
    f32x4_t v = {0, 0, 0, 0};
#pragma unroll 4
    for (int i = group; i < count + own_count; i += kGroups) {
        const int s = i < count ? i : a.prefix_splits + i - count;
        v += *reinterpret_cast<const f32x4_t *>(p + s * (DIM + kPartExtra) + 4 * at) * factor[s];
    }
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

// The same with a wavefront to a row and query head, where there are many of these: nothing waits for another, and a wavefront's loads are all on their way.
template <int DT, int DIM> __device__ static inline void join_row(const AttendArgs &a, int row) {
    typedef typename Elem<DT>::type T;
    constexpr int kEach = DIM / 64;
    typedef float FV __attribute__((ext_vector_type(kEach)));
    const int lane = threadIdx.x & 63;
    const float *p = a.parts + (int64_t)row * a.slots * (DIM + kPartExtra), *own = p + a.prefix_splits * (DIM + kPartExtra);
    // (a lane to a slot, and one more slot each where there are more than 64; what is read of results that there are not is not used)
    float bases[4], sums[4], m = -3.4028234663852886e38f, l = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i * 64 < a.slots) {
            const int s = min(i * 64 + lane, a.slots - 1);
            bases[i] = p[s * (DIM + kPartExtra) + DIM];
            sums[i] = p[s * (DIM + kPartExtra) + DIM + 1];
        }
    const int own_count = uniform(max(min(__builtin_bit_cast(int, own[DIM + 2]), a.splits), 0));
    const int count = __builtin_bit_cast(int, own[DIM + 3]) != 0 ? uniform(max(min(__builtin_bit_cast(int, p[DIM + 2]), a.prefix_splits), 0)) : 0;
    if (count == 0 && own_count <= 1) return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i * 64 < a.slots) {
            const int s = i * 64 + lane;
            if (s < count || (s >= a.prefix_splits && s - a.prefix_splits < own_count)) m = fmaxf(m, bases[i]);
        }
    for (int s = 1; s < 64; s *= 2) m = fmaxf(m, __shfl_xor(m, s));
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i * 64 < a.slots) {
            const int s = i * 64 + lane;
            const bool mine = s < count || (s >= a.prefix_splits && s - a.prefix_splits < own_count);
            bases[i] = mine ? __builtin_amdgcn_exp2f(bases[i] - m) : 0.f;
            l += mine ? sums[i] * bases[i] : 0.f;
        }
    for (int s = 1; s < 64; s *= 2) l += __shfl_xor(l, s);
    FV v = {};
    const int all_parts = count + own_count;
    for (int i0 = 0; i0 < all_parts; i0 += 8) {           // (behind the last that one again, which counts for nothing)
        FV x[8];
        float f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = min(i0 + k, all_parts - 1), s = i < count ? i : a.prefix_splits + i - count, at = s >> 6;
            const float factor = at == 0 ? bases[0] : at == 1 ? bases[1] : at == 2 ? bases[2] : bases[3];
            x[k] = *reinterpret_cast<const FV *>(p + s * (DIM + kPartExtra) + kEach * lane);
            f[k] = i0 + k < all_parts ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, factor), s & 63)) : 0.f;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) v += x[k] * f[k];
    }
    ElemVec<DT, kEach> y;
#pragma unroll
    for (int i = 0; i < kEach; ++i) y[i] = (T)(l == 0 ? 0.f : v[i] / l);
    *reinterpret_cast<ElemVec<DT, kEach> *>(static_cast<T *>(a.out) + (int64_t)row * DIM + kEach * lane) = y;
}
template <int DT, int DIM>
__global__ __launch_bounds__(256) void kv_attend_join_rows(AttendArgs a, int all) {
    const int row = blockIdx.x * 4 + uniform(threadIdx.x >> 6);
    if (row < all) join_row<DT, DIM>(a, row);
}
// Of two rows and query heads a wavefront, those that have more than one part.  (16 prompts behind a prefix, 72600 of them, a seventh with parts: the whole call
// 203 us, with one a wavefront 208, with 4 205, 8 212, 16 224.)
constexpr int kJoinRows = 2;
template <int DT, int DIM>
__global__ __launch_bounds__(256) void kv_attend_join_some(AttendArgs a, int all) {
    const int lane = threadIdx.x & 63, first = (blockIdx.x * 4 + uniform(threadIdx.x >> 6)) * kJoinRows;
    const bool mine = lane < kJoinRows && first + lane < all;
    const int parts = mine ? __builtin_bit_cast(int, a.parts[(int64_t)(first + lane) * a.slots * (DIM + kPartExtra) + DIM + 2]) : 0;
    for (uint64_t left = __ballot(parts > 1); left; left &= left - 1) join_row<DT, DIM>(a, first + __builtin_ctzll(left));
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

template <int DT, int DIM, int SEEN> static hipError_t launch_attend_dim(const AttendArgs &a, hipStream_t st) {
    if (a.many) {
        kv_attend_many<DT, DIM, SEEN><<<(unsigned)(a.tail ? (a.many_tiles + a.tail) * a.kv_heads : a.many_tiles * a.kv_heads * a.splits), 256, 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.tiles) kv_attend<DT, DIM, SEEN><<<(unsigned)(a.tiles * a.kv_heads * a.splits), 64 * kAttendWaves, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const int all = a.rows * a.q_heads;
    if (a.tail) kv_attend_join_some<DT, DIM><<<(unsigned)((all + 4 * kJoinRows - 1) / (4 * kJoinRows)), 256, 0, st>>>(a, all);
    else kv_attend_join<DT, DIM><<<(unsigned)(a.rows * a.q_heads), 256, 0, st>>>(a);
    return hipGetLastError();
}
template <int DT> static hipError_t launch_attend_type(const AttendArgs &a, int dim, hipStream_t st) {
    return dim == 64 ? launch_attend_dim<DT, 64, kAll>(a, st) : dim == 128 ? launch_attend_dim<DT, 128, kAll>(a, st) : launch_attend_dim<DT, 256, kAll>(a, st);
}

// The order costs a loop over the requests, and is for tiles that take many steps.
static bool longest_first(const nnv_attention_desc &d, int requests) { return requests < 64 && (int64_t)d.table_blocks * d.block_tokens > 1024; }

static AttendArgs with_sizes(const nnv_attention_desc &d, const AttendArgs &args) {
    AttendArgs a = args;
    a.many = attend_many(d, a.requests, a.rows);
    a.tiles = a.many ? 2 * a.requests : attend_tiles(a.requests, a.rows, a.group, kTileRows);
    a.many_tiles = attend_tiles(a.requests, a.rows, a.group, kManyRows);
    a.splits = attend_splits(d, a.requests, a.rows);
    a.group_inverse = ((1u << 21) + a.group - 1) / a.group;
    a.ordered = longest_first(d, a.requests);
    return a;
}

hipError_t launch_kv_attention(const nnv_attention_desc &d, const AttendArgs &args, void *ws, hipStream_t st) {
    AttendArgs a = with_sizes(d, args);
    a.parts = static_cast<float *>(ws);
    return d.dtype == NNV_F16 ? launch_attend_type<NNV_F16>(a, d.head_dim, st) : launch_attend_type<NNV_BF16>(a, d.head_dim, st);
}

// ---- a prefix read once for the requests that share it, and what each has behind it ------------------------------------------

// Where requests have 256 pairs and more on average, their tiles go over the prefix by themselves: it is converted for 128 pairs at a time either way, and nothing is to
// be joined (16 requests of up to 256 rows behind 4096 tokens, 32 heads of 128 and 8 of keys: 230 us, in two parts 328).
static bool shared_by_request(const nnv_attention_desc &d, int requests, int rows) { return (int64_t)rows * (d.q_heads / d.kv_heads) >= (int64_t)2 * kManyRows * requests; }

// Of these, where the longest go first, how many splits the tiles have that are left when the chip has been filled for the last time: 2 to 8 within 128 MB of partial
// results; 0: tiles are cut alike, if at all.
static int tail_splits(const nnv_attention_desc &d, int requests, int rows) {
    if (!shared_by_request(d, requests, rows) || !attend_many(d, requests, rows) || !longest_first(d, requests) || d.kv_heads > 64) return 0;
    const int64_t fit = ((int64_t)128 << 20) / ((int64_t)rows * d.q_heads * (d.head_dim + kPartExtra) * 4);
    return fit < 2 || 8 * kv_attention_groups(d, requests, rows) >= 1 << 24 ? 0 : fit < 8 ? (int)fit : 8;
}

// Otherwise prefixes and what is behind them are two parts, whose results are joined.  The prefix goes by 128 pairs, converted once for them, where a group has as
// many on average as fill a wavefront's part of those.
struct SharedSizes { bool many; int units, least, prefix, own, slots; int64_t prefix_groups, own_many, own_few; };
static SharedSizes shared_sizes(const nnv_attention_desc &d, int requests, int rows, int groups) {
    const int group = d.q_heads / d.kv_heads;
    const int64_t capacity = (int64_t)d.table_blocks * d.block_tokens, pairs = (int64_t)rows * group, each = (int64_t)rows * d.q_heads * (d.head_dim + kPartExtra) * 4;
    const bool own_many = attend_many(d, requests, rows) && pairs >= (int64_t)2 * kManyPairs * requests;      // (of fewer on average, nearly all are few)
    SharedSizes s{};
    s.many = own_many || pairs >= (int64_t)kManyPairs * groups;
    auto within = [&](int64_t splits, int64_t most) {     // of memory (one result each of a prefix and behind it there is at least, whatever these take), and of what the join takes
        splits = splits < most ? splits : most;
        splits = splits < kMostSplits ? splits : kMostSplits;
        while (splits > 1 && splits * each > (int64_t)128 << 20) splits = splits / 2;
        return (int)(splits < 1 ? 1 : splits);
    };
    const int64_t tile = s.many ? kManyRows : kTileRows, prefix_tiles = pairs / tile + groups + 1;
    // 384 workgroups for prefixes: the chip holds 512 of these, and the others' places are for what is behind (96 requests behind five prefixes of up to 16001
    // tokens: 256 140 us, 320 132, 384 115, 448 117, 512 120); 256 where parts are short
    // (64 requests behind 8192 tokens: parts of 256 tokens 51 us, of 512 42; the other way round 191 requests of 3 rows behind up to 481 tokens and heads of 256: parts of 128
    // tokens 30 us, of 512 43); by 16 pairs a round of the wavefronts at least.
    s.units = (384 + d.kv_heads - 1) / d.kv_heads;
    s.least = s.many && d.head_dim == 256 ? 2 : 4;
    if (groups > 64) s.prefix = within((s.units + prefix_tiles - 1) / prefix_tiles, capacity / kFewest + 1);
    else s.prefix = within(s.units, capacity / 128 + 1);
    // (parts are no more than units where tiles are no more than half of those: see find_part)
    s.prefix_groups = (groups > 64 ? prefix_tiles * s.prefix : prefix_tiles <= s.units / 2 ? s.units : s.units + prefix_tiles) * d.kv_heads;
    const int64_t own_tile = own_many ? kManyRows : kTileRows, full = pairs / own_tile, least = requests < rows ? requests : rows;
    const int64_t own_tiles = (full > least ? full : least > 0 ? least : 1) * d.kv_heads;
    s.own = within((512 + own_tiles - 1) / own_tiles, capacity / kFewest + 1);
    auto own_groups = [&] {
        s.own_many = own_many ? (int64_t)attend_tiles(requests, rows, group, kManyRows) * d.kv_heads * s.own : 0;
        s.own_few = (own_many ? 2 * (int64_t)requests : attend_tiles(requests, rows, group, kTileRows)) * d.kv_heads * s.own;
        return s.own_many + s.own_few;
    };
    while (own_groups() + s.prefix_groups >= 1 << 24 && s.own > 1) s.own /= 2;
    if (own_groups() + s.prefix_groups >= 1 << 24 && groups > 64 && s.prefix > 1) s.prefix = 1, s.prefix_groups = prefix_tiles * d.kv_heads;
    s.slots = s.prefix + s.own;
    return s;
}

int64_t kv_attention_shared_groups(const nnv_attention_desc &d, int requests, int rows, int groups) {
    if (!groups || shared_by_request(d, requests, rows)) return kv_attention_groups(d, requests, rows);
    const SharedSizes s = shared_sizes(d, requests, rows, groups);
    const int64_t all = s.prefix_groups + s.own_many + s.own_few, join = ((int64_t)rows * d.q_heads + 3) / 4;
    return all > join ? all : join;
}

size_t kv_attention_shared_workspace_bytes(const nnv_attention_desc &d, int requests, int rows, int groups) {
    if (!groups) return kv_attention_workspace_bytes(d, requests, rows);
    if (const int s = tail_splits(d, requests, rows)) return (size_t)rows * d.q_heads * s * (d.head_dim + kPartExtra) * 4;
    if (shared_by_request(d, requests, rows)) return kv_attention_workspace_bytes(d, requests, rows);
    return (size_t)rows * d.q_heads * shared_sizes(d, requests, rows, groups).slots * (d.head_dim + kPartExtra) * 4;
}

template <int DT, int DIM> static hipError_t launch_shared_dim(const nnv_attention_desc &d, const AttendArgs &args, hipStream_t st) {
    AttendArgs a = with_sizes(d, args);
    if (!a.n_groups) return launch_attend_dim<DT, DIM, kAll>(a, st);
    if (shared_by_request(d, a.requests, a.rows)) {
        if (const int splits = tail_splits(d, a.requests, a.rows)) {
            a.splits = a.slots = splits;
            a.tail = (d.head_dim == 64 ? 768 : d.head_dim == 128 ? 512 : 256) / a.kv_heads;
        }
        return launch_attend_dim<DT, DIM, kBoth>(a, st);
    }
    const SharedSizes s = shared_sizes(d, a.requests, a.rows, a.n_groups);
    a.slots = s.slots;
    a.prefix_splits = s.prefix;
    a.prefix_units = s.units;
    a.prefix_least = s.least;
    a.prefix_short = s.many ? 8 : 4;
    a.prefix_groups = (int)s.prefix_groups;
    a.own_many = (int)s.own_many;
    a.many = s.own_many > 0;
    a.tiles = (int)(s.own_few / ((int64_t)a.kv_heads * s.own));
    a.splits = s.own;
    const unsigned groups = (unsigned)(s.prefix_groups + s.own_many + s.own_few);
    if (!s.many) {
        kv_attend_shared<DT, DIM, false><<<groups, 256, 0, st>>>(a);
    } else if constexpr (DIM == 256) {
        // heads of 256 leave room for one workgroup of these a compute unit, and the others would have no more: a launch each (114 requests of a token behind 164, 16 heads
        // to a key head: in one launch 64 us, in these 54)
        kv_attend_many<DT, DIM, kPrefix><<<(unsigned)s.prefix_groups, 256, 0, st>>>(a);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (s.own_many) kv_attend_many<DT, DIM, kOwn><<<(unsigned)s.own_many, 256, 0, st>>>(a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        kv_attend<DT, DIM, kOwn><<<(unsigned)s.own_few, 64 * kAttendWaves, 0, st>>>(a);
    } else {
        kv_attend_shared<DT, DIM, true><<<groups, 256, 0, st>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int all = a.rows * a.q_heads;
    // (behind 4096 tokens, by wavefronts and by workgroups: 8192 rows and heads 64.2 us, 67.7; 4096 42.7, 43.8; 2048 30.9, 30.8; 256 16.5, 16.4)
    if (all >= 4096) kv_attend_join_rows<DT, DIM><<<(unsigned)((all + 3) / 4), 256, 0, st>>>(a, all);
    else kv_attend_join_shared<DT, DIM><<<(unsigned)all, 256, 0, st>>>(a);
    return hipGetLastError();
}
template <int DT> static hipError_t launch_shared_type(const nnv_attention_desc &d, const AttendArgs &a, hipStream_t st) {
    return d.head_dim == 64 ? launch_shared_dim<DT, 64>(d, a, st) : d.head_dim == 128 ? launch_shared_dim<DT, 128>(d, a, st) : launch_shared_dim<DT, 256>(d, a, st);
}

hipError_t launch_kv_attention_shared(const nnv_attention_desc &d, const AttendArgs &args, void *ws, hipStream_t st) {
    AttendArgs a = args;
    a.parts = static_cast<float *>(ws);
    return d.dtype == NNV_F16 ? launch_shared_type<NNV_F16>(d, a, st) : launch_shared_type<NNV_BF16>(d, a, st);
}

// ---- the blocks that a row and key head's list names -------------------------------------------------------------------------

// kv_attend, whose steps go through the list.  One row over 64 blocks of 64 tokens: 7.7 us and the join, a chain of starts, list, table and codes; 64 rows over up to 32 of them, 134 MB: 31 us,
// 4.3 TB/s, vector instructions 46 % of busy time and 41 % of the wavefronts' time spent waiting.

static int64_t listed_tiles(const nnv_attention_desc &d, int rows) { return (int64_t)rows * ((d.q_heads / d.kv_heads + kTileRows - 1) / kTileRows); }
int64_t kv_attention_blocks_groups(const nnv_attention_desc &d, int rows) { return listed_tiles(d, rows) * d.kv_heads; }

static int listed_splits(const nnv_attention_desc &d, int rows, int keep) {
    const int64_t groups = kv_attention_blocks_groups(d, rows), most = ((int64_t)keep * d.block_tokens + kFewestListed - 1) / kFewestListed;
    const int64_t each = (int64_t)rows * d.q_heads * (d.head_dim + kPartExtra) * 4;
    // (64 rows and 8 heads over up to 2048 tokens: 512 workgroups 31 us, 1024 with a join 37, 2048 41)
    int64_t s = (512 + groups - 1) / groups;
    if (s > most) s = most;
    if (s > kMostSplits) s = kMostSplits;
    while (s > 1 && (s * each > (int64_t)256 << 20 || s * groups >= 1 << 24)) s = s / 2;
    return (int)(s < 1 ? 1 : s);
}

size_t kv_attention_blocks_workspace_bytes(const nnv_attention_desc &d, int rows, int keep) {
    const int s = listed_splits(d, rows, keep);
    return s == 1 ? 0 : (size_t)rows * d.q_heads * s * (d.head_dim + kPartExtra) * 4;
}

template <int DT, int DIM> static hipError_t launch_listed_dim(const AttendArgs &a, hipStream_t st) {
    kv_attend<DT, DIM, kListed><<<(unsigned)((int64_t)a.tiles * a.kv_heads * a.splits), 64 * kAttendWaves, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    kv_attend_join<DT, DIM><<<(unsigned)(a.rows * a.q_heads), 256, 0, st>>>(a);
    return hipGetLastError();
}
template <int DT> static hipError_t launch_listed_type(const AttendArgs &a, int dim, hipStream_t st) {
    return dim == 64 ? launch_listed_dim<DT, 64>(a, st) : dim == 128 ? launch_listed_dim<DT, 128>(a, st) : launch_listed_dim<DT, 256>(a, st);
}

hipError_t launch_kv_attention_blocks(const nnv_attention_desc &d, const AttendArgs &args, void *ws, hipStream_t st) {
    AttendArgs a = args;
    a.tiles = (int)listed_tiles(d, a.rows);
    a.splits = listed_splits(d, a.rows, a.keep);
    a.parts = static_cast<float *>(ws);
    a.group_inverse = ((1u << 21) + a.group - 1) / a.group;
    return d.dtype == NNV_F16 ? launch_listed_type<NNV_F16>(a, d.head_dim, st) : launch_listed_type<NNV_BF16>(a, d.head_dim, st);
}

}  // namespace nnv

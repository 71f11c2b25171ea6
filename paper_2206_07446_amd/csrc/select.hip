// What attention over selected blocks reads before it: the bounds of the blocks' keys, and of each row the blocks that its queries select by them.
#include "nnv_internal.h"
#include "serving.h"
#include "lowbits.h"

namespace nnv {

namespace {

// A request: its first row, the row behind its last, its tokens.
struct Found { int request, start, end, length; };

// The last of `count` requests whose place, which rises with its start, is at or before `at` (the first if there is none).  A wavefront compares 64 of them at a
// time; what a request has beside its start comes with the last round, so that a chain of loads is one link long for up to 64 requests.
template <typename S, typename P> __device__ inline Found last_place(int count, int64_t at, const int32_t *lengths, S start_of, P place) {
    const int lane = threadIdx.x & 63;
    int lo = 0, span = count;
    for (;;) {
        const int each = (span + 63) / 64, i = lane * each < span ? lo + lane * each : lo;
        const bool mine = lane * each < span;
        const int start = start_of(i), end = each == 1 ? start_of(i + 1) : 0, length = each == 1 ? lengths[i] : 0;
        const int n = max(__builtin_popcountll(__ballot(mine && place(i, start) <= at)), 1);
        lo = __builtin_amdgcn_readfirstlane(lo + (n - 1) * each);
        span = __builtin_amdgcn_readfirstlane(min(each, span - (n - 1) * each));
        if (each == 1) return {lo, __builtin_amdgcn_readlane(start, n - 1), __builtin_amdgcn_readlane(end, n - 1), __builtin_amdgcn_readlane(length, n - 1)};
    }
}

}  // namespace

// ---- bounds -------------------------------------------------------------------------------------

typedef int16_t i16x2_t __attribute__((ext_vector_type(2)));

// bfloat16 pairs as 16-bit numbers of the same order, and back: the bits below the sign are turned where it is set.
__device__ static inline uint32_t ordered(uint32_t pair) {
    const i16x2_t sign = __builtin_bit_cast(i16x2_t, pair) >> 15;
    return pair ^ (__builtin_bit_cast(uint32_t, sign) & 0x7fff7fffu);
}
__device__ static inline uint32_t larger(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2_t, a), __builtin_bit_cast(i16x2_t, b)));
}

// Joins lanes that differ in bits MASK and up of their number, of 2 COUNT values each: of each pair one lane goes on with the lower half of the values, the other with
// the upper.  -> where what is left lies among the values.
template <int COUNT, int MASK> __device__ static inline int join_lanes(uint32_t (&v)[32], int lane) {
    if constexpr (MASK >= 64) {
        return 0;
    } else {
        const bool upper = lane & MASK;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const uint32_t keep = upper ? v[COUNT + i] : v[i], send = upper ? v[i] : v[COUNT + i];
            v[i] = larger(keep, (uint32_t)__shfl_xor((int)send, MASK));
        }
        return (upper ? COUNT : 0) + join_lanes<COUNT / 2, MASK * 2>(v, lane);
    }
}

// A wavefront takes a block's head.  A lane reads the 32 codes of one token that share a scale, 16 bytes, and keeps their largest values, and the largest of
// their complements, which are the complements of the smallest: values of e2m1 have two significant bits, and bfloat16 holds them all as they are.  Lanes of other
// tokens are then joined by halves: each step hands over half of what is left, so that 64 values over 16 lanes cost 30 exchanges and not 128.
// Bound by the chain of starts, table and codes: 64 blocks of 64 tokens and 8 heads of 128 4.3 us, 576 of 32 tokens and 8 heads of 64 (6 MB) 5.2.
template <int DIM>
__global__ __launch_bounds__(256) void kv_bounds(BoundsArgs a) {
    constexpr int kGroups = DIM / 32, kTokens = 64 / kGroups;      // lanes of a token, tokens of a round
    const int lane = threadIdx.x & 63, g = lane % kGroups, place = lane / kGroups;
    const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= (int64_t)a.units * a.kv_heads) return;
    const int u = (int)(unit / a.kv_heads), head = (int)(unit % a.kv_heads);
    auto start_of = [&](int i) { return min(max(a.starts[i], 0), a.rows); };
    // f tokens touch at most f / block + 2 blocks
    const Found f = last_place(a.requests, u, a.lengths, start_of, [&](int i, int start) { return (int64_t)(start >> a.block_log) + 2 * (int64_t)i; });
    const int request = f.request, start = f.start, fresh = f.end - start, block = 1 << a.block_log;
    const int length = min(max(f.length, 0), a.width << a.block_log);
    const int column = (max(length - fresh, 0) >> a.block_log) + (u - (start >> a.block_log) - 2 * request);
    if (fresh <= 0 || u - (start >> a.block_log) - 2 * request < 0 || ((int64_t)column << a.block_log) >= length) return;
    const int id = a.table[(int64_t)request * a.width + column];
    if (id < 0 || id >= a.blocks) return;
    const KvLayout at{DIM, block};
    const char *keys = a.cache + ((int64_t)id * a.kv_heads + head) * at.head_bytes();
    const int held = min(length - (column << a.block_log), block);
    uint32_t v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = 0x80008000u;
    // four rounds are on their way together; behind the last token that one again, which changes nothing
    for (int t0 = 0; t0 < held; t0 += 4 * kTokens) {
        i32x4_t codes[4];
        uint32_t byte[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = min(t0 + i * kTokens + place, held - 1);
            codes[i] = *reinterpret_cast<const i32x4_t *>(keys + t * (DIM / 2) + g * 16);
            byte[i] = (uint8_t)keys[at.key_scale_at() + t * kGroups + g];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (t0 + i * kTokens >= held) break;
            const float scale = scale_of_byte(min(max(byte[i], 1u), kMostE2m1Byte<NNV_BF16>));
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t pairs[4] = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i][w], scale, 0)),
                                           __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i][w], scale, 1)),
                                           __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i][w], scale, 2)),
                                           __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i][w], scale, 3))};
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const uint32_t x = ordered(pairs[p]);
                    v[w * 4 + p] = larger(v[w * 4 + p], x);
                    v[16 + w * 4 + p] = larger(v[16 + w * 4 + p], ~x);
                }
            }
        }
    }
    const int from = join_lanes<16, kGroups>(v, lane);
    constexpr int kLeft = 32 / kTokens;                              // pairs left to a lane: 1, 2 or 4
    const bool low = from >= 16;
    uint32_t *out = reinterpret_cast<uint32_t *>(a.bounds + (((int64_t)id * a.kv_heads + head) * 2 + low) * DIM + g * 32) + (from & 15);
#pragma unroll
    for (int i = 0; i < kLeft; ++i) out[i] = ordered(low ? ~v[i] : v[i]);
}

hipError_t launch_kv_bounds(const BoundsArgs &a, int dim, hipStream_t st) {
    const unsigned groups = (unsigned)(((int64_t)a.units * a.kv_heads + 3) / 4);
    if (dim == 64) kv_bounds<64><<<groups, 256, 0, st>>>(a);
    else if (dim == 128) kv_bounds<128><<<groups, 256, 0, st>>>(a);
    else kv_bounds<256><<<groups, 256, 0, st>>>(a);
    return hipGetLastError();
}

// ---- selection ----------------------------------------------------------------------------------

typedef double f64x2_t __attribute__((ext_vector_type(2)));
constexpr int kMostKeys = 4096;                          // of a tile's rows, where one workgroup scores and picks

typedef double f64x4_t __attribute__((ext_vector_type(4)));

// Numbers in the order of 64-bit keys; a NaN counts as -infinity.  Key 0 is no block's.
__device__ static inline uint64_t key_of(double v) {
    v = v == v ? v + 0.0 : -INFINITY;                                // (-0 as 0)
    const uint64_t bits = __builtin_bit_cast(uint64_t, v);
    return bits >> 63 ? ~bits : bits | (uint64_t)1 << 63;
}

// Bits that any lane of a wavefront has.
__device__ static inline uint32_t wave_or(uint32_t v) {
    v |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, false);       // lanes xor 1
    v |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, false);       // xor 2
    v |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, false);      // mirrored halves of a row
    v |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, false);      // mirrored row
    auto row = [&](int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); };
    return (row(0) | row(16)) | (row(32) | row(48));
}

// The `keep` largest of `visible` keys, the lowest blocks where keys are equal, in ascending order, by a wavefront whose lanes hold EACH of them.  The smallest key
// kept is found bit by bit, from the first that is not the same in all: each bit is one count over the keys.
template <int EACH> __device__ static inline void pick_by_wave(const uint64_t *keys, int visible, int first, int last, int keep, int32_t *out) {
    const int lane = threadIdx.x & 63;
    uint64_t key[EACH], set = 0, clear = 0;
    int kept = 0;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        const int b = j * 64 + lane;
        key[j] = b < visible ? keys[b] : 0;
        if (key[j] && (b < first || b >= visible - last)) key[j] = ~(uint64_t)0;
        if (key[j] && ~key[j]) {                          // (those that are always kept are all ones)
            set |= key[j];
            clear |= ~key[j];
        }
        kept += __builtin_popcountll(__ballot(key[j] != 0));
    }
    auto count = [&](uint64_t least) {
        int n = 0;
#pragma unroll
        for (int j = 0; j < EACH; ++j) n += __builtin_popcountll(__ballot(key[j] >= least));
        return n;
    };
    uint64_t least = 1;
    if (kept > keep) {
        set = wave_or((uint32_t)set) | (uint64_t)wave_or((uint32_t)(set >> 32)) << 32;
        const uint64_t differ = set & (wave_or((uint32_t)clear) | (uint64_t)wave_or((uint32_t)(clear >> 32)) << 32);
        const int top = differ ? 63 - __builtin_clzll(differ) : -1;
        least = top < 0 ? set : top == 63 ? 0 : set & ~(((uint64_t)2 << top) - 1);
        for (int bit = top; bit >= 0; --bit) {
            const uint64_t next = least | (uint64_t)1 << bit;
            const int n = count(next);
            if (n < keep) continue;
            least = next;
            kept = n;
            if (n == keep) break;
        }
    }
    // of the keys that are `least`, so many as fit are taken, the first ones
    int equal = kept > keep ? keep - count(least + 1) : 0x7fffffff, place = 0;      // (a key of all ones cannot be one too many: first + last <= keep)
    const uint64_t before = ((uint64_t)1 << lane) - 1;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        const uint64_t same = __ballot(key[j] == least);
        const bool take = key[j] > least || (key[j] == least && __builtin_popcountll(same & before) < equal);
        const uint64_t taken = __ballot(take);
        if (take) out[place + __builtin_popcountll(taken & before)] = j * 64 + lane;
        place += __builtin_popcountll(taken);
        equal -= __builtin_popcountll(same);
    }
    for (int i = place + lane; i < keep; i += 64) out[i] = -1;
}

// Scores of a tile of whole rows with a head's blocks: max(q hi, q lo) is max(q, 0) hi + min(q, 0) lo, so that a score is one product over 2 DIM, on the
// matrix cores in float64: 16 blocks x 4 values x 4 query heads (4x4x4, four of them in an instruction) or x 16 (16x16x4).  Lane l holds of block, and of query
// head, l % 16 (l % 4) the eight values from 32 s + 8 (l / 16): products sum over values in any order.  Queries lie in the LDS as they enter, the same for all
// wavefronts; the bounds of a wavefront's next 16 blocks are on their way while it computes.
//
// 64 rows over up to 512 blocks, 4 heads of 128 to a key head, 68 MB: 26 us, 2.6 TB/s: lookups 4 us, queries 2, four rounds of bounds 2 to 2.5 each, the pick; neither loads nor
// products bound alone (in two launches, 30 us, it took as long with either left out).  1000 rows of 8 heads of 64 over up to 282 blocks: 25 us, the matrix cores 10.4 of it (products of max(q, 0) and min(q, 0)
// apart cost twice those of a score; the float64 rate of 16x16x4 is that of vector instructions).
//
// EACH: where it is not 0, a workgroup of eight wavefronts takes all blocks of its tile (up to 64 EACH of a row), keeps their keys in the LDS and picks from them, a
// wavefront a row; otherwise one of four takes a chunk of the blocks and keys go to memory, for kv_pick.
template <int DT, int DIM, int COLS, int EACH>
__global__ __launch_bounds__(EACH ? 512 : 256, DIM == 256 ? 2 : EACH ? 4 : DIM == 128 ? 3 : 4) void kv_scores(SelectArgs a) {
    typedef typename Elem<DT>::type T;
    constexpr int kSteps = DIM / 32, kThreads = EACH ? 512 : 256, kRound = kThreads / 4;      // kRound: blocks that the wavefronts take at a time
    constexpr bool kPick = EACH != 0;
    __shared__ uint64_t keys[kPick ? kMostKeys : 1];
    __shared__ f64x2_t queries[DIM / 4][4][COLS];                    // max(q, 0) and min(q, 0) of value 32 s + 8 g + e at [8 s + e][g]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane / 16, col = lane % COLS;
    // (chunks last: workgroups go to the chip's eight parts in turn, and of two chunks the second, which fewer requests reach, would keep half of them idle)
    const int tiles = a.tiles, head = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads, u = rest % tiles, chunk = rest / tiles;
    if (kPick && rest >= tiles) {                        // (rows of no request are in no tile)
        const int begin = min(max(a.starts[0], 0), a.rows), end = min(max(a.starts[a.requests], 0), a.rows);
        const int64_t each = (int64_t)a.kv_heads * a.keep;
        for (int row = blockIdx.x - tiles * a.kv_heads; row < a.rows; row += a.kv_heads)
            if (row < begin || row >= end)
                for (int64_t i = threadIdx.x; i < each; i += kThreads) a.selected[row * each + i] = -1;
        return;
    }
    auto start_of = [&](int i) { return min(max(a.starts[i], a.row0), a.row0 + a.rows); };
    // a row at a time is found by itself; tiles of several begin at floor((starts[i] - row0) / tile_rows) + i
    const bool single = a.tile_rows == 1, wide = a.group > COLS;      // wide: a row's heads in several products
    // (eight values a thread, neighbours to one place after the other)
    constexpr int kParts = (COLS * 4 * kSteps + kThreads - 1) / kThreads;
    ElemVec<DT, 8> parts[kParts];
    auto part_of = [&](int k, int &at, int &part, int &s) {
        const int i = k * kThreads + threadIdx.x;
        at = i % COLS;
        part = i / COLS % 4;
        s = i / (COLS * 4);
        return i < COLS * 4 * kSteps;
    };
    auto load_queries = [&](int c, int tile0, int rows) {
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            int at, part, s;
            const bool is = part_of(k, at, part, s);
            const int row = wide || single ? 0 : at / a.group, h = wide ? c * COLS + at : at - row * a.group;
            parts[k] = ElemVec<DT, 8>{};
            if (is && row < rows && h < a.group)
                parts[k] = *reinterpret_cast<const ElemVec<DT, 8> *>(static_cast<const T *>(a.q) + ((int64_t)(tile0 + row) * a.q_heads + head * a.group + h) * DIM + s * 32 + part * 8);
        }
    };
    auto fill_queries = [&] {
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            int at, part, s;
            if (!part_of(k, at, part, s)) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = a.flip ? -(float)parts[k][e] : (float)parts[k][e];
                const float none = v == v ? 0.f : v;         // (a NaN stays one, and with it the head's sum)
                queries[8 * s + e][part][at] = f64x2_t{(double)(v > 0 ? v : none), (double)(v < 0 ? v : none)};
            }
        }
    };
    int last = -1;                                                   // the last token that a row sees
    if (single) {
        load_queries(0, a.row0 + u, 1);
        last = a.positions[a.row0 + u];
    }
    const Found f = last_place(a.requests, single ? a.row0 + u : u, a.lengths, start_of,
                               [&](int i, int start) { return single ? (int64_t)start : (int64_t)((start - a.row0) / a.tile_rows) + i; });
    const int local = single ? a.row0 + u - f.start : u - ((f.start - a.row0) / a.tile_rows + f.request);
    const int tile0 = f.start + local * a.tile_rows, rows = min(f.end - tile0, a.tile_rows);
    if (local < 0 || rows <= 0) {
        if (kPick && single)
            for (int i = threadIdx.x; i < a.keep; i += kThreads) a.selected[((int64_t)(a.row0 + u) * a.kv_heads + head) * a.keep + i] = -1;
        return;
    }
    const int length = min(max(f.length, 0), a.width << a.block_log);
    if (!single) {
        load_queries(0, tile0, rows);
        last = lane < rows ? a.positions[tile0 + lane] : -1;          // (16 rows at most)
    }
    // the first bounds do not wait for the positions: up to these, blocks of the request are read
    const int first_block = chunk * a.chunk_blocks, held_end = min(first_block + a.chunk_blocks, (length + (1 << a.block_log) - 1) >> a.block_log);
    if (!kPick && first_block >= held_end) return;
    const int32_t *table = a.table + (int64_t)f.request * a.width;

    struct Bounds { i32x4_t hi[kSteps], lo[kSteps]; bool is; };
    auto id_of = [&](int b0) { return table[min(b0 + lane % 16, held_end - 1)]; };
    auto load = [&](int b0, int id, Bounds &b) {
        b.is = b0 + lane % 16 < held_end && id >= 0 && id < a.blocks;
        const __bf16 *p = a.bounds + ((int64_t)(b.is ? id : 0) * a.kv_heads + head) * 2 * DIM + g * 8;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            b.hi[s] = *reinterpret_cast<const i32x4_t *>(p + s * 32);
            b.lo[s] = *reinterpret_cast<const i32x4_t *>(p + DIM + s * 32);
        }
    };
    const int begin = first_block + wave * 16, window = min(a.group, COLS);      // columns of a row
    Bounds first, second;
    int id_next = 0;
    if (begin < held_end) {
        load(begin, id_of(begin), first);
        id_next = id_of(min(begin + kRound, held_end - 1));
    }
    const int seen = min(last, length - 1);               // of row `lane` (of the only one, in all lanes)
    if (!single)
        for (int s = 1; s < 16; s *= 2) last = max(last, __shfl_xor(last, s));
    last = min(__builtin_amdgcn_readfirstlane(last), length - 1);
    const int end_block = min(held_end, last < 0 ? 0 : (last >> a.block_log) + 1);
    if (!kPick && first_block >= end_block) return;
    for (int c = 0; c * COLS < (wide ? a.group : 1); ++c) {
        if (c) {
            __syncthreads();
            if (begin < end_block) {
                load(begin, id_of(begin), first);
                id_next = id_of(min(begin + kRound, held_end - 1));
            }
        }
        if (c) load_queries(c, tile0, rows);
        fill_queries();
        __syncthreads();
        const int pair = c * COLS + col, row = wide ? 0 : col / a.group;
        const bool there = wide ? pair < a.group : row < rows;
        auto round = [&](int b0, const Bounds &now, Bounds &next) {
            const int after = min(b0 + kRound, held_end - 1);        // (behind the last block, that one again)
            load(after, id_next, next);
            id_next = id_of(min(after + kRound, held_end - 1));
            asm volatile("" ::: "memory");             // queries are read again each round: kept, they would take the registers of another wavefront
            f64x4_t sum = {0, 0, 0, 0}, more = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t wh = now.hi[s][e / 2], wl = now.lo[s][e / 2];
                    const double x = (double)__builtin_bit_cast(float, e % 2 ? wh & 0xffff0000u : wh << 16);
                    const double y = (double)__builtin_bit_cast(float, e % 2 ? wl & 0xffff0000u : wl << 16);
                    const f64x2_t q = queries[8 * s + e][g][col];
                    if constexpr (COLS == 4) {
                        sum[e % 4] = __builtin_amdgcn_mfma_f64_4x4x4f64(x, q[0], sum[e % 4], 0, 0, 0);
                        more[e % 4] = __builtin_amdgcn_mfma_f64_4x4x4f64(y, q[1], more[e % 4], 0, 0, 0);
                    } else {
                        sum = __builtin_amdgcn_mfma_f64_16x16x4f64(x, q[0], sum, 0, 0, 0);
                        more = __builtin_amdgcn_mfma_f64_16x16x4f64(y, q[1], more, 0, 0, 0);
                    }
                }
            sum += more;
            if (COLS == 4) sum[0] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
            // over the columns of a row, into its first: windows of twice the width, then one that ends where the row does
            const uint64_t valid = __ballot(now.is);
#pragma unroll
            for (int r = 0; r < (COLS == 4 ? 1 : 4); ++r) {
                double v = there ? fmax(sum[r], -INFINITY) : -INFINITY;       // (a sum that is no number: -infinity)
                int w = 1;
                for (; 2 * w <= window; w *= 2) v = fmax(v, __shfl(v, lane + w));
                if (w < window) v = fmax(v, __shfl(v, lane + window - w));
                // lane: 16x16x4 holds block 4 r + g, 4x4x4 block 4 (lane / 4 % 4) + g of query head lane % COLS
                const int in = COLS == 4 ? lane / 4 % 4 * 4 + g : 4 * r + g, block = b0 + in;
                if (col == row * window && row < rows && block < end_block) {
                    uint64_t *to = kPick ? keys + row * a.width + block : a.scores + ((int64_t)(tile0 + row - a.row0) * a.kv_heads + head) * a.width + block;
                    const uint64_t key = valid >> in & 1 ? key_of(v) : 0;
                    *to = c && *to > key ? *to : key;
                }
            }
        };
        // two rounds at a time, so that bounds stay in the registers that they were loaded into
        for (int b0 = begin; b0 < end_block; b0 += 2 * kRound) {
            round(b0, first, second);
            if (b0 + kRound < end_block) round(b0 + kRound, second, first);
        }
    }
    if constexpr (kPick) {
        __syncthreads();
        for (int r = wave; r < rows; r += kThreads / 64) {
            const int own = __builtin_amdgcn_readlane(seen, r);
            pick_by_wave<EACH>(keys + r * a.width, own < 0 ? 0 : (own >> a.block_log) + 1, a.first, a.last, a.keep,
                               a.selected + ((int64_t)(tile0 + r) * a.kv_heads + head) * a.keep);
        }
    }
}

// The `keep` largest keys of a row and head, the lowest blocks where keys are equal, in ascending order.  The smallest key kept is found bit by bit, from the
// first that is not the same in all: each bit is one count over the keys, which stay in registers.
template <int THREADS, int EACH>
__global__ __launch_bounds__(THREADS) void kv_pick(SelectArgs a) {
    constexpr int kWaves = THREADS / 64;
    __shared__ int counts[2][EACH][kWaves];
    __shared__ int total[2][kWaves];
    __shared__ uint32_t bits[4][kWaves];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int row = a.row0 + (int)(blockIdx.x / a.kv_heads), head = blockIdx.x % a.kv_heads;
    // (the scores of all of the table's columns do not wait for how many the row sees)
    const uint64_t *scores = a.scores + ((int64_t)(row - a.row0) * a.kv_heads + head) * a.width;
    uint64_t key[EACH];
#pragma unroll
    for (int j = 0; j < EACH; ++j) key[j] = scores[min(j * THREADS + t, a.width - 1)];
    const int position = a.positions[row];
    Found f{};
    if (a.requests) f = last_place(a.requests, row, a.lengths, [&](int i) { return a.starts[i]; }, [](int, int start) { return (int64_t)start; });
    const int length = f.start <= row && row < f.end ? min(max(f.length, 0), a.width << a.block_log) : 0;
    const int last = min(position, length - 1), visible = last < 0 ? 0 : (last >> a.block_log) + 1;
    int32_t *out = a.selected + ((int64_t)row * a.kv_heads + head) * a.keep;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        const int b = j * THREADS + t;
        if (b >= visible) key[j] = 0;
        if (key[j] && (b < a.first || b >= visible - a.last)) key[j] = ~(uint64_t)0;
    }
    int turn = 0;
    auto count = [&](uint64_t least) {
        int n = 0;
#pragma unroll
        for (int j = 0; j < EACH; ++j) n += __builtin_popcountll(__ballot(key[j] >= least));
        if constexpr (kWaves == 1) return n;
        if (lane == 0) total[turn][wave] = n;
        __syncthreads();
        int all = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) all += total[turn][w];
        turn ^= 1;
        return all;
    };
    uint64_t least = 1;
    int kept = count(1);
    if (kept > a.keep) {
        // (those that are always kept are all ones)
        uint64_t set = 0, clear = 0;
#pragma unroll
        for (int j = 0; j < EACH; ++j)
            if (key[j] && ~key[j]) {
                set |= key[j];
                clear |= ~key[j];
            }
        uint32_t any[4] = {wave_or((uint32_t)set), wave_or((uint32_t)(set >> 32)), wave_or((uint32_t)clear), wave_or((uint32_t)(clear >> 32))};
        if constexpr (kWaves > 1) {
            if (lane < 4) bits[lane][wave] = lane == 0 ? any[0] : lane == 1 ? any[1] : lane == 2 ? any[2] : any[3];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int w = 0; w < kWaves; ++w) any[i] |= bits[i][w];
        }
        set = any[0] | (uint64_t)any[1] << 32;
        const uint64_t differ = set & (any[2] | (uint64_t)any[3] << 32);
        const int top = differ ? 63 - __builtin_clzll(differ) : -1;
        least = top == 63 ? 0 : set & ~(((uint64_t)2 << max(top, 0)) - 1);
        if (top < 0) least = set;                         // all the same
        for (int bit = top; bit >= 0; --bit) {
            const uint64_t next = least | (uint64_t)1 << bit;
            const int n = count(next);
            if (n < a.keep) continue;
            least = next;
            kept = n;
            if (n == a.keep) break;
        }
    }
    // of the keys that are `least`, so many more than fit are left out, the last ones
    const int chosen = min(kept, a.keep);
    const int above = kept > a.keep ? count(least + 1) : 0;         // (a key of all ones cannot be one too many: first + last <= keep)
    const int equal = chosen - above;
    // places: of an element, those chosen before it; of the elements before its own round and wavefront by counts in the LDS
    auto places = [&](auto want, int which, int (&before)[EACH]) {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const uint64_t set = __ballot(want(j));
            before[j] = __builtin_popcountll(set & (((uint64_t)1 << lane) - 1));
            if (lane == 0) counts[which][j][wave] = __builtin_popcountll(set);
        }
        __syncthreads();
        int sum = 0;
#pragma unroll
        for (int j = 0; j < EACH; ++j)
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                if (w == wave) before[j] += sum;
                sum += counts[which][j][w];
            }
    };
    int before[EACH];
    bool take[EACH];
    if (kept > a.keep) {
        places([&](int j) { return key[j] == least; }, 0, before);
#pragma unroll
        for (int j = 0; j < EACH; ++j) take[j] = key[j] > least || (key[j] == least && before[j] < equal);
    } else {
#pragma unroll
        for (int j = 0; j < EACH; ++j) take[j] = key[j] >= least;
    }
    places([&](int j) { return take[j]; }, 1, before);
#pragma unroll
    for (int j = 0; j < EACH; ++j)
        if (take[j]) out[before[j]] = j * THREADS + t;
    for (int i = chosen + t; i < a.keep; i += THREADS) out[i] = -1;
}

// The same with a wavefront to a row and head, where there are many: nothing waits for another at every bit.
template <int EACH>
__global__ __launch_bounds__(256) void kv_pick_rows(SelectArgs a) {
    const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= (int64_t)a.rows * a.kv_heads) return;
    const int row = a.row0 + (int)(unit / a.kv_heads), head = (int)(unit % a.kv_heads);
    const int position = a.positions[row];
    Found f{};
    if (a.requests) f = last_place(a.requests, row, a.lengths, [&](int i) { return a.starts[i]; }, [](int, int start) { return (int64_t)start; });
    const int length = f.start <= row && row < f.end ? min(max(f.length, 0), a.width << a.block_log) : 0;
    const int last = min(position, length - 1), visible = last < 0 ? 0 : (last >> a.block_log) + 1;
    pick_by_wave<EACH>(a.scores + unit * a.width, visible, a.first, a.last, a.keep, a.selected + ((int64_t)row * a.kv_heads + head) * a.keep);
}

constexpr int64_t kScoreBytes = (int64_t)256 << 20;

// Rows whose scores are kept at a time.
static int select_rows(const nnv_attention_desc &d, int rows) {
    const int64_t each = (int64_t)d.kv_heads * d.table_blocks * 8, fit = kScoreBytes / each;
    return (int)(fit < 1 ? 1 : fit < rows ? fit : rows);
}
size_t kv_select_workspace_bytes(const nnv_attention_desc &d, int rows) {
    return (size_t)select_rows(d, rows) * d.kv_heads * d.table_blocks * 8;
}

template <int DT, int DIM> static hipError_t launch_select_dim(const SelectArgs &args, int step, hipStream_t st) {
    SelectArgs a = args;
    const int all = a.rows;
    const bool narrow = a.group <= 4 && all <= a.requests;           // a row a request: no more columns than one has
    a.tile_rows = narrow || a.group > 16 ? 1 : 16 / a.group;
    for (int row0 = 0; row0 < all; row0 += step) {
        a.row0 = row0;
        a.rows = all - row0 < step ? all - row0 : step;
        const int64_t tiles = a.tile_rows == 1 ? a.rows : (int64_t)a.rows / a.tile_rows + a.requests;
        a.tiles = (int)tiles;
        // One launch for single rows of up to 1024 blocks that keep the chip busy with a workgroup each (64 rows over up to 512 blocks 30.0 -> 26.4 us), and wherever there
        // is little to do; not for prompts, whose scores wait for the matrix cores (1000 rows over up to 282 blocks: 49 us, in two launches 36).
        const int64_t units = tiles * a.kv_heads;
        if (a.requests && a.width <= 1024 && a.width * a.tile_rows <= kMostKeys && (narrow ? units >= 256 || a.width <= 256 : units < 512 && a.width <= 256) && all == a.rows) {
            a.chunks = 1;
            a.chunk_blocks = a.width;
            const unsigned picks = (unsigned)((tiles + (a.tile_rows > 1)) * a.kv_heads);
            if (a.width <= 512) narrow ? kv_scores<DT, DIM, 4, 8><<<picks, 512, 0, st>>>(a) : kv_scores<DT, DIM, 16, 8><<<picks, 512, 0, st>>>(a);
            else narrow ? kv_scores<DT, DIM, 4, 16><<<picks, 512, 0, st>>>(a) : kv_scores<DT, DIM, 16, 16><<<picks, 512, 0, st>>>(a);
            return hipGetLastError();
        }
        // as many chunks as make 1536 workgroups, of 64 to 1024 blocks, by the tiles that there are at least
        const int64_t whole = a.rows / a.tile_rows, least = a.requests < a.rows ? a.requests : a.rows, there = (whole > least ? whole : least) * a.kv_heads;
        int64_t parts = 1536 / (there ? there : 1);
        if (parts < (a.width + 1023) / 1024) parts = (a.width + 1023) / 1024;
        int64_t blocks = ((a.width + parts - 1) / parts + 63) / 64 * 64;
        while (tiles * a.kv_heads * ((a.width + blocks - 1) / blocks) >= 1 << 24) blocks *= 2;
        a.chunk_blocks = (int)blocks;
        a.chunks = (int)((a.width + blocks - 1) / blocks);
        const unsigned groups = (unsigned)(tiles * a.kv_heads * a.chunks);
        if (a.requests) {
            if (narrow) kv_scores<DT, DIM, 4, 0><<<groups, 256, 0, st>>>(a);
            else kv_scores<DT, DIM, 16, 0><<<groups, 256, 0, st>>>(a);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        const unsigned picks = (unsigned)a.rows * a.kv_heads;
        // (4775 rows and heads over up to 788 blocks: workgroups of 256 33 us, a wavefront each 24; 1612 over up to 2233: of 1024 60, 40)
        if (picks >= 512 && a.width <= 4096) {
            const unsigned fours = (picks + 3) / 4;
            if (a.width <= 512) kv_pick_rows<8><<<fours, 256, 0, st>>>(a);
            else if (a.width <= 1024) kv_pick_rows<16><<<fours, 256, 0, st>>>(a);
            else if (a.width <= 2048) kv_pick_rows<32><<<fours, 256, 0, st>>>(a);
            else kv_pick_rows<64><<<fours, 256, 0, st>>>(a);
        } else if (a.width <= 512) kv_pick<64, 8><<<picks, 64, 0, st>>>(a);
        else if (a.width <= 2048) kv_pick<256, 8><<<picks, 256, 0, st>>>(a);
        else if (a.width <= 8192) kv_pick<1024, 8><<<picks, 1024, 0, st>>>(a);
        else kv_pick<1024, 32><<<picks, 1024, 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <int DT> static hipError_t launch_select_type(const SelectArgs &a, int dim, int step, hipStream_t st) {
    return dim == 64 ? launch_select_dim<DT, 64>(a, step, st) : dim == 128 ? launch_select_dim<DT, 128>(a, step, st) : launch_select_dim<DT, 256>(a, step, st);
}
hipError_t launch_kv_select(const nnv_attention_desc &d, const SelectArgs &a, hipStream_t st) {
    const int step = select_rows(d, a.rows);
    return d.dtype == NNV_F16 ? launch_select_type<NNV_F16>(a, d.head_dim, step, st) : launch_select_type<NNV_BF16>(a, d.head_dim, step, st);
}

}  // namespace nnv

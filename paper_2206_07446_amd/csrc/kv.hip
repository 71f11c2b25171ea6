// A serving step's plan, and the cache of keys and values held in 4 bits: norms and rotations with the append, and reading back.
#include "nnv_internal.h"
#include "serving.h"
#include "lowbits.h"

namespace nnv {

// ---- the plan of a step -------------------------------------------------------------------------

// Counts are added up to kMany and no further: more than any launch has rows or any cache blocks, so that nothing wraps around.
constexpr int kMany = 1 << 30;
__device__ static inline int add_up(int a, int b) { return (int)min((uint32_t)a + (uint32_t)b, (uint32_t)kMany); }

// Exclusive sum over the workgroup's threads of counts of 0 to kMany; total is everybody's.  Lanes of a wavefront by shifts within rows of 16 and broadcasts
// between those, wavefronts through the LDS (scratch, by turns one of two).
template <int THREADS> __device__ static inline int block_scan(int v, int *scratch, int &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int incl = v;
    incl = add_up(incl, __builtin_amdgcn_update_dpp(0, incl, 0x111, 0xf, 0xf, false));
    incl = add_up(incl, __builtin_amdgcn_update_dpp(0, incl, 0x112, 0xf, 0xf, false));
    incl = add_up(incl, __builtin_amdgcn_update_dpp(0, incl, 0x114, 0xf, 0xf, false));
    incl = add_up(incl, __builtin_amdgcn_update_dpp(0, incl, 0x118, 0xf, 0xf, false));
    incl = add_up(incl, __builtin_amdgcn_update_dpp(0, incl, 0x142, 0xa, 0xf, false));
    incl = add_up(incl, __builtin_amdgcn_update_dpp(0, incl, 0x143, 0xc, 0xf, false));
    if (lane == 63) scratch[wave] = incl;
    __syncthreads();
    int before = __shfl_up(incl, 1);
    if (lane == 0) before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) {
        if (i < wave) before = add_up(before, scratch[i]);
        total = add_up(total, scratch[i]);
    }
    return before;
}

// The last of a chunk's requests whose `from` is at `at` or before it.
template <int CHUNK> __device__ static inline int last_from(const int *from, int last, int at) {
    int i = 0;
#pragma unroll
    for (int step = CHUNK / 2; step; step /= 2)
        if (i + step <= last && from[i + step] <= at) i += step;
    return i;
}

// Every workgroup sums over all requests, a chunk of EACH to a thread at a time (two prefix sums: rows, then blocks needed), and writes the rows of its
// own range and its share of the new table entries; the requests' own outputs are written by the workgroup whose turn the chunk is.
// No workgroup waits for another: what one needs of another's table entries it takes from the free list itself.
// Bound by the latency of a chunk's loads (those of the next are on their way), two scans, a search.
template <int THREADS, int EACH>
__global__ __launch_bounds__(THREADS) void kv_plan(PlanArgs a, int rows_each) {
    constexpr int kPlanThreads = THREADS, kPlanEach = EACH, kPlanChunk = kPlanThreads * EACH;
    __shared__ int scratch[2][kPlanThreads / 64];
    __shared__ int s_start[kPlanChunk], s_held[kPlanChunk], s_entry[kPlanChunk];   // s_entry: blocks that the requests before this one ask for
    __shared__ bool s_granted[kPlanChunk];
    const int t = threadIdx.x, block = 1 << a.block_log;
    const int64_t capacity = (int64_t)a.width << a.block_log;
    auto read = [&](const int32_t *p, int c0, int (&v)[kPlanEach]) {
        if (EACH > 1 && c0 + (t + 1) * kPlanEach <= a.requests) {
            __builtin_memcpy(v, p + c0 + t * kPlanEach, sizeof(v));
            return;
        }
#pragma unroll
        for (int j = 0; j < kPlanEach; ++j) {
            const int i = c0 + t * kPlanEach + j;
            v[j] = i < a.requests ? p[i] : 0;
        }
    };
    int held_next[kPlanEach], fresh_next[kPlanEach];
    read(a.held, 0, held_next);
    read(a.fresh, 0, fresh_next);
    const int count = max(0, min(*a.free_count, a.blocks));
    auto free_block = [&](int place) { return a.free_blocks[count - 1 - place]; };
    const int r0 = min(blockIdx.x * (int64_t)rows_each, (int64_t)a.rows), r1 = min(r0 + rows_each, a.rows);
    int rows_before = 0, need_before = 0, taken = 0;
    for (int c0 = 0, chunk = 0; c0 < a.requests; c0 += kPlanChunk, ++chunk) {
        int held[kPlanEach], fresh[kPlanEach], sum = 0;
#pragma unroll
        for (int j = 0; j < kPlanEach; ++j) {
            held[j] = held_next[j];
            fresh[j] = fresh_next[j];
            sum = add_up(sum, max(min(fresh[j], kMany), 0));
        }
        if (c0 + kPlanChunk < a.requests) {
            read(a.held, c0 + kPlanChunk, held_next);
            read(a.fresh, c0 + kPlanChunk, fresh_next);
        }
        int chunk_rows, chunk_need, start[kPlanEach], need[kPlanEach], wanted = 0;
        int at = add_up(rows_before, block_scan<THREADS>(sum, scratch[0], chunk_rows));
        bool fits[kPlanEach];
#pragma unroll
        for (int j = 0; j < kPlanEach; ++j) {
            const int64_t all = (int64_t)held[j] + fresh[j];
            start[j] = at;
            at = add_up(at, max(min(fresh[j], kMany), 0));
            fits[j] = held[j] >= 0 && fresh[j] >= 0 && all <= capacity && at <= a.rows;
            need[j] = fits[j] ? (int)(((all + block - 1) >> a.block_log) - (((int64_t)held[j] + block - 1) >> a.block_log)) : 0;
            wanted = add_up(wanted, need[j]);
        }
        int entry = block_scan<THREADS>(wanted, scratch[1], chunk_need);
        const bool mine = chunk % gridDim.x == blockIdx.x;
#pragma unroll
        for (int j = 0; j < kPlanEach; ++j) {
            const int i = c0 + t * kPlanEach + j, upto = add_up(add_up(need_before, entry), need[j]);
            const bool granted = fits[j] && (need[j] == 0 || upto <= count);
            if (granted && need[j]) taken = upto;
            s_start[t * kPlanEach + j] = min(start[j], a.rows);
            s_held[t * kPlanEach + j] = held[j];
            s_entry[t * kPlanEach + j] = entry;
            s_granted[t * kPlanEach + j] = granted;
            if (mine && i < a.requests) {
                a.starts[i] = min(start[j], a.rows);
                a.lengths[i] = granted ? held[j] + fresh[j] : (int)max((int64_t)0, min((int64_t)held[j], capacity));
            }
            entry = add_up(entry, need[j]);
        }
        __syncthreads();
        const int last = min(kPlanChunk, a.requests - c0) - 1;
        // new table entries: a workgroup writes its share of the chunk's, up to where the free list ends
        const int entries = max(0, min(chunk_need, count - need_before)), share = (int)(((int64_t)entries + gridDim.x - 1) / gridDim.x);
        const int e1 = (int)min((int64_t)entries, (int64_t)share * (blockIdx.x + 1));
        for (int64_t e = (int64_t)share * blockIdx.x + t; e < e1; e += kPlanThreads) {
            const int i = last_from<kPlanChunk>(s_entry, last, (int)e);
            if (!s_granted[i]) continue;
            const int column = (int)((((int64_t)s_held[i] + block - 1) >> a.block_log) + (e - s_entry[i]));
            a.table[(int64_t)(c0 + i) * a.width + column] = free_block(need_before + (int)e);
        }
        const int lo = max(r0, rows_before), hi = min(r1, add_up(rows_before, chunk_rows));
        for (int r = lo + t; r < hi; r += kPlanThreads) {
            const int i = last_from<kPlanChunk>(s_start, last, r);
            int32_t position = -1;
            int64_t slot = -1;
            if (s_granted[i]) {
                position = s_held[i] + (r - s_start[i]);
                const int b = position >> a.block_log, old = (int)(((int64_t)s_held[i] + block - 1) >> a.block_log);
                const int id = b < old ? a.table[(int64_t)(c0 + i) * a.width + b] : free_block(need_before + s_entry[i] + b - old);
                if (id >= 0 && id < a.blocks) slot = ((int64_t)id << a.block_log) + (position & (block - 1));
            }
            a.positions[r] = position;
            a.slots[r] = slot;
        }
        rows_before = add_up(rows_before, chunk_rows);
        need_before = add_up(need_before, chunk_need);
        __syncthreads();
    }
    for (int r = max(r0, rows_before) + t; r < r1; r += kPlanThreads) {
        a.positions[r] = -1;
        a.slots[r] = -1;
    }
    if (blockIdx.x) return;
    // the pops end where the last admitted request's do
#pragma unroll
    for (int s = 1; s < 64; s *= 2) taken = max(taken, __shfl_xor(taken, s));
    if ((t & 63) == 0) scratch[0][t >> 6] = taken;
    __syncthreads();
    if (t) return;
    for (int i = 1; i < kPlanThreads / 64; ++i) taken = max(taken, scratch[0][i]);
    *a.left = count - taken;
    a.starts[a.requests] = min(rows_before, a.rows);
}

hipError_t launch_kv_plan(const PlanArgs &a, hipStream_t st) {
    // A workgroup per 1024 rows, as many as the chip holds at a time.  A request to a thread and all of them in one chunk where that can be: us with 256
    // threads x 1, 256 x 4, 1024 x 1, x 2, x 4, of one row a request: 64 requests 4.4, 5.4, 5.6, 6.3, 7.2; 1024: 10.4, 7.7, 5.6, 6.4, 7.3;
    // 2000: 16.3, 10.7, 8.3, 6.4, 7.5; 3000: 21.5, 13.0, 10.9, 9.7, 7.6; 9000: 55, 27, 26, 19, 16.
    const int wanted = (int)((a.rows + (int64_t)1023) / 1024), groups = wanted < 1 ? 1 : wanted > 512 ? 512 : wanted;
    const int each = (int)((a.rows + (int64_t)groups - 1) / groups);
    if (a.requests <= 256) kv_plan<256, 1><<<groups, 256, 0, st>>>(a, each);
    else if (a.requests <= 1024) kv_plan<1024, 1><<<groups, 1024, 0, st>>>(a, each);
    else if (a.requests <= 2048) kv_plan<1024, 2><<<groups, 1024, 0, st>>>(a, each);
    else kv_plan<1024, 4><<<groups, 1024, 0, st>>>(a, each);
    return hipGetLastError();
}

// ---- the cache ----------------------------------------------------------------------------------

// Byte of a token's eight codes from value d0 of a head (a multiple of 8) in its block; of heads of 64 the second four
// lie 8 bytes further.
template <int DIM> __device__ static inline int key_codes_at(int token, int d0) { return token * (DIM / 2) + d0 / 2; }
template <int DIM> __device__ static inline int value_codes_at(int token, int d0) {
    return (((token >> 2) * 16 + d0 / (DIM / 16)) * 4 + (token & 3)) * (DIM / 32) + (d0 % (DIM / 16)) / 2;
}
template <int DIM> __device__ static inline int key_scale_at(int token, int d0) { return token * (DIM / 32) + d0 / 32; }
template <int DIM> __device__ static inline int value_scale_at(int token, int d0) { return ((token >> 2) * (DIM / 32) + d0 / 32) * 4 + (token & 3); }

template <int DIM> __device__ static inline void store_value_codes(char *p, int token, int d0, uint32_t codes) {
    char *at = p + value_codes_at<DIM>(token, d0);
    if constexpr (DIM == 64) {
        *reinterpret_cast<uint16_t *>(at) = (uint16_t)codes;
        *reinterpret_cast<uint16_t *>(at + 8) = (uint16_t)(codes >> 16);
    } else {
        *reinterpret_cast<uint32_t *>(at) = codes;
    }
}
template <int DIM> __device__ static inline uint32_t load_value_codes(const char *p, int token, int d0) {
    const char *at = p + value_codes_at<DIM>(token, d0);
    if constexpr (DIM == 64) return *reinterpret_cast<const uint16_t *>(at) | (uint32_t)*reinterpret_cast<const uint16_t *>(at + 8) << 16;
    else return *reinterpret_cast<const uint32_t *>(at);
}

// Eight of the 32 values of a group, four lanes to a group, -> their codes and the group's scale byte.
template <int DT> __device__ static inline uint32_t e2m1_codes8(const float (&v)[8], uint32_t &byte) {
    float x[8];
    auto most = [&] {
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = max(amax, __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu);
        amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
        return max(amax, (uint32_t)__shfl_xor((int)amax, 2));
    };
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v[i];
    uint32_t amax = most();
    if (__any(amax >= kInfBits)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = e2m1_input(x[i]);
        amax = most();
    }
    byte = e2m1_scale_byte<DT>(amax);
    const float scale = scale_of_byte(byte);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
    return w;
}

__device__ static inline void load8f(const float *p, float (&v)[8]) {
    const f32x4_t a = reinterpret_cast<const f32x4_t *>(p)[0], b = reinterpret_cast<const f32x4_t *>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
// Rounded; zeros where the row is none.
template <int DT> __device__ static inline void store8(typename Elem<DT>::type *p, const float (&v)[8], bool there = true) {
    ElemVec<DT, 8> x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (typename Elem<DT>::type)v[i];
    i32x4_t words = __builtin_bit_cast(i32x4_t, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) words[i] = there ? words[i] : 0;
    *reinterpret_cast<i32x4_t *>(p) = words;
}

// What norm and rotation of values d0 .. d0 + 7 of HEADS heads of a row read, eight values of the rotation's other half with their weights among them.  FAST: these lie in one
// half of the rotated part, or behind it, and come in one load each; the head itself is read in the place of weights and angles
// that there are not.  The first part does not wait for the row's position, so that a thread's chain of loads has two links.
template <int DT, int DIM, bool FAST, int HEADS> struct RopeInput {
    typedef typename Elem<DT>::type T;
    ElemVec<DT, 8> x[HEADS], other_x[HEADS];
    float w[8], other_w[8], cs[8], sn[8];
    int half, other;
    bool turns, low;
    static __device__ ElemVec<DT, 8> eight(const T *p) {
        if constexpr (FAST) return *reinterpret_cast<const ElemVec<DT, 8> *>(p);
        ElemVec<DT, 8> v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p[i];
        return v;
    }
    // of heads `head`, .. `more` further ones (the last of them again where a thread takes more)
    __device__ void load_values(const T *head, int more, int d0) {
#pragma unroll
        for (int n = 0; n < HEADS; ++n) x[n] = eight(head + (n ? min(n, more) * DIM : 0) + d0);
    }
    __device__ void load_rest(const T *head, int more, int d0, const float *weight, const RopeArgs &a) {
        half = a.rotary / 2;
        turns = d0 < a.rotary;
        low = d0 < half;
        if constexpr (FAST) {
            other = !turns || a.interleaved ? d0 : low ? d0 + half : d0 - half;
#pragma unroll
            for (int n = 0; n < HEADS; ++n) other_x[n] = eight(head + (n ? min(n, more) * DIM : 0) + other);
            const float *none = reinterpret_cast<const float *>(head);
            load8f(weight ? weight + d0 : none, w);
            load8f(weight ? weight + other : none, other_w);
        } else {
            if (weight) load8f(weight + d0, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int d = d0 + i, at = d >= a.rotary ? d : a.interleaved ? d ^ 1 : d < half ? d + half : d - half;
#pragma unroll
                for (int n = 0; n < HEADS; ++n) other_x[n][i] = head[(n ? min(n, more) * DIM : 0) + at];
                if (weight) other_w[i] = weight[at];
            }
        }
    }
    __device__ void load_angles(const T *head, int d0, const float *angles, const RopeArgs &a) {
        if constexpr (FAST) {
            const float *none = reinterpret_cast<const float *>(head);
            const int angle = !turns ? 0 : a.interleaved ? d0 / 2 : low ? d0 : other, more = a.interleaved || !a.rotary ? 0 : 4;
            const float *c = a.rotary ? angles + angle : none, *s = a.rotary ? angles + half + angle : none;
            const f32x4_t c0 = *reinterpret_cast<const f32x4_t *>(c), c1 = *reinterpret_cast<const f32x4_t *>(c + more);
            const f32x4_t s0 = *reinterpret_cast<const f32x4_t *>(s), s1 = *reinterpret_cast<const f32x4_t *>(s + more);
#pragma unroll
            for (int i = 0; i < 4; ++i) { cs[i] = c0[i]; cs[4 + i] = c1[i]; sn[i] = s0[i]; sn[4 + i] = s1[i]; }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int d = d0 + i, angle = a.interleaved ? d >> 1 : d < half ? d : d - half;
                if (d < a.rotary) { cs[i] = angles[angle]; sn[i] = angles[half + angle]; }
            }
        }
    }
    // In F (float for queries, double for keys), DIM / 8 lanes to a head.
    template <typename F> __device__ void norm_rope(int n, int d0, bool norm, const RopeArgs &a, F (&h)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = (F)(float)x[n][i];
        F inv = 1;
        if (norm) {
            F sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += h[i] * h[i];
#pragma unroll
            for (int s = 1; s < DIM / 8; s *= 2) sum += __shfl_xor(sum, s);
            inv = (F)1 / sqrt(sum / (F)DIM + (F)a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = h[i] * inv * (F)w[i];
        }
        if (!turns) return;
        if (FAST && a.interleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const F x0 = h[2 * i], x1 = h[2 * i + 1];
                h[2 * i] = x0 * (F)cs[i] - x1 * (F)sn[i];
                h[2 * i + 1] = x1 * (F)cs[i] + x0 * (F)sn[i];
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int d = d0 + i;
            if (!FAST && d >= a.rotary) continue;
            const bool lower = FAST ? low : a.interleaved ? !(d & 1) : d < half;
            F p = (F)(float)other_x[n][i];
            if (norm) p = p * inv * (F)other_w[i];
            h[i] = h[i] * (F)cs[i] + p * (F)(lower ? -sn[i] : sn[i]);
        }
    }
};

// A thread takes eight values of two query heads of a row, so that weights and angles are read once for them, or of one key or value head.  (8191 rows of
// 32 heads of 128: queries alone 36.1 us with one head a thread, 28.7 with two, 27.9 with four, 23 at the rate of a copy; 64 rows are the same with all.)
// Workgroups of queries, of keys and of values are apart: the keys' float64 is then not waited for by others of its wavefront.  Bound by the traffic of
// the rows, or of a few rows by the chain of loads.
constexpr int kQueryHeads = 2;
template <int DT, int DIM, bool FAST>
__global__ __launch_bounds__(256) void qk_norm_rope(RopeArgs a, uint32_t query_groups, uint32_t key_groups) {
    typedef typename Elem<DT>::type T;
    constexpr uint32_t kLanes = DIM / 8;
    uint32_t group = blockIdx.x;
    const int d0 = (threadIdx.x % kLanes) * 8;
    auto is_there = [&](int position) { return position >= 0 && (a.rotary == 0 || position < a.max_position); };
    if (group < query_groups) {
        const uint32_t unit = (group * 256 + threadIdx.x) / kLanes, per_row = ((uint32_t)a.q_heads + kQueryHeads - 1) / kQueryHeads,
                       row = unit / per_row, first = unit % per_row * kQueryHeads;
        if (row >= (uint32_t)a.rows) return;
        const int position = a.positions[row], more = a.q_heads - 1 - (int)first;
        const T *head = static_cast<const T *>(a.q) + row * a.ldq + (int64_t)first * DIM;
        RopeInput<DT, DIM, FAST, kQueryHeads> in;
        in.load_values(head, more, d0);
        in.load_rest(head, more, d0, a.q_weight, a);
        const bool there = is_there(position);
        in.load_angles(head, d0, a.rope + (there ? (int64_t)position * a.rotary : 0), a);
        T *out = static_cast<T *>(a.q_out) + ((int64_t)row * a.q_heads + first) * DIM + d0;
#pragma unroll
        for (int n = 0; n < kQueryHeads; ++n) {
            float v[8];
            in.template norm_rope<float>(n, d0, a.q_weight != nullptr, a, v);
            if (n == 0 || n <= more) store8<DT>(out + n * DIM, v, there);
        }
        return;
    }
    group -= query_groups;
    const bool key = group < key_groups;
    const uint32_t unit = ((key ? group : group - key_groups) * 256 + threadIdx.x) / kLanes, row = unit / (uint32_t)a.kv_heads, hk = unit % (uint32_t)a.kv_heads;
    if (row >= (uint32_t)a.rows) return;
    const int position = a.positions[row];
    const int64_t slot = a.cache ? a.slots[row] : -1;
    const T *head = static_cast<const T *>(key ? a.k : a.v) + row * (key ? a.ldk : a.ldv) + (int64_t)hk * DIM;
    RopeInput<DT, DIM, FAST, 1> in;
    in.load_values(head, 0, d0);
    bool there;
    float v[8];
    if (key) {
        in.load_rest(head, 0, d0, a.k_weight, a);
        there = is_there(position);
        in.load_angles(head, d0, a.rope + (there ? (int64_t)position * a.rotary : 0), a);
        double x[8];
        in.template norm_rope<double>(0, d0, a.k_weight != nullptr, a, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = float_odd(x[j]);
        if (a.k_out) store8<DT>(static_cast<T *>(a.k_out) + ((int64_t)row * a.kv_heads + hk) * DIM + d0, v, there);
    } else {
        there = is_there(position);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (float)in.x[0][j];
    }
    if (!there || slot < 0 || slot >= a.total_slots) return;
    uint32_t byte;
    const uint32_t codes = e2m1_codes8<DT>(v, byte);
    const KvLayout at{DIM, 1 << a.block_log};
    char *block = a.cache + ((slot >> a.block_log) * a.kv_heads + hk) * at.head_bytes();
    const int token = (int)(slot & (at.tokens - 1));
    if (key) {
        *reinterpret_cast<uint32_t *>(block + key_codes_at<DIM>(token, d0)) = codes;
        if (d0 % 32 == 0) block[at.key_scale_at() + key_scale_at<DIM>(token, d0)] = (char)byte;
    } else {
        store_value_codes<DIM>(block + at.value_at(), token, d0, codes);
        if (d0 % 32 == 0) block[at.value_scale_at() + value_scale_at<DIM>(token, d0)] = (char)byte;
    }
}

template <int DT, int DIM> static hipError_t launch_rope_dim(const RopeArgs &a, hipStream_t st) {
    auto groups = [&](int heads) { return (unsigned)(((int64_t)a.rows * heads * (DIM / 8) + 255) / 256); };
    const unsigned queries = a.q ? groups((a.q_heads + kQueryHeads - 1) / kQueryHeads) : 0, keys = a.k ? groups(a.kv_heads) : 0, all = queries + keys + (a.cache ? keys : 0);
    const bool turns = a.rotary % (a.interleaved ? 8 : 16) == 0;
    const bool fast = turns && (!a.q || a.ldq % 8 == 0) && (!a.k || (a.ldk % 8 == 0 && a.ldv % 8 == 0));
    if (fast) qk_norm_rope<DT, DIM, true><<<all, 256, 0, st>>>(a, queries, keys);
    else qk_norm_rope<DT, DIM, false><<<all, 256, 0, st>>>(a, queries, keys);
    return hipGetLastError();
}

template <int DT> static hipError_t launch_rope_type(const RopeArgs &a, int dim, hipStream_t st) {
    return dim == 64 ? launch_rope_dim<DT, 64>(a, st) : dim == 128 ? launch_rope_dim<DT, 128>(a, st) : launch_rope_dim<DT, 256>(a, st);
}

hipError_t launch_qk_norm_rope(const RopeArgs &a, int dim, int dtype, hipStream_t st) {
    return dtype == NNV_F16 ? launch_rope_type<NNV_F16>(a, dim, st) : launch_rope_type<NNV_BF16>(a, dim, st);
}

// A thread reads eight values of a head of a slot: keys, then values.  Bound by what it writes (8191 rows of 6 heads of 64, 16 MB: 6 us).
template <int DT, int DIM>
__global__ __launch_bounds__(256) void kv_read(int n, const int64_t *__restrict__ slots, const char *__restrict__ cache, void *k, void *v, int kv_heads,
                                               int block_log, int64_t total_slots) {
    typedef typename Elem<DT>::type T;
    constexpr int kLanes = DIM / 8;
    const int64_t unit = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kLanes;
    const int both = k && v ? 2 : 1;
    const int64_t i = unit / (both * kv_heads);
    if (i >= n) return;
    const int part = (int)(unit % (both * kv_heads)), d0 = (threadIdx.x % kLanes) * 8;
    const bool key = both == 2 ? part < kv_heads : k != nullptr;
    const int hk = part % kv_heads;
    const int64_t slot = slots[i];
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (slot >= 0 && slot < total_slots) {
        const KvLayout at{DIM, 1 << block_log};
        const char *block = cache + ((slot >> block_log) * kv_heads + hk) * at.head_bytes();
        const int token = (int)(slot & (at.tokens - 1));
        const uint32_t codes = key ? *reinterpret_cast<const uint32_t *>(block + key_codes_at<DIM>(token, d0))
                                   : load_value_codes<DIM>(block + at.value_at(), token, d0);
        const uint32_t byte = (uint8_t)(key ? block[at.key_scale_at() + key_scale_at<DIM>(token, d0)]
                                            : block[at.value_scale_at() + value_scale_at<DIM>(token, d0)]);
        const float scale = scale_of_byte(min(max(byte, 1u), kMostE2m1Byte<DT>));
        const auto p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
        const auto p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
        x[0] = p0[0]; x[1] = p0[1]; x[2] = p1[0]; x[3] = p1[1];
        x[4] = p2[0]; x[5] = p2[1]; x[6] = p3[0]; x[7] = p3[1];
    }
    store8<DT>(static_cast<T *>(key ? k : v) + (i * kv_heads + hk) * DIM + d0, x);
}

template <int DT, int DIM>
static hipError_t launch_read_dim(int n, const int64_t *slots, const char *cache, void *k, void *v, int kv_heads, int block_log, int64_t total_slots, hipStream_t st) {
    const int64_t threads = (int64_t)n * (k && v ? 2 : 1) * kv_heads * (DIM / 8);
    kv_read<DT, DIM><<<(unsigned)((threads + 255) / 256), 256, 0, st>>>(n, slots, cache, k, v, kv_heads, block_log, total_slots);
    return hipGetLastError();
}

hipError_t launch_kv_read(int n, const int64_t *slots, const char *cache, void *k, void *v, int kv_heads, int dim, int block_log, int64_t total_slots,
                          int dtype, hipStream_t st) {
#define NNV_READ(DT, DIM) launch_read_dim<DT, DIM>(n, slots, cache, k, v, kv_heads, block_log, total_slots, st)
    if (dtype == NNV_F16) return dim == 64 ? NNV_READ(NNV_F16, 64) : dim == 128 ? NNV_READ(NNV_F16, 128) : NNV_READ(NNV_F16, 256);
    return dim == 64 ? NNV_READ(NNV_BF16, 64) : dim == 128 ? NNV_READ(NNV_BF16, 128) : NNV_READ(NNV_BF16, 256);
#undef NNV_READ
}

}  // namespace nnv

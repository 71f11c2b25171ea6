// A serving step's plan, and the cache of keys and values held in 4 bits: norms and rotations with the append, and reading back.
#include "nnv_internal.h"
#include "serving.h"
#include "lowbits.h"

namespace nnv {

// ---- the plan of a step -------------------------------------------------------------------------

constexpr int kPlanThreads = 256, kPlanEach = 4, kPlanChunk = kPlanThreads * kPlanEach;

// Counts are added up to kMany and no further: more than any launch has rows or any cache blocks, so that nothing wraps around.
constexpr int kMany = 1 << 30;
__device__ static inline int add_up(int a, int b) { return (int)min((uint32_t)a + (uint32_t)b, (uint32_t)kMany); }

// Exclusive sum over the workgroup's threads of counts of 0 to kMany; total is everybody's.  Lanes of a wavefront by shifts within rows of 16 and broadcasts
// between those, wavefronts through the LDS (scratch, by turns one of two).
__device__ static inline int block_scan(int v, int *scratch, int &total) {
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
    for (int i = 0; i < kPlanThreads / 64; ++i) {
        if (i < wave) before = add_up(before, scratch[i]);
        total = add_up(total, scratch[i]);
    }
    return before;
}

// The last of a chunk's requests whose `from` is at `at` or before it.
__device__ static inline int last_from(const int *from, int last, int at) {
    int i = 0;
#pragma unroll
    for (int step = kPlanChunk / 2; step; step /= 2)
        if (i + step <= last && from[i + step] <= at) i += step;
    return i;
}

// Every workgroup sums over all requests, 1024 at a time (two prefix sums: rows, then blocks needed), and writes the rows of its
// own range and its share of the new table entries; the requests' own outputs are written by the workgroup whose turn the chunk is.
// No workgroup waits for another: what one needs of another's table entries it takes from the free list itself.
// Bound by the latency of a chunk's loads (those of the next are on their way), two scans, a search.
__global__ __launch_bounds__(kPlanThreads) void kv_plan(PlanArgs a, int rows_each) {
    __shared__ int scratch[2][kPlanThreads / 64];
    __shared__ int s_start[kPlanChunk], s_held[kPlanChunk], s_entry[kPlanChunk];   // s_entry: blocks that the requests before this one ask for
    __shared__ bool s_granted[kPlanChunk];
    const int t = threadIdx.x, block = 1 << a.block_log;
    const int64_t capacity = (int64_t)a.width << a.block_log;
    auto read = [&](const int32_t *p, int c0, int (&v)[kPlanEach]) {
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
        int at = add_up(rows_before, block_scan(sum, scratch[0], chunk_rows));
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
        int entry = block_scan(wanted, scratch[1], chunk_need);
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
            const int i = last_from(s_entry, last, (int)e);
            if (!s_granted[i]) continue;
            const int column = (int)((((int64_t)s_held[i] + block - 1) >> a.block_log) + (e - s_entry[i]));
            a.table[(int64_t)(c0 + i) * a.width + column] = free_block(need_before + (int)e);
        }
        const int lo = max(r0, rows_before), hi = min(r1, add_up(rows_before, chunk_rows));
        for (int r = lo + t; r < hi; r += kPlanThreads) {
            const int i = last_from(s_start, last, r);
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
    // a workgroup per 1024 rows, as many as the chip holds at a time
    const int wanted = (int)((a.rows + (int64_t)1023) / 1024), groups = wanted < 1 ? 1 : wanted > 512 ? 512 : wanted;
    const int each = (int)((a.rows + (int64_t)groups - 1) / groups);
    kv_plan<<<groups, kPlanThreads, 0, st>>>(a, each);
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
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = e2m1_input(v[i]);
        amax = max(amax, __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu);
    }
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
    byte = e2m1_scale_byte<DT>(amax);
    const float scale = scale_of_byte(byte);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
    return w;
}

template <int DT, bool FAST> __device__ static inline void load8(const typename Elem<DT>::type *p, float (&v)[8]) {
    if constexpr (FAST) {
        const ElemVec<DT, 8> x = *reinterpret_cast<const ElemVec<DT, 8> *>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)p[i];
    }
}
__device__ static inline void load8f(const float *p, float (&v)[8]) {
    const f32x4_t a = reinterpret_cast<const f32x4_t *>(p)[0], b = reinterpret_cast<const f32x4_t *>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
template <int DT> __device__ static inline void store8(typename Elem<DT>::type *p, const float (&v)[8]) {
    ElemVec<DT, 8> x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (typename Elem<DT>::type)v[i];
    *reinterpret_cast<ElemVec<DT, 8> *>(p) = x;
}

// Norm and rotation of values d0 .. d0 + 7 of a head in F (float for queries, double for keys), DIM / 8 lanes to a head.
// FAST: eight values lie in one half of the rotated part, or behind it, and come in one load.
template <typename F, int DT, int DIM, bool FAST>
__device__ static inline void norm_rope8(const typename Elem<DT>::type *head, int d0, const float *weight, const float *angles, const RopeArgs &a, F (&h)[8]) {
    float x[8], w[8];
    load8<DT, FAST>(head + d0, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = (F)x[i];
    F inv = 1;
    if (weight) {
        F sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += h[i] * h[i];
#pragma unroll
        for (int s = 1; s < DIM / 8; s *= 2) sum += __shfl_xor(sum, s);
        inv = (F)1 / sqrt(sum / (F)DIM + (F)a.eps);
        load8f(weight + d0, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = h[i] * inv * (F)w[i];
    }
    if (d0 >= a.rotary) return;
    const int half = a.rotary / 2;
    F turned[8];
    if constexpr (FAST) {
        float c[8], s[8], o[8];
        if (a.interleaved) {
            const f32x4_t cc = *reinterpret_cast<const f32x4_t *>(angles + d0 / 2), ss = *reinterpret_cast<const f32x4_t *>(angles + half + d0 / 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                turned[2 * i] = h[2 * i] * (F)cc[i] - h[2 * i + 1] * (F)ss[i];
                turned[2 * i + 1] = h[2 * i + 1] * (F)cc[i] + h[2 * i] * (F)ss[i];
            }
        } else {
            const bool low = d0 < half;
            const int other = low ? d0 + half : d0 - half, angle = low ? d0 : other;
            load8<DT, true>(head + other, o);
            if (weight) load8f(weight + other, w);
            load8f(angles + angle, c);
            load8f(angles + half + angle, s);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                F p = (F)o[i];
                if (weight) p = p * inv * (F)w[i];
                turned[i] = low ? h[i] * (F)c[i] - p * (F)s[i] : h[i] * (F)c[i] + p * (F)s[i];
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int d = d0 + i;
            turned[i] = h[i];
            if (d >= a.rotary) continue;
            const bool low = a.interleaved ? !(d & 1) : d < half;
            const int other = a.interleaved ? d ^ 1 : low ? d + half : d - half;
            const int angle = a.interleaved ? d >> 1 : low ? d : other;
            F p = (F)(float)head[other];
            if (weight) p = p * inv * (F)weight[other];
            const F c = (F)angles[angle], s = (F)angles[half + angle];
            turned[i] = low ? h[i] * c - p * s : h[i] * c + p * s;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = turned[i];
}

// A thread takes eight values of a head of a row.  Workgroups of queries, of keys and of values are apart: the keys' float64 is then not
// waited for by others of its wavefront.  What a thread reads is asked for before it is known whether the row is one, so that the
// chain of loads is a position and its angles, no more.  Bound by the traffic of the rows.
template <int DT, int DIM, bool FAST>
__global__ __launch_bounds__(256) void qk_norm_rope(RopeArgs a, uint32_t query_groups, uint32_t key_groups) {
    typedef typename Elem<DT>::type T;
    constexpr uint32_t kLanes = DIM / 8;
    const uint32_t group = blockIdx.x;
    const int d0 = (threadIdx.x % kLanes) * 8;
    if (group < query_groups) {
        const uint32_t unit = (group * 256 + threadIdx.x) / kLanes, row = unit / (uint32_t)a.q_heads, h = unit % (uint32_t)a.q_heads;
        if (row >= (uint32_t)a.rows) return;
        const int position = a.positions[row];
        const bool there = position >= 0 && (a.rotary == 0 || position < a.max_position);
        float v[8];
        norm_rope8<float, DT, DIM, FAST>(static_cast<const T *>(a.q) + row * a.ldq + (int64_t)h * DIM, d0, a.q_weight,
                                         a.rope + (there ? (int64_t)position * a.rotary : 0), a, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = there ? v[i] : 0.f;
        store8<DT>(static_cast<T *>(a.q_out) + ((int64_t)row * a.q_heads + h) * DIM + d0, v);
        return;
    }
    const bool key = group < query_groups + key_groups;
    const uint32_t unit = ((group - query_groups - (key ? 0 : key_groups)) * 256 + threadIdx.x) / kLanes;
    const uint32_t row = unit / (uint32_t)a.kv_heads, hk = unit % (uint32_t)a.kv_heads;
    if (row >= (uint32_t)a.rows) return;
    const int position = a.positions[row];
    const int64_t slot = a.cache ? a.slots[row] : -1;
    const bool there = position >= 0 && (a.rotary == 0 || position < a.max_position);
    float v[8];
    if (key) {
        double x[8];
        norm_rope8<double, DT, DIM, FAST>(static_cast<const T *>(a.k) + row * a.ldk + (int64_t)hk * DIM, d0, a.k_weight,
                                          a.rope + (there ? (int64_t)position * a.rotary : 0), a, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = there ? float_odd(x[i]) : 0.f;
        if (a.k_out) store8<DT>(static_cast<T *>(a.k_out) + ((int64_t)row * a.kv_heads + hk) * DIM + d0, v);
    } else {
        load8<DT, FAST>(static_cast<const T *>(a.v) + row * a.ldv + (int64_t)hk * DIM + d0, v);
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
    const unsigned queries = a.q ? groups(a.q_heads) : 0, keys = a.k ? groups(a.kv_heads) : 0, all = queries + keys + (a.cache ? keys : 0);
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

// A thread reads eight values of a head of a slot: keys, then values.
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

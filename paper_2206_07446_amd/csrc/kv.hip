// A serving step's plan, and the cache of keys and values held in 4 bits: norms and rotations with the append, and reading back.
#include "nnv_internal.h"
#include "serving.h"
#include "lowbits.h"

namespace nnv {

// ---- the plan of a step -------------------------------------------------------------------------

constexpr int kPlanThreads = 256, kPlanEach = 4, kPlanChunk = kPlanThreads * kPlanEach;

// Exclusive sum over the workgroup's threads; total is everybody's.
__device__ static inline int64_t block_scan(int64_t v, int64_t *scratch, int64_t &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t incl = v;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const int64_t o = __shfl_up(incl, s);
        if (lane >= s) incl += o;
    }
    __syncthreads();                       // the scratch of the scan before has been read
    if (lane == 63) scratch[wave] = incl;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < kPlanThreads / 64; ++i) {
        if (i < wave) before += scratch[i];
        total += scratch[i];
    }
    return before + incl - v;
}

// Every workgroup sums over all requests, 1024 at a time (two prefix sums: rows, then blocks needed), and writes the rows of its
// own range; the requests' own outputs and table entries are written by the workgroup whose turn the chunk is.
// No workgroup waits for another: what one needs of another's table entries it takes from the free list itself.
// Bound by the latency of a chunk's loads and two scans.
__global__ __launch_bounds__(kPlanThreads) void kv_plan(PlanArgs a, int rows_each) {
    __shared__ int64_t scratch[kPlanThreads / 64];
    __shared__ int s_start[kPlanChunk], s_held[kPlanChunk], s_pop[kPlanChunk];     // s_pop: place in the pops, -1 of a request not admitted
    const int t = threadIdx.x, block = 1 << a.block_log;
    const int64_t capacity = (int64_t)a.width << a.block_log;
    const int count = max(0, min(*a.free_count, a.blocks));
    const int64_t r0 = (int64_t)blockIdx.x * rows_each, r1 = min((int64_t)a.rows, r0 + rows_each);
    int64_t rows_before = 0, need_before = 0, taken = 0;
    auto free_block = [&](int64_t place) { return a.free_blocks[count - 1 - place]; };
    for (int c0 = 0, chunk = 0; c0 < a.requests; c0 += kPlanChunk, ++chunk) {
        int held[kPlanEach], fresh[kPlanEach];
        int64_t sum = 0;
#pragma unroll
        for (int j = 0; j < kPlanEach; ++j) {
            const int i = c0 + t * kPlanEach + j;
            held[j] = i < a.requests ? a.held[i] : 0;
            fresh[j] = i < a.requests ? a.fresh[i] : 0;
            sum += max(fresh[j], 0);
        }
        int64_t chunk_rows, chunk_need;
        int64_t start[kPlanEach], need[kPlanEach];
        int64_t at = rows_before + block_scan(sum, scratch, chunk_rows);
        int64_t wanted = 0;
        bool fits[kPlanEach];
#pragma unroll
        for (int j = 0; j < kPlanEach; ++j) {
            const int64_t all = (int64_t)held[j] + fresh[j];
            start[j] = at;
            at += max(fresh[j], 0);
            fits[j] = held[j] >= 0 && fresh[j] >= 0 && all <= capacity && at <= a.rows;
            need[j] = fits[j] ? ((all + block - 1) >> a.block_log) - (((int64_t)held[j] + block - 1) >> a.block_log) : 0;
            wanted += need[j];
        }
        int64_t pop = need_before + block_scan(wanted, scratch, chunk_need);
        const bool mine = chunk % gridDim.x == blockIdx.x;
#pragma unroll
        for (int j = 0; j < kPlanEach; ++j) {
            const int i = c0 + t * kPlanEach + j;
            const bool granted = fits[j] && (need[j] == 0 || pop + need[j] <= count);
            if (granted && need[j]) taken = pop + need[j];
            s_start[t * kPlanEach + j] = (int)min(start[j], (int64_t)a.rows);
            s_held[t * kPlanEach + j] = held[j];
            s_pop[t * kPlanEach + j] = granted ? (int)pop : -1;
            if (mine && i < a.requests) {
                a.starts[i] = (int)min(start[j], (int64_t)a.rows);
                a.lengths[i] = granted ? held[j] + fresh[j] : (int)max((int64_t)0, min((int64_t)held[j], capacity));
                if (granted) {
                    int32_t *entry = a.table + (int64_t)i * a.width + (((int64_t)held[j] + block - 1) >> a.block_log);
                    for (int64_t b = 0; b < need[j]; ++b) entry[b] = free_block(pop + b);
                }
            }
            pop += need[j];
        }
        __syncthreads();
        const int64_t lo = max(r0, rows_before), hi = min(r1, rows_before + chunk_rows);
        const int last = min(kPlanChunk, a.requests - c0) - 1;
        for (int64_t r = lo + t; r < hi; r += kPlanThreads) {
            int i = 0;                     // the last request that starts at r or before
            for (int step = kPlanChunk / 2; step; step /= 2)
                if (i + step <= last && s_start[i + step] <= r) i += step;
            const int first = s_pop[i];
            int32_t position = -1;
            int64_t slot = -1;
            if (first >= 0) {
                position = s_held[i] + (int)(r - s_start[i]);
                const int b = position >> a.block_log, old = (s_held[i] + block - 1) >> a.block_log;
                const int id = b < old ? a.table[(int64_t)(c0 + i) * a.width + b] : free_block(first + b - old);
                if (id >= 0 && id < a.blocks) slot = ((int64_t)id << a.block_log) + (position & (block - 1));
            }
            a.positions[r] = position;
            a.slots[r] = slot;
        }
        rows_before += chunk_rows;
        need_before += chunk_need;
        __syncthreads();
    }
    for (int64_t r = max(r0, rows_before) + t; r < r1; r += kPlanThreads) {
        a.positions[r] = -1;
        a.slots[r] = -1;
    }
    if (blockIdx.x) return;
    // the pops end where the last admitted request's do
#pragma unroll
    for (int s = 1; s < 64; s *= 2) taken = max(taken, __shfl_xor(taken, s));
    if ((t & 63) == 0) scratch[t >> 6] = taken;
    __syncthreads();
    if (t) return;
    for (int i = 1; i < kPlanThreads / 64; ++i) taken = max(taken, scratch[i]);
    *a.left = (int)(count - taken);
    a.starts[a.requests] = (int)min(rows_before, (int64_t)a.rows);
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

// A thread takes eight values of a head of a row, queries first, then keys, then values; heads [first, first + heads) of them.
// Bound by the traffic of the rows.
template <int DT, int DIM, bool FAST>
__global__ __launch_bounds__(256) void qk_norm_rope(RopeArgs a, int first, int heads) {
    typedef typename Elem<DT>::type T;
    constexpr int kLanes = DIM / 8;
    const int64_t unit = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kLanes;
    const int64_t row = unit / heads;
    if (row >= a.rows) return;
    const int h = first + (int)(unit % heads), d0 = (threadIdx.x % kLanes) * 8;
    const int position = a.positions[row];
    const bool there = position >= 0 && (a.rotary == 0 || position < a.max_position);
    const float *angles = a.rope + (int64_t)position * a.rotary;
    if (h < a.q_heads) {
        float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (there) norm_rope8<float, DT, DIM, FAST>(static_cast<const T *>(a.q) + row * a.ldq + (int64_t)h * DIM, d0, a.q_weight, angles, a, v);
        store8<DT>(static_cast<T *>(a.q_out) + (row * a.q_heads + h) * DIM + d0, v);
        return;
    }
    const bool key = h < a.q_heads + a.kv_heads;
    const int hk = key ? h - a.q_heads : h - a.q_heads - a.kv_heads;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (there && key) {
        double x[8];
        norm_rope8<double, DT, DIM, FAST>(static_cast<const T *>(a.k) + row * a.ldk + (int64_t)hk * DIM, d0, a.k_weight, angles, a, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = float_odd(x[i]);
    } else if (there) {
        load8<DT, FAST>(static_cast<const T *>(a.v) + row * a.ldv + (int64_t)hk * DIM + d0, v);
    }
    if (key && a.k_out) store8<DT>(static_cast<T *>(a.k_out) + (row * a.kv_heads + hk) * DIM + d0, v);
    if (!a.cache || !there) return;
    const int64_t slot = a.slots[row];
    if (slot < 0 || slot >= a.total_slots) return;
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
    const int first = a.q ? 0 : a.q_heads, heads = (a.q ? a.q_heads : 0) + (a.k ? (a.cache ? 2 : 1) * a.kv_heads : 0);
    const int64_t threads = (int64_t)a.rows * heads * (DIM / 8);
    const bool turns = a.rotary % (a.interleaved ? 8 : 16) == 0;
    const bool fast = turns && (!a.q || a.ldq % 8 == 0) && (!a.k || (a.ldk % 8 == 0 && a.ldv % 8 == 0));
    const unsigned grid = (unsigned)((threads + 255) / 256);
    if (fast) qk_norm_rope<DT, DIM, true><<<grid, 256, 0, st>>>(a, first, heads);
    else qk_norm_rope<DT, DIM, false><<<grid, 256, 0, st>>>(a, first, heads);
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

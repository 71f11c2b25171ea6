// The step between two blocks of a language model: the block's output, behind its own norm, its gate and a factor, onto the residual
// stream, and the next block's norm of that sum, in one pass.
//
// r = x + scale * gate * (y / sqrt(mean(y^2) + eps) * post),  h = r / sqrt(mean(r^2) + eps) * pre
//
// A row stays in the registers of the threads that read it, so that each input is read once and each output written once: bound by that traffic, and for a
// few rows by the chain of loads, two sums over the row and the stores.  8191 rows of 5120 (float32 stream, gates, both norms, 503 MB): 99 us, 5.1 TB/s, the rate of a
// copy; 64 rows of 4096: 4.5 us, of which a launch that does nothing takes 3.5 to 4.
#include <type_traits>
#include "nnv_internal.h"
#include "serving.h"
#include "lowbits.h"

namespace nnv {

// Values of a row that a thread holds: CHUNKS times eight.  VEC: neighbours in one load, where rows and strides are multiples of eight; otherwise
// values that lie `threads` apart, so that the lanes of a wavefront still read neighbours.
template <bool VEC, int CHUNKS> struct RowPlaces {
    int n, threads, at;
    __device__ int first(int c) const { return (c * threads + at) * 8; }
    __device__ int one(int c, int i) const { return (c * 8 + i) * threads + at; }
    template <typename T> __device__ void load(const T *p, float (&v)[CHUNKS][8]) const {
        typedef T T8 __attribute__((ext_vector_type(8)));
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            if constexpr (VEC) {
                T8 x = {};
                if (first(c) < n) x = *reinterpret_cast<const T8 *>(p + first(c));
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = (float)x[i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = one(c, i) < n ? (float)p[one(c, i)] : 0.f;
            }
        }
    }
    template <typename T> __device__ void store(T *p, const float (&v)[CHUNKS][8]) const {
        typedef T T8 __attribute__((ext_vector_type(8)));
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            if constexpr (VEC) {
                T8 x;
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = (T)v[c][i];
                if (first(c) < n) *reinterpret_cast<T8 *>(p + first(c)) = x;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (one(c, i) < n) p[one(c, i)] = (T)v[c][i];
            }
        }
    }
};

// Sum over a wavefront, the same in all lanes, in an order that depends on nothing.
__device__ static inline float wave_sum(float v) {
    auto moved = [&](auto step) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(step)::value, 0xf, 0xf, false)); };
    v += moved(std::integral_constant<int, 0xb1>{});      // lanes xor 1
    v += moved(std::integral_constant<int, 0x4e>{});      // xor 2
    v += moved(std::integral_constant<int, 0x141>{});     // mirrored halves of a row
    v += moved(std::integral_constant<int, 0x140>{});     // mirrored row
    const int bits = __builtin_bit_cast(int, v);
    auto row = [&](int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(bits, lane)); };
    return (row(0) + row(16)) + (row(32) + row(48));
}
__device__ static inline double wave_sum(double v) {
#pragma unroll
    for (int s = 1; s < 64; s *= 2) v += __shfl_xor(v, s);
    return v;
}

// Over the threads of a row: a wavefront, or the workgroup.  (Two scratches by turns, so that one barrier a sum is enough.)
template <typename F> __device__ static inline F row_sum(F v, bool alone, F *scratch) {
    v = wave_sum(v);
    if (alone) return v;
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    if ((threadIdx.x & 63) == 0) scratch[wave] = v;
    __syncthreads();
    F sum = scratch[0];
    for (int i = 1; i < waves; ++i) sum += scratch[i];
    return sum;
}

// 1 / sqrt(mean(v^2) + eps).  Squares that leave float32's range, on either side, are added up again in float64; a row of zeros without eps stays one.  Of a row below
// 2^-128 or so the reciprocal is no float32: it is the product of `factor` and a power of two that moves no bit of v, 1 where the squares are in range.
struct Inverse { float twos, factor; };
template <int CHUNKS> __device__ static inline Inverse inverse_rms(const float (&v)[CHUNKS][8], int n, float eps, bool alone, float *scratch, double *scratch_wide) {
    float sum = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(v[c][i], v[c][i], sum);
    sum = row_sum(sum, alone, scratch);
    if (sum > 0x1p-80f && sum < INFINITY) return {1.f, 1.f / sqrtf(sum / (float)n + eps)};
    double wide = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) wide += (double)v[c][i] * (double)v[c][i];
    wide = row_sum(wide, alone, scratch_wide) / n + (double)eps;
    if (wide == 0) return {1.f, 0.f};
    const double inverse = 1.0 / sqrt(wide);                 // (twos: not 1 only where what they take off or add lies beyond the range of a result)
    const float twos = inverse > 0x1p100 ? 0x1p64f : inverse < 0x1p-100 ? 0x1p-64f : 1.f;
    return {twos, (float)(inverse / (double)twos)};
}

template <int XT, int YT, bool VEC, int CHUNKS>
__global__ __launch_bounds__(1024) void residual_norm(ResidualArgs a) {
    typedef typename Elem<XT>::type X;
    typedef typename Elem<YT>::type Y;
    __shared__ float scratch[2][16];
    __shared__ double scratch_wide[2][16];
    const bool alone = a.threads == 64;                   // a wavefront to a row
    const int64_t row = alone ? (int64_t)blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6) : blockIdx.x;
    if (row >= a.m) return;
    const RowPlaces<VEC, CHUNKS> at{a.n, a.threads, alone ? (int)(threadIdx.x & 63) : (int)threadIdx.x};
    float r[CHUNKS][8], y[CHUNKS][8], w[CHUNKS][8];
    at.load(static_cast<const X *>(a.x) + row * a.ldx, r);
    if (a.y) {
        at.load(static_cast<const Y *>(a.y) + row * a.ldy, y);
        const int64_t which = !a.gate ? 0 : a.index ? a.index[row] : a.gates == 1 ? 0 : row;
        const bool adds = !a.gate || (which >= 0 && which < a.gates);
        if (a.gate) at.load(static_cast<const Y *>(a.gate) + (adds ? which : 0) * a.ldg, w);
        if (a.post) {
            float weight[CHUNKS][8];
            at.load(a.post, weight);
            const Inverse inverse = inverse_rms(y, a.n, a.eps, alone, scratch[0], scratch_wide[0]);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) y[c][i] = y[c][i] * inverse.twos * inverse.factor * weight[c][i];
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float part = a.gate ? y[c][i] * w[c][i] : y[c][i];
                r[c][i] = adds ? fmaf(part, a.scale, r[c][i]) : r[c][i];
            }
        at.store(static_cast<X *>(a.x_out) + row * a.ldo, r);
    }
    if (!a.pre) return;
    at.load(a.pre, w);
    const Inverse inverse = inverse_rms(r, a.n, a.eps, alone, scratch[1], scratch_wide[1]);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) r[c][i] = r[c][i] * inverse.twos * inverse.factor * w[c][i];
    const int64_t h = row * a.ldh;
    if (a.h_dtype == NNV_F32) at.store(static_cast<float *>(a.h) + h, r);
    else if (a.h_dtype == NNV_F16) at.store(static_cast<_Float16 *>(a.h) + h, r);
    else at.store(static_cast<__bf16 *>(a.h) + h, r);
}

template <int XT, int YT, bool VEC> static hipError_t launch_residual_types(const ResidualArgs &args, hipStream_t st) {
    ResidualArgs a = args;
    const int eights = (a.n + 7) / 8;
    // (two loads of eight a thread where there are many rows: 8191 rows of 5120 99 us, with one 103, with four 151, spilt; 1024 threads for the 640 that have work 107)
    const int wanted = eights > 64 && a.m >= 512 ? 2 : 1;
    const int each = (eights + wanted - 1) / wanted, threads = each > 1024 ? 1024 : (each + 63) / 64 * 64, chunks = (eights + threads - 1) / threads;
    a.threads = threads;
    const unsigned group = threads == 64 ? 256u : (unsigned)threads, rows = threads == 64 ? 4u : 1u, groups = (unsigned)((a.m + (int64_t)rows - 1) / rows);
    if (chunks == 1) residual_norm<XT, YT, VEC, 1><<<groups, group, 0, st>>>(a);
    else if (chunks == 2) residual_norm<XT, YT, VEC, 2><<<groups, group, 0, st>>>(a);
    else residual_norm<XT, YT, VEC, 4><<<groups, group, 0, st>>>(a);
    return hipGetLastError();
}
template <int XT> static hipError_t launch_residual_x(const ResidualArgs &a, int y_dtype, bool vec, hipStream_t st) {
#define NNV_RESIDUAL(YT) (vec ? launch_residual_types<XT, YT, true>(a, st) : launch_residual_types<XT, YT, false>(a, st))
    return y_dtype == NNV_F32 ? NNV_RESIDUAL(NNV_F32) : y_dtype == NNV_F16 ? NNV_RESIDUAL(NNV_F16) : NNV_RESIDUAL(NNV_BF16);
#undef NNV_RESIDUAL
}

hipError_t launch_residual_norm(const nnv_residual_desc &d, const ResidualArgs &a, hipStream_t st) {
    const bool one = a.m == 1;                            // (its strides are not looked at)
    auto eights = [&](int64_t stride, bool used) { return !used || one || stride % 8 == 0; };
    const bool vec = a.n % 8 == 0 && eights(a.ldx, true) && eights(a.ldy, a.y) && eights(a.ldo, a.y) && (!a.y || !a.gate || a.gates == 1 || a.ldg % 8 == 0) &&
                     eights(a.ldh, a.pre);
    return d.x_dtype == NNV_F32 ? launch_residual_x<NNV_F32>(a, d.y_dtype, vec, st)
         : d.x_dtype == NNV_F16 ? launch_residual_x<NNV_F16>(a, d.y_dtype, vec, st) : launch_residual_x<NNV_BF16>(a, d.y_dtype, vec, st);
}

}  // namespace nnv

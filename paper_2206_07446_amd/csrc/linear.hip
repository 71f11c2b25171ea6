// Products with weights held in 8 bits: y = x W^T + bias, e4m3 codes with a power-of-two scale for 128 inputs of
// a row of x and for each 128 x 128 block of W.
//
// Both operands lie in memory as the matrix instructions read them.  A piece is 16 rows x 128 inputs, 2 KB: lane l of a wavefront
// holds row l % 16, inputs 32 (l / 16) .. + 31 of the block, as two halves of 16 bytes each at [half][l].  One piece is an operand of a
// 16x16x128 instruction, two pieces (32 rows) are those of two 32x32x64 instructions; a copy of consecutive bytes
// to the LDS and reads of 16 bytes a lane from there meet no bank twice.
// The scales go into the instructions as the bytes that they are kept as; sums stay in the instructions' float32 accumulators over
// the whole reduction.
#include "nnv_internal.h"
#include "serving.h"
#include "lowbits.h"

namespace nnv {

constexpr int kPieceBytes = 2048;

static inline int blocks128(int v) { return (v + 127) / 128; }
static inline int scale_words(int k) { return (blocks128(k) + 3) / 4; }      // 32-bit words of scale bytes of a row of blocks

size_t linear_codes_bytes(int rows, int k) { return (size_t)((rows + 15) / 16) * blocks128(k) * kPieceBytes; }

size_t linear_transformed_bytes(const nnv_linear_desc &d) {
    return linear_codes_bytes(blocks128(d.n) * 128, d.k) + align_up((size_t)blocks128(d.n) * scale_words(d.k) * 4, 256);
}

// Workspace: codes of x, then its scales: [16 rows][word][row of the 16], a byte per block.
size_t linear_workspace_bytes(const nnv_linear_desc &d, int m) {
    return linear_codes_bytes(m, d.k) + align_up((size_t)((m + 15) / 16) * scale_words(d.k) * 64, 256);
}

template <int DT> __device__ static inline float load_as_float(const void *p, int64_t i) {
    return (float)static_cast<const typename Elem<DT>::type *>(p)[i];
}

// 16 consecutive inputs of a row from `at`, `left` of which are there.
template <int DT, bool VEC> __device__ static inline void load16(const void *p, int64_t at, int left, float (&v)[16]) {
    if (VEC && left >= 16) {
        const auto *q = reinterpret_cast<const ElemVec<DT, 8> *>(static_cast<const typename Elem<DT>::type *>(p) + at);
        const ElemVec<DT, 8> a = q[0], b = q[1];
#pragma unroll
        for (int i = 0; i < 8; ++i) { v[i] = (float)a[i]; v[8 + i] = (float)b[i]; }
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = i < left ? load_as_float<DT>(p, at + i) : 0.f;
}

__device__ static inline uint32_t amax_bits16(const float (&v)[16]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu);
    return m;
}

__device__ static inline i32x4_t codes16(const float (&v)[16], uint32_t byte, uint32_t amax) {
    const float inv = inverse_of_byte(byte);
    i32x4_t c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t w = e4m3_code4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3], inv);
        if (amax >= kInfBits) w = e4m3_nan_where(w, v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        c[i] = (int)w;
    }
    return c;
}

// x -> codes and scales.  A workgroup takes 16 rows x 2 blocks, 8 threads a row's block: a wavefront reads 256-byte runs of 8
// rows and writes 128-byte runs of a piece.  Bound by the traffic of x.
template <int DT, bool VEC>
__global__ __launch_bounds__(256) void linear_quantise(const void *__restrict__ x, int64_t ldx, int m, int k, char *__restrict__ codes,
                                                       char *__restrict__ scales) {
    const int t = threadIdx.x, part = t & 7, r = (t >> 3) & 15, kblocks = (k + 127) / 128;
    const int kb = blockIdx.x * 2 + (t >> 7), tile = blockIdx.y;
    const int64_t row = (int64_t)tile * 16 + r;
    if (kb >= kblocks || row >= m) return;                 // the 8 threads of a row's block leave together
    float v[16];
    const int at = kb * 128 + part * 16;
    load16<DT, VEC>(x, row * ldx + at, k - at, v);
    uint32_t amax = amax_bits16(v);
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 4));
    const uint32_t byte = e4m3_scale_byte(amax);
    char *piece = codes + ((int64_t)tile * kblocks + kb) * kPieceBytes;
    *reinterpret_cast<i32x4_t *>(piece + (part & 1) * 1024 + (r + 16 * (part >> 1)) * 16) = codes16(v, byte, amax);
    if (part == 0) scales[(((int64_t)tile * ((kblocks + 3) / 4) + kb / 4) * 16 + r) * 4 + kb % 4] = (char)byte;
}

// Raw weights -> codes and scales, a block of 128 x 128 a workgroup.  Bound by the traffic of the raw weights.
template <int DT, bool VEC>
__global__ __launch_bounds__(256) void linear_pack(const void *__restrict__ w, int n, int k, char *__restrict__ codes, char *__restrict__ scales) {
    const int t = threadIdx.x, part = t & 7, r = t >> 3, kblocks = (k + 127) / 128;
    const int kb = blockIdx.x, nb = blockIdx.y, at = kb * 128 + part * 16;
    float v[4][16];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = nb * 128 + i * 32 + r;
        load16<DT, VEC>(w, (int64_t)row * k + at, row < n ? k - at : 0, v[i]);
        amax = max(amax, amax_bits16(v[i]));
    }
    for (int s = 1; s < 64; s *= 2) amax = max(amax, (uint32_t)__shfl_xor((int)amax, s));
    __shared__ uint32_t most[4];
    if ((t & 63) == 0) most[t >> 6] = amax;
    __syncthreads();
    amax = max(max(most[0], most[1]), max(most[2], most[3]));
    const uint32_t byte = e4m3_scale_byte(amax);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 32 + r;
        char *piece = codes + ((int64_t)(nb * 8 + row / 16) * kblocks + kb) * kPieceBytes;
        *reinterpret_cast<i32x4_t *>(piece + (part & 1) * 1024 + (row % 16 + 16 * (part >> 1)) * 16) = codes16(v[i], byte, amax);
    }
    // the last block writes the bytes of its word that stand for no block
    const int words = (kblocks + 3) / 4;
    if (t == 0) scales[((int64_t)nb * words + kb / 4) * 4 + kb % 4] = (char)byte;
    if (kb == kblocks - 1 && t > 0 && t < 4 && kb % 4 + t < 4) scales[((int64_t)nb * words + kb / 4) * 4 + kb % 4 + t] = 0;
}

struct LinearArgs {
    const char *w, *w_scales, *x, *x_scales;
    const float *bias;
    void *y;
    int64_t ldy;
    int m, n, kblocks;
};

template <int DT> __device__ static inline void store4(const LinearArgs &a, int64_t row, int col, f32x4_t v) {
    if (row >= a.m) return;
    typename Elem<DT>::type *y = static_cast<typename Elem<DT>::type *>(a.y) + row * a.ldy + col;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (col + i < a.n) y[i] = (typename Elem<DT>::type)(v[i] + (a.bias ? a.bias[col + i] : 0.f));
}

__device__ static inline i32x8_t load_piece(const char *p, int lane) {
    const i32x4_t lo = *reinterpret_cast<const i32x4_t *>(p + lane * 16), hi = *reinterpret_cast<const i32x4_t *>(p + 1024 + lane * 16);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// Eight codes (two words) as bfloat16 values, the scale in: exact, an e4m3 code has four significant bits.
__device__ static inline bf16x8_t bf16_of_codes(int w0, int w1, float scale) {
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true);
    return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ static inline float scale_at(uint32_t word, int kb) { return scale_of_byte((word >> (8 * (kb % 4))) & 255); }

// Few rows: a workgroup holds 16 outputs x 16 MT rows and splits the reduction over its wavefronts, which read weights straight
// from memory into registers and add their sums in the LDS in a fixed order.  The codes go to the matrix cores as
// bfloat16: their 8-bit instructions line the products of a few inputs up to the largest and cut off what is 2^17 below it
// (sums 1.3e-5 off in the 2-norm on normal inputs, 2^-16 of the sum of magnitudes at most), those of bfloat16 add in float32.
// The conversions cost nothing here, where the weights' traffic is what bounds.
template <int DT, int MT>
__global__ __launch_bounds__(256) void linear_rows(LinearArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, words = (a.kblocks + 3) / 4;
    const int tile = blockIdx.x, first = blockIdx.y * MT, tiles = (a.m + 15) / 16;
    f32x4_t acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = f32x4_t{0, 0, 0, 0};
    const char *w = a.w + (int64_t)tile * a.kblocks * kPieceBytes;
    const uint32_t *ws = reinterpret_cast<const uint32_t *>(a.w_scales) + (int64_t)(tile / 8) * words;
    for (int kb = wave; kb < a.kblocks; kb += 4) {
        const i32x8_t wp = load_piece(w + (int64_t)kb * kPieceBytes, lane);
        const float sw = scale_at(ws[kb / 4], kb);
        bf16x8_t wv[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) wv[s] = bf16_of_codes(wp[2 * s], wp[2 * s + 1], sw);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int64_t mt = min(first + i, tiles - 1);
            const i32x8_t xp = load_piece(a.x + (mt * a.kblocks + kb) * kPieceBytes, lane);
            const float sx = scale_at(reinterpret_cast<const uint32_t *>(a.x_scales)[(mt * words + kb / 4) * 16 + lane % 16], kb);
#pragma unroll
            for (int s = 0; s < 4; ++s)
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[s], bf16_of_codes(xp[2 * s], xp[2 * s + 1], sx), acc[i], 0, 0, 0);
        }
    }
    __shared__ f32x4_t part[3][MT][64];
    if (wave)
#pragma unroll
        for (int i = 0; i < MT; ++i) part[wave - 1][i][lane] = acc[i];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const f32x4_t s = (acc[i] + part[0][i][lane]) + (part[1][i][lane] + part[2][i][lane]);
        store4<DT>(a, (int64_t)(first + i) * 16 + lane % 16, tile * 16 + 4 * (lane / 16), s);
    }
}

template <int DT> static hipError_t launch_rows(const LinearArgs &a, hipStream_t st) {
    const int tiles = (a.m + 15) / 16, ntiles = (a.n + 15) / 16;
    if (tiles == 1) linear_rows<DT, 1><<<dim3(ntiles, 1), 256, 0, st>>>(a);
    else linear_rows<DT, 4><<<dim3(ntiles, (tiles + 3) / 4), 256, 0, st>>>(a);
    return hipGetLastError();
}

template <int DT> static hipError_t launch_quantise(const void *x, int64_t ldx, int m, int k, char *codes, char *scales, hipStream_t st) {
    const dim3 grid((blocks128(k) + 1) / 2, (m + 15) / 16);
    if (ldx * (int64_t)sizeof(typename Elem<DT>::type) % 16 == 0) linear_quantise<DT, true><<<grid, 256, 0, st>>>(x, ldx, m, k, codes, scales);
    else linear_quantise<DT, false><<<grid, 256, 0, st>>>(x, ldx, m, k, codes, scales);
    return hipGetLastError();
}

template <int DT> static hipError_t launch_pack(const void *w, int n, int k, char *codes, char *scales, hipStream_t st) {
    const dim3 grid(blocks128(k), blocks128(n));
    if (k * sizeof(typename Elem<DT>::type) % 16 == 0) linear_pack<DT, true><<<grid, 256, 0, st>>>(w, n, k, codes, scales);
    else linear_pack<DT, false><<<grid, 256, 0, st>>>(w, n, k, codes, scales);
    return hipGetLastError();
}

hipError_t launch_linear_pack(const nnv_linear_desc &d, const void *raw, void *tx, hipStream_t st) {
    char *codes = static_cast<char *>(tx), *scales = codes + linear_codes_bytes(blocks128(d.n) * 128, d.k);
    if (d.raw_dtype == NNV_F32) return launch_pack<NNV_F32>(raw, d.n, d.k, codes, scales, st);
    if (d.raw_dtype == NNV_F16) return launch_pack<NNV_F16>(raw, d.n, d.k, codes, scales, st);
    return launch_pack<NNV_BF16>(raw, d.n, d.k, codes, scales, st);
}

hipError_t launch_linear(const nnv_linear_desc &d, int m, const void *x, int64_t ldx, const void *tx, const float *bias, void *y, int64_t ldy, void *ws,
                         hipStream_t st) {
    LinearArgs a;
    a.w = static_cast<const char *>(tx);
    a.w_scales = a.w + linear_codes_bytes(blocks128(d.n) * 128, d.k);
    char *codes = static_cast<char *>(ws), *scales = codes + linear_codes_bytes(m, d.k);
    a.x = codes; a.x_scales = scales;
    a.bias = bias; a.y = y; a.ldy = ldy; a.m = m; a.n = d.n; a.kblocks = blocks128(d.k);
    hipError_t e = d.x_dtype == NNV_F32 ? launch_quantise<NNV_F32>(x, ldx, m, d.k, codes, scales, st)
                 : d.x_dtype == NNV_F16 ? launch_quantise<NNV_F16>(x, ldx, m, d.k, codes, scales, st)
                                        : launch_quantise<NNV_BF16>(x, ldx, m, d.k, codes, scales, st);
    if (e != hipSuccess) return e;
    return d.y_dtype == NNV_F32 ? launch_rows<NNV_F32>(a, st) : d.y_dtype == NNV_F16 ? launch_rows<NNV_F16>(a, st) : launch_rows<NNV_BF16>(a, st);
}

}  // namespace nnv

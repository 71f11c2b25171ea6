// Products with weights held in 8 bits: y = x W^T + bias, e4m3 codes with a power-of-two scale for 128 inputs of
// a row of x and for each 128 x 128 block of W.
//
// Both operands lie in memory as the matrix instructions read them.  A piece is 16 rows x 64 inputs (a step), 1 KB: lane l of half a
// wavefront has row l % 16, inputs 32 (l / 16) .. + 31 of the step, as two halves of 16 bytes at [half][l].  Two pieces are an operand of
// 32 rows of a 32x32x64 instruction, or two steps of 16 rows for 16x16x32 ones; a copy of consecutive bytes to the LDS and reads of 16
// bytes a lane from there meet no bank twice.  Pieces lie by rows of 16 and then by steps; those of the weights by 128 rows, steps, and the
// eight pieces of a step, so that what a tile reads of a step is 8 KB in one place.
// The scales go into the instructions as the bytes that they are kept as; sums stay in the instructions' float32 accumulators over
// the whole reduction.
#include "nnv_internal.h"
#include "serving.h"
#include "lowbits.h"
#include "buf.h"

namespace nnv {

constexpr int kPieceBytes = 1024;

static inline int blocks128(int v) { return (v + 127) / 128; }
// Blocks of the reduction as they are held: an even number of them, the last one zeros where it has to be.
static inline int held_blocks(int k) { return (blocks128(k) + 1) / 2 * 2; }
static inline int scale_words(int k) { return (blocks128(k) + 3) / 4; }      // 32-bit words of scale bytes of a row of blocks

size_t linear_codes_bytes(int rows, int k) { return (size_t)((rows + 15) / 16) * held_blocks(k) * 2 * kPieceBytes; }

size_t linear_transformed_bytes(const nnv_linear_desc &d) {
    return linear_codes_bytes(blocks128(d.n) * 128, d.k) + align_up((size_t)blocks128(d.n) * scale_words(d.k) * 4, 256);
}

// Workspace: codes of x, then its scales: [16 rows][word][row of the 16], a byte per block; then parts of sums.
static size_t linear_x_bytes(int m, int k) { return linear_codes_bytes(m, k) + align_up((size_t)((m + 15) / 16) * scale_words(k) * 64, 256); }
template <int DT> __device__ static inline float load_as_float(const void *p, int64_t i) {
    return (float)static_cast<const typename Elem<DT>::type *>(p)[i];
}

// 16 consecutive inputs of a row from `at`, `left` of which are there.  Rows may begin anywhere: loads and stores of 16 bytes need no alignment (6 rows
// of 842 by 5376: 14.4 us with a load for each input, 8.4 so).
template <int DT> __device__ static inline void load16(const void *p, int64_t at, int left, float (&v)[16]) {
    if (left >= 16) {
        const auto *q = static_cast<const typename Elem<DT>::type *>(p) + at;
        ElemVec<DT, 8> a, b;
        __builtin_memcpy(&a, q, sizeof(a));
        __builtin_memcpy(&b, q + 8, sizeof(b));
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

// Where inputs 16 part .. + 15 of a row's block lie in their piece.
__device__ static inline int code_at(int row, int part) { return (part & 1) * 512 + (row + 16 * (part / 2 % 2)) * 16; }

// x -> codes and scales.  A workgroup takes 16 rows x 2 blocks, 8 threads a row's block: a wavefront reads 256-byte runs of 8
// rows and writes 128-byte runs of two pieces.  Bound by the traffic of x (4096 x 4096 bfloat16, 51 MB: 11 us).
template <int DT>
__global__ __launch_bounds__(256) void linear_quantise(const void *__restrict__ x, int64_t ldx, int m, int k, char *__restrict__ codes,
                                                       char *__restrict__ scales) {
    const int t = threadIdx.x, part = t & 7, r = (t >> 3) & 15, kblocks = (k + 127) / 128, held = (kblocks + 1) / 2 * 2;
    const int kb = blockIdx.x * 2 + (t >> 7), tile = blockIdx.y;
    const int64_t row = (int64_t)tile * 16 + r;
    if (row >= m) return;                                  // the 8 threads of a row's block leave together
    float v[16];
    const int at = kb * 128 + part * 16;
    load16<DT>(x, row * ldx + at, k - at, v);
    uint32_t amax = amax_bits16(v);
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 4));
    const uint32_t byte = e4m3_scale_byte(amax);
    char *piece = codes + (((int64_t)tile * held + kb) * 2 + part / 4) * kPieceBytes;
    *reinterpret_cast<i32x4_t *>(piece + code_at(r, part)) = codes16(v, byte, amax);
    if (part == 0) scales[(((int64_t)tile * ((kblocks + 3) / 4) + kb / 4) * 16 + r) * 4 + kb % 4] = (char)byte;
}

// Raw weights -> codes and scales, a block of 128 x 128 a workgroup.  Bound by the traffic of the raw weights (4096 x 8192 float32, 168 MB: 26 us,
// the last-level cache serving some of it).
template <int DT>
__global__ __launch_bounds__(256) void linear_pack(const void *__restrict__ w, int n, int k, char *__restrict__ codes, char *__restrict__ scales) {
    const int t = threadIdx.x, part = t & 7, r = t >> 3, kblocks = (k + 127) / 128, held = (kblocks + 1) / 2 * 2;
    const int kb = blockIdx.x, nb = blockIdx.y, at = kb * 128 + part * 16;
    float v[4][16];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = nb * 128 + i * 32 + r;
        load16<DT>(w, (int64_t)row * k + at, row < n ? k - at : 0, v[i]);
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
        char *piece = codes + ((((int64_t)nb * held + kb) * 2 + part / 4) * 8 + row / 16) * kPieceBytes;
        *reinterpret_cast<i32x4_t *>(piece + code_at(row % 16, part)) = codes16(v[i], byte, amax);
    }
    // the last block writes the bytes of its word that stand for no block
    const int words = (kblocks + 3) / 4;
    if (t == 0) scales[((int64_t)nb * words + kb / 4) * 4 + kb % 4] = (char)byte;
    if (kb == held - 1 && t > 0 && t < 4 && kb % 4 + t < 4) scales[((int64_t)nb * words + kb / 4) * 4 + kb % 4 + t] = 0;
}

struct LinearArgs {
    const char *w, *w_scales, *x, *x_scales;
    const float *bias;
    void *y;
    int64_t ldy;
    int m, n, kblocks, held;      // blocks of the reduction, and as they are held
    float *parts;           // [splits][m][n rounded up to 4]: sums of the reduction's parts, where it is split
    int splits;
};

template <int DT> __device__ static inline void store4(const LinearArgs &a, int64_t row, int col, f32x4_t v) {
    if (row >= a.m || col >= a.n) return;
    typename Elem<DT>::type *y = static_cast<typename Elem<DT>::type *>(a.y) + row * a.ldy + col;
    if (col + 4 <= a.n) {
        ElemVec<DT, 4> out;
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = (typename Elem<DT>::type)(v[i] + (a.bias ? a.bias[col + i] : 0.f));
        __builtin_memcpy(y, &out, sizeof(out));
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (col + i < a.n) y[i] = (typename Elem<DT>::type)(v[i] + (a.bias ? a.bias[col + i] : 0.f));
}

template <int DT> __device__ static inline void store8(const LinearArgs &a, int64_t row, int col, f32x4_t lo, f32x4_t hi) {
    if (DT != NNV_F32 && col + 8 <= a.n && row < a.m) {
        ElemVec<DT, 8> out;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            out[i] = (typename Elem<DT>::type)(lo[i] + (a.bias ? a.bias[col + i] : 0.f));
            out[4 + i] = (typename Elem<DT>::type)(hi[i] + (a.bias ? a.bias[col + 4 + i] : 0.f));
        }
        __builtin_memcpy(static_cast<typename Elem<DT>::type *>(a.y) + row * a.ldy + col, &out, sizeof(out));
        return;
    }
    store4<DT>(a, row, col, lo);
    store4<DT>(a, row, col + 4, hi);
}

// What a wavefront's lanes have written to the LDS is there for the others of it.
__device__ static inline void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Two pieces, `apart` bytes apart: a block of 16 rows, a row and 32 inputs a lane.
__device__ static inline i32x8_t load_block(const char *p, int apart, int lane) {
    p += lane / 32 * apart + lane % 32 * 16;
    const i32x4_t lo = *reinterpret_cast<const i32x4_t *>(p), hi = *reinterpret_cast<const i32x4_t *>(p + 512);
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

// 32 consecutive inputs of a row as words of their storage type; `left` of them are there.
template <int DX> struct Inputs32 { uint32_t word[DX == NNV_F32 ? 32 : 16]; };
template <int DX> __device__ static inline void load32(const void *p, int64_t at, int left, Inputs32<DX> &v) {
    typedef typename Elem<DX>::type T;
    constexpr int kWords = DX == NNV_F32 ? 32 : 16, kEach = 32 / kWords;
    const T *q = static_cast<const T *>(p) + at;
#pragma unroll
    for (int i = 0; i < kWords; ++i) v.word[i] = 0;
    if (left >= 32) {
        __builtin_memcpy(v.word, q, sizeof(v.word));
    } else if (left > 0) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            if (i >= left) continue;
            if constexpr (kEach == 1) v.word[i] = __builtin_bit_cast(uint32_t, q[i]);
            else v.word[i / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, q[i]) << (16 * (i % 2));
        }
    }
}

// Bits of the largest magnitude, as those of a float32.
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
template <int DX> __device__ static inline uint32_t amax_bits32(const Inputs32<DX> &v) {
    if constexpr (DX == NNV_F32) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) m = max(m, v.word[i] & 0x7fffffffu);
        return m;
    } else {
        u16x2_t m = {0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_t, v.word[i] & 0x7fff7fffu));
        const uint16_t most = m[0] > m[1] ? m[0] : m[1];
        return __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(typename Elem<DX>::type, most));
    }
}

// Their codes, by the instructions that divide by a power of two and round once.
typedef short i16x2_t __attribute__((ext_vector_type(2)));
template <int DX> __device__ static inline i32x8_t codes32(const Inputs32<DX> &v, uint32_t byte, uint32_t amax) {
    const float scale = scale_of_byte(byte);
    i32x8_t codes;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        i16x2_t c = {0, 0};
        if constexpr (DX == NNV_F32) {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, __builtin_bit_cast(float, v.word[4 * i]), __builtin_bit_cast(float, v.word[4 * i + 1]), scale, false);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, __builtin_bit_cast(float, v.word[4 * i + 2]), __builtin_bit_cast(float, v.word[4 * i + 3]), scale, true);
        } else if constexpr (DX == NNV_F16) {
            typedef ElemVec<NNV_F16, 2> H;
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(c, __builtin_bit_cast(H, v.word[2 * i]), scale, false);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(c, __builtin_bit_cast(H, v.word[2 * i + 1]), scale, true);
        } else {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2_t, v.word[2 * i]), scale, false);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2_t, v.word[2 * i + 1]), scale, true);
        }
        codes[i] = __builtin_bit_cast(int, c);
        if (amax >= kInfBits) {
            auto value = [&](int j) {
                if constexpr (DX == NNV_F32) return __builtin_bit_cast(float, v.word[j]);
                else return (float)__builtin_bit_cast(typename Elem<DX>::type, (uint16_t)(v.word[j / 2] >> (16 * (j % 2))));
            };
            codes[i] = (int)e4m3_nan_where((uint32_t)codes[i], value(4 * i), value(4 * i + 1), value(4 * i + 2), value(4 * i + 3));
        }
    }
    return codes;
}

// Up to 16 rows: a workgroup holds 16 NT outputs x all rows and splits the reduction over its wavefronts, which read weights straight
// from memory into registers, blocks ahead, and add their sums in the LDS in a fixed order.  x is rounded here, by every
// workgroup for itself (a launch of its own takes 2.5 us); what a lane reads of x is its part of the operand.  The codes go to the matrix cores as
// bfloat16: their 8-bit instructions line the products of eight neighbouring inputs up to the largest and hold them to 2^-13 of it (sums 1.3e-5 off
// in the 2-norm on normal inputs, 2^-10 of the sum of magnitudes at most), those of bfloat16 add in float32.
// The conversions cost nothing here, where the weights' traffic is what bounds.
constexpr int kRowWaves = 8;
template <int DT, int DX, int NT>
__global__ __launch_bounds__(64 * kRowWaves) void linear_rows(LinearArgs a, const void *__restrict__ x, int64_t ldx, int k) {
    constexpr int kAhead = NT == 1 ? 4 : 2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), words = (a.kblocks + 3) / 4, tile = blockIdx.x * NT;
    const int row = lane % 16, quarter = lane / 16;
    f32x4_t acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4_t{0, 0, 0, 0};
    const char *w = a.w + (int64_t)(tile / 8) * a.held * 16 * kPieceBytes + tile % 8 * kPieceBytes;
    const uint32_t *w_scales = reinterpret_cast<const uint32_t *>(a.w_scales) + (int64_t)(tile / 8) * words;
    i32x8_t ring[kAhead][NT];
    Inputs32<DX> inputs[2];
    auto fetch_weights = [&](int kb, i32x8_t (&v)[NT]) {
#pragma unroll
        for (int t = 0; t < NT; ++t) v[t] = load_block(w + ((int64_t)kb * 16 + t) * kPieceBytes, 8 * kPieceBytes, lane);
    };
    auto fetch_inputs = [&](int kb, Inputs32<DX> &v) {
        const int at = kb * 128 + quarter * 32;
        load32<DX>(x, row * ldx + at, row < a.m ? k - at : 0, v);
    };
    const int last = a.kblocks - 1;                      // behind it, it is loaded again (see linear_waves)
#pragma unroll
    for (int d = 0; d < kAhead; ++d) {
        const int kb = min(wave + kRowWaves * d, last);
        fetch_weights(kb, ring[d]);
        if (d < 2) fetch_inputs(kb, inputs[d]);
    }
    for (int base = wave; base < a.kblocks; base += kRowWaves * kAhead) {
#pragma unroll
        for (int d = 0; d < kAhead; ++d) {
            const int kb = base + kRowWaves * d, later = kb + kRowWaves * kAhead;
            if (kb < a.kblocks) {
                const Inputs32<DX> v = inputs[d % 2];
                fetch_inputs(min(kb + 2 * kRowWaves, last), inputs[d % 2]);
                uint32_t amax = amax_bits32(v);
                amax = max(amax, (uint32_t)__shfl_xor((int)amax, 16));
                amax = max(amax, (uint32_t)__shfl_xor((int)amax, 32));
                const uint32_t byte = e4m3_scale_byte(amax);
                const i32x8_t xp = codes32(v, byte, amax);
                const float sw = scale_at(w_scales[kb / 4], kb), sx = scale_of_byte(byte);
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const bf16x8_t xv = bf16_of_codes(xp[2 * s], xp[2 * s + 1], sx);
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of_codes(ring[d][t][2 * s], ring[d][t][2 * s + 1], sw), xv, acc[t], 0, 0, 0);
                }
            }
            fetch_weights(min(later, last), ring[d]);
        }
    }
    __shared__ f32x4_t part[kRowWaves][NT][64];
#pragma unroll
    for (int t = 0; t < NT; ++t) part[wave][t][lane] = acc[t];
    __syncthreads();
    if (wave >= NT) return;
    f32x4_t sum = part[0][wave][lane];
#pragma unroll
    for (int i = 1; i < kRowWaves; ++i) sum += part[i][wave][lane];
    store4<DT>(a, row, (tile + wave) * 16 + 4 * quarter, sum);
}

// Many rows: a workgroup of WN x WM wavefronts holds 32 FN WN outputs x 32 FM WM rows, a wavefront 32 FN x 32 FM of them in registers.
// Steps of 64 inputs go from memory to the LDS without registers, three steps ahead, into four buffers in turn: arrays of their
// own, by which the compiler sees that reading one need not wait for loads into another.  4096 x 12288 x 4096 by tiles of 256: 162-173 us, 2.4-2.5 PFLOP/s;
// 256 x 4096 x 8192 by tiles of 128 in four parts: 15.8 us, the same with loads seven steps ahead.
// EXACT: codes become bfloat16 on their way from the LDS, as in linear_rows; else they enter the 8-bit instructions, at twice the rate: for
// 16-bit results, whose own rounding is coarser than what those lose on inputs of like size (see linear_rows; a caller who needs more asks for float32).
template <int WN, int WM, int FN, int FM> struct TileShape {
    static constexpr int kWaves = WN * WM, kN = 32 * FN * WN, kM = 32 * FM * WM, kPieces = (kN + kM) / 16, kLoads = kPieces / kWaves;
    static_assert(kPieces % kWaves == 0, "every wavefront loads as many pieces");
};

// A wait until at most n loads from memory are out, and no operation of the LDS.
constexpr int wait_loads(int n) { return (n & 15) | (n >> 4 << 14) | (7 << 4); }

__device__ static inline i32x8_t lds_operand(const char *p) {
    const i32x4_t lo = *reinterpret_cast<const i32x4_t *>(p), hi = *reinterpret_cast<const i32x4_t *>(p + 512);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// The products of a step of 64 inputs; the scales in the lowest bytes of sw and sx(j).
template <bool EXACT, int FN, int FM, typename F>
__device__ static inline void multiply(const i32x8_t (&w)[FN], const i32x8_t (&x)[FM], uint32_t sw, F sx, f32x16_t (&acc)[FN][FM]) {
    if constexpr (EXACT) {
        const float fw = scale_of_byte(sw & 255);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            bf16x8_t wv[FN], xv[FM];
#pragma unroll
            for (int i = 0; i < FN; ++i) wv[i] = bf16_of_codes(w[i][2 * s], w[i][2 * s + 1], fw);
#pragma unroll
            for (int j = 0; j < FM; ++j) xv[j] = bf16_of_codes(x[j][2 * s], x[j][2 * s + 1], scale_of_byte(sx(j) & 255));
#pragma unroll
            for (int i = 0; i < FN; ++i)
#pragma unroll
                for (int j = 0; j < FM; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wv[i], xv[j], acc[i][j], 0, 0, 0);
        }
    } else {
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const int bx = (int)sx(j);
#pragma unroll
            for (int i = 0; i < FN; ++i) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[i], x[j], acc[i][j], 0, 0, 0, (int)sw, 0, bx);
        }
    }
}

template <int DT, bool EXACT, int WN, int WM, int FN, int FM>
__global__ __launch_bounds__(64 * WN * WM) void linear_tile(LinearArgs a) {
    typedef TileShape<WN, WM, FN, FM> Shape;
    __shared__ __attribute__((aligned(16))) char buf0[Shape::kPieces * kPieceBytes], buf1[Shape::kPieces * kPieceBytes], buf2[Shape::kPieces * kPieceBytes],
        buf3[Shape::kPieces * kPieceBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wn = wave % WN, wm = wave / WN;
    const int ntiles = (a.n + Shape::kN - 1) / Shape::kN, mtiles = (a.m + Shape::kM - 1) / Shape::kM;
    const int tile = xcd_logical_tile(ntiles * mtiles * a.splits);
    if (tile < 0) return;
    // four columns of tiles at a time, so that the workgroups of an XCD at any moment share rows and weights in its L2
    const int split = tile / (ntiles * mtiles), at = tile % (ntiles * mtiles), band = at / (4 * mtiles), in_band = at % (4 * mtiles);
    const int width = min(4, ntiles - 4 * band), n0 = (4 * band + in_band % width) * Shape::kN, m0 = in_band / width * Shape::kM;
    const int words = (a.kblocks + 3) / 4, words_each = (words + a.splits - 1) / a.splits;
    const int pair0 = split * words_each * 2, pair1 = min(a.held / 2, pair0 + words_each * 2);      // the split's pairs of blocks, four steps each
    const int last_step = 4 * pair1 - 1;

    // sources of this wavefront's pieces, at step 0
    const char *source[Shape::kLoads];
    int apart[Shape::kLoads];                            // bytes from a step to the next
    const uint32_t lane_at = lane * 16;
#pragma unroll
    for (int i = 0; i < Shape::kLoads; ++i) {
        const int piece = wave * Shape::kLoads + i;
        const bool weights = piece < Shape::kN / 16;
        const int last = weights ? ((a.n + 127) / 128) * 8 - 1 : (a.m + 15) / 16 - 1;
        const int64_t rows = min(weights ? n0 / 16 + piece : m0 / 16 + piece - Shape::kN / 16, last);
        source[i] = weights ? a.w + (rows / 8 * a.held * 16 + rows % 8) * kPieceBytes : a.x + rows * a.held * 2 * kPieceBytes;
        apart[i] = weights ? 8 * kPieceBytes : kPieceBytes;
    }
    auto fetch = [&](int step, char *buf) {              // steps behind the last fetch the last again: the counts below stay what they are
        const int64_t s = min(step, last_step);
#pragma unroll
        for (int i = 0; i < Shape::kLoads; ++i)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(source[i] + s * apart[i] + lane_at),
                                             (__attribute__((address_space(3))) void *)(buf + (wave * Shape::kLoads + i) * kPieceBytes), 16, 0, 0);
    };
    // scale words of four blocks: of the wavefront's outputs (one block of 128 or a part of it to 32 FN of them) and of its rows
    const int n_wave = n0 + wn * 32 * FN, m_wave = m0 + wm * 32 * FM;
    const uint32_t *w_scales = reinterpret_cast<const uint32_t *>(a.w_scales) + (int64_t)min(n_wave / 128, (a.n + 127) / 128 - 1) * words;
    const uint32_t *x_scales[FM];
#pragma unroll
    for (int f = 0; f < FM; ++f) {
        const int row = min(m_wave + 32 * f + lane % 32, (a.m + 15) / 16 * 16 - 1);
        x_scales[f] = reinterpret_cast<const uint32_t *>(a.x_scales) + (int64_t)(row / 16) * words * 16 + row % 16;
    }
    f32x16_t acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;

    uint32_t sw, sx[FM], sw_next, sx_next[FM];
    auto fetch_scales = [&](int pair) {
        const int word = min(pair / 2, words - 1);
        sw_next = w_scales[word] >> (pair % 2 * 16);
#pragma unroll
        for (int f = 0; f < FM; ++f) sx_next[f] = x_scales[f][(int64_t)word * 16];
    };
    fetch_scales(pair0);
    fetch(4 * pair0, buf0);
    fetch(4 * pair0 + 1, buf1);
    fetch(4 * pair0 + 2, buf2);
    __builtin_amdgcn_s_waitcnt(wait_loads(3 * Shape::kLoads) | (15 << 8));   // the scales have come: said here, so that the loop does not wait for more
    const int read_at = (lane % 32 / 16) * kPieceBytes + (lane % 16 + 16 * (lane / 32)) * 16;

    auto compute = [&](const char *buf, int byte) {
        const char *wp = buf + wn * FN * 2 * kPieceBytes + read_at, *xp = buf + (Shape::kN / 16 + wm * FM * 2) * kPieceBytes + read_at;
        i32x8_t w[FN], x[FM];
#pragma unroll
        for (int i = 0; i < FN; ++i) w[i] = lds_operand(wp + i * 2 * kPieceBytes);
#pragma unroll
        for (int j = 0; j < FM; ++j) x[j] = lds_operand(xp + j * 2 * kPieceBytes);
        multiply<EXACT, FN, FM>(w, x, sw >> (8 * byte), [&](int j) { return sx[j] >> (8 * byte); }, acc);
    };
    // A step: its loads have come (those of the two after it may be out), and everybody has read the buffer that is loaded into next.
#define NNV_STEP(S, BUF, INTO)                        \
    {                                                 \
        asm volatile("" ::: "memory");                \
        __builtin_amdgcn_s_waitcnt(kWaitTwoSteps);    \
        __builtin_amdgcn_s_barrier();                 \
        asm volatile("" ::: "memory");                \
        fetch(4 * pair + S + 3, INTO);                \
        compute(BUF, S / 2);                          \
    }
    constexpr int kWaitTwoSteps = wait_loads(2 * Shape::kLoads);
    for (int pair = pair0; pair < pair1; ++pair) {
        sw = sw_next;
#pragma unroll
        for (int f = 0; f < FM; ++f) sx[f] = sx_next[f] >> (pair % 2 * 16);
        fetch_scales(pair + 1);
        NNV_STEP(0, buf0, buf3)
        NNV_STEP(1, buf1, buf0)
        NNV_STEP(2, buf2, buf1)
        NNV_STEP(3, buf3, buf2)
    }
#undef NNV_STEP
    __builtin_amdgcn_s_waitcnt(0);       // nothing may come into the LDS after the workgroup

    // A lane holds row lane % 32 of a 32 x 32 tile, outputs 8 (r / 4) + 4 (lane / 32) + r % 4: 32 rows at a time go through the wavefront's share of the
    // LDS, fours of outputs xor-ed with the row so that neither side meets a bank twice, and out in whole lines.
    __builtin_amdgcn_s_barrier();        // everybody has read the buffers
    constexpr int kFours = 8 * FN, kShare = 32 * kFours * 16, kShares = Shape::kPieces * kPieceBytes / kShare;
    static_assert(4 * kShares >= Shape::kWaves, "a share of the buffers for every wavefront");
    const int which = wave / kShares;
    f32x4_t *share = reinterpret_cast<f32x4_t *>((which == 0 ? buf0 : which == 1 ? buf1 : which == 2 ? buf2 : buf3) + wave % kShares * kShare);
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const int r0 = lane % 32;
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                share[r0 * kFours + ((8 * i + r / 2 + lane / 32) ^ (r0 & 15))] = f32x4_t{acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]};
        wave_fence();
        if (a.splits > 1) {
            const int quads = (a.n + 3) / 4;
#pragma unroll
            for (int e = lane; e < 32 * kFours; e += 64) {
                const int r = e / kFours, four = e % kFours, row = m_wave + 32 * j + r, col = n_wave + 4 * four;
                if (row < a.m && col < a.n)
                    *reinterpret_cast<f32x4_t *>(a.parts + (((int64_t)split * a.m + row) * quads + col / 4) * 4) = share[r * kFours + (four ^ (r & 15))];
            }
        } else {
#pragma unroll
            for (int e = lane; e < 16 * kFours; e += 64) {
                const int r = e / (kFours / 2), eight = e % (kFours / 2);
                store8<DT>(a, m_wave + 32 * j + r, n_wave + 8 * eight, share[r * kFours + ((2 * eight) ^ (r & 15))],
                           share[r * kFours + ((2 * eight + 1) ^ (r & 15))]);
            }
        }
        wave_fence();
    }
}

// In between: a workgroup holds 32 FN outputs x 32 FM rows and its four wavefronts split the reduction, each with all of them in
// registers; a step's operands come from memory a step ahead, and nothing is shared until the sums are added in the LDS.  A tile read by one
// wavefront needs no LDS on its way in and no barrier, and the more of the reduction stays in one workgroup the fewer partial sums are
// written: a launch fills the chip with small tiles or short parts.
template <int DT, bool EXACT, int FN, int FM>
__global__ __launch_bounds__(256, 2) void linear_waves(LinearArgs a) {
    constexpr int kN = 32 * FN, kM = 32 * FM, kQuads = FN * FM * 4, kAhead = 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ntiles = (a.n + kN - 1) / kN, mtiles = (a.m + kM - 1) / kM;
    const int tile = xcd_logical_tile(ntiles * mtiles * a.splits);
    if (tile < 0) return;
    const int split = tile / (ntiles * mtiles), at = tile % (ntiles * mtiles), n0 = at / mtiles * kN, m0 = at % mtiles * kM;
    const int words = (a.kblocks + 3) / 4, words_each = (words + a.splits - 1) / a.splits;
    const int step0 = split * words_each * 8, step1 = min(2 * a.held, step0 + words_each * 8);

    const int r16 = lane % 32 / 16, inside = (lane % 16 + 16 * (lane / 32)) * 16;
    const char *w = a.w + ((int64_t)(n0 / 128) * a.held * 16 + n0 / 16 % 8 + r16) * kPieceBytes + inside;
    const uint32_t *w_scales = reinterpret_cast<const uint32_t *>(a.w_scales) + (int64_t)(n0 / 128) * words;
    const char *x[FM];
    const uint32_t *x_scales[FM];
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const int64_t rows = min(m0 / 16 + 2 * j + r16, (a.m + 15) / 16 - 1);
        x[j] = a.x + rows * a.held * 2 * kPieceBytes + inside;
        x_scales[j] = reinterpret_cast<const uint32_t *>(a.x_scales) + rows * words * 16 + lane % 16;
    }
    struct Operands { i32x8_t w[FN], x[FM]; uint32_t sw, sx[FM]; };
    auto load16x2 = [](const char *p) {
        const i32x4_t lo = *reinterpret_cast<const i32x4_t *>(p), hi = *reinterpret_cast<const i32x4_t *>(p + 512);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto fetch = [&](int step, Operands &o) {
        const int64_t s = step;
#pragma unroll
        for (int i = 0; i < FN; ++i) o.w[i] = load16x2(w + s * 8 * kPieceBytes + i * 2 * kPieceBytes);
#pragma unroll
        for (int j = 0; j < FM; ++j) o.x[j] = load16x2(x[j] + s * kPieceBytes);
        const int word = step / 8;
        o.sw = w_scales[word];
#pragma unroll
        for (int j = 0; j < FM; ++j) o.sx[j] = x_scales[j][(int64_t)word * 16];
    };
    f32x16_t acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
    // a step behind the last is loaded as the last again: a load that some rounds leave out would make every round wait for all on their way
    Operands ring[kAhead];
    const int last = step1 - 1;
    if (step0 < step1)
#pragma unroll
        for (int d = 0; d < kAhead; ++d) fetch(min(step0 + wave + 4 * d, last), ring[d]);
    for (int base = step0 + wave; base < step1; base += 4 * kAhead) {
#pragma unroll
        for (int d = 0; d < kAhead; ++d) {
            const int step = base + 4 * d;
            if (step < step1) {
                const int byte = step / 2 % 4;
                multiply<EXACT, FN, FM>(ring[d].w, ring[d].x, ring[d].sw >> (8 * byte), [&](int j) { return ring[d].sx[j] >> (8 * byte); }, acc);
            }
            fetch(min(step + 4 * kAhead, last), ring[d]);
        }
    }
    // all sums into the LDS, a quarter of each out of it by every wavefront
    __shared__ f32x4_t part[4][kQuads][64];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                part[wave][(i * FM + j) * 4 + q][lane] = f32x4_t{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kQuads / 4; ++e) {
        const int quad = wave * (kQuads / 4) + e, i = quad / 4 / FM, j = quad / 4 % FM, q = quad % 4;
        const f32x4_t v = (part[0][quad][lane] + part[1][quad][lane]) + (part[2][quad][lane] + part[3][quad][lane]);
        const int row = m0 + 32 * j + lane % 32, col = n0 + 32 * i + 8 * q + 4 * (lane / 32);
        if (a.splits == 1) store4<DT>(a, row, col, v);
        else if (row < a.m && col < a.n) *reinterpret_cast<f32x4_t *>(a.parts + (((int64_t)split * a.m + row) * ((a.n + 3) / 4) + col / 4) * 4) = v;
    }
}

// Adds the parts of a split reduction in their order, four outputs a thread.
template <int DT> __global__ __launch_bounds__(256) void linear_join(LinearArgs a) {
    const int quads = (a.n + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)a.m * quads) return;
    f32x4_t v = {0, 0, 0, 0};
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) v += *reinterpret_cast<const f32x4_t *>(a.parts + ((int64_t)s * a.m * quads + i) * 4);
    store4<DT>(a, i / quads, (int)(i % quads) * 4, v);
}

// How a product runs.  Times of whole calls in us, bfloat16, weights not in the caches, best of each kind:
//   m, n, k               rows   waves   tile 128   tile 256
//   16,  4096, 8192       13.6    13.3       14.5       27
//   16, 12288, 4096       14.4    16.0       18.3       22       one row: rows 12.6
//   64,  4096, 8192         -     15.2       16.7       28       waves in 4 parts 15.2, 2 16.0, 1 19.3
//   128, 4096, 8192         -     20.1       20.5       32
//   256, 4096, 8192         -     27.1       25.4       36       tile 128 in 4 parts 25.4, 2 32, 1 46, 8 29
//   256, 12288, 4096        -     42         32         38       tile 128 in 1 part 32, 2 37
//   512, 4096, 8192         -     47         36         43       tile 128 in 2 parts 36, 1 49
//   1024, 4096, 8192        -     91         55         55
//   1024, 12288, 4096       -    137         68         54
//   4096, 12288, 4096       -      -         207        173
//   1024, 1024, 1024        -     10.3       11.8       19.6
enum LinearWay { kRows, kWaves, kTile128, kTile256 };
struct LinearPlan { LinearWay way; int splits; };
static LinearPlan linear_plan(const nnv_linear_desc &d, int m) {
    auto count = [&](int rows, int outputs) { return (int64_t)((m + rows - 1) / rows) * ((d.n + outputs - 1) / outputs); };
    auto parts = [&](int64_t tiles, int shortest) {      // so that tiles fill 256 compute units, four parts at most, none shorter than so many inputs
        const int64_t s = 256 / tiles, most = d.k / shortest < 4 ? d.k / shortest : 4;
        return (int)(s > most ? most < 1 ? 1 : most : s < 1 ? 1 : s);
    };
    if (m <= 16) return {kRows, 1};
    if (count(256, 256) >= 192) return {kTile256, 1};
    if (m >= 128 && count(128, 128) >= 48 && (d.k >= 2048 || count(128, 128) >= 160)) return {kTile128, parts(count(128, 128), 1024)};
    return {kWaves, parts(count(32, 64), 2048)};
}

template <int DT, int DX> static hipError_t launch_rows(const LinearArgs &a, const void *x, int64_t ldx, int k, hipStream_t st) {
    // As many outputs to a workgroup as leave three workgroups to four compute units.  Four rows, us with 16, 32, 64 outputs:
    // n 4096, k 8192: 11.8, 12.3, 14.5;  6144, 4096: 10.3, 8.9, 9.2;  8192, 8192: 19.6, 15.1, 18.4;  12288, 4096: 17.9, 15.9, 12.6
    if (a.n >= 192 * 64) linear_rows<DT, DX, 4><<<(a.n + 63) / 64, 64 * kRowWaves, 0, st>>>(a, x, ldx, k);
    else if (a.n >= 192 * 32) linear_rows<DT, DX, 2><<<(a.n + 31) / 32, 64 * kRowWaves, 0, st>>>(a, x, ldx, k);
    else linear_rows<DT, DX, 1><<<(a.n + 15) / 16, 64 * kRowWaves, 0, st>>>(a, x, ldx, k);
    return hipGetLastError();
}

// y's type is known; x is rounded in a launch of its own unless there are a few rows of it.
template <int DT> static hipError_t launch_product(const LinearArgs &a, LinearWay way, hipStream_t st) {
    constexpr bool kExact = DT == NNV_F32;
    auto grid = [&](int rows, int outputs) { return xcd_grid(((a.n + outputs - 1) / outputs) * ((a.m + rows - 1) / rows) * a.splits); };
    if (way == kWaves) linear_waves<DT, kExact, 2, 1><<<grid(32, 64), 256, 0, st>>>(a);
    else if (way == kTile128) linear_tile<DT, kExact, 2, 2, 2, 2><<<grid(128, 128), 256, 0, st>>>(a);
    else linear_tile<DT, kExact, 2, 4, 4, 2><<<grid(256, 256), 512, 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    linear_join<DT><<<(unsigned)(((int64_t)a.m * ((a.n + 3) / 4) + 255) / 256), 256, 0, st>>>(a);
    return hipGetLastError();
}

template <int DT> static hipError_t launch_quantise(const void *x, int64_t ldx, int m, int k, char *codes, char *scales, hipStream_t st) {
    const dim3 grid((blocks128(k) + 1) / 2, (m + 15) / 16);
    linear_quantise<DT><<<grid, 256, 0, st>>>(x, ldx, m, k, codes, scales);
    return hipGetLastError();
}

template <int DT> static hipError_t launch_pack(const void *w, int n, int k, char *codes, char *scales, hipStream_t st) {
    const dim3 grid(held_blocks(k), blocks128(n));
    linear_pack<DT><<<grid, 256, 0, st>>>(w, n, k, codes, scales);
    return hipGetLastError();
}

size_t linear_workspace_bytes(const nnv_linear_desc &d, int m) {
    const LinearPlan plan = linear_plan(d, m);
    const int splits = plan.splits;
    if (plan.way == kRows) return 0;
    return linear_x_bytes(m, d.k) + (splits == 1 ? 0 : (size_t)splits * m * ((d.n + 3) / 4) * 16);
}

// f with a storage type as a constant.
template <int DT> struct TypeConstant { static constexpr int value = DT; };
template <typename F> static hipError_t with_type(int dtype, F f) {
    return dtype == NNV_F32 ? f(TypeConstant<NNV_F32>{}) : dtype == NNV_F16 ? f(TypeConstant<NNV_F16>{}) : f(TypeConstant<NNV_BF16>{});
}

hipError_t launch_linear_pack(const nnv_linear_desc &d, const void *raw, void *tx, hipStream_t st) {
    char *codes = static_cast<char *>(tx), *scales = codes + linear_codes_bytes(blocks128(d.n) * 128, d.k);
    return with_type(d.raw_dtype, [&](auto dt) { return launch_pack<dt.value>(raw, d.n, d.k, codes, scales, st); });
}

hipError_t launch_linear(const nnv_linear_desc &d, int m, const void *x, int64_t ldx, const void *tx, const float *bias, void *y, int64_t ldy, void *ws,
                         hipStream_t st) {
    LinearArgs a;
    a.w = static_cast<const char *>(tx);
    a.w_scales = a.w + linear_codes_bytes(blocks128(d.n) * 128, d.k);
    char *codes = static_cast<char *>(ws), *scales = codes + linear_codes_bytes(m, d.k);
    a.x = codes; a.x_scales = scales;
    a.bias = bias; a.y = y; a.ldy = ldy; a.m = m; a.n = d.n; a.kblocks = blocks128(d.k); a.held = held_blocks(d.k);
    const LinearPlan plan = linear_plan(d, m);
    a.splits = plan.splits;
    a.parts = reinterpret_cast<float *>(codes + linear_x_bytes(m, d.k));
    if (plan.way == kRows)
        return with_type(d.y_dtype, [&](auto dt) { return with_type(d.x_dtype, [&](auto dx) { return launch_rows<dt.value, dx.value>(a, x, ldx, d.k, st); }); });
    const hipError_t e = with_type(d.x_dtype, [&](auto dx) { return launch_quantise<dx.value>(x, ldx, m, d.k, codes, scales, st); });
    if (e != hipSuccess) return e;
    return with_type(d.y_dtype, [&](auto dt) { return launch_product<dt.value>(a, plan.way, st); });
}

}  // namespace nnv

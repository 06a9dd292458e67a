// Quantisation of rows to four-bit floating point with a scale per 32 elements, and back.
//
// A block's scale is the power of two 2^(floor(log2 amax) - 2): divided by it the largest element lies in [4, 8), and the
// largest code is 6.  floor(log2 amax) is the exponent field of the fp32 value, so the scale byte is that field minus 2 (at least
// 0: subnormal blocks keep the smallest scale).  The conversion instruction divides by the scale, rounds to nearest even and
// limits to +-6 in one step for two elements (compared with the definition over every scale, halfway values among the elements).
#include "fff_device.h"
#include "fff_mx4.h"

namespace fff {
namespace {

// bits of |v| in fp32 order (a NaN above infinity)
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    const uint32_t e = amax >> 23;
    return e == 255 ? 255u : (e > 2 ? e - 2 : 0u);
}

// eight values -> eight codes, the first in the low bits
__device__ __forceinline__ uint32_t pack_codes(const float* f, uint32_t scale) {
    const float s = __uint_as_float(scale << 23);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[0], f[1], s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[2], f[3], s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[4], f[5], s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[6], f[7], s, 3);
    return scale == 255u ? 0u : r;
}

template <int XOR> __device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    constexpr int perm = XOR == 1 ? 0xB1 : 0x4E;     // lanes [1,0,3,2] or [2,3,0,1] of every four
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, perm, 0xf, 0xf, false));
}

// Eight consecutive elements of a row from element c on; zeros behind its end.
template <bool BF16> __device__ __forceinline__ void load_eight(const char* row, int64_t c, int64_t cols, float* f) {
    constexpr int es = BF16 ? 2 : 4;
    if (c + 8 <= cols) {
        if (BF16) {
            widen<true>(load_any(row + c * es), f);
        } else {
            widen<false>(load_any(row + c * es), f);
            widen<false>(load_any(row + c * es + 16), f + 4);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = c + i < cols ? Elem<BF16>::load(row, c + i) : 0.0f;
    }
}

// A lane takes eight elements of a row, four lanes a block; a thread keeps its place in the row and strides over rows, so
// that the division into row and place is made once.
template <bool BF16>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const char* __restrict__ src, uint8_t* __restrict__ codes,
                                                           uint8_t* __restrict__ scales, int64_t rows, int64_t cols, int64_t row_step) {
    constexpr int es = BF16 ? 2 : 4;
    const int64_t nb = (cols + kMxBlock - 1) / kMxBlock;
    const int64_t pieces = 4 * nb;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t r0 = id / pieces, c = id - r0 * pieces;
    if (r0 >= row_step) return;                    // (whole groups of four lanes)
    for (int64_t r = r0; r < rows; r += row_step) {
        float f[8];
        load_eight<BF16>(src + r * cols * es, 8 * c, cols, f);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, magnitude(f[i]));
        m = quad_max<2>(quad_max<1>(m));
        const uint32_t s = scale_byte(m);
        *(uint32_t*)(codes + r * nb * 16 + 4 * c) = pack_codes(f, s);
        if ((c & 3) == 0) scales[r * nb + c / 4] = (uint8_t)s;
    }
}

// The transposed matrix: 64 columns x 128 rows a block, a lane one column's 32 rows (read row by row, 64 columns of a row at once, all 32 on their way together),
// a wave one block of 32 of each column.  The codes cross LDS so that a column's four blocks leave as 64 bytes in a piece.
constexpr int kTransRows = 128, kTransCols = 64;
template <bool BF16>
__global__ __launch_bounds__(256) void mx4_quantize_columns_kernel(const char* __restrict__ src, uint8_t* __restrict__ codes,
                                                                   uint8_t* __restrict__ scales, int64_t rows, int64_t cols,
                                                                   int64_t col_tiles, int64_t row_tiles) {
    __shared__ uint4 part[kTransCols * 5];         // four blocks of a column, five apart
    __shared__ uint8_t part_s[kTransCols * 4];
    constexpr int es = BF16 ? 2 : 4;
    const int64_t nb = (rows + kMxBlock - 1) / kMxBlock;
    const int64_t per = col_tiles * row_tiles;
    const int64_t b = blockIdx.x / per, at = blockIdx.x - b * per;
    const int64_t c0 = at % col_tiles * kTransCols, kb0 = at / col_tiles * (kTransRows / kMxBlock);
    src += b * rows * cols * es;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int64_t r0 = (kb0 + wv) * kMxBlock, c = c0 + lane < cols ? c0 + lane : cols - 1;
    if (r0 < rows) {
        float f[32];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) f[i] = Elem<BF16>::load(src, (r0 + i < rows ? r0 + i : rows - 1) * cols + c);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            f[i] = r0 + i < rows ? f[i] : 0.0f;
            m = max(m, magnitude(f[i]));
        }
        const uint32_t s = scale_byte(m);
        part[lane * 5 + wv] = make_uint4(pack_codes(f, s), pack_codes(f + 8, s), pack_codes(f + 16, s), pack_codes(f + 24, s));
        part_s[lane * 4 + wv] = (uint8_t)s;
    }
    __syncthreads();
    const int64_t to = c0 + (tid >> 2), kb = kb0 + (tid & 3);
    if (to >= cols || kb >= nb) return;
    const int64_t o = (b * cols + to) * nb + kb;
    *(uint4*)(codes + o * 16) = part[(tid >> 2) * 5 + (tid & 3)];
    scales[o] = part_s[tid];
}

// Eight elements a lane, as in mx4_quantize_kernel.
template <bool BF16>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                             char* __restrict__ out, int64_t rows, int64_t cols, int64_t row_step) {
    constexpr int es = BF16 ? 2 : 4;
    const int64_t nb = (cols + kMxBlock - 1) / kMxBlock;
    const int64_t pieces = (cols + 7) / 8;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t r0 = id / pieces, c = id - r0 * pieces;
    if (r0 >= row_step) return;
    for (int64_t r = r0; r < rows; r += row_step) {
        const uint32_t w = *(const uint32_t*)(codes + r * nb * 16 + 4 * c);
        const float s = __uint_as_float((uint32_t)scales[r * nb + c / 4] << 23);
        char* const o = out + (r * cols + 8 * c) * es;
        if (BF16) {
            const bf16x2_t v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1),
                                   __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3)};
            if (8 * c + 8 <= cols) {
                store_any(o, __builtin_bit_cast(uint4, v));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (8 * c + i < cols) ((__bf16*)o)[i] = v[i / 2][i % 2];
            }
        } else {
            float f[8];
#define FFF_PAIR(I)                                                        \
    {                                                                      \
        const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, I);  \
        f[2 * I] = v[0];                                                   \
        f[2 * I + 1] = v[1];                                               \
    }
            FFF_PAIR(0) FFF_PAIR(1) FFF_PAIR(2) FFF_PAIR(3)
#undef FFF_PAIR
            if (8 * c + 8 <= cols) {
                store_any(o, narrow<false>(f));
                store_any(o + 16, narrow<false>(f + 4));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (8 * c + i < cols) ((float*)o)[i] = f[i];
            }
        }
    }
}

__global__ __launch_bounds__(256) void pad_rows_kernel(const uint16_t* __restrict__ src, uint16_t* __restrict__ dst, int64_t rows, int64_t cols,
                                                       int64_t row_step) {
    const int64_t pieces = (cols + kMxBlock - 1) / kMxBlock * 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t r0 = id / pieces, c = id - r0 * pieces;
    if (r0 >= row_step) return;
    for (int64_t r = r0; r < rows; r += row_step) {
        const uint16_t* const row = src + r * cols;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (8 * c + 8 <= cols) {
            v = load_any(row + 8 * c);
        } else {
            uint16_t e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = 8 * c + i < cols ? row[8 * c + i] : (uint16_t)0;
            v = __builtin_bit_cast(uint4, e);
        }
        *(uint4*)(dst + (r * pieces + c) * 8) = v;
    }
}

// Rows a pass over the grid takes (every one of its `pieces` places has a thread) and the blocks for them: as many threads as the compute units
// hold at once, fewer for small matrices.
int64_t rows_a_pass(int64_t rows, int64_t pieces, int64_t* blocks) {
    const int64_t threads = (int64_t)device_info().cus * 2048;
    int64_t step = threads / pieces;
    if (step < 1) step = 1;
    if (step > rows) step = rows;
    *blocks = (step * pieces + 255) / 256;
    return step;
}

}  // namespace

hipError_t launch_mx4_quantize(const void* src, uint8_t* codes, uint8_t* scales, bool transpose, int64_t batch, int64_t rows,
                               int64_t cols, bool bf16, hipStream_t s) {
    if (transpose) {
        const int64_t ct = (cols + kTransCols - 1) / kTransCols, rt = (rows + kTransRows - 1) / kTransRows;
        note_launch("mx4_quantize_columns_kernel<%s>", bf16 ? "bf16" : "f32");
        const dim3 grid((unsigned)(batch * ct * rt));
        if (bf16) mx4_quantize_columns_kernel<true><<<grid, 256, 0, s>>>((const char*)src, codes, scales, rows, cols, ct, rt);
        else mx4_quantize_columns_kernel<false><<<grid, 256, 0, s>>>((const char*)src, codes, scales, rows, cols, ct, rt);
        return hipGetLastError();
    }
    rows *= batch;
    int64_t blocks;
    const int64_t step = rows_a_pass(rows, 4 * mx_blocks(cols), &blocks);
    note_launch("mx4_quantize_kernel<%s>", bf16 ? "bf16" : "f32");
    if (bf16) mx4_quantize_kernel<true><<<dim3((unsigned)blocks), 256, 0, s>>>((const char*)src, codes, scales, rows, cols, step);
    else mx4_quantize_kernel<false><<<dim3((unsigned)blocks), 256, 0, s>>>((const char*)src, codes, scales, rows, cols, step);
    return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, void* out, int64_t rows, int64_t cols, bool bf16,
                                 hipStream_t s) {
    int64_t blocks;
    const int64_t step = rows_a_pass(rows, (cols + 7) / 8, &blocks);
    note_launch("mx4_dequantize_kernel<%s>", bf16 ? "bf16" : "f32");
    if (bf16) mx4_dequantize_kernel<true><<<dim3((unsigned)blocks), 256, 0, s>>>(codes, scales, (char*)out, rows, cols, step);
    else mx4_dequantize_kernel<false><<<dim3((unsigned)blocks), 256, 0, s>>>(codes, scales, (char*)out, rows, cols, step);
    return hipGetLastError();
}

hipError_t launch_pad_rows(const uint16_t* src, uint16_t* dst, int64_t rows, int64_t cols, hipStream_t s) {
    int64_t blocks;
    const int64_t step = rows_a_pass(rows, 4 * mx_blocks(cols), &blocks);
    note_launch("pad_rows_kernel");
    pad_rows_kernel<<<dim3((unsigned)blocks), 256, 0, s>>>(src, dst, rows, cols, step);
    return hipGetLastError();
}

}  // namespace fff

// Products with four-bit matrices: out = act(A W^T + b), and leaf networks of k leaves per token.
//
// W is [N, K] in blocks of 32 along K.  The operand of a matrix instruction is a row of W per lane: lane (j, g) of a wave
// (j = lane mod 16, g = lane / 16) takes block 4 c + g of row j in step c, 16 bytes of codes and one scale byte, so a step covers
// 128 elements of K and every load is a whole block.  K is only an order of summation, so the rows of A are read the same way.
//   A in bf16: the lane's 32 codes become four operands of v_mfma_f32_16x16x32_bf16 (eight elements of K per lane each): the
//     conversion instruction multiplies by the scale, and code times scale is exact in bf16 (infinity from 2^128 on, which scales 253 and 254 reach).
//   A in four bits: the 16 bytes are the operand of v_mfma_scale_f32_16x16x128_f8f6f4 as they are, with a scale byte per lane.
// Rows of W are the rows of the result, rows of A its columns: lane (j, g) ends with four consecutive outputs of token j.
#include "fff_device.h"
#include "fff_mx4.h"

#include <type_traits>

namespace fff {
namespace {

// an address that is the same in all lanes, in scalar registers
__device__ __forceinline__ const char* uniform(const char* p) {
    const uint64_t v = (uint64_t)p;
    return (const char*)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)v) | (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(v >> 32)) << 32);
}
// four bytes a lane straight to LDS: lane i's land at lds + 4 i
__device__ __forceinline__ void load_word_to_lds(const char* src, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(src) : "memory");
}
// load_to_lds from a base that the wave shares
__device__ __forceinline__ void load_to_lds_from(const char* base, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}

typedef int i32x8_t __attribute__((ext_vector_type(8)));

enum { kDense, kHidden, kOutput };

struct Args {
    const char* a;               // rows of bf16, or codes
    const uint8_t* a_scales;
    int64_t a_row;               // bytes from row to row
    const uint8_t* w;
    const uint8_t* w_scales;
    const void* bias;            // may be null
    char* out;
    int64_t T, N;                // rows of A, rows of W (of one leaf)
    int64_t out_row;             // elements from row to row of out (hidden activations: of each of a row's two values)
    int Kb, pieces;              // blocks of a row of W; whole pieces of 16 bytes of a bf16 row
    int act;
    bool out_bf16, out_vec;      // out_vec: four consecutive outputs are one aligned store
    // leaf networks
    const int32_t* idx;          // [T, k]
    const float* weight;         // [T, k] or null
    const int32_t* perm;         // slot -> pair t k + i
    const int32_t* tile_leaf;    // [tiles]
    const int32_t* tile_slot;    // [tiles] first slot
    const int32_t* start;        // [E + 1] first slot of a leaf
    const int32_t* n_tiles;
    int64_t E;
    int k;
    int parts;                   // blocks that share a tile's rows (output launches)
};

__device__ __forceinline__ bf16x8_t dequantise8(uint32_t codes, float scale) {
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
    const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
    const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

template <int BYTE = 0>
__device__ __forceinline__ f32x4_t mfma4(const uint4& w, uint32_t ws, const uint4& a, uint32_t as, const f32x4_t& acc) {
    const i32x8_t vw = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0}, va = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(vw, va, acc, 4, 4, BYTE, (int)ws, BYTE, (int)as);
}

// One step of 128 elements: a block of 32 of this lane's row of W against VALUES rows of each of MT rows of A (A in bf16: four pieces each).
template <bool A4, int MT, int VALUES>
__device__ __forceinline__ void multiply128(const uint4& w, uint32_t ws, const uint4 (&a)[VALUES][MT][A4 ? 1 : 4], const uint32_t (&as)[MT], f32x4_t (&acc)[MT]) {
    if constexpr (A4) {
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[m] = mfma4(w, ws, a[0][m][0], as[m], acc[m]);
    } else {
        const float s = __uint_as_float(ws << 23);
        const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const bf16x8_t f = dequantise8(q[u], s);
#pragma unroll
            for (int v = 0; v < VALUES; ++v)
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, __builtin_bit_cast(bf16x8_t, a[v][m][u]), acc[m], 0, 0, 0);
        }
    }
}

// The same with its loads, at a row's end: block b may lie behind it, and the block may be cut (pieces of bf16 rows): zeros there.
template <bool A4, int MT, int VALUES>
__device__ __forceinline__ void step128(const uint8_t* w_row, const uint8_t* ws_row, const char* const (&a_row)[MT],
                                        const uint8_t* const (&as_row)[MT], int b, int Kb, int pieces, f32x4_t (&acc)[MT]) {
    constexpr int kPieces = A4 ? 1 : 4;
    const bool in = b < Kb;
    const int bb = in ? b : Kb - 1;
    const uint4 w = keep_if(in, *(const uint4*)(w_row + 16 * (int64_t)bb));
    const uint32_t ws = in ? ws_row[bb] : 0u;
    uint4 a[VALUES][MT][kPieces];
    uint32_t as[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            const int p = kPieces * bb + u;
            const bool there = in && (A4 || p < pieces);
#pragma unroll
            for (int v = 0; v < VALUES; ++v) a[v][m][u] = keep_if(there, *(const uint4*)(a_row[m] + 64 * (int64_t)Kb * v + 16 * (int64_t)(there ? p : 0)));
        }
        if constexpr (A4) as[m] = in ? as_row[m][bb] : 0u;
    }
    multiply128<A4, MT, VALUES>(w, ws, a, as, acc);
}

// The steps wv, wv + waves, ... of the rows' steps, the loads of several of them (few rows of A: four) on their way at once: a wave has few steps, and
// one after the other they are a chain of memory round trips.  VALUES = 2: rows of hidden activations, a row of first values and one of second ones, 64 Kb bytes each.
template <bool A4, int MT, int VALUES>
__device__ __forceinline__ void wave_steps(const uint8_t* w_row, const uint8_t* ws_row, const char* const (&a_row)[MT],
                                           const uint8_t* const (&as_row)[MT], int Kb, int pieces, int g, int wv, int waves,
                                           f32x4_t (&acc)[MT]) {
    constexpr int kRows = MT * VALUES, kBatch = A4 ? (MT == 4 ? 2 : 4) : (kRows == 1 ? 4 : kRows == 2 ? 2 : 1), kPieces = A4 ? 1 : 4;
    const int steps = (Kb + 3) / 4;
    const int whole = A4 ? Kb / 4 : pieces / 16;       // steps without an end of a row in them
    int c = wv;
    for (; c < whole; c += kBatch * waves) {
        uint4 w[kBatch], a[kBatch][VALUES][MT][kPieces];
        uint32_t ws[kBatch], as[kBatch][MT];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int s = c + u * waves;
            if (u > 0 && s >= whole) break;
            const int b = 4 * s + g;
            w[u] = *(const uint4*)(w_row + 16 * (int64_t)b);
            ws[u] = ws_row[b];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
#pragma unroll
                for (int v = 0; v < VALUES; ++v)
#pragma unroll
                    for (int q = 0; q < kPieces; ++q) a[u][v][m][q] = *(const uint4*)(a_row[m] + 64 * (int64_t)Kb * v + 16 * (int64_t)(kPieces * b + q));
                if constexpr (A4) as[u][m] = as_row[m][b];
            }
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (u > 0 && c + u * waves >= whole) break;
            multiply128<A4, MT, VALUES>(w[u], ws[u], a[u], as[u], acc);
        }
    }
    for (c = whole + (wv + waves - whole % waves) % waves; c < steps; c += waves)      // (the first of this wave's behind the whole ones)
        step128<A4, MT, VALUES>(w_row, ws_row, a_row, as_row, 4 * c + g, Kb, pieces, acc);
}

__device__ __forceinline__ float bias_at(const Args& a, const void* bias, int64_t n) {
    if (!bias) return 0.0f;
    return a.out_bf16 ? bf16_to_f32(((const uint16_t*)bias)[n]) : ((const float*)bias)[n];
}

// GELU of results that end in bf16: v Phi(v), with Phi(-x) = 2^q(x), x = |v|, and q a polynomial of degree nine fitted to log2 Phi(-x) on [0, 14.5] so that the
// error of Phi(-x) is a part of it, however small it is: less than 2^-16 of it for x <= 5, 2^-15 to 7, 2^-12 to 11, 2^-10 to 14.5, where single precision
// ends (half a step of bf16: 2^-8).  Behind it q falls on, and 2^q is zero.  A form of the error function with an absolute bound (3e-7 of erfc) is as long, and nine
// steps of bf16 off at v = -5 (4096 x 4096 x 4096: 127 us with either; the library's error function takes a fifth more).
__device__ __forceinline__ float gelu_bulk(float v) {
    const float x = fabsf(v);
    float q = fmaf(x, -2.15122642e-9f, 1.54943689e-7f);
    q = fmaf(q, x, -4.88549659e-6f);
    q = fmaf(q, x, 8.94168485e-5f);
    q = fmaf(q, x, -1.06638416e-3f);
    q = fmaf(q, x, 8.87488251e-3f);
    q = fmaf(q, x, -5.44875760e-2f);
    q = fmaf(q, x, -4.58109131e-1f);
    q = fmaf(q, x, -1.15133097f);
    q = fmaf(q, x, -9.99995044e-1f);
    const float e = __builtin_amdgcn_exp2f(q);
    return v * (v >= 0.0f ? 1.0f - e : e);
}
// Of results in fp32: erfc, where 1 + erf would cancel below zero.
__device__ __forceinline__ float gelu_f32(float v) { return 0.5f * v * erfcf(v * -0.70710678118654752440f); }
// (ReLU by a comparison: a maximum with 0 would turn NaN, which a block of scale 255 stands for, into 0)
__device__ __forceinline__ float apply(float v, int act, bool bf16) {
    if (act == 0) return v < 0.0f ? 0.0f : v;
    return act == 2 ? v : bf16 ? gelu_bulk(v) : gelu_f32(v);
}

// four consecutive outputs n .. n + 3 of a row, those below `limit`
__device__ __forceinline__ void store4(char* out, bool bf16, bool vec, int64_t at, int64_t n, int64_t limit, const float* v) {
    if (bf16) {
        uint16_t* const o = (uint16_t*)out + at;
        if (vec && n + 4 <= limit) {
            *(uint2*)(o + n) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (n + q < limit) o[n + q] = f32_to_bf16(v[q]);
        }
    } else {
        float* const o = (float*)out + at;
        if (vec && n + 4 <= limit) {
            *(float4*)(o + n) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (n + q < limit) o[n + q] = v[q];
        }
    }
}

// Hidden activations are held as two bf16 values, the first 16 bits of the fp32 value and what they leave, rounded: within 2^-15 of it, where one value, within 2^-8,
// would cost results in bf16 half of their accuracy (of 8192 tokens through 2 of 16 leaves, 768 - 2048 - 768: 2.3e-3 off on average, 1.7e-3 with two, which is the rounding of the
// results alone; 169 and 211 us).  Infinities and NaN are the first value alone.  A row is its first values, then its second ones.
__device__ __forceinline__ float first_value(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }
__device__ __forceinline__ float second_value(float v) { return fabsf(v) < __builtin_inff() ? v - first_value(v) : 0.0f; }
__device__ __forceinline__ uint32_t first_values(float a, float b) { return __float_as_uint(a) >> 16 | (__float_as_uint(b) & 0xffff0000u); }
__device__ __forceinline__ uint32_t second_values(float a, float b) { return pack_bf16x2(second_value(a), second_value(b)); }
// four of a row of `width`, at a multiple of four
__device__ __forceinline__ void store_hidden4(char* out, int64_t row, int64_t width, int64_t n, const float* v) {
    uint16_t* const o = (uint16_t*)out + row * 2 * width + n;
    *(uint2*)o = make_uint2(first_values(v[0], v[1]), first_values(v[2], v[3]));
    *(uint2*)(o + width) = make_uint2(second_values(v[0], v[1]), second_values(v[2], v[3]));
}
// eight, at a multiple of eight
__device__ __forceinline__ void store_hidden8(char* out, int64_t row, int64_t width, int64_t n, const float* v) {
    uint16_t* const o = (uint16_t*)out + row * 2 * width + n;
    *(uint4*)o = make_uint4(first_values(v[0], v[1]), first_values(v[2], v[3]), first_values(v[4], v[5]), first_values(v[6], v[7]));
    *(uint4*)(o + width) = make_uint4(second_values(v[0], v[1]), second_values(v[2], v[3]), second_values(v[4], v[5]), second_values(v[6], v[7]));
}

// eight, at a multiple of eight; vec: rows are whole aligned pieces of 16 bytes
__device__ __forceinline__ void store8(char* out, bool bf16, bool vec, int64_t at, int64_t n, int64_t limit, const float* v) {
    if (vec && n + 8 <= limit) {
        if (bf16) {
            *(uint4*)((uint16_t*)out + at + n) = narrow<true>(v);
        } else {
            *(uint4*)((float*)out + at + n) = narrow<false>(v);
            *(uint4*)((float*)out + at + n + 4) = narrow<false>(v + 4);
        }
        return;
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        if (n + q >= limit) break;
        if (bf16) ((uint16_t*)out)[at + n + q] = f32_to_bf16(v[q]);
        else ((float*)out)[at + n + q] = v[q];
    }
}

// 16 rows of W against 16 MT rows of A per block, K shared out among its waves.
//   kDense         rows of A as they come, rows of out too
//   kHidden        a tile of one leaf's slots: rows of A are the slots' tokens; out is h [slot][two values][32 blocks]
//   kOutput        a tile of one leaf's slots, or half of one: rows of A are h; out is y [pair] in fp32, or with k = 1 the token's row
template <bool A4, int MT, int MODE, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 4) void mx4_rows_kernel(const Args a) {
    __shared__ f32x4_t part[WAVES][MT][kWave];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, j = lane & 15, g = lane >> 4;
    const int64_t n_blocks = (a.N + 15) / 16;
    int64_t nb = blockIdx.x % n_blocks, tile = blockIdx.x / n_blocks, part_of = 0;
    if (MODE == kOutput && a.parts > 1) {
        part_of = tile % a.parts;
        tile /= a.parts;
    }
    const int64_t n0 = nb * 16;
    const int64_t w_row_bytes = (int64_t)a.Kb * 16;
    const int64_t n = n0 + j < a.N ? n0 + j : a.N - 1;
    int64_t leaf = 0, first = 0, rows = 0;     // first row of A (slot, pair, token) and how many there are
    if constexpr (MODE == kDense) {
        first = tile * (16 * MT);
        rows = a.T - first;
    } else {
        if (tile >= *a.n_tiles) return;
        leaf = a.tile_leaf[tile];
        first = a.tile_slot[tile] + part_of * (16 * MT);
        rows = a.start[leaf + 1] - first;
        if (rows <= 0) return;
    }
    if (rows > 16 * MT) rows = 16 * MT;
    f32x4_t acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const char* a_row[MT];
    const uint8_t* as_row[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        int64_t r = 16 * m + j < rows ? 16 * m + j : rows - 1;
        r += first;
        if constexpr (MODE == kHidden) r = a.perm[r] / a.k;
        a_row[m] = a.a + r * a.a_row;
        as_row[m] = A4 ? a.a_scales + r * a.Kb : nullptr;
    }
    wave_steps<A4, MT, MODE == kOutput ? 2 : 1>(a.w + (leaf * a.N + n) * w_row_bytes, a.w_scales + (leaf * a.N + n) * a.Kb, a_row, as_row, a.Kb, a.pieces, g, wv, WAVES, acc);
#pragma unroll
    for (int m = 0; m < MT; ++m) part[wv][m][lane] = acc[m];
    __syncthreads();
    for (int m = wv; m < MT; m += WAVES) {
        f32x4_t v = part[0][m][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += part[w][m][lane];
        const int64_t row = 16 * m + j;
        if (row >= rows) continue;
        float o[4];
        const int64_t n4 = n0 + 4 * g;
        if constexpr (MODE == kDense) {
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = n4 + q < a.N ? apply(v[q] + bias_at(a, a.bias, n4 + q), a.act, a.out_bf16) : 0.f;
            store4(a.out, a.out_bf16, a.out_vec, (first + row) * a.out_row, n4, a.N, o);
        } else if constexpr (MODE == kHidden) {
            const uint16_t* const bias = (const uint16_t*)a.bias + leaf * a.N;
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = n4 + q < a.N ? apply(v[q] + bf16_to_f32(bias[n4 + q]), a.act, true) : 0.f;
            // (the row of h is whole blocks of 32: zeros behind the leaf's width)
            store_hidden4(a.out, first + row, a.out_row, n4, o);
            if (n4 + 16 >= a.N && n4 + 16 < a.out_row) {
                const float z[4] = {0.f, 0.f, 0.f, 0.f};
                store_hidden4(a.out, first + row, a.out_row, n4 + 16, z);
            }
        } else {
            const uint16_t* const bias = (const uint16_t*)a.bias + leaf * a.N;
            const int64_t pair = a.perm[first + row];
            const float scale = a.k == 1 && a.weight ? a.weight[pair] : 1.0f;
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = n4 + q < a.N ? (v[q] + bf16_to_f32(bias[n4 + q])) * scale : 0.f;
            store4(a.out, a.out_bf16, a.out_vec, pair * a.out_row, n4, a.N, o);
        }
    }
}

// ---- tiles through LDS -------------------------------------------------------------------------------------
//
// Many rows of A: a block of four waves takes 16 MT rows of A against 128 rows of W, a wave all of these rows of A against 32 of W (so that codes
// are converted once a block).  A stage is 64 elements of K of bf16 rows (128 bytes of a row of A, 32 of W), 256 of codes (128 bytes of either): one is
// multiplied while the next is on its way straight from memory to LDS.  Three blocks (of codes two) share a compute unit, and one multiplies while another
// waits or ends.  What that is worth, in us, for 16384 x 768 x 2048 with GELU, 16384 x 2048 x 768 and 4096 x 4096 x 4096 of bf16 rows: 78, 53, 139; two blocks
// with three stages 92, 61, 141; before both, on another card, a wave on 64 x 64 results and eight waves on 256 x 256 of them, half of which read
// while the others multiply, took 116, 61, 145 and 97, 65, 138 where this shape took 106, 59, 134.
// 8192 x 4096 x 4096 of codes: 109; three stages of 128 elements (twice the barriers) 152 where this took 116.
// Scale bytes come in panels of 32 blocks (1024 elements of K) of every row, with the first stage that they belong to: a row's scales of one stage are
// a few bytes in a line of their own, so that fetching them stage by stage cost as much as the codes (8192 x 4096 x 4096, four bits both: 121 us without
// such loads, 174 with them), and a panel of the whole K before the first stage was a third of a short K's time (16384 x 768 x 2048: 87 -> 71 us).
//
// Lane (j, g) multiplies, of a stage of bf16 rows, elements 16 g + 8 u .. + 7 in step u (pieces 2 g + u of A, four bytes of codes); of a stage of codes,
// block 2 g + u.  Pieces of 16 bytes in LDS are turned within their row as tile_swz has it, so that the 16 lanes of a pass of an operand read meet every
// bank once; the turn is made by the lanes' source addresses, since a load to LDS writes lane after lane.  Rows of 32 bytes, read eight bytes a lane, need none.
__device__ const uint4 g_zero_piece = {0, 0, 0, 0};
constexpr int kPanel = 32;       // blocks whose scales come together

template <int ROW> __device__ __forceinline__ int turn(int row) { return ROW == 128 ? lds_rot(row) : 0; }
template <int ROW> __device__ __forceinline__ int lds_slot(int row, int piece) {
    constexpr int n = ROW / 16;
    return row * n + ((piece + turn<ROW>(row)) & (n - 1));
}
template <bool A4, int MT> struct TileShape {
    static constexpr int kThreads = 256, kWaves = 4, NT = 2, kRows = 16 * MT, kCols = 128;
    static constexpr int kARow = 128, kWRow = A4 ? 128 : 32;           // bytes of a row in a stage
    static constexpr int kRing = 2;                                                // stages in LDS
    static constexpr int kStageBlocks = A4 ? 8 : 2;                               // blocks of 32 in a stage
    static constexpr int kABytes = kRows * kARow, kWBytes = kCols * kWRow, kStage = kABytes + kWBytes;
    static constexpr int kALoads = kABytes / 1024 / kWaves, kWLoads = kWBytes / 1024 / kWaves;   // a wave's loads of 1 KB a stage
    static_assert(kALoads * 1024 * kWaves == kABytes && kWLoads * 1024 * kWaves == kWBytes, "whole loads a wave");
    static constexpr int kScaleRows = kCols + (A4 ? 128 : 0);      // (rows behind the last: its scales again)
    static constexpr int kPanelBytes = kScaleRows * kPanel, kPanelStages = kPanel / kStageBlocks, kPanelLoads = kPanelBytes / 1024 / kWaves, kPanelWords = kPanelBytes / 256 / kWaves;
    static constexpr int kLds = kRing * kStage + 2 * kPanelBytes;
};

// Rows of hidden activations (kOutput) are the first values of 8 MT slots and then their second ones, whose sums meet at the end: W is read and converted once for both.
template <bool A4, int MODE, bool WIDE, int MT>
__global__ __launch_bounds__(256, A4 ? 2 : 3) void mx4_tile_kernel(const Args a, const uint32_t max_row_tiles, const uint32_t col_tiles) {
    typedef TileShape<A4, MT> S;
    constexpr int NT = S::NT, kSlots = MODE == kOutput ? S::kRows / 2 : S::kRows;
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), j = lane & 15, g = lane >> 4;
    // an XCD takes a contiguous range of tiles, kGroup row tiles against all columns at a time
    constexpr uint32_t kGroup = 4;
    // (of the tiles that there are: a grid for the most that leaves can have leaves one XCD a part of its range)
    const uint32_t row_tiles = MODE == kDense ? max_row_tiles : (uint32_t)(*a.n_tiles * a.parts);
    const uint32_t share = (row_tiles * col_tiles + kXcds - 1) / kXcds, id = (blockIdx.x % kXcds) * share + blockIdx.x / kXcds;
    if (blockIdx.x / kXcds >= share || id >= row_tiles * col_tiles) return;
    const uint32_t group = id / (kGroup * col_tiles), in = id - group * kGroup * col_tiles;
    const uint32_t tall = row_tiles - kGroup * group < kGroup ? row_tiles - kGroup * group : kGroup;
    const int64_t rt = kGroup * group + in % tall, ct = in / tall;
    const int64_t n0 = ct * S::kCols;
    int64_t leaf = 0, first, rows;
    if constexpr (MODE == kDense) {
        first = rt * S::kRows;
        rows = a.T - first;
    } else {
        leaf = a.tile_leaf[rt / a.parts];
        first = a.tile_slot[rt / a.parts] + rt % a.parts * kSlots;
        rows = a.start[leaf + 1] - first;
        if (rows <= 0) return;
    }
    if (rows > kSlots) rows = kSlots;
    const auto a_index = [&](int64_t r) -> int64_t {
        if (MODE == kOutput) r &= kSlots - 1;
        r = (r < rows ? r : rows - 1) + first;
        if constexpr (MODE == kHidden) r = a.perm[r] / a.k;
        return r;
    };
    const auto w_index = [&](int64_t n) -> int64_t { return leaf * a.N + (n0 + n < a.N ? n0 + n : a.N - 1); };

    // Sources of this lane's pieces in stage 0: bytes from a base that the wave shares (from any address where WIDE says that the
    // rows of A reach further than 32 bits).
    const char* const a_base = uniform(MODE == kHidden ? a.a : a.a + first * a.a_row);
    const int64_t w_row = (int64_t)a.Kb * 16;
    const char* const w_base = uniform((const char*)a.w + (leaf * a.N + n0) * w_row);
    typedef typename std::conditional<WIDE, int64_t, uint32_t>::type Offset;
    Offset a_off[S::kALoads];
    uint32_t w_off[S::kWLoads];
    const auto a_piece = [&](int i) {
        constexpr int n = S::kARow / 16;
        return (lane - turn<S::kARow>((i * S::kWaves + wv) * (64 / n) + lane / n)) & (n - 1);
    };
    const auto w_piece = [&](int i) {
        constexpr int n = S::kWRow / 16;
        return (lane - turn<S::kWRow>((i * S::kWaves + wv) * (64 / n) + lane / n)) & (n - 1);
    };
#pragma unroll
    for (int i = 0; i < S::kALoads; ++i) {
        const int in_tile = (i * S::kWaves + wv) * (1024 / S::kARow) + lane / (S::kARow / 16);
        const int64_t r = a_index(in_tile);
        a_off[i] = (Offset)((MODE == kHidden ? r : r - first) * a.a_row + 16 * a_piece(i));
        if (MODE == kOutput && in_tile >= kSlots) a_off[i] += (Offset)(64 * a.Kb);
    }
#pragma unroll
    for (int i = 0; i < S::kWLoads; ++i) {
        const int64_t r = (i * S::kWaves + wv) * (1024 / S::kWRow) + lane / (S::kWRow / 16);
        w_off[i] = (uint32_t)((n0 + r < a.N ? r : a.N - 1 - n0) * w_row + 16 * w_piece(i));
    }

    const int stages = (a.Kb + S::kStageBlocks - 1) / S::kStageBlocks;
    const int a_pieces = A4 ? a.Kb : a.pieces;
    const int whole = a_pieces / (S::kARow / 16) < a.Kb / S::kStageBlocks ? a_pieces / (S::kARow / 16) : a.Kb / S::kStageBlocks;
    const uint32_t lds0 = lds_address(lds) + wv * 1024;
    // Scales of a panel of all rows, zeros behind a row's end (zero codes times 2^-127): straight to LDS, 16 bytes a lane where rows of scales are whole
    // aligned pieces, else four, or through registers where they are not even that.
    const uintptr_t scale_bits = (uintptr_t)a.w_scales | (A4 ? (uintptr_t)a.a_scales : 0) | (uintptr_t)a.Kb;
    const int scale_width = scale_bits % 16 == 0 ? 16 : scale_bits % 4 == 0 ? 4 : 1;
    const auto scales_of = [&](int row) { return row < S::kCols ? a.w_scales + w_index(row) * a.Kb : a.a_scales + a_index(row - S::kCols) * a.Kb; };
    const auto fetch_panel = [&](int panel) {
        const int b0 = panel * kPanel, to = S::kRing * S::kStage + (panel & 1) * S::kPanelBytes;
        if (scale_width == 16) {
#pragma unroll
            for (int i = 0; i < S::kPanelLoads; ++i)
                load_to_lds(b0 + 16 * (lane % 2) < a.Kb ? (const char*)scales_of((i * S::kWaves + wv) * 32 + lane / 2) + 16 * (lane % 2) + b0 : (const char*)&g_zero_piece,
                            __builtin_amdgcn_readfirstlane(lds_address(lds) + to + (i * S::kWaves + wv) * 1024));
            return;
        }
        if (scale_width == 4) {
#pragma unroll 1
            for (int i = 0; i < S::kPanelWords; ++i) {
                const int first = (i * S::kWaves + wv) * 64, at = first + lane, b = b0 + 4 * (at % 8);
                load_word_to_lds(b < a.Kb ? (const char*)scales_of(at / 8) + b : (const char*)&g_zero_piece,
                                 __builtin_amdgcn_readfirstlane(lds_address(lds) + to + 4 * first));
            }
            return;
        }
#pragma unroll 1
        for (int at = tid; at < S::kScaleRows * 8; at += S::kThreads) {
            const int b = b0 + 4 * (at % 8);
            const uint8_t* const src = scales_of(at / 8) + b;
            uint32_t q = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) q |= (uint32_t)(b + e < a.Kb ? src : (const uint8_t*)&g_zero_piece)[e] << (8 * e);
            *(uint32_t*)(lds + to + 4 * at) = q;
        }
    };
    const auto fetch = [&](int c, int buf) {
        if (c % S::kPanelStages == 0) fetch_panel(c / S::kPanelStages);
        const uint32_t at = __builtin_amdgcn_readfirstlane(lds0 + buf * S::kStage);
        const char* const as = a_base + (int64_t)c * S::kARow;
        const char* const ws = w_base + (int64_t)c * S::kWRow;
        if (c < whole) {
#pragma unroll
            for (int i = 0; i < S::kALoads; ++i) {
                if constexpr (WIDE) load_to_lds(as + a_off[i], at + i * S::kWaves * 1024);
                else load_to_lds_from(as, a_off[i], at + i * S::kWaves * 1024);
            }
#pragma unroll
            for (int i = 0; i < S::kWLoads; ++i) load_to_lds_from(ws, w_off[i], at + S::kABytes + i * S::kWaves * 1024);
        } else {        // the end of the rows: zeros behind it
            const char* const zero = (const char*)&g_zero_piece;
#pragma unroll
            for (int i = 0; i < S::kALoads; ++i)
                load_to_lds(c * (S::kARow / 16) + a_piece(i) < a_pieces ? as + a_off[i] : zero, at + i * S::kWaves * 1024);
#pragma unroll
            for (int i = 0; i < S::kWLoads; ++i)
                load_to_lds(c * (S::kWRow / 16) + w_piece(i) < a.Kb ? ws + w_off[i] : zero, at + S::kABytes + i * S::kWaves * 1024);
        }
    };
    f32x4_t acc[NT][MT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[n][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    constexpr int kLoads = S::kALoads + S::kWLoads, kSteps = 2;
    uint4 fa[kSteps][MT], fw[A4 ? 2 : 1][NT];        // (bf16 rows: fw[.].xy are the codes of both steps of a stage)
    uint32_t as[MT], ws[NT];      // (A4: the bytes of both steps)
    const auto read = [&](int c, int buf) {
        const uint4* const la = (const uint4*)(lds + buf * S::kStage);
        const char* const lw = lds + buf * S::kStage + S::kABytes;
        const uint8_t* const scales = (const uint8_t*)lds + S::kRing * S::kStage + (c / S::kPanelStages & 1) * S::kPanelBytes + c * S::kStageBlocks % kPanel;
        const int b = A4 ? 2 * g : g >> 1;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int row = 16 * (wv * NT + n) + j;
            if constexpr (A4) {
#pragma unroll
                for (int u = 0; u < 2; ++u) fw[u][n] = ((const uint4*)lw)[lds_slot<128>(row, 2 * g + u)];
                ws[n] = *(const uint16_t*)(scales + row * kPanel + b);
            } else {
                const uint2 v = *(const uint2*)(lw + row * 32 + 8 * g);
                fw[0][n].x = v.x;
                fw[0][n].y = v.y;
                ws[n] = scales[row * kPanel + b];
            }
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int row = 16 * m + j;
#pragma unroll
            for (int u = 0; u < kSteps; ++u) fa[u][m] = la[lds_slot<128>(row, 2 * g + u)];
            if constexpr (A4) as[m] = *(const uint16_t*)(scales + (S::kCols + row) * kPanel + b);
        }
    };
    const auto multiply = [&]() {
#pragma unroll
        for (int u = 0; u < kSteps; ++u)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if constexpr (A4) {
#pragma unroll
                    for (int m = 0; m < MT; ++m) acc[n][m] = u == 0 ? mfma4<0>(fw[u][n], ws[n], fa[u][m], as[m], acc[n][m]) : mfma4<1>(fw[u][n], ws[n], fa[u][m], as[m], acc[n][m]);
                } else {
                    const bf16x8_t f = dequantise8(u == 0 ? fw[0][n].x : fw[0][n].y, __uint_as_float(ws[n] << 23));
#pragma unroll
                    for (int m = 0; m < MT; ++m)
                        acc[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, __builtin_bit_cast(bf16x8_t, fa[u][m]), acc[n][m], 0, 0, 0);
                }
            }
    };
    const auto barrier = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll 1
    for (int c = 0; c < S::kRing && c < stages; ++c) fetch(c, c);
    if (stages >= S::kRing) wait_loads<(S::kRing - 1) * kLoads>();
    else wait_loads<0>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
    int buf = 0;
    for (int c = 0; c < stages; ++c) {
        read(c, buf);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        wait_loads<0>();               // this wave's part of stage c + 1 is there
        barrier();
        if (c + S::kRing < stages) fetch(c + S::kRing, buf);      // (everybody has read stage c)
        multiply();
        buf = buf == S::kRing - 1 ? 0 : buf + 1;
    }

    // Results through LDS, half of the wave's rows at a time, so that they leave as whole rows of 16 NT columns, eight a lane, from a loop:
    // written out for every accumulator the epilogue was more code than the instruction cache takes, and fetching it took longer than
    // the stages of a short K.
    constexpr int kLanes = 2 * NT;
    constexpr int kHalf = MT / 2, kPitch = 16 * NT + 4, kRowsAtOnce = 64 / kLanes;
    static_assert(S::kWaves * 16 * kHalf * kPitch * 4 <= S::kLds, "results fit where the stages were");
    float* const part = (float*)lds + wv * 16 * kHalf * kPitch;
    if constexpr (MODE == kOutput) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int m = 0; m < MT / 2; ++m) acc[n][m] += acc[n][m + MT / 2];
    }
    const int64_t limit = MODE == kHidden ? a.out_row : a.N;
    const int64_t n8 = n0 + 16 * NT * wv + 8 * (lane % kLanes);
    float bias[8];
#pragma unroll
    for (int q = 0; q < 8; ++q)
        bias[q] = n8 + q >= a.N ? 0.f : MODE == kDense ? bias_at(a, a.bias, n8 + q) : bf16_to_f32(((const uint16_t*)a.bias)[leaf * a.N + n8 + q]);
    __syncthreads();
    for (int half = 0; half < (MODE == kOutput ? 1 : 2); ++half) {
#pragma unroll
        for (int m = 0; m < kHalf; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) *(f32x4_t*)(part + (16 * m + j) * kPitch + 16 * n + 4 * g) = half == 0 ? acc[n][m] : acc[n][m + kHalf];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int64_t row0 = 16 * half * kHalf;
#pragma unroll 1
        for (int r = lane / kLanes; r < 16 * kHalf; r += kRowsAtOnce) {
            if (row0 + r >= rows || n8 >= limit) continue;
            int64_t to = first + row0 + r;
            float scale = 1.0f;
            if constexpr (MODE == kOutput) {
                to = a.perm[to];
                if (a.k == 1 && a.weight) scale = a.weight[to];
            }
            const float* const v = part + r * kPitch + 8 * (lane % kLanes);
            float o[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                o[q] = v[q] + bias[q];
                if constexpr (MODE == kOutput) o[q] *= scale;
                else o[q] = apply(o[q], a.act, MODE == kHidden || a.out_bf16);
                if constexpr (MODE == kHidden) o[q] = n8 + q < a.N ? o[q] : 0.f;
            }
            if constexpr (MODE == kHidden) store_hidden8(a.out, to, a.out_row, n8, o);
            else store8(a.out, a.out_bf16, a.out_vec, to * a.out_row, n8, limit, o);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

template <bool A4, int MODE, int MT> hipError_t launch_tiles(Args a, int64_t row_tiles, hipStream_t s) {
    typedef TileShape<A4, MT> S;
    const int64_t col_tiles = ((MODE == kHidden ? a.out_row : a.N) + S::kCols - 1) / S::kCols;
    const int64_t blocks = (row_tiles * a.parts * col_tiles + kXcds - 1) / kXcds * kXcds;
    a.out_vec = a.out_row % (a.out_bf16 ? 8 : 4) == 0 && ((uintptr_t)a.out & 15) == 0;
    // rows of A within 32 bits of the first that a block reaches: its own always (K <= 2^22; hidden rows 2^18 bytes), any token's not always
    const bool wide = MODE == kHidden && a.T * a.a_row >= (int64_t)1 << 32;
    note_launch("mx4_tile_kernel<%s,%d,%s>", A4 ? "mx4" : "bf16", S::kRows, MODE == kDense ? "dense" : MODE == kHidden ? "hidden" : "output");
    const auto kernel = wide ? mx4_tile_kernel<A4, MODE, MODE == kHidden, MT> : mx4_tile_kernel<A4, MODE, false, MT>;
    const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds);
    if (e != hipSuccess) return e;
    kernel<<<dim3((unsigned)blocks), S::kThreads, S::kLds, s>>>(a, (uint32_t)row_tiles, (uint32_t)col_tiles);
    return hipGetLastError();
}

// Rows of A a tile: 128 once there are enough such tiles for two a compute unit, else 64 (us with 64 / 128; K = N = 4096: 1024 bf16 rows, 256 tiles of 128,
// 45 / 50, 2048 rows 76 / 67; of codes 20 / 23, 37 / 31; 4096 bf16 rows of 768, 2048 results, 512 tiles: 21 / 22).
int tile_rows_for(int64_t rows, int64_t cols) { return ((rows + 127) / 128) * ((cols + 127) / 128) >= 2 * device_info().cus ? 128 : 64; }

template <bool A4, int MODE> hipError_t launch_tiles(Args a, int64_t row_tiles, int tile_rows, hipStream_t s) {
    a.parts = MODE == kOutput ? tile_rows / 64 : 1;
    if constexpr (MODE != kOutput) {
        if (tile_rows == 64) return launch_tiles<A4, MODE, 4>(a, row_tiles, s);
    }
    return launch_tiles<A4, MODE, 8>(a, row_tiles, s);
}

// ---- a block a token ---------------------------------------------------------------------------------------
//
// Narrow leaves: one launch, no scratch.  All hidden activations of the token's k leaves (a wave's share of D, four tiles of 16 neurons at a
// time, the waves' sums met in LDS), then all its outputs (a wave's tiles of 16, the whole sum over the pairs).  Bound by the latency of the two
// dependent reads of weights.
constexpr int kTokenWaves = 8, kTokenTiles = 4;

// Steps c0, c0 + stride, ... of one row of A (in global memory or LDS; VALUES = 2: of hidden activations) against up to NT tiles of 16 rows of W,
// whose first blocks are `first` of its matrix.
template <int VALUES, class Index, int NT>
__device__ __forceinline__ void tiles_steps(const uint8_t* w_base, const uint8_t* ws_base, const Index (&first)[NT], int tiles,
                                            const char* a_row, int Kb, int pieces, int g, int c0, int stride, f32x4_t (&acc)[NT]) {
    const int steps = (Kb + 3) / 4;
    for (int c = c0; c < steps; c += stride) {
        const int b = 4 * c + g;
        const bool in = b < Kb;
        const int bb = in ? b : Kb - 1;
        uint4 w[NT], x[VALUES][4];
        uint32_t ws[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (t >= tiles) break;
            const Index at = first[t] + bb;
            w[t] = ((const uint4*)w_base)[at];
            ws[t] = ws_base[at];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const bool there = in && 4 * bb + u < pieces;
#pragma unroll
            for (int v = 0; v < VALUES; ++v) x[v][u] = keep_if(there, *(const uint4*)(a_row + 64 * (int64_t)Kb * v + 16 * (int64_t)(there ? 4 * bb + u : 0)));
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (t >= tiles) break;
            w[t] = keep_if(in, w[t]);
            ws[t] = in ? ws[t] << 23 : 0u;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (t >= tiles) break;
                const bf16x8_t f = dequantise8(u == 0 ? w[t].x : u == 1 ? w[t].y : u == 2 ? w[t].z : w[t].w, __uint_as_float(ws[t]));
#pragma unroll
                for (int v = 0; v < VALUES; ++v) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, __builtin_bit_cast(bf16x8_t, x[v][u]), acc[t], 0, 0, 0);
            }
    }
}

__global__ __launch_bounds__(64 * kTokenWaves) void mx4_token_kernel(const Args a, const Args b) {
    extern __shared__ __align__(16) uint16_t h[];          // [k][two values][h_row]
    __shared__ float part[2][kTokenWaves][16 * kTokenTiles];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, j = lane & 15, g = lane >> 4;
    const int64_t t = blockIdx.x;
    const int h_row = (int)a.out_row, h_tiles = h_row / 16;
    int round = 0;
    for (int i = 0; i < a.k; ++i) {
        const uint32_t e = (uint32_t)__builtin_amdgcn_readfirstlane(a.idx[t * a.k + i]);
        if (e >= a.E) continue;                            // (not read below)
        const int64_t row0 = (int64_t)e * a.N;
        for (int t0 = 0; t0 < h_tiles; t0 += kTokenTiles, round ^= 1) {
            uint32_t first[kTokenTiles];                   // (leaves of few bytes)
            f32x4_t acc[kTokenTiles];
#pragma unroll
            for (int u = 0; u < kTokenTiles; ++u) {
                const int n = 16 * (t0 + u) + j;
                first[u] = (uint32_t)((n < a.N ? n : (int)a.N - 1) * a.Kb);
                acc[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
            tiles_steps<1>(a.w + row0 * a.Kb * 16, a.w_scales + row0 * a.Kb, first, h_tiles - t0 < kTokenTiles ? h_tiles - t0 : kTokenTiles, a.a + t * a.a_row, a.Kb, a.pieces, g, wv, kTokenWaves, acc);
            if (j == 0) {
#pragma unroll
                for (int u = 0; u < kTokenTiles; ++u) *(f32x4_t*)&part[round][wv][16 * u + 4 * g] = acc[u];
            }
            __syncthreads();
            const int n = 16 * t0 + tid;
            if (tid < 16 * kTokenTiles && n < h_row) {
                float v = part[round][0][tid];
#pragma unroll
                for (int w = 1; w < kTokenWaves; ++w) v += part[round][w][tid];
                v = n < a.N ? apply(v + bf16_to_f32(((const uint16_t*)a.bias)[(int64_t)e * a.N + n]), a.act, true) : 0.f;
                h[2 * i * h_row + n] = (uint16_t)(__float_as_uint(v) >> 16);
                h[(2 * i + 1) * h_row + n] = f32_to_bf16(second_value(v));
            }
        }
    }
    __syncthreads();
    const int64_t o_tiles = (b.N + 15) / 16;
    for (int64_t t0 = (int64_t)wv * kTokenTiles; t0 < o_tiles; t0 += kTokenWaves * kTokenTiles) {
        const int tiles = o_tiles - t0 < kTokenTiles ? (int)(o_tiles - t0) : kTokenTiles;
        f32x4_t sum[kTokenTiles];
#pragma unroll
        for (int u = 0; u < kTokenTiles; ++u) sum[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < b.k; ++i) {
            const uint32_t e = (uint32_t)__builtin_amdgcn_readfirstlane(b.idx[t * b.k + i]);
            if (e >= b.E) continue;
            const int64_t row0 = (int64_t)e * b.N;
            const float scale = b.weight ? b.weight[t * b.k + i] : 1.0f;
            uint32_t first[kTokenTiles];
            f32x4_t acc[kTokenTiles];
#pragma unroll
            for (int u = 0; u < kTokenTiles; ++u) {
                const int n = 16 * ((int)t0 + u) + j;
                first[u] = (uint32_t)((n < b.N ? n : (int)b.N - 1) * b.Kb);
                acc[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
            tiles_steps<2>(b.w + row0 * b.Kb * 16, b.w_scales + row0 * b.Kb, first, tiles, (const char*)(h + 2 * i * h_row), b.Kb, b.pieces, g, 0, 1, acc);
            if (j == 0) {
#pragma unroll
                for (int u = 0; u < kTokenTiles; ++u)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int64_t n = 16 * (t0 + u) + 4 * g + q;
                        if (n < b.N) sum[u][q] = fmaf(scale, acc[u][q] + bf16_to_f32(((const uint16_t*)b.bias)[(int64_t)e * b.N + n]), sum[u][q]);
                    }
            }
        }
        if (j == 0) {
#pragma unroll
            for (int u = 0; u < kTokenTiles; ++u) {
                const float o[4] = {sum[u][0], sum[u][1], sum[u][2], sum[u][3]};
                store4(b.out, true, b.out_vec, t * b.out_row, 16 * (t0 + u) + 4 * g, b.N, o);
            }
        }
    }
}

// ---- few pairs of wide leaves ------------------------------------------------------------------------------
//
// Nothing to group: a block takes 16 NT columns of one pair's hidden activations (HIDDEN; h [pair]) or of one token's
// outputs (its pairs one after another, each wave's part times the pair's weight), K shared out among its waves.  Bound by the bytes of the weights.
template <bool HIDDEN, int NT>
__global__ __launch_bounds__(64 * kTokenWaves, 4) void mx4_direct_kernel(const Args a) {
    __shared__ float part[kTokenWaves][16 * NT];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, j = lane & 15, g = lane >> 4;
    const int64_t width = HIDDEN ? a.out_row : a.N, n_blocks = (width + 16 * NT - 1) / (16 * NT);
    const int64_t item = blockIdx.x / n_blocks, n0 = (blockIdx.x - item * n_blocks) * (16 * NT);
    const int k = HIDDEN ? 1 : a.k, steps = (a.Kb + 3) / 4;
    if (HIDDEN && (uint32_t)a.idx[item] >= a.E) return;            // (nobody reads its row)
    const int tiles = width - n0 < 16 * NT ? (int)((width - n0 + 15) / 16) : NT;
    f32x4_t sum[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) sum[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < k; ++i) {
        const int64_t pair = item * k + i;
        const uint32_t e = (uint32_t)__builtin_amdgcn_readfirstlane(a.idx[pair]);
        if (e >= a.E) continue;
        const int64_t row0 = (int64_t)e * a.N;
        int64_t first[NT];
        f32x4_t acc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int64_t n = n0 + 16 * t + j;
            first[t] = (n < a.N ? n : a.N - 1) * a.Kb;
            acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        // (step c of pair i is step i * steps + c of the sum: waves that pair i leaves without a step begin with pair i + 1)
        tiles_steps<HIDDEN ? 1 : 2>(a.w + row0 * a.Kb * 16, a.w_scales + row0 * a.Kb, first, tiles, a.a + (HIDDEN ? pair / a.k : pair) * a.a_row, a.Kb, a.pieces, g,
                        (wv + kTokenWaves - i * steps % kTokenWaves) % kTokenWaves, kTokenWaves, acc);
        const float scale = !HIDDEN && a.weight ? a.weight[pair] : 1.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int q = 0; q < 4; ++q) sum[t][q] = fmaf(scale, acc[t][q], sum[t][q]);
    }
    if (j == 0) {
#pragma unroll
        for (int t = 0; t < NT; ++t) *(f32x4_t*)&part[wv][16 * t + 4 * g] = sum[t];
    }
    __syncthreads();
    const int64_t n = n0 + tid;
    if (tid >= 16 * NT || n >= width) return;
    float v = part[0][tid];
#pragma unroll
    for (int w = 1; w < kTokenWaves; ++w) v += part[w][tid];
    for (int i = 0; i < k; ++i) {
        const int64_t pair = item * k + i;
        const uint32_t e = (uint32_t)a.idx[pair];
        if (e >= a.E || n >= a.N) continue;
        const float scale = a.weight ? a.weight[pair] : 1.0f, bias = bf16_to_f32(((const uint16_t*)a.bias)[(int64_t)e * a.N + n]);
        v = HIDDEN ? apply(v + bias, a.act, true) : fmaf(scale, bias, v);
    }
    if (HIDDEN && n >= a.N) v = 0.f;
    uint16_t* const out = (uint16_t*)a.out + item * (HIDDEN ? 2 : 1) * a.out_row + n;
    if constexpr (HIDDEN) {
        out[0] = (uint16_t)(__float_as_uint(v) >> 16);
        out[a.out_row] = f32_to_bf16(second_value(v));
    } else {
        out[0] = f32_to_bf16(v);
    }
}

// Columns a block: 64 where that leaves a block for every compute unit.
template <bool HIDDEN> hipError_t launch_direct(const Args& a, int64_t items, hipStream_t s) {
    const int64_t width = HIDDEN ? a.out_row : a.N;
    const auto blocks = [&](int nt) { return (width + 16 * nt - 1) / (16 * nt) * items; };
    const int nt = blocks(4) >= device_info().cus ? 4 : blocks(2) >= device_info().cus ? 2 : 1;
    note_launch("mx4_direct_kernel<%s,%d>", HIDDEN ? "hidden" : "output", nt);
    const dim3 grid((unsigned)blocks(nt));
    if (nt == 4) mx4_direct_kernel<HIDDEN, 4><<<grid, 64 * kTokenWaves, 0, s>>>(a);
    else if (nt == 2) mx4_direct_kernel<HIDDEN, 2><<<grid, 64 * kTokenWaves, 0, s>>>(a);
    else mx4_direct_kernel<HIDDEN, 1><<<grid, 64 * kTokenWaves, 0, s>>>(a);
    return hipGetLastError();
}

// ---- grouping of the pairs by leaf -------------------------------------------------------------------------
//
// rank[p] = place of pair p among its leaf's; which pair gets which place depends on the order of the atomics, and
// nothing else does: a row's sums do not know its place in a tile.
constexpr int kGroupPairs = 1024;         // pairs of a block
constexpr int kGroupLdsLeaves = 8192;     // leaves whose counts fit LDS

// Counts of a block's pairs meet in LDS first (LDS: E <= kGroupLdsLeaves): 16384 pairs on 16 leaves, all by atomics on memory, took 46 us.
template <bool LDS>
__global__ __launch_bounds__(256) void group_count_kernel(const int32_t* __restrict__ idx, int64_t P, int E, int32_t* __restrict__ count,
                                                          int32_t* __restrict__ rank) {
    extern __shared__ int32_t own[];
    const int64_t p0 = (int64_t)blockIdx.x * kGroupPairs + threadIdx.x;
    if (!LDS) {
#pragma unroll
        for (int i = 0; i < kGroupPairs / 256; ++i) {
            const int64_t p = p0 + 256 * i;
            const uint32_t e = p < P ? (uint32_t)idx[p] : ~0u;
            if (e < (uint32_t)E) rank[p] = atomicAdd(count + e, 1);
        }
        return;
    }
    for (int e = threadIdx.x; e < E; e += 256) own[e] = 0;
    __syncthreads();
    uint32_t e[kGroupPairs / 256];
    int32_t r[kGroupPairs / 256];
#pragma unroll
    for (int i = 0; i < kGroupPairs / 256; ++i) {
        e[i] = p0 + 256 * i < P ? (uint32_t)idx[p0 + 256 * i] : ~0u;
        if (e[i] < (uint32_t)E) r[i] = atomicAdd(own + e[i], 1);
    }
    __syncthreads();
    for (int l = threadIdx.x; l < E; l += 256)
        if (own[l]) own[l] = atomicAdd(count + l, own[l]);      // from here on the places before the block's
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kGroupPairs / 256; ++i)
        if (e[i] < (uint32_t)E) rank[p0 + 256 * i] = own[e[i]] + r[i];
}

// exclusive sums over a block of 1024 threads
__device__ __forceinline__ void block_scan(int32_t& x, int32_t& y, int32_t (&sums)[2][16]) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int32_t x0 = x, y0 = y;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t u = __shfl_up(x, d, 64), v = __shfl_up(y, d, 64);
        x += lane >= d ? u : 0;
        y += lane >= d ? v : 0;
    }
    if (lane == 63) {
        sums[0][wv] = x;
        sums[1][wv] = y;
    }
    __syncthreads();
    x -= x0;
    y -= y0;
    for (int w = 0; w < wv; ++w) {
        x += sums[0][w];
        y += sums[1][w];
    }
}

// start[E + 1], tile_start[E + 1]: exclusive sums of the counts and of the tiles of `tile_rows` slots
__device__ __forceinline__ void scan_leaves(const int32_t* count, int64_t E, int tile_rows, int32_t* start, int32_t* tile_start, int32_t (&sums)[2][16]) {
    const int tid = threadIdx.x;
    const int64_t per = (E + 1023) / 1024, e0 = tid * per < E ? tid * per : E, e1 = e0 + per < E ? e0 + per : E;
    int32_t c = 0, t = 0;
    for (int64_t e = e0; e < e1; ++e) {
        c += count[e];
        t += (count[e] + tile_rows - 1) / tile_rows;
    }
    block_scan(c, t, sums);
    for (int64_t e = e0; e < e1; ++e) {
        const int32_t n = count[e];
        start[e] = c;
        tile_start[e] = t;
        c += n;
        t += (n + tile_rows - 1) / tile_rows;
    }
    if (e0 < E && e1 == E) {
        start[E] = c;
        tile_start[E] = t;
    }
}

__global__ __launch_bounds__(1024) void group_scan_kernel(const int32_t* __restrict__ count, int64_t E, int tile_rows, int32_t* __restrict__ start,
                                                          int32_t* __restrict__ tile_start) {
    __shared__ int32_t sums[2][16];
    scan_leaves(count, E, tile_rows, start, tile_start, sums);
}

__device__ __forceinline__ void place(int64_t p, uint32_t e, int32_t r, int tile_rows, const int32_t* start, const int32_t* tile_start,
                                      int32_t* __restrict__ perm, int32_t* __restrict__ tile_leaf, int32_t* __restrict__ tile_slot) {
    const int32_t slot = start[e] + r;
    perm[slot] = (int32_t)p;
    if (r % tile_rows == 0) {
        const int32_t tile = tile_start[e] + r / tile_rows;
        tile_leaf[tile] = (int32_t)e;
        tile_slot[tile] = slot;
    }
}

__global__ __launch_bounds__(256) void group_place_kernel(const int32_t* __restrict__ idx, int64_t P, int64_t E, int tile_rows,
                                                          const int32_t* __restrict__ rank, const int32_t* __restrict__ start,
                                                          const int32_t* __restrict__ tile_start, int32_t* __restrict__ perm,
                                                          int32_t* __restrict__ tile_leaf, int32_t* __restrict__ tile_slot) {
    const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (p >= P) return;
    const uint32_t e = (uint32_t)idx[p];
    if (e < E) place(p, e, rank[p], tile_rows, start, tile_start, perm, tile_leaf, tile_slot);
}

// Two launches while all blocks' counts are few: each block's own, then every block adds up those before it, scans the leaves and places its pairs.
// A leaf's counts are a thread's, so the work is quadratic in the blocks (pairs of 1, 4 and 16 leaves, whole forward, two launches / four: 65536 24.2 / 25.6 us,
// 27.2 / 28.2, 28.4 / 29.9; 131072 37.1 / 37.9, 46.1 / 45.1, 47.2 / 46.9; 262144 71.8 / 70.5, 80.8 / 76.3, 80.0 / 76.7; of one leaf 8 million 5357 / 2733).
constexpr int64_t kGroupWords = 8192, kGroupTwoLeaves = 4000, kGroupTwoBlocks = 128;     // counts of all blocks; leaves whose four tables fit 64 KB of LDS
__global__ __launch_bounds__(1024) void group_hist_kernel(const int32_t* __restrict__ idx, int64_t P, int E, int32_t* __restrict__ counts) {
    extern __shared__ int32_t own[];
    for (int e = threadIdx.x; e < E; e += 1024) own[e] = 0;
    __syncthreads();
    const int64_t p = (int64_t)blockIdx.x * kGroupPairs + threadIdx.x;
    const uint32_t e = p < P ? (uint32_t)idx[p] : ~0u;
    if (e < (uint32_t)E) atomicAdd(own + e, 1);
    __syncthreads();
    for (int l = threadIdx.x; l < E; l += 1024) counts[(int64_t)blockIdx.x * E + l] = own[l];
}

__global__ __launch_bounds__(1024) void group_spread_kernel(const int32_t* __restrict__ idx, int64_t P, int E, int tile_rows,
                                                            const int32_t* __restrict__ counts, int32_t* __restrict__ start,
                                                            int32_t* __restrict__ tile_start, int32_t* __restrict__ perm,
                                                            int32_t* __restrict__ tile_leaf, int32_t* __restrict__ tile_slot) {
    extern __shared__ int32_t own[];          // places before this block's [E], all [E], start [E + 1], tile_start [E + 1]
    __shared__ int32_t sums[2][16];
    int32_t *const all = own + E, *const lds_start = all + E, *const lds_tiles = lds_start + E + 1;
    for (int e = threadIdx.x; e < E; e += 1024) {
        int32_t before = 0, total = 0;
#pragma unroll 8
        for (int b = 0; b < (int)gridDim.x; ++b) {
            const int32_t n = counts[(int64_t)b * E + e];
            before += b < (int)blockIdx.x ? n : 0;
            total += n;
        }
        own[e] = before;
        all[e] = total;
    }
    __syncthreads();
    scan_leaves(all, E, tile_rows, lds_start, lds_tiles, sums);
    __syncthreads();
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= E; e += 1024) {
            start[e] = lds_start[e];
            tile_start[e] = lds_tiles[e];
        }
    const int64_t p = (int64_t)blockIdx.x * kGroupPairs + threadIdx.x;
    const uint32_t e = p < P ? (uint32_t)idx[p] : ~0u;
    if (e < (uint32_t)E) place(p, e, atomicAdd(own + e, 1), tile_rows, lds_start, lds_tiles, perm, tile_leaf, tile_slot);
}

// All of it in one block, for few pairs: counts, sums and places in LDS (a second pass of atomics gives the places).
constexpr int64_t kGroupOnePairs = 4096, kGroupOneLeaves = 4096;
__global__ __launch_bounds__(1024) void group_one_kernel(const int32_t* __restrict__ idx, int P, int E, int tile_rows, int32_t* __restrict__ start,
                                                         int32_t* __restrict__ tile_start, int32_t* __restrict__ perm, int32_t* __restrict__ tile_leaf,
                                                         int32_t* __restrict__ tile_slot) {
    extern __shared__ int32_t counts[];      // counts [E], start [E + 1], tile_start [E + 1]
    __shared__ int32_t sums[2][16];
    int32_t *const lds_start = counts + E, *const lds_tiles = lds_start + E + 1;
    for (int e = threadIdx.x; e < E; e += 1024) counts[e] = 0;
    __syncthreads();
    for (int p = threadIdx.x; p < P; p += 1024) {
        const uint32_t e = (uint32_t)idx[p];
        if (e < (uint32_t)E) atomicAdd(counts + e, 1);
    }
    __syncthreads();
    scan_leaves(counts, E, tile_rows, lds_start, lds_tiles, sums);
    __syncthreads();
    for (int e = threadIdx.x; e <= E; e += 1024) {
        start[e] = lds_start[e];
        tile_start[e] = lds_tiles[e];
        if (e < E) counts[e] = 0;
    }
    __syncthreads();
    for (int p = threadIdx.x; p < P; p += 1024) {
        const uint32_t e = (uint32_t)idx[p];
        if (e < (uint32_t)E) place(p, e, atomicAdd(counts + e, 1), tile_rows, lds_start, lds_tiles, perm, tile_leaf, tile_slot);
    }
}

// out[t] = sum over the token's pairs of weight * y[pair], in the order of the pairs, V columns a thread
template <int V>
__global__ __launch_bounds__(256) void combine_kernel(const int32_t* __restrict__ idx, const float* __restrict__ weight, const float* __restrict__ y,
                                                      uint16_t* __restrict__ out, int64_t T, int64_t O, int64_t E, int k) {
    const int64_t cols = O / V, id = (int64_t)blockIdx.x * 256 + threadIdx.x, t = id / cols, o = (id - t * cols) * V;
    if (t >= T) return;
    float v[V];
#pragma unroll
    for (int q = 0; q < V; ++q) v[q] = 0;
#pragma unroll 4
    for (int i = 0; i < k; ++i) {
        const bool there = (uint32_t)idx[t * k + i] < E;
        const float g = weight ? weight[t * k + i] : 1.0f;
        float f[V];
        if constexpr (V == 8) {
            const float* const row = y + (t * k + i) * O + o;
            widen<false>(*(const uint4*)row, f);
            widen<false>(*(const uint4*)(row + 4), f + 4);
        } else {
            f[0] = y[(t * k + i) * O + o];
        }
#pragma unroll
        for (int q = 0; q < V; ++q) v[q] = there ? fmaf(g, f[q], v[q]) : v[q];
    }
    if constexpr (V == 8) *(uint4*)(out + t * O + o) = narrow<true>(v);
    else out[t * O + o] = f32_to_bf16(v[0]);
}

// k = 1: the rows of tokens without a leaf
__global__ __launch_bounds__(256) void clear_kernel(const int32_t* __restrict__ idx, uint16_t* __restrict__ out, int64_t T, int64_t O, int64_t E) {
    for (int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); t < T; t += (int64_t)gridDim.x * 4) {
        if ((uint32_t)idx[t] < E) continue;
        for (int64_t o = threadIdx.x & 63; o < O; o += 64) out[t * O + o] = 0;
    }
}

template <bool A4, int MODE> hipError_t launch_rows(Args a, int64_t tiles, int mt, hipStream_t s) {
    a.parts = MODE == kOutput && mt == 4 ? 2 : 1;          // (rows of two values: half as many at a time)
    mt /= a.parts;
    const int64_t blocks = (a.N + 15) / 16 * tiles * a.parts;
    note_launch("mx4_rows_kernel<%s,%d,%s>", A4 ? "mx4" : "bf16", mt,
                MODE == kDense ? "dense" : MODE == kHidden ? "hidden" : "output");
    const dim3 grid((unsigned)blocks);
    if constexpr (MODE != kOutput) {
        if (mt == 4) {
            mx4_rows_kernel<A4, 4, MODE, 4><<<grid, 256, 0, s>>>(a);
            return hipGetLastError();
        }
    }
    if (mt == 1) mx4_rows_kernel<A4, 1, MODE, 8><<<grid, 512, 0, s>>>(a);
    else mx4_rows_kernel<A4, 2, MODE, 8><<<grid, 512, 0, s>>>(a);
    return hipGetLastError();
}

// Times in us of a product by mx4_rows_kernel and by mx4_tile_kernel, fitted to both over 16 .. 256 rows, 4096 x 4096 and 1024 x 768 matrices (bf16 rows and
// codes; within about 10 %): the one grows with its rows from a launch's time on, the other is a chain of stages along K until its tiles fill the
// chip more than once.  (4096 x 4096, bf16 rows: 96 of them 31 / 31 us, 128 36 / 31; codes: 64 11.7 / 13.8, 96 17.6 / 13.6; 768 x 2048, bf16 rows: 256
// 9.0 / 10.4, 512 15.4 / 10.7; codes: 256 5.5 / 7.8, 1024 12.8 / 8.5.)
double rows_us(bool a4, double rows, int64_t N, int64_t K) { return 4.2 + rows * (double)N * (double)K * (a4 ? 7.9e-9 : 1.55e-8); }
// Hidden activations (`two_values`) count as two rows, and a block's stages are those of 128 rows from the first tile on (up to 4096 pairs, four shapes
// with 4, 16 and 64 leaves: 0.01 us an element of K; with it the faster of both launches is chosen, or one less than a seventh behind it).
double tiles_us(bool a4, double rows64, int64_t N, int64_t K, bool two_values = false) {
    const double tiles = (two_values ? 2 : 1) * rows64 * (double)((N + 127) / 128) / 512, few = two_values ? 1.7 : 1;
    return (a4 ? 6 : 7) + (double)K * (a4 ? 0.0019 : 0.0059) * (tiles > few ? tiles : few);
}

// Rows of A a block of mx4_rows_kernel takes, in tiles of 16: the most that leave blocks for three quarters of the compute units (1024 x 768, bf16 rows, one, two
// and four tiles: 64 rows 4.4, 4.9, 6.6 us; 128 5.9, 5.0, 6.6; 256 8.2, 7.2, 6.7).
int rows_tile(int64_t rows, int64_t N) {
    const auto fills = [&](int mt) { return (rows + 16 * mt - 1) / (16 * mt) * ((N + 15) / 16) >= kSmallEnoughBlocks; };
    return rows > 32 && fills(4) ? 4 : rows > 16 && fills(2) ? 2 : 1;
}

// whether a launch of mx4_rows_kernel, 512 threads a block, takes so many tiles of rows
bool rows_fit(int64_t tiles, int64_t N) { return tiles * ((N + 15) / 16) < kMaxMx4Blocks / 2; }

int64_t align256(int64_t bytes) { return (bytes + 255) / 256 * 256; }

struct LeafScratch {
    int64_t count, start, tile_start, rank, perm, tile_leaf, tile_slot, h, y, total;
    LeafScratch(int64_t P, int64_t O, int64_t E, int k, int L) {
        int64_t o = 0;
        const auto take = [&](int64_t bytes) {
            const int64_t at = o;
            o += align256(bytes);
            return at;
        };
        const int64_t tiles = P / 16 + (E < P ? E : P) + 1;
        count = take(4 * (E > kGroupWords ? E : kGroupWords));
        start = take(4 * (E + 1));
        tile_start = take(4 * (E + 1));
        rank = take(4 * P);
        perm = take(4 * P);
        tile_leaf = take(4 * tiles);
        tile_slot = take(4 * tiles);
        h = take(4 * P * kMxBlock * mx_blocks(L));
        y = take(k > 1 ? 4 * P * O : 0);
        total = o;
    }
};

}  // namespace

hipError_t launch_mx4_product(const Mx4Product& p, hipStream_t s) {
    Args a{};
    const bool a4 = p.a_scales != nullptr;
    a.a = (const char*)p.a;
    a.a_scales = p.a_scales;
    a.a_row = a4 ? 16 * mx_blocks(p.K) : 2 * p.lda;
    a.w = p.w;
    a.w_scales = p.w_scales;
    a.bias = p.bias;
    a.out = (char*)p.out;
    a.T = p.T;
    a.N = p.N;
    a.out_row = p.N;
    a.Kb = (int)mx_blocks(p.K);
    a.pieces = (int)(p.lda / 8);
    a.act = p.act;
    a.out_bf16 = p.out_bf16;
    a.out_vec = p.N % 4 == 0 && ((uintptr_t)p.out & (p.out_bf16 ? 7 : 15)) == 0;
    const int mt = rows_tile(p.T, p.N);
    if (tiles_us(a4, (double)((p.T + 63) / 64), p.N, p.K) < rows_us(a4, (double)p.T, p.N, p.K) || !rows_fit((p.T + 16 * mt - 1) / (16 * mt), p.N)) {
        const int tile_rows = tile_rows_for(p.T, p.N);
        const int64_t tiles = (p.T + tile_rows - 1) / tile_rows;
        return a4 ? launch_tiles<true, kDense>(a, tiles, tile_rows, s) : launch_tiles<false, kDense>(a, tiles, tile_rows, s);
    }
    const int64_t tiles = (p.T + 16 * mt - 1) / (16 * mt);
    return a4 ? launch_rows<true, kDense>(a, tiles, mt, s) : launch_rows<false, kDense>(a, tiles, mt, s);
}

int64_t mx4_leaves_scratch_bytes(int64_t T, int64_t O, int64_t E, int k, int L) { return LeafScratch(T * k, O, E, k, L).total; }

hipError_t launch_mx4_leaves(const Mx4Leaves& p, void* scratch, hipStream_t s) {
    const int64_t P = p.T * p.k;
    const LeafScratch at(P, p.O, p.E, p.k, p.L);
    char* const base = (char*)scratch;
    const auto words = [&](int64_t o) { return (int32_t*)(base + o); };
    uint16_t* const h = (uint16_t*)(base + at.h);
    const int64_t h_row = kMxBlock * mx_blocks(p.L);
    Args a{};
    a.a = (const char*)p.x;
    a.a_row = 2 * p.ldx;
    a.w = p.w1;
    a.w_scales = p.s1;
    a.bias = p.b1;
    a.out = (char*)h;
    a.T = p.T;
    a.N = p.L;
    a.out_row = h_row;
    a.Kb = (int)mx_blocks(p.D);
    a.pieces = (int)(p.ldx / 8);
    a.act = p.act;
    a.out_bf16 = true;
    a.idx = p.idx;
    a.weight = p.weight;
    a.E = p.E;
    a.k = p.k;
    Args b = a;
    b.a = (const char*)h;
    b.a_row = 4 * h_row;
    b.w = p.w2;
    b.w_scales = p.s2;
    b.bias = p.b2;
    b.out = (char*)p.out;
    b.N = p.O;
    b.out_row = p.O;
    b.Kb = (int)mx_blocks(p.L);
    b.pieces = (int)(h_row / 8);
    b.out_vec = p.O % 4 == 0 && ((uintptr_t)p.out & 7) == 0;
    hipError_t e;
    // Few pairs, or few of them a leaf: grouping gains nothing.  Leaves of few bytes go a block a token (one launch); others are spread over the chip.
    const int64_t leaf_bytes = (int64_t)p.L * 16 * a.Kb + p.O * 16 * b.Kb, h_bytes = 4 * h_row * p.k;
    if ((P <= 32 || P <= 4 * p.E) && p.k * leaf_bytes <= 256 * 1024 && h_bytes <= 64 * 1024) {
        note_launch("mx4_token_kernel");
        if (h_bytes > 56 * 1024 && (e = hipFuncSetAttribute((const void*)mx4_token_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)h_bytes)) != hipSuccess) return e;
        mx4_token_kernel<<<dim3((unsigned)p.T), 64 * kTokenWaves, (size_t)h_bytes, s>>>(a, b);
        return hipGetLastError();
    }
    if (P <= 32) {
        if ((e = launch_direct<true>(a, P, s)) != hipSuccess) return e;
        return launch_direct<false>(b, p.T, s);
    }
    const int64_t met = p.E < P ? p.E : P;
    const int mt = P / p.E <= 16 ? 1 : P / p.E <= 32 ? 2 : 4;
    const double rows = 16.0 * mt * (double)(P / (16 * mt) + met), rows64 = (double)(P / 64 + met);
    const bool large = tiles_us(false, rows64, p.L, p.D) + tiles_us(false, rows64, p.O, p.L, true) < rows_us(false, rows, p.L, p.D) + rows_us(false, 2 * rows, p.O, p.L) ||
                       !rows_fit(2 * (P / (16 * mt) + met), p.L > p.O ? p.L : p.O);
    int tile_rows = large ? tile_rows_for(P, p.L < p.O ? p.L : p.O) : 16 * mt;
    if (tile_rows == 128 && 2 * (P / 128 + met) * ((p.O + 127) / 128) > kMaxMx4Tiles) tile_rows = 64;       // (blocks of the second product)
    const int64_t tiles = P / tile_rows + met;
    int32_t *const count = words(at.count), *const start = words(at.start), *const tile_start = words(at.tile_start);
    int32_t *const rank = words(at.rank), *const perm = words(at.perm), *const tile_leaf = words(at.tile_leaf), *const tile_slot = words(at.tile_slot);
    if (P <= kGroupOnePairs && p.E <= kGroupOneLeaves) {
        note_launch("group_one_kernel");
        group_one_kernel<<<1, 1024, (size_t)(3 * p.E + 2) * 4, s>>>(p.idx, (int)P, (int)p.E, tile_rows, start, tile_start, perm, tile_leaf, tile_slot);
    } else if (p.E <= kGroupTwoLeaves && P <= kGroupTwoBlocks * kGroupPairs && (P + kGroupPairs - 1) / kGroupPairs * p.E <= kGroupWords) {
        const dim3 blocks((unsigned)((P + kGroupPairs - 1) / kGroupPairs));
        note_launch("group_hist_kernel");
        group_hist_kernel<<<blocks, 1024, (size_t)p.E * 4, s>>>(p.idx, P, (int)p.E, count);
        note_launch("group_spread_kernel");
        group_spread_kernel<<<blocks, 1024, (size_t)(4 * p.E + 2) * 4, s>>>(p.idx, P, (int)p.E, tile_rows, count, start, tile_start, perm, tile_leaf,
                                                                             tile_slot);
    } else {
        if ((e = launch_zero(count, (p.E + 3) / 4 * 4, s)) != hipSuccess) return e;   // (whole pieces: the region is of 256 bytes)
        note_launch("group kernels");
        const dim3 blocks((unsigned)((P + kGroupPairs - 1) / kGroupPairs));
        if (p.E <= kGroupLdsLeaves) group_count_kernel<true><<<blocks, 256, (size_t)p.E * 4, s>>>(p.idx, P, (int)p.E, count, rank);
        else group_count_kernel<false><<<blocks, 256, 0, s>>>(p.idx, P, (int)p.E, count, rank);
        group_scan_kernel<<<1, 1024, 0, s>>>(count, p.E, tile_rows, start, tile_start);
        group_place_kernel<<<dim3((unsigned)((P + 255) / 256)), 256, 0, s>>>(p.idx, P, p.E, tile_rows, rank, start, tile_start, perm, tile_leaf, tile_slot);
    }
    if ((e = hipGetLastError()) != hipSuccess) return e;
    a.perm = b.perm = perm;
    a.tile_leaf = b.tile_leaf = tile_leaf;
    a.tile_slot = b.tile_slot = tile_slot;
    a.start = b.start = start;
    a.n_tiles = b.n_tiles = tile_start + p.E;
    float* const y = p.k > 1 ? (float*)(base + at.y) : nullptr;
    if (y) {
        b.out = (char*)y;
        b.out_bf16 = false;
        b.out_vec = p.O % 4 == 0;
    }
    if (large) {
        if ((e = launch_tiles<false, kHidden>(a, tiles, tile_rows, s)) != hipSuccess) return e;
        if ((e = launch_tiles<false, kOutput>(b, tiles, tile_rows, s)) != hipSuccess) return e;
    } else {
        if ((e = launch_rows<false, kHidden>(a, tiles, mt, s)) != hipSuccess) return e;
        if ((e = launch_rows<false, kOutput>(b, tiles, mt, s)) != hipSuccess) return e;
    }
    if (!y) {
        note_launch("clear_kernel");
        clear_kernel<<<dim3((unsigned)(p.T < 4096 ? (p.T + 3) / 4 : 1024)), 256, 0, s>>>(p.idx, p.out, p.T, p.O, p.E);
        return hipGetLastError();
    }
    const int v = p.O % 8 == 0 && ((uintptr_t)p.out & 15) == 0 ? 8 : 1;
    note_launch("combine_kernel<%d>", v);
    const int64_t most = ((kMaxMx4Blocks - 1) * 256) / (p.O / v);       // tokens of a launch
    for (int64_t t = 0; t < p.T; t += most) {
        const int64_t n = p.T - t < most ? p.T - t : most;
        const dim3 grid((unsigned)((n * (p.O / v) + 255) / 256));
        const int32_t* const idx = p.idx + t * p.k;
        const float *const weight = p.weight ? p.weight + t * p.k : nullptr, *const from = y + t * p.k * p.O;
        if (v == 8) combine_kernel<8><<<grid, 256, 0, s>>>(idx, weight, from, p.out + t * p.O, n, p.O, p.E, p.k);
        else combine_kernel<1><<<grid, 256, 0, s>>>(idx, weight, from, p.out + t * p.O, n, p.O, p.E, p.k);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace fff

// Products with four-bit matrices: out = act(A W^T + b), and leaf networks of k leaves per token.
//
// W is [N, K] in blocks of 32 along K.  The operand of a matrix instruction is a row of W per lane: lane (j, g) of a wave
// (j = lane mod 16, g = lane / 16) takes block 4 c + g of row j in step c, 16 bytes of codes and one scale byte, so a step covers
// 128 elements of K and every load is a whole block.  K is only an order of summation, so the rows of A are read the same way.
//   A in bf16: the lane's 32 codes become four operands of v_mfma_f32_16x16x32_bf16 (eight elements of K per lane each): the
//     conversion instruction multiplies by the scale, and code times scale is exact in bf16.
//   A in four bits: the 16 bytes are the operand of v_mfma_scale_f32_16x16x128_f8f6f4 as they are, with a scale byte per lane.
// Rows of W are the rows of the result, rows of A its columns: lane (j, g) ends with four consecutive outputs of token j.
#include "fff_device.h"
#include "fff_mx4.h"

namespace fff {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

enum { kDense, kHidden, kOutput, kHiddenDirect, kOutputDirect };

struct Args {
    const char* a;               // rows of bf16, or codes
    const uint8_t* a_scales;
    int64_t a_row;               // bytes from row to row
    const uint8_t* w;
    const uint8_t* w_scales;
    const void* bias;            // may be null
    char* out;
    int64_t T, N;                // rows of A, rows of W (of one leaf)
    int64_t out_row;             // elements from row to row of out
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
};

__device__ __forceinline__ bf16x8_t dequantise8(uint32_t codes, float scale) {
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
    const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
    const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ f32x4_t mfma4(const uint4& w, uint32_t ws, const uint4& a, uint32_t as, const f32x4_t& acc) {
    const i32x8_t vw = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0}, va = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(vw, va, acc, 4, 4, 0, (int)ws, 0, (int)as);
}

// One step of 128 elements: block b of this lane's row of W against MT rows of A.  TAIL: b may lie behind the row's end, and
// the block may be cut (pieces of bf16 rows): zeros there.
template <bool A4, int MT, bool TAIL>
__device__ __forceinline__ void step128(const uint8_t* w_row, const uint8_t* ws_row, const char* const (&a_row)[MT],
                                        const uint8_t* const (&as_row)[MT], int b, int Kb, int pieces, f32x4_t (&acc)[MT]) {
    const bool in = !TAIL || b < Kb;
    const int bb = in ? b : Kb - 1;
    const uint4 w = keep_if(in, *(const uint4*)(w_row + 16 * (int64_t)bb));
    const uint32_t ws = in ? ws_row[bb] : 0u;
    if constexpr (A4) {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const uint4 a = keep_if(in, *(const uint4*)(a_row[m] + 16 * (int64_t)bb));
            acc[m] = mfma4(w, ws, a, in ? as_row[m][bb] : 0u, acc[m]);
        }
    } else {
        const float s = __uint_as_float(ws << 23);
        uint4 a[MT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int p = 4 * bb + u;
                a[m][u] = keep_if(in && (!TAIL || p < pieces), *(const uint4*)(a_row[m] + 16 * (int64_t)(!TAIL || p < pieces ? p : 0)));
            }
        const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const bf16x8_t f = dequantise8(q[u], s);
#pragma unroll
            for (int m = 0; m < MT; ++m)
                acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, __builtin_bit_cast(bf16x8_t, a[m][u]), acc[m], 0, 0, 0);
        }
    }
}

// The steps wv, wv + waves, ... of the rows' steps.
template <bool A4, int MT>
__device__ __forceinline__ void wave_steps(const uint8_t* w_row, const uint8_t* ws_row, const char* const (&a_row)[MT],
                                           const uint8_t* const (&as_row)[MT], int Kb, int pieces, int g, int wv, int waves,
                                           f32x4_t (&acc)[MT]) {
    const int steps = (Kb + 3) / 4;
    const int whole = A4 ? Kb / 4 : pieces / 16;       // steps without an end of a row in them
    int c = wv;
    for (; c < whole; c += waves) step128<A4, MT, false>(w_row, ws_row, a_row, as_row, 4 * c + g, Kb, pieces, acc);
    for (; c < steps; c += waves) step128<A4, MT, true>(w_row, ws_row, a_row, as_row, 4 * c + g, Kb, pieces, acc);
}

__device__ __forceinline__ float bias_at(const Args& a, const void* bias, int64_t n) {
    if (!bias) return 0.0f;
    return a.out_bf16 ? bf16_to_f32(((const uint16_t*)bias)[n]) : ((const float*)bias)[n];
}

__device__ __forceinline__ float apply(float v, int act) { return act == 2 ? v : activate(v, act); }

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

// 16 rows of W against 16 MT rows of A per block, K shared out among its waves.
//   kDense         rows of A as they come, rows of out too
//   kHidden        a tile of one leaf's slots: rows of A are the slots' tokens; out is h [slot][32 blocks]
//   kOutput        a tile of one leaf's slots: rows of A are h; out is y [pair] in fp32, or with k = 1 the token's row
//   kHiddenDirect  a tile is one pair: h [pair], times the pair's weight
//   kOutputDirect  a tile is one token: the sum over its pairs as one product along k rows of h and of W
template <bool A4, int MT, int MODE, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void mx4_rows_kernel(const Args a) {
    __shared__ f32x4_t part[WAVES][MT][kWave];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, j = lane & 15, g = lane >> 4;
    const int64_t n_blocks = (a.N + 15) / 16;
    const int64_t nb = blockIdx.x % n_blocks, tile = blockIdx.x / n_blocks;
    const int64_t n0 = nb * 16;
    const int64_t w_row_bytes = (int64_t)a.Kb * 16;
    const int64_t n = n0 + j < a.N ? n0 + j : a.N - 1;
    int64_t leaf = 0, first = 0, rows = 0;     // first row of A (slot, pair, token) and how many there are
    if constexpr (MODE == kDense) {
        first = tile * (16 * MT);
        rows = a.T - first;
    } else if constexpr (MODE == kHidden || MODE == kOutput) {
        if (tile >= *a.n_tiles) return;
        leaf = a.tile_leaf[tile];
        first = a.tile_slot[tile];
        rows = a.start[leaf + 1] - first;
    } else {
        first = tile;
        rows = 1;
    }
    if (rows > 16 * MT) rows = 16 * MT;
    f32x4_t acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const char* a_row[MT];
    const uint8_t* as_row[MT];
    if constexpr (MODE == kOutputDirect) {
        // step c of pair i is step i * steps + c of the sum
        const int steps = (a.Kb + 3) / 4, whole = a.pieces / 16;
        for (int u = wv; u < a.k * steps; u += WAVES) {
            const int i = u / steps, c = u - i * steps;
            const int64_t pair = first * a.k + i;
            const uint32_t e = (uint32_t)a.idx[pair];
            if (e >= a.E) continue;
            const uint8_t* const w_row = a.w + ((int64_t)e * a.N + n) * w_row_bytes;
            const uint8_t* const ws_row = a.w_scales + ((int64_t)e * a.N + n) * a.Kb;
            a_row[0] = a.a + pair * a.a_row;
            if (c < whole) step128<A4, MT, false>(w_row, ws_row, a_row, as_row, 4 * c + g, a.Kb, a.pieces, acc);
            else step128<A4, MT, true>(w_row, ws_row, a_row, as_row, 4 * c + g, a.Kb, a.pieces, acc);
        }
    } else {
        if constexpr (MODE == kHiddenDirect) {
            const uint32_t e = (uint32_t)a.idx[first];
            if (e >= a.E) return;              // (kOutputDirect does not read its row)
            leaf = e;
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            int64_t r = 16 * m + j < rows ? 16 * m + j : rows - 1;
            r += first;
            if constexpr (MODE == kHidden) r = a.perm[r] / a.k;
            if constexpr (MODE == kHiddenDirect) r = first / a.k;
            a_row[m] = a.a + r * a.a_row;
            as_row[m] = A4 ? a.a_scales + r * a.Kb : nullptr;
        }
        wave_steps<A4, MT>(a.w + (leaf * a.N + n) * w_row_bytes, a.w_scales + (leaf * a.N + n) * a.Kb, a_row, as_row, a.Kb, a.pieces, g, wv,
                           WAVES, acc);
    }
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
            for (int q = 0; q < 4; ++q) o[q] = n4 + q < a.N ? apply(v[q] + bias_at(a, a.bias, n4 + q), a.act) : 0.f;
            store4(a.out, a.out_bf16, a.out_vec, (first + row) * a.out_row, n4, a.N, o);
        } else if constexpr (MODE == kHidden || MODE == kHiddenDirect) {
            const uint16_t* const bias = (const uint16_t*)a.bias + leaf * a.N;
            const float scale = MODE == kHiddenDirect && a.weight ? a.weight[first] : 1.0f;
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = n4 + q < a.N ? apply(v[q] + bf16_to_f32(bias[n4 + q]), a.act) * scale : 0.f;
            // (the row of h is whole blocks of 32: zeros behind the leaf's width)
            store4(a.out, true, true, (first + row) * a.out_row, n4, a.out_row, o);
            if (n4 + 16 >= a.N && n4 + 16 < a.out_row) {
                const float z[4] = {0.f, 0.f, 0.f, 0.f};
                store4(a.out, true, true, (first + row) * a.out_row, n4 + 16, a.out_row, z);
            }
        } else if constexpr (MODE == kOutput) {
            const uint16_t* const bias = (const uint16_t*)a.bias + leaf * a.N;
            const int64_t pair = a.perm[first + row];
            const float scale = a.k == 1 && a.weight ? a.weight[pair] : 1.0f;
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = n4 + q < a.N ? (v[q] + bf16_to_f32(bias[n4 + q])) * scale : 0.f;
            store4(a.out, a.out_bf16, a.out_vec, pair * a.out_row, n4, a.N, o);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = v[q];
            for (int i = 0; i < a.k; ++i) {
                const uint32_t e = (uint32_t)a.idx[first * a.k + i];
                if (e >= a.E) continue;
                const float scale = a.weight ? a.weight[first * a.k + i] : 1.0f;
                const uint16_t* const bias = (const uint16_t*)a.bias + (int64_t)e * a.N;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (n4 + q < a.N) o[q] = fmaf(scale, bf16_to_f32(bias[n4 + q]), o[q]);
            }
            store4(a.out, true, a.out_vec, first * a.out_row, n4, a.N, o);
        }
    }
}

// ---- tiles through LDS -------------------------------------------------------------------------------------
//
// Many rows of A: a block of WM x WN waves takes 16 MT WM rows of A against 16 NT WN rows of W, a wave 16 MT x 16 NT results.  A stage is 128
// elements of K (bf16 rows: 256 bytes of a row of A, 64 of W) or 256 (codes: 128 bytes of either); two stages, one on its way
// straight to LDS while the other is multiplied.  Scale bytes go to registers, a stage ahead too.
//
// Pieces of 16 bytes in LDS are turned within their row so that the 16 lanes of a pass of an operand read (rows
// {0-3, 12-15} of one g with rows {4-11} of its neighbour, then the others) meet every bank once; the turn is made by
// the lanes' source addresses, since a load to LDS writes lane after lane:
//   128-byte rows, pieces 2 g + u: tile_swz's; 256-byte rows, pieces 4 g + u: (row & 3) + 8 (row >> 3 & 1) further; 64-byte rows, piece g:
//   2 (row >> 3 & 1) further.
__device__ const uint4 g_zero_piece = {0, 0, 0, 0};

template <int ROW> __device__ __forceinline__ int turn(int row) {
    return ROW == 256 ? (row & 3) + 8 * ((row >> 3) & 1) : ROW == 128 ? lds_rot(row) : 2 * ((row >> 3) & 1);
}
template <int ROW> __device__ __forceinline__ int lds_slot(int row, int piece) {
    constexpr int n = ROW / 16;
    return row * n + ((piece + turn<ROW>(row)) & (n - 1));
}

// `count` scale bytes of a row from block b on, the first in the low byte; zeros behind the row's Kb
template <int COUNT> __device__ __forceinline__ uint32_t load_scales(const uint8_t* row, int b, int Kb) {
    typedef uint32_t u32_any __attribute__((aligned(1)));
    typedef uint16_t u16_any __attribute__((aligned(1)));
    if (b + COUNT <= Kb) return COUNT == 4 ? *(const u32_any*)(row + b) : (uint32_t) * (const u16_any*)(row + b);
    uint32_t v = 0;
#pragma unroll
    for (int i = 0; i < COUNT; ++i)
        if (b + i < Kb) v |= (uint32_t)row[b + i] << (8 * i);
    return v;
}

template <bool A4, int WM, int WN, int MT, int NT> struct TileShape {
    static constexpr int kThreads = 64 * WM * WN, kWaves = WM * WN, kRows = 16 * MT * WM, kCols = 16 * NT * WN;
    static constexpr int kARow = A4 ? 128 : 256, kWRow = A4 ? 128 : 64;         // bytes of a row in a stage
    static constexpr int kStepBlocks = A4 ? 8 : 4;                                // blocks of 32 in a stage
    static constexpr int kABytes = kRows * kARow, kWBytes = kCols * kWRow, kStage = kABytes + kWBytes;
    static constexpr int kALoads = kABytes / 1024 / kWaves, kWLoads = kWBytes / 1024 / kWaves;   // a wave's loads of 1 KB a stage
    static_assert(kALoads * 1024 * kWaves == kABytes && kWLoads * 1024 * kWaves == kWBytes, "whole loads a wave");
};

template <bool A4, int MODE, int WM, int WN, int MT, int NT>
__global__ __launch_bounds__(64 * WM * WN, 2) void mx4_tile_kernel(const Args a, const int64_t row_tiles, const int64_t col_tiles) {
    typedef TileShape<A4, WM, WN, MT, NT> S;
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, j = lane & 15, g = lane >> 4;
    const int wm = wv / WN, wn = wv % WN;
    // an XCD takes a contiguous range of tiles, eight row tiles against all columns at a time
    const int64_t id = xcd_contiguous_block();
    if (id >= row_tiles * col_tiles) return;
    const int64_t group = id / (8 * col_tiles), in = id - group * 8 * col_tiles;
    const int64_t tall = row_tiles - 8 * group < 8 ? row_tiles - 8 * group : 8;
    const int64_t rt = 8 * group + in % tall, ct = in / tall;
    const int64_t n0 = ct * S::kCols;
    int64_t leaf = 0, first, rows;
    if constexpr (MODE == kDense) {
        first = rt * S::kRows;
        rows = a.T - first;
    } else {
        if (rt >= *a.n_tiles) return;
        leaf = a.tile_leaf[rt];
        first = a.tile_slot[rt];
        rows = a.start[leaf + 1] - first;
    }
    if (rows > S::kRows) rows = S::kRows;
    const auto a_index = [&](int64_t r) -> int64_t {
        r = (r < rows ? r : rows - 1) + first;
        if constexpr (MODE == kHidden) r = a.perm[r] / a.k;
        return r;
    };
    const auto w_index = [&](int64_t n) -> int64_t { return leaf * a.N + (n0 + n < a.N ? n0 + n : a.N - 1); };
    const int64_t w_row_bytes = (int64_t)a.Kb * 16;

    // sources of this lane's pieces: piece `p` of its rows in stage 0
    const char* a_src[S::kALoads];
    const char* w_src[S::kWLoads];
    int a_piece[S::kALoads], w_piece[S::kWLoads];
#pragma unroll
    for (int i = 0; i < S::kALoads; ++i) {
        constexpr int n = S::kARow / 16;
        const int row = (i * S::kWaves + wv) * (64 / n) + lane / n;
        a_piece[i] = (lane - turn<S::kARow>(row)) & (n - 1);
        a_src[i] = a.a + a_index(row) * a.a_row + 16 * a_piece[i];
    }
#pragma unroll
    for (int i = 0; i < S::kWLoads; ++i) {
        constexpr int n = S::kWRow / 16;
        const int row = (i * S::kWaves + wv) * (64 / n) + lane / n;
        w_piece[i] = (lane - turn<S::kWRow>(row)) & (n - 1);
        w_src[i] = (const char*)a.w + w_index(row) * w_row_bytes + 16 * w_piece[i];
    }
    // rows of scales of this lane's operands
    const uint8_t* ws_row[NT];
    const uint8_t* as_row[MT];
#pragma unroll
    for (int n = 0; n < NT; ++n) ws_row[n] = a.w_scales + w_index(16 * (wn * NT + n) + j) * a.Kb;
#pragma unroll
    for (int m = 0; m < MT; ++m) as_row[m] = A4 ? a.a_scales + a_index(16 * (wm * MT + m) + j) * a.Kb : nullptr;

    const int stages = (a.Kb + S::kStepBlocks - 1) / S::kStepBlocks;
    const int a_pieces = A4 ? a.Kb : a.pieces;
    const char* const zero = (const char*)&g_zero_piece;
    const uint32_t lds0 = lds_address(lds);
    uint32_t w_scale[NT], a_scale[MT];
    const auto fetch = [&](int c, int buf) {
        const int64_t a_off = (int64_t)c * S::kARow, w_off = (int64_t)c * S::kWRow;
#pragma unroll
        for (int n = 0; n < NT; ++n) w_scale[n] = A4 ? load_scales<2>(ws_row[n], 8 * c + 2 * g, a.Kb) : load_scales<4>(ws_row[n], 4 * c, a.Kb);
        if constexpr (A4) {
#pragma unroll
            for (int m = 0; m < MT; ++m) a_scale[m] = load_scales<2>(as_row[m], 8 * c + 2 * g, a.Kb);
        }
        const uint32_t at = lds0 + buf * S::kStage;
#pragma unroll
        for (int i = 0; i < S::kALoads; ++i)
            load_to_lds(c * (S::kARow / 16) + a_piece[i] < a_pieces ? a_src[i] + a_off : zero, __builtin_amdgcn_readfirstlane(at + (i * S::kWaves + wv) * 1024));
#pragma unroll
        for (int i = 0; i < S::kWLoads; ++i)
            load_to_lds(c * (S::kWRow / 16) + w_piece[i] < a.Kb ? w_src[i] + w_off : zero,
                        __builtin_amdgcn_readfirstlane(at + S::kABytes + (i * S::kWaves + wv) * 1024));
    };

    f32x4_t acc[NT][MT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[n][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    fetch(0, 0);
    for (int c = 0; c < stages; ++c) {
        // the stage is there (this wave's part, then everybody's), and nobody reads the other buffer any more
        wait_loads<0>();
        uint32_t ws[NT], as[MT];
#pragma unroll
        for (int n = 0; n < NT; ++n) ws[n] = w_scale[n];
#pragma unroll
        for (int n = 0; n < NT; ++n) asm volatile("" : "+v"(ws[n]));      // (the compiler waits for its loads here, not behind the next stage's)
        if constexpr (A4) {
#pragma unroll
            for (int m = 0; m < MT; ++m) as[m] = a_scale[m];
#pragma unroll
            for (int m = 0; m < MT; ++m) asm volatile("" : "+v"(as[m]));
        }
        __syncthreads();
        if (c + 1 < stages) fetch(c + 1, (c + 1) & 1);
        const uint4* const la = (const uint4*)(lds + (c & 1) * S::kStage);
        const uint4* const lw = (const uint4*)(lds + (c & 1) * S::kStage + S::kABytes);
        if constexpr (A4) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint4 fa[MT];
#pragma unroll
                for (int m = 0; m < MT; ++m) fa[m] = la[lds_slot<128>(16 * (wm * MT + m) + j, 2 * g + u)];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint4 fw = lw[lds_slot<128>(16 * (wn * NT + n) + j, 2 * g + u)];
#pragma unroll
                    for (int m = 0; m < MT; ++m) acc[n][m] = mfma4(fw, u ? ws[n] >> 8 : ws[n], fa[m], u ? as[m] >> 8 : as[m], acc[n][m]);
                }
            }
        } else {
            uint4 fw[NT];
            float s[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                fw[n] = lw[lds_slot<64>(16 * (wn * NT + n) + j, g)];
                s[n] = __uint_as_float(((ws[n] >> (8 * g)) & 255u) << 23);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                bf16x8_t fa[MT];
#pragma unroll
                for (int m = 0; m < MT; ++m) fa[m] = __builtin_bit_cast(bf16x8_t, la[lds_slot<256>(16 * (wm * MT + m) + j, 4 * g + u)]);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const bf16x8_t f = dequantise8(u == 0 ? fw[n].x : u == 1 ? fw[n].y : u == 2 ? fw[n].z : fw[n].w, s[n]);
#pragma unroll
                    for (int m = 0; m < MT; ++m) acc[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, fa[m], acc[n][m], 0, 0, 0);
                }
            }
        }
    }

#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int64_t row = 16 * (wm * MT + m) + j;
        if (row >= rows) continue;
        int64_t to = first + row;
        float scale = 1.0f;
        if constexpr (MODE == kOutput) {
            to = a.perm[to];
            if (a.k == 1 && a.weight) scale = a.weight[to];
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int64_t n4 = n0 + 16 * (wn * NT + n) + 4 * g;
            const int64_t limit = MODE == kHidden ? a.out_row : a.N;
            if (n4 >= limit) continue;
            float o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float v = acc[n][m][q];
                if constexpr (MODE == kDense) o[q] = n4 + q < a.N ? apply(v + bias_at(a, a.bias, n4 + q), a.act) : 0.f;
                else if constexpr (MODE == kHidden) o[q] = n4 + q < a.N ? apply(v + bf16_to_f32(((const uint16_t*)a.bias)[leaf * a.N + n4 + q]), a.act) : 0.f;
                else o[q] = n4 + q < a.N ? (v + bf16_to_f32(((const uint16_t*)a.bias)[leaf * a.N + n4 + q])) * scale : 0.f;
            }
            store4(a.out, MODE == kHidden || a.out_bf16, MODE == kHidden || a.out_vec, to * a.out_row, n4, limit, o);
        }
    }
}

template <bool A4, int MODE, int WM, int WN, int MT, int NT> hipError_t launch_tiles(const Args& a, int64_t row_tiles, hipStream_t s) {
    typedef TileShape<A4, WM, WN, MT, NT> S;
    const int64_t width = MODE == kHidden ? a.out_row : a.N;
    const int64_t col_tiles = (width + S::kCols - 1) / S::kCols;
    const int64_t blocks = (row_tiles * col_tiles + kXcds - 1) / kXcds * kXcds;
    if (blocks >= (int64_t)1 << 31) return hipErrorInvalidConfiguration;
    note_launch("mx4_tile_kernel<%s,%d,%d,%s>", A4 ? "mx4" : "bf16", S::kRows, S::kCols, MODE == kDense ? "dense" : MODE == kHidden ? "hidden" : "output");
    const auto kernel = mx4_tile_kernel<A4, MODE, WM, WN, MT, NT>;
    const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * S::kStage);
    if (e != hipSuccess) return e;
    kernel<<<dim3((unsigned)blocks), S::kThreads, 2 * S::kStage, s>>>(a, row_tiles, col_tiles);
    return hipGetLastError();
}

// ---- grouping of the pairs by leaf -------------------------------------------------------------------------
//
// rank[p] = place of pair p among its leaf's; which pair gets which place depends on the order of the atomics, and
// nothing else does: a row's sums do not know its place in a tile.
__global__ __launch_bounds__(256) void group_count_kernel(const int32_t* __restrict__ idx, int64_t P, int64_t E, int32_t* __restrict__ count,
                                                          int32_t* __restrict__ rank) {
    const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (p >= P) return;
    const uint32_t e = (uint32_t)idx[p];
    if (e < E) rank[p] = atomicAdd(count + e, 1);
}

// start[E + 1], tile_start[E + 1]: exclusive sums of the counts and of the tiles of `tile_rows` slots
__global__ __launch_bounds__(1024) void group_scan_kernel(const int32_t* __restrict__ count, int64_t E, int tile_rows, int32_t* __restrict__ start,
                                                          int32_t* __restrict__ tile_start) {
    __shared__ int32_t sum[2][1024];
    const int tid = threadIdx.x;
    const int64_t per = (E + 1023) / 1024, e0 = tid * per, e1 = e0 + per < E ? e0 + per : E;
    int32_t c = 0, t = 0;
    for (int64_t e = e0; e < e1; ++e) {
        c += count[e];
        t += (count[e] + tile_rows - 1) / tile_rows;
    }
    sum[0][tid] = c;
    sum[1][tid] = t;
    __syncthreads();
    for (int d = 1; d < 1024; d <<= 1) {
        const int32_t v0 = tid >= d ? sum[0][tid - d] : 0, v1 = tid >= d ? sum[1][tid - d] : 0;
        __syncthreads();
        sum[0][tid] += v0;
        sum[1][tid] += v1;
        __syncthreads();
    }
    c = sum[0][tid] - c;
    t = sum[1][tid] - t;
    for (int64_t e = e0; e < e1; ++e) {
        start[e] = c;
        tile_start[e] = t;
        c += count[e];
        t += (count[e] + tile_rows - 1) / tile_rows;
    }
    if (tid == 1023) {
        start[E] = sum[0][1023];
        tile_start[E] = sum[1][1023];
    }
}

__global__ __launch_bounds__(256) void group_place_kernel(const int32_t* __restrict__ idx, int64_t P, int64_t E, int tile_rows,
                                                          const int32_t* __restrict__ rank, const int32_t* __restrict__ start,
                                                          const int32_t* __restrict__ tile_start, int32_t* __restrict__ perm,
                                                          int32_t* __restrict__ tile_leaf, int32_t* __restrict__ tile_slot) {
    const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (p >= P) return;
    const uint32_t e = (uint32_t)idx[p];
    if (e >= E) return;
    const int32_t r = rank[p], slot = start[e] + r;
    perm[slot] = (int32_t)p;
    if (r % tile_rows == 0) {
        const int32_t tile = tile_start[e] + r / tile_rows;
        tile_leaf[tile] = (int32_t)e;
        tile_slot[tile] = slot;
    }
}

// out[t] = sum over the token's pairs of weight * y[pair], in the order of the pairs; y may be null (k = 1): only the
// rows of tokens without a leaf are written, with zeros
__global__ __launch_bounds__(256) void combine_kernel(const int32_t* __restrict__ idx, const float* __restrict__ weight, const float* __restrict__ y,
                                                      uint16_t* __restrict__ out, int64_t T, int64_t O, int64_t E, int k) {
    const int64_t t = blockIdx.x;
    if (!y) {
        if ((uint32_t)idx[t] < E) return;
        for (int64_t o = threadIdx.x; o < O; o += 256) out[t * O + o] = 0;
        return;
    }
    for (int64_t o = threadIdx.x; o < O; o += 256) {
        float v = 0;
        for (int i = 0; i < k; ++i) {
            if ((uint32_t)idx[t * k + i] >= E) continue;
            v = fmaf(weight ? weight[t * k + i] : 1.0f, y[(t * k + i) * O + o], v);
        }
        out[t * O + o] = f32_to_bf16(v);
    }
}

template <bool A4, int MODE> hipError_t launch_rows(const Args& a, int64_t tiles, int mt, hipStream_t s) {
    const int64_t blocks = (a.N + 15) / 16 * tiles;
    if (blocks >= (int64_t)1 << 31) return hipErrorInvalidConfiguration;
    note_launch("mx4_rows_kernel<%s,%d,%s>", A4 ? "mx4" : "bf16", mt,
                MODE == kDense ? "dense" : MODE == kHidden ? "hidden" : MODE == kOutput ? "output" : MODE == kHiddenDirect ? "hidden,direct" : "output,direct");
    const dim3 grid((unsigned)blocks);
    if constexpr (MODE == kHiddenDirect || MODE == kOutputDirect) {
        mx4_rows_kernel<A4, 1, MODE, 8><<<grid, 512, 0, s>>>(a);
    } else {
        if (mt == 1) mx4_rows_kernel<A4, 1, MODE, 8><<<grid, 512, 0, s>>>(a);
        else if (mt == 2) mx4_rows_kernel<A4, 2, MODE, 8><<<grid, 512, 0, s>>>(a);
        else mx4_rows_kernel<A4, 4, MODE, 4><<<grid, 256, 0, s>>>(a);
    }
    return hipGetLastError();
}

int rows_tile(int64_t rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }

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
        count = take(4 * E);
        start = take(4 * (E + 1));
        tile_start = take(4 * (E + 1));
        rank = take(4 * P);
        perm = take(4 * P);
        tile_leaf = take(4 * tiles);
        tile_slot = take(4 * tiles);
        h = take(2 * P * kMxBlock * mx_blocks(L));
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
    if (p.T >= 128) {
        if (a4) return launch_tiles<true, kDense, 2, 4, 4, 4>(a, (p.T + 127) / 128, s);
        return launch_tiles<false, kDense, 2, 4, 4, 4>(a, (p.T + 127) / 128, s);
    }
    const int mt = rows_tile(p.T);
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
    b.a_row = 2 * h_row;
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
    if (P <= 32) {
        if ((e = launch_rows<false, kHiddenDirect>(a, P, 1, s)) != hipSuccess) return e;
        return launch_rows<false, kOutputDirect>(b, p.T, 1, s);
    }
    const bool large = P / p.E >= 64;
    const int mt = rows_tile(P / p.E);
    const int tile_rows = large ? 128 : 16 * mt;
    const int64_t tiles = P / tile_rows + (p.E < P ? p.E : P);
    int32_t *const count = words(at.count), *const start = words(at.start), *const tile_start = words(at.tile_start);
    int32_t *const rank = words(at.rank), *const perm = words(at.perm), *const tile_leaf = words(at.tile_leaf), *const tile_slot = words(at.tile_slot);
    if ((e = launch_zero(count, (p.E + 3) / 4 * 4, s)) != hipSuccess) return e;   // (whole pieces: the region is of 256 bytes)
    const dim3 pairs((unsigned)((P + 255) / 256));
    note_launch("group_kernels");
    group_count_kernel<<<pairs, 256, 0, s>>>(p.idx, P, p.E, count, rank);
    group_scan_kernel<<<1, 1024, 0, s>>>(count, p.E, tile_rows, start, tile_start);
    group_place_kernel<<<pairs, 256, 0, s>>>(p.idx, P, p.E, tile_rows, rank, start, tile_start, perm, tile_leaf, tile_slot);
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
        if ((e = launch_tiles<false, kHidden, 2, 4, 4, 4>(a, tiles, s)) != hipSuccess) return e;
        if ((e = launch_tiles<false, kOutput, 2, 4, 4, 4>(b, tiles, s)) != hipSuccess) return e;
    } else {
        if ((e = launch_rows<false, kHidden>(a, tiles, mt, s)) != hipSuccess) return e;
        if ((e = launch_rows<false, kOutput>(b, tiles, mt, s)) != hipSuccess) return e;
    }
    note_launch("combine_kernel");
    combine_kernel<<<dim3((unsigned)p.T), 256, 0, s>>>(p.idx, p.weight, y, p.out, p.T, p.O, p.E, p.k);
    return hipGetLastError();
}

}  // namespace fff

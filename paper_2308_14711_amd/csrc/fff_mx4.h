// Four-bit matrices (blocks of 32 elements along a row: 16 bytes of codes, one scale byte), and the operators on routed experts:
// what their translation units share.
#pragma once
#include "fff_internal.h"

namespace fff {

constexpr int kMxBlock = 32;                       // elements that share a scale
constexpr int64_t kMaxExperts = 4096;              // of launch_route
constexpr int kMaxChoices = 32;                    // experts per token
constexpr int64_t kMaxMx4Blocks = 1 << 24;         // a launch ends at 2^32 threads: fewer blocks of 256
constexpr int64_t kMaxMx4Tiles = kMaxMx4Blocks - 8;  // of a product: as many blocks for each of the eight XCDs
constexpr int64_t kMaxMx4Row = (int64_t)1 << 34;   // elements of a row to quantise or read back: its pieces are threads of a launch
inline int64_t mx_blocks(int64_t cols) { return (cols + kMxBlock - 1) / kMxBlock; }

// fff_mx4.hip
hipError_t launch_mx4_quantize(const void* src, uint8_t* codes, uint8_t* scales, bool transpose, int64_t batch, int64_t rows,
                               int64_t cols, bool bf16, hipStream_t s);
hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, void* out, int64_t rows, int64_t cols, bool bf16,
                                 hipStream_t s);
// dst [rows, 32 mx_blocks(cols)] <- src [rows, cols], zeros behind a row's end (bf16)
hipError_t launch_pad_rows(const uint16_t* src, uint16_t* dst, int64_t rows, int64_t cols, hipStream_t s);

// fff_mx4_product.hip
struct Mx4Product {
    const void* a;              // bf16 rows of lda elements (whole aligned pieces of 16 bytes), or codes
    const uint8_t* a_scales;    // null: bf16 rows
    int64_t lda;                // bf16 rows only
    const uint8_t* w;
    const uint8_t* w_scales;
    const void* bias;           // null: none
    void* out;
    int64_t T, K, N;
    int act;                    // fff_act
    bool out_bf16;
};
hipError_t launch_mx4_product(const Mx4Product& p, hipStream_t s);

struct Mx4Leaves {
    const uint16_t* x;          // rows of ldx elements, whole aligned pieces of 16 bytes
    int64_t ldx;
    const uint8_t *w1, *s1, *w2, *s2;
    const uint16_t *b1, *b2;
    const int32_t* idx;         // [T, k]
    const float* weight;        // null: ones
    uint16_t* out;
    int64_t T, D, O, E;
    int k, L, act;
};
int64_t mx4_leaves_scratch_bytes(int64_t T, int64_t O, int64_t E, int k, int L);
hipError_t launch_mx4_leaves(const Mx4Leaves& p, void* scratch, hipStream_t s);

// fff_moe_route.hip
struct Route {
    const void* logits;
    const uint8_t* mask;
    int64_t T, E;
    int k;
    bool normalise, bf16;
};
int64_t route_scratch_bytes(int64_t T, int64_t E);
hipError_t launch_route(const Route& r, int32_t* idx, float* weight, int32_t* count, float* prob_mean, float* loss, void* scratch,
                        hipStream_t s);
hipError_t launch_route_backward(const Route& r, const int32_t* idx, const int32_t* count, const float* dweight, const float* dloss,
                                 void* dlogits, hipStream_t s);

}  // namespace fff

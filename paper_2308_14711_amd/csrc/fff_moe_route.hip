// Choice of k experts per token from gating logits, their mixture weights, per-expert counts and balance losses, and the gradient.
//
// One pass over the logits: a group of G lanes (a power of two) holds a token's row in V registers a lane, takes its maximum and
// sum of exponentials, and picks the k largest one after another (the maximum over the group, then the lowest index that holds it).  What the
// losses need of all tokens -- sum over tokens of p, the counts, sum of lse^2 -- stays in registers and LDS over the tokens of a block
// and leaves as one row per block; a second launch adds the rows of the blocks up, always in the same order.
// The gradient is one pass as well: with c[e] = dloss[0] E f[e] / n, p and lse from the logits again,
//   dlogits[e] = p[e] (c[e] - sum_j c[j] p[j] + 2 dloss[1] lse / n) + the weights' part on the k chosen.
// Both are bound by the bytes of the logits (and their gradient).
#include "fff_device.h"
#include "fff_mx4.h"

namespace fff {
namespace {

constexpr int kRouteWaves = 4;
constexpr int kMaxRouteBlocks = 512;

struct RouteArgs {
    const void* logits;
    const uint8_t* mask;
    int32_t* idx;                // forward: out, backward: in
    float* weight;
    const int32_t* count;        // backward
    const float* dweight;
    const float* dloss;
    void* dlogits;
    float* part_p;               // [blocks][E] sums of p; null: no statistics
    int32_t* part_count;         // [blocks][E]
    float* part_z;               // [blocks] sums of lse^2
    int32_t* part_n;             // [blocks] tokens
    int32_t* ticket;             // cleared for the second launch
    int64_t T;
    int E, k, lanes;             // lanes: G
    bool normalise;
};

template <int CTRL> __device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
template <int CTRL> __device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, false); }
__device__ __forceinline__ uint32_t word(float v) { return __float_as_uint(v); }
__device__ __forceinline__ uint32_t word(int v) { return (uint32_t)v; }
__device__ __forceinline__ void unword(uint32_t w, float& v) { v = __uint_as_float(w); }
__device__ __forceinline__ void unword(uint32_t w, int& v) { v = (int)w; }

// v of all lanes of the group (G consecutive lanes), combined in the same way in each of them
template <class T, class OP> __device__ __forceinline__ T group_reduce(T v, int G, OP op) {
    if (G >= 2) v = op(v, dpp<0xB1>(v));         // [1,0,3,2]
    if (G >= 4) v = op(v, dpp<0x4E>(v));         // [2,3,0,1]
    if (G >= 8) v = op(v, dpp<0x141>(v));        // mirror of eight
    if (G >= 16) v = op(v, dpp<0x140>(v));       // mirror of sixteen
    if (G >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(word(v), word(v), false, false);
        T x, y;
        unword(r[0], x);
        unword(r[1], y);
        v = op(x, y);
    }
    if (G >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(word(v), word(v), false, false);
        T x, y;
        unword(r[0], x);
        unword(r[1], y);
        v = op(x, y);
    }
    return v;
}
__device__ __forceinline__ float group_max(float v, int G) { return group_reduce(v, G, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float group_add(float v, int G) { return group_reduce(v, G, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ int group_min(int v, int G) { return group_reduce(v, G, [](int a, int b) { return min(a, b); }); }

// Element of the row that register v of lane gi holds: whole pieces of 16 bytes, lane after lane, or (VEC = false: rows that
// are not whole aligned pieces) single elements.
template <bool BF16, bool VEC> __device__ __forceinline__ int element(int v, int gi, int G) {
    constexpr int VE = BF16 ? 8 : 4;
    return VEC ? (v / VE * G + gi) * VE + v % VE : v * G + gi;
}

template <bool BF16, int V, bool VEC> __device__ __forceinline__ void load_row(const RouteArgs& a, int64_t t, int gi, float (&l)[V]) {
    constexpr int VE = BF16 ? 8 : 4, es = BF16 ? 2 : 4;
    const char* const row = (const char*)a.logits + t * a.E * es;
    const float ninf = -__builtin_inff();
    if (VEC) {
#pragma unroll
        for (int v = 0; v < V; v += VE) {
            const int e = element<BF16, VEC>(v, gi, a.lanes);
            const uint4 q = *(const uint4*)(row + (e < a.E ? e : 0) * es);
            widen<BF16>(q, l + v);
#pragma unroll
            for (int i = 0; i < VE; ++i)
                if (e >= a.E) l[v + i] = ninf;
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = element<BF16, VEC>(v, gi, a.lanes);
            l[v] = Elem<BF16>::load(row, e < a.E ? e : 0);
            if (e >= a.E) l[v] = ninf;
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) l[v] = l[v] != l[v] ? ninf : l[v];
}

// exp(l - m) for l <= m, m > -infinity; logits of +infinity share the row.  The product with log2(e) is carried in two parts: rounded to
// one, it would leave a relative error of up to 2^-19 where l lies far below m.
__device__ __forceinline__ float relative(float l, float m) {
    constexpr float kLog2e = 1.44269504f, kLog2eRest = 1.925963033e-8f;
    const float x = fmaxf(l - m, -200.0f);       // (exp(-200) is 0 in fp32)
    const float y = x * kLog2e;
    const float rest = fmaf(x, kLog2eRest, fmaf(x, kLog2e, -y));
    const float r = __builtin_amdgcn_exp2f(y);
    const float v = fmaf(r, rest * 0.693147181f, r);
    return m == __builtin_inff() ? (l == m ? 1.0f : 0.0f) : v;
}

// order of LDS accesses within a wave (they execute in order; the compiler must keep them so)
__device__ __forceinline__ void wave_sync() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

template <bool BF16, int V, bool VEC>
__global__ __launch_bounds__(64 * kRouteWaves) void route_kernel(const RouteArgs a) {
    extern __shared__ float lds[];               // statistics: kRouteWaves x E sums, E counts
    __shared__ float pick_w[64 * kRouteWaves * 8];
    __shared__ int32_t pick_i[64 * kRouteWaves * 8];
    __shared__ float block_z[kRouteWaves];
    __shared__ int32_t block_n[kRouteWaves];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int G = a.lanes, gi = lane & (G - 1), rows = 64 / G, E = a.E, k = a.k;
    const bool stats = a.part_p != nullptr;
    int32_t* const counts = (int32_t*)(lds + kRouteWaves * E);
    // slots of this group: k <= E <= G V and k <= 32
    float* const my_w = pick_w + (tid / G) * k;
    int32_t* const my_i = pick_i + (tid / G) * k;
    const float ninf = -__builtin_inff();
    float acc[V], z = 0;
    int n = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] = 0;
    if (stats) {
        for (int e = tid; e < E; e += 64 * kRouteWaves) counts[e] = 0;
        __syncthreads();
    }
    const int64_t step = (int64_t)gridDim.x * kRouteWaves * rows;
    // (rows past the end and masked ones run along as empty rows: the lanes of a wave stay together)
    for (int64_t t0 = ((int64_t)blockIdx.x * kRouteWaves + wv) * rows; t0 < a.T; t0 += step) {
        const int64_t t = t0 + lane / G;
        const bool there = t < a.T, on = there && (!a.mask || a.mask[t]);
        float l[V];
        load_row<BF16, V, VEC>(a, there ? t : a.T - 1, gi, l);
        float m = ninf;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!on) l[v] = ninf;
            m = fmaxf(m, l[v]);
        }
        m = group_max(m, G);
        const bool any = m > ninf;
        if (stats) {
            float p[V], s = 0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                p[v] = any ? relative(l[v], m) : 0.0f;
                s += p[v];
            }
            s = group_add(s, G);
            const float inv = any ? 1.0f / s : 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] = fmaf(p[v], inv, acc[v]);
            if (any && gi == 0) {
                const float lse = m + logf(s);
                z = fmaf(lse, lse, z);
                ++n;
            }
        }
        float total = 0;
        if (!a.normalise) {
#pragma unroll
            for (int v = 0; v < V; ++v) total += any ? relative(l[v], m) : 0.0f;
            total = group_add(total, G);
        }
        float chosen = 0;
        for (int i = 0; i < k; ++i) {
            float best = ninf;
#pragma unroll
            for (int v = 0; v < V; ++v) best = fmaxf(best, l[v]);
            best = group_max(best, G);
            int at = 0x7fffffff;
#pragma unroll
            for (int v = V - 1; v >= 0; --v)
                if (l[v] == best) at = element<BF16, VEC>(v, gi, G);
            at = group_min(at, G);
            const bool found = best > ninf;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (element<BF16, VEC>(v, gi, G) == at) l[v] = ninf;
            const float w = found ? relative(best, m) : 0.0f;
            chosen += w;
            if (gi == 0) {
                my_w[i] = w;
                my_i[i] = found ? at : -1;
                if (stats && found) atomicAdd(counts + at, 1);
            }
        }
        wave_sync();
        const float by = a.normalise ? chosen : total;
        if (there)
            for (int i = gi; i < k; i += G) {
                a.idx[t * k + i] = my_i[i];
                a.weight[t * k + i] = any ? my_w[i] / by : 0.0f;
            }
        wave_sync();
    }
    if (!stats) return;
    // the groups of a wave hold the same columns: their sums, then the waves'
    for (int d = G; d < 64; d <<= 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) acc[v] += __shfl_xor(acc[v], d, 64);
    }
    for (int d = 1; d < 64; d <<= 1) {
        z += __shfl_xor(z, d, 64);
        n += __shfl_xor(n, d, 64);
    }
    if (lane < G) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = element<BF16, VEC>(v, gi, G);
            if (e < E) lds[wv * E + e] = acc[v];
        }
    }
    if (lane == 0) {
        block_z[wv] = z;
        block_n[wv] = n;
    }
    __syncthreads();
    for (int e = tid; e < E; e += 64 * kRouteWaves) {
        float s = lds[e];
#pragma unroll
        for (int w = 1; w < kRouteWaves; ++w) s += lds[w * E + e];
        a.part_p[(int64_t)blockIdx.x * E + e] = s;
        a.part_count[(int64_t)blockIdx.x * E + e] = counts[e];
    }
    if (tid == 0) {
        a.part_z[blockIdx.x] = (block_z[0] + block_z[1]) + (block_z[2] + block_z[3]);
        a.part_n[blockIdx.x] = (block_n[0] + block_n[1]) + (block_n[2] + block_n[3]);
        if (blockIdx.x == 0) *a.ticket = 0;
    }
}

// 64 experts a block: sums over the rows of the first launch, then (the block that comes last) the losses.
__global__ __launch_bounds__(256) void route_finish_kernel(const float* __restrict__ part_p, const int32_t* __restrict__ part_count,
                                                           const float* __restrict__ part_z, const int32_t* __restrict__ part_n, int blocks,
                                                           int E, int k, int32_t* __restrict__ count, float* __restrict__ prob_mean,
                                                           float* __restrict__ loss, float* __restrict__ share, int32_t* __restrict__ ticket) {
    __shared__ float sum_p[4][64];
    __shared__ int32_t sum_c[4][64];
    __shared__ float sum_z[4];
    __shared__ int32_t sum_n[4];
    __shared__ bool last;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int e = blockIdx.x * 64 + lane;
    float p = 0, z = 0;
    int32_t c = 0, n = 0;
    if (e < E)
        for (int b = wv; b < blocks; b += 4) {
            p += part_p[(int64_t)b * E + e];
            c += part_count[(int64_t)b * E + e];
        }
    for (int b = tid; b < blocks; b += 256) {
        z += part_z[b];
        n += part_n[b];
    }
    for (int d = 1; d < 64; d <<= 1) {
        z += __shfl_xor(z, d, 64);
        n += __shfl_xor(n, d, 64);
    }
    sum_p[wv][lane] = p;
    sum_c[wv][lane] = c;
    if (lane == 0) {
        sum_z[wv] = z;
        sum_n[wv] = n;
    }
    __syncthreads();
    z = (sum_z[0] + sum_z[1]) + (sum_z[2] + sum_z[3]);
    n = (sum_n[0] + sum_n[1]) + (sum_n[2] + sum_n[3]);
    if (wv == 0) {
        p = (sum_p[0][lane] + sum_p[1][lane]) + (sum_p[2][lane] + sum_p[3][lane]);
        c = (sum_c[0][lane] + sum_c[1][lane]) + (sum_c[2][lane] + sum_c[3][lane]);
        const float mean = n > 0 ? p / (float)n : 0.0f;
        if (e < E) {
            if (count) count[e] = c;
            if (prob_mean) prob_mean[e] = mean;
        }
        if (blockIdx.x == 0 && lane == 0 && count) count[E] = n;
        float f = e < E && n > 0 ? (float)c / ((float)n * (float)k) * mean : 0.0f;
        f = wave_sum(f);
        if (lane == 0 && loss) {
            __hip_atomic_store(share + blockIdx.x, f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
        }
    }
    __syncthreads();
    if (!loss || !last || tid != 0) return;
    float s = 0;
    for (int b = 0; b < (int)gridDim.x; ++b) s += __hip_atomic_load(share + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    loss[0] = (float)E * s;
    loss[1] = n > 0 ? z / (float)n : 0.0f;
}

// what a call without tokens leaves
__global__ __launch_bounds__(256) void route_empty_kernel(int E, int32_t* __restrict__ count, float* __restrict__ prob_mean, float* __restrict__ loss) {
    const int e = blockIdx.x * 256 + threadIdx.x;
    if (count && e <= E) count[e] = 0;
    if (prob_mean && e < E) prob_mean[e] = 0;
    if (loss && e < 2) loss[e] = 0;
}

template <bool BF16, int V, bool VEC>
__global__ __launch_bounds__(64 * kRouteWaves) void route_backward_kernel(const RouteArgs a) {
    constexpr int VE = BF16 ? 8 : 4, es = BF16 ? 2 : 4;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int G = a.lanes, gi = lane & (G - 1), rows = 64 / G, E = a.E, k = a.k;
    const float ninf = -__builtin_inff();
    float pull[V], pull_z = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) pull[v] = 0;
    if (a.dloss) {
        const int n = a.count[E];
        if (n > 0) {
            const float by = a.dloss[0] * (float)E / ((float)n * (float)k) / (float)n;
            pull_z = 2.0f * a.dloss[1] / (float)n;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int e = element<BF16, VEC>(v, gi, G);
                pull[v] = e < E ? by * (float)a.count[e] : 0.0f;
            }
        }
    }
    const int64_t step = (int64_t)gridDim.x * kRouteWaves * rows;
    for (int64_t t0 = ((int64_t)blockIdx.x * kRouteWaves + wv) * rows; t0 < a.T; t0 += step) {
        const int64_t t = t0 + lane / G;
        const bool there = t < a.T, on = there && (!a.mask || a.mask[t]);
        const int64_t tt = there ? t : a.T - 1;
        float l[V], d[V];
        load_row<BF16, V, VEC>(a, tt, gi, l);
        float m = ninf;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!on) l[v] = ninf;
            m = fmaxf(m, l[v]);
        }
        m = group_max(m, G);
        const bool any = m > ninf;
        float s = 0, dot = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            l[v] = any ? relative(l[v], m) : 0.0f;
            s += l[v];
            dot = fmaf(l[v], pull[v], dot);
        }
        s = group_add(s, G);
        dot = group_add(dot, G);
        const float inv = any ? 1.0f / s : 0.0f;
        dot *= inv;
        const float zz = any && pull_z != 0.0f ? pull_z * (m + logf(s)) : 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] = l[v] > 0.0f ? l[v] * inv * (pull[v] - dot + zz) : 0.0f;
        if (a.dweight && any) {
            // the chosen experts' shares, then their part of the gradient
            const char* const row = (const char*)a.logits + tt * E * es;
            float sum = 0, mean = 0;
            for (int i = 0; i < k; ++i) {
                const uint32_t e = (uint32_t)a.idx[tt * k + i];
                if (e >= (uint32_t)E) continue;
                const float x = Elem<BF16>::load(row, e);
                const float w = x == x ? relative(x, m) : 0.0f;
                sum += w;
                mean = fmaf(w, a.dweight[tt * k + i], mean);
            }
            const float by = a.normalise ? (sum > 0.0f ? 1.0f / sum : 0.0f) : inv;
            mean *= by;
            if (!a.normalise) {
#pragma unroll
                for (int v = 0; v < V; ++v) d[v] = fmaf(-l[v] * inv, mean, d[v]);
            }
            for (int i = 0; i < k; ++i) {
                const int e = a.idx[tt * k + i];
                if ((uint32_t)e >= (uint32_t)E) continue;
                const float g = a.dweight[tt * k + i] - (a.normalise ? mean : 0.0f);
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (element<BF16, VEC>(v, gi, G) == e) d[v] = fmaf(l[v] * by, g, d[v]);
            }
        }
        if (!there) continue;
        char* const out = (char*)a.dlogits + t * E * es;
        if (VEC) {
#pragma unroll
            for (int v = 0; v < V; v += VE) {
                const int e = element<BF16, VEC>(v, gi, G);
                if (e < E) *(uint4*)(out + e * es) = narrow<BF16>(d + v);
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int e = element<BF16, VEC>(v, gi, G);
                if (e < E) Elem<BF16>::store(out, e, d[v]);
            }
        }
    }
}

// Registers a lane (a power of two, 8 at least) and lanes a row.
void route_shape(int64_t E, int* V, int* G) {
    *V = E <= 512 ? 8 : E <= 1024 ? 16 : E <= 2048 ? 32 : 64;
    int g = 1;
    while (g * *V < E) g *= 2;
    *G = g;
}

// A block's share of the tokens: enough blocks to cover the chip, but no more rows of partial sums than they are worth.
int route_blocks(int64_t T, int G) {
    const int64_t rows = kRouteWaves * (64 / G);
    const int64_t b = (T + rows - 1) / rows;
    return (int)(b > kMaxRouteBlocks ? kMaxRouteBlocks : b);
}

template <class F> hipError_t with_shape(bool bf16, int V, bool vec, F f) {
    const auto type = [&](auto B) {
        const auto size = [&](auto X) {
            if (V == 8) return f(B, std::integral_constant<int, 8>(), X);
            if (V == 16) return f(B, std::integral_constant<int, 16>(), X);
            if (V == 32) return f(B, std::integral_constant<int, 32>(), X);
            return f(B, std::integral_constant<int, 64>(), X);
        };
        return vec ? size(std::true_type()) : size(std::false_type());
    };
    return bf16 ? type(std::true_type()) : type(std::false_type());
}

struct RouteScratch {
    int64_t part_p, part_count, part_z, part_n, share, ticket, total;
    RouteScratch(int64_t T, int64_t E) {
        int V, G;
        route_shape(E, &V, &G);
        const int64_t blocks = T > 0 ? route_blocks(T, G) : 0;
        int64_t o = 0;
        const auto take = [&](int64_t words) {
            const int64_t at = o;
            o += (4 * words + 255) / 256 * 256;
            return at;
        };
        part_p = take(blocks * E);
        part_count = take(blocks * E);
        part_z = take(blocks);
        part_n = take(blocks);
        share = take((E + 63) / 64);
        ticket = take(1);
        total = o;
    }
};

RouteArgs common_args(const Route& r, int* V, bool* vec) {
    RouteArgs a{};
    a.logits = r.logits;
    a.mask = r.mask;
    a.T = r.T;
    a.E = (int)r.E;
    a.k = r.k;
    a.normalise = r.normalise;
    route_shape(r.E, V, &a.lanes);
    *vec = vec_ok(r.logits, r.E, r.bf16);
    return a;
}

}  // namespace

int64_t route_scratch_bytes(int64_t T, int64_t E) { return RouteScratch(T, E).total; }

hipError_t launch_route(const Route& r, int32_t* idx, float* weight, int32_t* count, float* prob_mean, float* loss, void* scratch,
                        hipStream_t s) {
    const bool stats = count || prob_mean || loss;
    if (r.T == 0) {
        if (!stats) return hipSuccess;
        note_launch("route_empty_kernel");
        route_empty_kernel<<<dim3((unsigned)((r.E + 256) / 256)), 256, 0, s>>>((int)r.E, count, prob_mean, loss);
        return hipGetLastError();
    }
    int V;
    bool vec;
    RouteArgs a = common_args(r, &V, &vec);
    a.idx = idx;
    a.weight = weight;
    const RouteScratch at(r.T, r.E);
    char* const base = (char*)scratch;
    if (stats) {
        a.part_p = (float*)(base + at.part_p);
        a.part_count = (int32_t*)(base + at.part_count);
        a.part_z = (float*)(base + at.part_z);
        a.part_n = (int32_t*)(base + at.part_n);
        a.ticket = (int32_t*)(base + at.ticket);
    }
    const int blocks = route_blocks(r.T, a.lanes);
    const size_t lds = stats ? (size_t)(kRouteWaves + 1) * r.E * 4 : 0;
    note_launch("route_kernel<%s,%d,%s>", r.bf16 ? "bf16" : "f32", V, vec ? "pieces" : "elements");
    hipError_t e = with_shape(r.bf16, V, vec, [&](auto B, auto N, auto X) {
        const auto kernel = route_kernel<decltype(B)::value, decltype(N)::value, decltype(X)::value>;
        if (lds > 32 * 1024) {
            const hipError_t rc = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (rc != hipSuccess) return rc;
        }
        kernel<<<dim3((unsigned)blocks), 64 * kRouteWaves, lds, s>>>(a);
        return hipGetLastError();
    });
    if (e != hipSuccess || !stats) return e;
    note_launch("route_finish_kernel");
    route_finish_kernel<<<dim3((unsigned)((r.E + 63) / 64)), 256, 0, s>>>(a.part_p, a.part_count, a.part_z, a.part_n, blocks, a.E, a.k, count,
                                                                          prob_mean, loss, (float*)(base + at.share), a.ticket);
    return hipGetLastError();
}

hipError_t launch_route_backward(const Route& r, const int32_t* idx, const int32_t* count, const float* dweight, const float* dloss,
                                 void* dlogits, hipStream_t s) {
    int V;
    bool vec;
    RouteArgs a = common_args(r, &V, &vec);
    vec = vec && vec_ok(dlogits, r.E, r.bf16);
    a.idx = const_cast<int32_t*>(idx);
    a.count = count;
    a.dweight = dweight;
    a.dloss = dloss;
    a.dlogits = dlogits;
    const int64_t rows = kRouteWaves * (64 / a.lanes);
    int64_t blocks = (r.T + rows - 1) / rows;
    if (blocks > 4 * kMaxRouteBlocks) blocks = 4 * kMaxRouteBlocks;
    note_launch("route_backward_kernel<%s,%d,%s>", r.bf16 ? "bf16" : "f32", V, vec ? "pieces" : "elements");
    return with_shape(r.bf16, V, vec, [&](auto B, auto N, auto X) {
        route_backward_kernel<decltype(B)::value, decltype(N)::value, decltype(X)::value><<<dim3((unsigned)blocks), 64 * kRouteWaves, 0, s>>>(a);
        return hipGetLastError();
    });
}

}  // namespace fff

// Choice of k experts per token from gating logits, their mixture weights, per-expert counts and balance losses, and the gradient.
//
// One pass over the logits: a group of G lanes (a power of two) holds a token's row in V registers a lane, takes its maximum and
// sum of exponentials, and picks the k largest: one after another (the maximum over the group, then the lowest index that holds it), or where k is
// larger all at once (the few that reach a bound below the k-th, each of which counts those before it).  What the
// losses need of all tokens -- sum over tokens of p, the counts, sum of lse^2 -- stays in registers and LDS over the tokens of a block
// and leaves as one row per block; a second launch adds the rows of the blocks up, always in the same order.
// The gradient is one pass as well: with c[e] = dloss[0] E f[e] / n, p and lse from the logits again,
//   dlogits[e] = p[e] (c[e] - sum_j c[j] p[j] + 2 dloss[1] lse / n) + the weights' part on the k chosen.
// The gradient is near the time of the bytes of the logits and their gradient (32768 x 512 in fp32, 134 MB: 34 us, 4.0 TB/s), the forward pass is vector
// work and waits for lanes and LDS (8 chosen there: 34 us, where bytes alone would take 13; vector units busy 54 % of the cycles).
#include "fff_device.h"
#include "fff_mx4.h"

namespace fff {
namespace {

constexpr int kBackwardWaves = 4;
constexpr int kMaxBackwardBlocks = 2048;
// Waves of a block of the forward kernel: as many as its registers leave room for on a compute unit, since a
// block leaves one row of partial sums (sixteen waves a block on 256 blocks instead of four on 512, 512 experts: 92 -> 70 us).
constexpr int route_waves(int V) { return V <= 16 ? 16 : V == 32 ? 8 : 4; }

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
template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false); }
__device__ __forceinline__ uint32_t word(uint32_t v) { return v; }
__device__ __forceinline__ void unword(uint32_t w, uint32_t& v) { v = w; }
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
// the larger of two that are no NaN (fmaxf spends an instruction on making one quiet)
__device__ __forceinline__ float larger(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, __builtin_inff()); }
__device__ __forceinline__ float group_max(float v, int G) { return group_reduce(v, G, [](float a, float b) { return larger(a, b); }); }
__device__ __forceinline__ float group_add(float v, int G) { return group_reduce(v, G, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ uint32_t group_max(uint32_t v, int G) { return group_reduce(v, G, [](uint32_t a, uint32_t b) { return max(a, b); }); }
__device__ __forceinline__ int group_min(int v, int G) { return group_reduce(v, G, [](int a, int b) { return min(a, b); }); }

// Element of the row that register v of lane gi holds: whole pieces of 16 bytes, lane after lane, or (VEC = false: rows that
// are not whole aligned pieces) single elements.
template <bool BF16, bool VEC> __device__ __forceinline__ int element(int v, int gi, int G) {
    constexpr int VE = BF16 ? 8 : 4;
    return VEC ? (v / VE * G + gi) * VE + v % VE : v * G + gi;
}

// A row as it lies in memory, asked for ahead of its use.
template <bool BF16, int V, bool VEC> struct RawRow {
    static constexpr int VE = BF16 ? 8 : 4, es = BF16 ? 2 : 4;
    uint4 q[VEC ? V / VE : 1];
    typename Elem<BF16>::type x[VEC ? 1 : V];
    uint8_t on;
    __device__ __forceinline__ void load(const RouteArgs& a, int64_t t, int gi) {
        t = t < a.T ? t : a.T - 1;
        const char* const row = (const char*)a.logits + t * a.E * es;
        on = a.mask ? a.mask[t] : 1;
        if constexpr (VEC) {
#pragma unroll
            for (int v = 0; v < V; v += VE) {
                const int e = element<BF16, VEC>(v, gi, a.lanes);
                q[v / VE] = *(const uint4*)(row + (e < a.E ? e : 0) * es);
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int e = element<BF16, VEC>(v, gi, a.lanes);
                x[v] = ((const typename Elem<BF16>::type*)row)[e < a.E ? e : 0];
            }
        }
    }
    // its logits: -infinity for NaN, behind the row's end and in a row that takes no part
    __device__ __forceinline__ void values(const RouteArgs& a, bool there, int gi, float (&l)[V]) const {
        const float ninf = -__builtin_inff();
        const bool row_on = there && on;
        if constexpr (VEC) {
#pragma unroll
            for (int v = 0; v < V; v += VE) {
                widen<BF16>(q[v / VE], l + v);
                const bool in = row_on && element<BF16, VEC>(v, gi, a.lanes) < a.E;
#pragma unroll
                for (int i = 0; i < VE; ++i) l[v + i] = in && l[v + i] == l[v + i] ? l[v + i] : ninf;
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                l[v] = Elem<BF16>::load(x, v);
                l[v] = row_on && element<BF16, VEC>(v, gi, a.lanes) < a.E && l[v] == l[v] ? l[v] : ninf;
            }
        }
    }
};

// exp(l - m) for l <= m, m finite.  With y the rounded product of x = l - m and log2(e), exp(x) = 2^y exp(x - y ln 2), and x - y ln 2, ln 2 in two parts, is what the
// product's rounding left: without it the error grows with m - l, 2^-24 (m - l) and more, as much again as the difference's own (32768 x 512 fp32 logits,
// k = 8, and the gradient: 67.7 us without, 69.3 with).
__device__ __forceinline__ float relative(float l, float m) {
    const float x = fmaxf(l - m, -200.0f);       // (exp(-200) is 0 in fp32)
    const float y = x * 1.44269504f;
    const float rest = fmaf(y, 1.904654e-9f, fmaf(y, -0.693147182f, x));
    const float r = __builtin_amdgcn_exp2f(y);
    return fmaf(r, rest, r);
}
// The same for any m: logits of +infinity share the row.
__device__ __forceinline__ float share_of(float l, float m) { return m == __builtin_inff() ? (l == m ? 1.0f : 0.0f) : relative(l, m); }
// All of a row's (zeros where it has none).
template <int V> __device__ __forceinline__ void shares_of(const float (&l)[V], float m, bool any, float (&p)[V]) {
    const float by = any ? m : 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = relative(l[v], by);
    if (__any(m == __builtin_inff())) {
#pragma unroll
        for (int v = 0; v < V; ++v) p[v] = share_of(l[v], by);
    }
}

// order of LDS accesses within a wave (they execute in order; the compiler must keep them so)
__device__ __forceinline__ void wave_sync() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// A value's bits in the order of values (-0 as 0), and back.  -infinity's are kNoKey.
constexpr uint32_t kNoKey = 0x007fffffu;
__device__ __forceinline__ uint32_t order_key(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// One by one the largest logits that a group holds; values of -infinity are none.  Values are compared as keys, whole numbers: a maximum is one
// instruction then (of floats two, the one before it making NaNs quiet).
//
// bf16 logits: value and index are one key, the index turned round in the low half, so that the largest key is the choice, ties included.  fp32: the lane
// whose largest key is the group's takes it from its registers, those of the fours that hold it; only where two lanes hold it the lower index is looked for.
// (32768 rows of 512 in fp32, 8 one by one: 46 us with floats, 41 with keys.)
// of a bf16 logit's key, whose low half is not its own
__device__ __forceinline__ float short_value(uint32_t key) { return key_value((key & 0xffff0000u) | (key & 0x80000000u ? 0u : 0xffffu)); }
constexpr int kReached = 64;
template <bool BF16, int V, bool VEC> struct Picker {
    uint32_t key[V];
    uint32_t four[BF16 ? 1 : V / 4];      // the largest of four registers each
    uint32_t mine;                        // of all
    __device__ __forceinline__ Picker(const float (&row)[V], int gi, int G) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            key[v] = order_key(row[v]);
            if constexpr (BF16) key[v] = (key[v] & 0xffff0000u) | (0xffffu - (uint32_t)element<BF16, VEC>(v, gi, G));
        }
        mine = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) mine = max(mine, key[v]);
    }
    // before the first of next()
    __device__ __forceinline__ void start() {
        if constexpr (!BF16) {
#pragma unroll
            for (int q = 0; q < V / 4; ++q) four[q] = max(max(key[4 * q], key[4 * q + 1]), max(key[4 * q + 2], key[4 * q + 3]));
        }
    }
    // the largest value, before the first choice
    __device__ __forceinline__ float largest(int G) const {
        const uint32_t best = group_max(mine, G);
        if constexpr (BF16) return best < 0x00800000u ? -__builtin_inff() : short_value(best);
        else return key_value(best);
    }
    // All k choices at once (16 lanes or more): the k-th largest of the lanes' largest is no more than the k-th choice, and few logits reach
    // it (512 of 32 lanes, k = 8: 9).  Those meet in LDS, a lane counts how many of them come before its own, and that is its slot.  False, with nothing
    // done, where a row of the wave has more than kReached of them.
    __device__ __forceinline__ bool all(int k, int gi, int G, uint64_t* reached, float* slot_value, int* slot_at, int32_t* counts) const {
        asm volatile("" : "+v"(gi));       // (indexes are formed where they are used, not kept in registers over the rows)
        uint32_t left = mine, bound = 0;
        for (int i = 0; i < k; ++i) {
            bound = group_max(left, G);
            left = left == bound ? 0u : left;
        }
        bound = max(bound, BF16 ? 0x00800000u : kNoKey + 1);
        int own = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) own += key[v] >= bound;
        // its place behind those of the lanes before it
        int upto = own;
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xf, 0xf, true);         // from one, two, four, eight lanes before, in sixteen
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xf, 0xf, true);
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xf, 0xf, true);
        upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xf, 0xf, true);
        if (G >= 32) upto += __builtin_amdgcn_update_dpp(0, upto, 0x142, 0xa, 0xf, false);        // sixteen's last to the next sixteen
        if (G == 64) upto += __builtin_amdgcn_update_dpp(0, upto, 0x143, 0xc, 0xf, false);
        const int n1 = __builtin_amdgcn_readlane(upto, 63);
        int n = n1, most = n1;
        if (G < 64) {
            const int n0 = __builtin_amdgcn_readlane(upto, 31);
            n = threadIdx.x & 32 ? n1 : n0;
            most = max(n0, n1);
        }
        if (G < 32) {
            const int n0 = __builtin_amdgcn_readlane(upto, 15), n2 = __builtin_amdgcn_readlane(upto, 47);
            n = threadIdx.x & 16 ? n : threadIdx.x & 32 ? n2 : n0;
            most = max(most, max(n0, n2));
        }
        if (most > kReached) return false;
        const int end = (most + 3) & ~3;
        for (int i = gi; i < end; i += G) reached[i] = 0;
        wave_sync();
        uint64_t* to = reached + (upto - own);
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (key[v] >= bound) *to++ = (uint64_t)key[v] << 32 | (BF16 ? 0u : (uint32_t)~element<BF16, VEC>(v, gi, G));
        wave_sync();
        for (int c = gi; c < end; c += G) {
            const uint64_t x = reached[c];
            int before = 0;
            for (int i = 0; i < end; i += 4) {
#pragma unroll
                for (int u = 0; u < 4; ++u) before += reached[i + u] > x;
            }
            if (c < n && before < k) {
                const uint32_t high = (uint32_t)(x >> 32);
                const int at = BF16 ? 0xffff - (int)(high & 0xffffu) : (int)~(uint32_t)x;
                slot_value[before] = BF16 ? short_value(high) : key_value(high);
                slot_at[before] = at;
                if (counts) atomicAdd(counts + at, 1);
            }
        }
        for (int i = n + gi; i < k; i += G) slot_at[i] = -1;
        return true;
    }
    // Whether there is one (`found`); its value; `at`: its index, in the one lane that answers true.
    __device__ __forceinline__ bool next(int gi, int G, float* value, int* at, bool* found) {
        const uint32_t best = group_max(mine, G);
        if constexpr (BF16) {
            mine = 0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                key[v] = key[v] == best ? 0u : key[v];
                mine = max(mine, key[v]);
            }
            *found = best >= 0x00800000u;          // (above -infinity's 0x007f....)
            *at = 0xffff - (int)(best & 0xffffu);
            *value = short_value(best);
            return gi == 0 && *found;
        } else {
            *value = key_value(best);
            *found = best > kNoKey;
            bool have = mine == best && *found;
            asm volatile("" : "+v"(gi));       // (as above)
            if (__popcll(__ballot(have)) != __popcll(__ballot(*found && gi == 0))) {     // two lanes hold it somewhere
                int lowest = 0x7fffffff;
#pragma unroll
                for (int v = V - 1; v >= 0; --v)
                    if (key[v] == best) lowest = element<BF16, VEC>(v, gi, G);
                const int first = group_min(have ? lowest : 0x7fffffff, G);       // (of all lanes)
                have = have && lowest == first;
            }
            bool open = have;
#pragma unroll
            for (int q = 0; q < V / 4; ++q) {
                const bool here = open && four[q] == best;
                if (!__any(here)) continue;
#pragma unroll
                for (int v = 4 * q; v < 4 * q + 4; ++v) {
                    const bool hit = open && key[v] == best;
                    *at = hit ? element<BF16, VEC>(v, gi, G) : *at;
                    key[v] = hit ? 0u : key[v];
                    open = open && !hit;
                }
                four[q] = max(max(key[4 * q], key[4 * q + 1]), max(key[4 * q + 2], key[4 * q + 3]));
            }
            mine = 0;
#pragma unroll
            for (int q = 0; q < V / 4; ++q) mine = max(mine, four[q]);
            return have;
        }
    }
};

template <bool BF16, int V, bool VEC, bool ONCE>
__global__ __launch_bounds__(64 * route_waves(V)) void route_kernel(const RouteArgs a) {
    constexpr int kWaves = route_waves(V);
    extern __shared__ float lds[];               // the slots chosen; statistics: kWaves x E sums, E counts
    __shared__ float block_z[kWaves];
    __shared__ int32_t block_n[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int G = a.lanes, rows = 64 / G, E = a.E, k = a.k;
    int gi = lane & (G - 1);
    const bool stats = a.part_p != nullptr;
    const int slots = kWaves * rows * k;
    float* const my_w = lds + (tid / G) * k;
    int32_t* const my_i = (int32_t*)lds + slots + (tid / G) * k;
    uint64_t* const reached = (uint64_t*)(lds + 2 * slots) + tid / G * kReached;
    float* const sums = lds + 2 * slots + (ONCE ? 2 * kWaves * rows * kReached : 0);
    int32_t* const counts = (int32_t*)sums + kWaves * E;
    float acc[V], z = 0;
    int n = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] = 0;
    if (stats) {
        for (int e = tid; e < E; e += 64 * kWaves) counts[e] = 0;
        __syncthreads();
    }
    const int64_t step = (int64_t)gridDim.x * kWaves * rows;
    int64_t t0 = ((int64_t)blockIdx.x * kWaves + wv) * rows;
    RawRow<BF16, V, VEC> raw;
    if (t0 < a.T) raw.load(a, t0 + lane / G, gi);
    // (rows past the end and masked ones run along as empty rows: the lanes of a wave stay together)
    for (; t0 < a.T; t0 += step) {
        if constexpr (V >= 16) asm volatile("" : "+v"(gi));        // (indexes are formed where they are used: kept over the rows they take registers)
        const int64_t t = t0 + lane / G;
        const bool there = t < a.T;
        float l[V];
        raw.values(a, there, gi, l);
        if (t0 + step < a.T) raw.load(a, t + step, gi);
        Picker<BF16, V, VEC> picker(l, gi, G);
        const float m = picker.largest(G);
        const bool any = m > -__builtin_inff();
        float total = 0;
        if (stats || !a.normalise) {
            float p[V];
            shares_of(l, m, any, p);
#pragma unroll
            for (int v = 0; v < V; ++v) total += p[v];
            total = group_add(total, G);
            if (stats) {
                const float inv = any ? 1.0f / total : 0.0f;
#pragma unroll
                for (int v = 0; v < V; ++v) acc[v] = fmaf(p[v], inv, acc[v]);
                if (any && gi == 0) {
                    const float lse = m + logf(total);
                    z = fmaf(lse, lse, z);
                    ++n;
                }
            }
        }
        bool done = false;
        if constexpr (ONCE) done = picker.all(k, gi, G, reached, my_w, my_i, stats ? counts : nullptr);
        if (!done) picker.start();
        for (int i = done ? k : 0; i < k; ++i) {
            float value;
            int at = 0;
            bool found;
            const bool mine = picker.next(gi, G, &value, &at, &found);
            if (mine || (!found && gi == 0)) {
                my_w[i] = value;
                my_i[i] = found ? at : -1;
                if (stats && found) atomicAdd(counts + at, 1);
            }
        }
        wave_sync();
        // a lane a slot (k <= G), or several
        float chosen = 0;
        if (a.normalise) {
            for (int i = gi; i < k; i += G) chosen += my_i[i] >= 0 ? share_of(my_w[i], m) : 0.0f;
            chosen = group_add(chosen, G);
        }
        const float by = a.normalise ? chosen : total;
        if (there)
            for (int i = gi; i < k; i += G) {
                const int e = my_i[i];
                a.idx[t * k + i] = e;
                a.weight[t * k + i] = e >= 0 ? share_of(my_w[i], m) / by : 0.0f;
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
            if (e < E) sums[wv * E + e] = acc[v];
        }
    }
    if (lane == 0) {
        block_z[wv] = z;
        block_n[wv] = n;
    }
    __syncthreads();
    for (int e = tid; e < E; e += 64 * kWaves) {
        float s = sums[e];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) s += sums[w * E + e];
        a.part_p[(int64_t)blockIdx.x * E + e] = s;
        a.part_count[(int64_t)blockIdx.x * E + e] = counts[e];
    }
    if (tid == 0) {
        z = 0;
        n = 0;
        for (int w = 0; w < kWaves; ++w) {
            z += block_z[w];
            n += block_n[w];
        }
        a.part_z[blockIdx.x] = z;
        a.part_n[blockIdx.x] = n;
        if (blockIdx.x == 0) *a.ticket = 0;
    }
}

// 64 experts a block: sums over the rows of the first launch (sixteen waves, every sixteenth row each), then (the block that comes last) the losses.
constexpr int kFinishWaves = 16;
__global__ __launch_bounds__(64 * kFinishWaves) void route_finish_kernel(const float* __restrict__ part_p, const int32_t* __restrict__ part_count,
                                                                         const float* __restrict__ part_z, const int32_t* __restrict__ part_n,
                                                                         int blocks, int E, int k, int32_t* __restrict__ count,
                                                                         float* __restrict__ prob_mean, float* __restrict__ loss,
                                                                         float* __restrict__ share, int32_t* __restrict__ ticket) {
    __shared__ float sum_p[kFinishWaves][64], sum_z[kFinishWaves];
    __shared__ int32_t sum_c[kFinishWaves][64], sum_n[kFinishWaves];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int e = blockIdx.x * 64 + lane;
    float p = 0, z = 0;
    int32_t c = 0, n = 0;
    if (e < E) {
#pragma unroll 8
        for (int b = wv; b < blocks; b += kFinishWaves) {
            p += part_p[(int64_t)b * E + e];
            c += part_count[(int64_t)b * E + e];
        }
    }
    if (tid < blocks) {           // (no more blocks than threads)
        z = part_z[tid];
        n = part_n[tid];
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
    if (wv != 0) return;
    z = sum_z[0];
    n = sum_n[0];
    p = sum_p[0][lane];
    c = sum_c[0][lane];
#pragma unroll
    for (int w = 1; w < kFinishWaves; ++w) {
        z += sum_z[w];
        n += sum_n[w];
        p += sum_p[w][lane];
        c += sum_c[w][lane];
    }
    const float mean = n > 0 ? p / (float)n : 0.0f;
    if (e < E) {
        if (count) count[e] = c;
        if (prob_mean) prob_mean[e] = mean;
    }
    if (blockIdx.x == 0 && lane == 0 && count) count[E] = n;
    if (!loss) return;
    const float f = wave_sum(e < E && n > 0 ? (float)c / ((float)n * (float)k) * mean : 0.0f);
    if (lane == 0) {
        __hip_atomic_store(share + blockIdx.x, f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const bool last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
        if (last) {
            float s = 0;
            for (int b = 0; b < (int)gridDim.x; ++b) s += __hip_atomic_load(share + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            loss[0] = (float)E * s;
            loss[1] = n > 0 ? z / (float)n : 0.0f;
        }
    }
}

// what a call without tokens leaves
__global__ __launch_bounds__(256) void route_empty_kernel(int E, int32_t* __restrict__ count, float* __restrict__ prob_mean, float* __restrict__ loss) {
    const int e = blockIdx.x * 256 + threadIdx.x;
    if (count && e <= E) count[e] = 0;
    if (prob_mean && e < E) prob_mean[e] = 0;
    if (loss && e < 2) loss[e] = 0;
}

// kSlots: slots of a row that a lane looks after (gi, gi + G, ...): one where k <= G, else up to eight (k <= E <= G V, and V = 8 where G < 32)
template <bool BF16, int V, bool VEC, int kSlots>
__global__ __launch_bounds__(64 * kBackwardWaves) void route_backward_kernel(const RouteArgs a) {
    extern __shared__ float patches[];           // G V words a group, zeros between rows
    constexpr int VE = BF16 ? 8 : 4, es = BF16 ? 2 : 4;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int G = a.lanes, rows = 64 / G, E = a.E, k = a.k;
    int gi = lane & (G - 1);
    // a row's logits, chosen experts and their gradients, asked for ahead of their use
    int64_t t0 = ((int64_t)blockIdx.x * kBackwardWaves + wv) * rows;
    RawRow<BF16, V, VEC> raw;
    uint32_t next_e[kSlots];
    float next_g[kSlots];
    const auto ask = [&](int64_t t) {
        raw.load(a, t, gi);
        if (!a.dweight) return;
        t = t < a.T ? t : a.T - 1;
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
            if (s * G >= k) break;
            const int i = gi + s * G;
            next_e[s] = i < k ? (uint32_t)a.idx[t * k + i] : ~0u;
            next_g[s] = i < k ? a.dweight[t * k + i] : 0.0f;
        }
    };
    if (t0 < a.T) ask(t0 + lane / G);
    float* const patch = patches + (tid / G) * (G * V);
    for (int i = lane; i < 64 * V; i += 64) patches[wv * 64 * V + i] = 0;
    wave_sync();
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
    const int64_t step = (int64_t)gridDim.x * kBackwardWaves * rows;
    for (; t0 < a.T; t0 += step) {
        if constexpr (V >= 16) asm volatile("" : "+v"(gi));        // (indexes are formed where they are used: kept over the rows they take registers)
        const int64_t t = t0 + lane / G;
        const bool there = t < a.T;
        const int64_t tt = there ? t : a.T - 1;
        const char* const row = (const char*)a.logits + tt * E * es;
        uint32_t slot_e[kSlots];
        float slot_g[kSlots], slot_x[kSlots];
        if (a.dweight) {
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
                if (s * G >= k) break;
                slot_e[s] = next_e[s];
                slot_g[s] = next_g[s];
                slot_x[s] = Elem<BF16>::load(row, slot_e[s] < (uint32_t)E ? slot_e[s] : 0);
            }
        }
        float l[V], d[V], m = -__builtin_inff();
        raw.values(a, there, gi, l);
#pragma unroll
        for (int v = 0; v < V; ++v) m = larger(m, l[v]);
        m = group_max(m, G);
        const bool any = m > -__builtin_inff();
        if (t0 + step < a.T) ask(t + step);
        float s = 0, dot = 0;
        shares_of(l, m, any, d);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            l[v] = d[v];
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
        if (a.dweight) {
            // The slots' part: a lane a slot, put to where the expert's lane reads it.  (Rows that take no part run along.)
            float sum = 0, mean = 0;
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
                if (s * G >= k) break;
                const bool good = any && slot_e[s] < (uint32_t)E && slot_x[s] == slot_x[s];
                slot_x[s] = good ? share_of(slot_x[s], m) : 0.0f;
                slot_g[s] = any && slot_e[s] < (uint32_t)E ? slot_g[s] : 0.0f;         // (no expert's: not read)
                sum += slot_x[s];
                mean = fmaf(slot_x[s], slot_g[s], mean);
            }
            sum = group_add(sum, G);
            mean = group_add(mean, G);
            const float by = a.normalise ? (sum > 0.0f ? 1.0f / sum : 0.0f) : inv;
            mean *= by;
            if (!a.normalise) {
#pragma unroll
                for (int v = 0; v < V; ++v) d[v] = fmaf(-l[v] * inv, mean, d[v]);
            }
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
                if (s * G >= k) break;
                if (any && slot_e[s] < (uint32_t)E) atomicAdd(patch + slot_e[s], slot_x[s] * by * (slot_g[s] - (a.normalise ? mean : 0.0f)));
            }
            wave_sync();
#pragma unroll
            for (int v = 0; v < V; ++v) d[v] += patch[element<BF16, VEC>(v, gi, G)];
            wave_sync();
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
                if (s * G >= k) break;
                if (slot_e[s] < (uint32_t)E) patch[slot_e[s]] = 0;
            }
            wave_sync();
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

// Registers a lane (a power of two, 8 at least) and lanes a row.  A row on fewer lanes shares the steps over the lanes among more rows of a wave, in the
// forward kernel also those of the choices, so that eight registers end at 64 experts there (65536 rows, forward and finish: 256 bf16 logits, k = 2 and 8,
// 30.1 and 39.6 us with eight, 23.5 and 30.4 with sixteen; 128: 19.2 and 25.0, 17.0 and 22.3; fp32 128, k = 8: 25.3, and 31.0 since eight lanes do not
// choose at once) and at 256 in the backward kernel (256 bf16 logits: 28.5, sixteen 32.3).
void route_shape(int64_t E, int64_t up_to_8, int* V, int* G) {
    *V = E <= up_to_8 ? 8 : E <= 1024 ? 16 : E <= 2048 ? 32 : 64;
    int g = 1;
    while (g * *V < E) g *= 2;
    *G = g;
}
// Rows of partial sums that scratch has room for, and blocks of the forward kernel: one a compute unit (50432 tokens, 128 experts: 14.7 us; two: 17.4).
constexpr int64_t kMaxPartRows = 256;
int route_blocks(int64_t T, int waves, int G) {
    const int64_t rows = waves * (64 / G), most = device_info().cus < kMaxPartRows ? device_info().cus : kMaxPartRows;
    const int64_t b = (T + rows - 1) / rows;
    return (int)(b > most ? most : b);
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
        const int64_t blocks = T > 0 ? (T < kMaxPartRows ? T : kMaxPartRows) : 0;
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

RouteArgs common_args(const Route& r, int64_t up_to_8, int* V, bool* vec) {
    RouteArgs a{};
    a.logits = r.logits;
    a.mask = r.mask;
    a.T = r.T;
    a.E = (int)r.E;
    a.k = r.k;
    a.normalise = r.normalise;
    route_shape(r.E, up_to_8, V, &a.lanes);
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
    // Choices one by one or at once (65536 rows of 256, us, one by one / at once: bf16 k = 2 30 / 33, 4 35 / 36, 8 45 / 41; fp32 k = 2 33 / 33, 4 41 / 35,
    // 8 60 / 40; 32768 fp32 rows of 512, k = 8: 45 / 33).  With k near the lanes' number too many logits reach the bound.
    const int late = r.bf16 ? 6 : 3;
    RouteArgs a = common_args(r, !r.bf16 && r.k >= late ? 128 : 64, &V, &vec);
    const bool at_once = a.lanes >= 16 && r.k >= late && 4 * r.k <= 3 * a.lanes;
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
    const int waves = route_waves(V), blocks = route_blocks(r.T, waves, a.lanes);
    const size_t lds = (size_t)waves * (64 / a.lanes) * 8 * (r.k + (at_once ? kReached : 0)) + (stats ? (size_t)(waves + 1) * r.E * 4 : 0);
    note_launch("route_kernel<%s,%d,%s>", r.bf16 ? "bf16" : "f32", V, vec ? "pieces" : "elements");
    hipError_t e = with_shape(r.bf16, V, vec, [&](auto B, auto N, auto X) {
        constexpr bool bf16 = decltype(B)::value, pieces = decltype(X)::value;
        constexpr int regs = decltype(N)::value;
        const auto kernel = at_once ? route_kernel<bf16, regs, pieces, true> : route_kernel<bf16, regs, pieces, false>;
        if (lds > 60 * 1024) {
            const hipError_t rc = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (rc != hipSuccess) return rc;
        }
        kernel<<<dim3((unsigned)blocks), 64 * waves, lds, s>>>(a);
        return hipGetLastError();
    });
    if (e != hipSuccess || !stats) return e;
    note_launch("route_finish_kernel");
    route_finish_kernel<<<dim3((unsigned)((r.E + 63) / 64)), 64 * kFinishWaves, 0, s>>>(a.part_p, a.part_count, a.part_z, a.part_n, blocks, a.E, a.k, count,
                                                                          prob_mean, loss, (float*)(base + at.share), a.ticket);
    return hipGetLastError();
}

hipError_t launch_route_backward(const Route& r, const int32_t* idx, const int32_t* count, const float* dweight, const float* dloss,
                                 void* dlogits, hipStream_t s) {
    int V;
    bool vec;
    RouteArgs a = common_args(r, 256, &V, &vec);
    vec = vec && vec_ok(dlogits, r.E, r.bf16);
    a.idx = const_cast<int32_t*>(idx);
    a.count = count;
    a.dweight = dweight;
    a.dloss = dloss;
    a.dlogits = dlogits;
    const int64_t rows = kBackwardWaves * (64 / a.lanes);
    int64_t blocks = (r.T + rows - 1) / rows;
    if (blocks > kMaxBackwardBlocks) blocks = kMaxBackwardBlocks;
    note_launch("route_backward_kernel<%s,%d,%s>", r.bf16 ? "bf16" : "f32", V, vec ? "pieces" : "elements");
    return with_shape(r.bf16, V, vec, [&](auto B, auto N, auto X) {
        constexpr bool bf16 = decltype(B)::value, pieces = decltype(X)::value;
        constexpr int regs = decltype(N)::value;
        const auto kernel = regs == 8 && r.k > a.lanes ? route_backward_kernel<bf16, regs, pieces, regs == 8 ? 8 : 1> : route_backward_kernel<bf16, regs, pieces, 1>;
        const size_t lds = (size_t)kBackwardWaves * 64 * decltype(N)::value * 4;
        if (lds > 60 * 1024) {
            const hipError_t rc = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (rc != hipSuccess) return rc;
        }
        kernel<<<dim3((unsigned)blocks), 64 * kBackwardWaves, lds, s>>>(a);
        return hipGetLastError();
    });
}

}  // namespace fff

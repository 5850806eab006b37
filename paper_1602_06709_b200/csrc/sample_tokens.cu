// One token of each row of logits: temperature, top-k, top-p and min-p, from a given random number.
//
//   d = (z - max z) / temperature,  weight = exp(d).  In the order of falling z (equal ones: rising id) the filters keep a first part of the
//   row: top_k tokens; of them those in front of which lies less than top_p of their weight; those with weight >= min_p.
//   Among the kept, in the order of their ids, the first whose cumulated weight exceeds uniform times the total.
//
// Which token that is depends on sums over up to all tokens, next to which one token's weight can be tiny: weights are taken
// in 64 bits (relative error 1e-14) and held as whole numbers of 2^-44 (less for rows of more than 2^18), so that sums do not depend on the
// order of additions and histograms can be built with atomics.
//
// A block takes a row; what it reads once it finds in L2 the next time.
//   Every row: the maximum, two 16-bit logits to an instruction.
//   Small top-k: the k-th largest of the threads' maxima is a bound that k tokens reach and few others; those go to a list in shared memory,
//     and everything else happens there, by comparing all pairs.
//   Other filters: a histogram over z, of weights or counts, says in which bin the part kept ends (with top-p: of the tokens whose weight is
//     not below (1 - top_p) / K of the total; the others together do not reach what top-p leaves out).  The bin's tokens go to the list; if
//     they do not fit, the bin is divided by the bits of its values, down to a single value.
//   What is kept is summed by pieces of consecutive ids, and the piece in which the random number falls is searched.
// The cost is the weights': one takes twelve operations in 64 bits, of which an SM does 64 a cycle, so a row that needs all of them takes three
// times as long as reading it.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "pcl_internal.h"
#include "pcl_ptx.cuh"

namespace pcl {

namespace {

constexpr int kBins = 2048;
constexpr int kList = 1024;                  // tokens of the list
constexpr int kPieces = 256;                 // pieces of consecutive ids, at most
constexpr int kWeightBits = 44;

struct SampleParams {
    int N, K, bits;                          // bits: a weight of 1 is 2^bits
    const void* logits;
    const float *uniform, *temperature, *top_p, *min_p;
    const int* top_k;
    int* token;
    float* logprob;
};

using u64 = unsigned long long;

// Sixteen bytes of logits.
template <class T> struct Vec;
template <> struct Vec<float> {
    static constexpr int E = 4, kLowBit = 0;                 // kLowBit: lowest bit that a value's fp32 form can have set
    static constexpr uint32_t kLeast = 0xff800000u;          // a word of -inf
    static __device__ __forceinline__ float get(const uint32_t (&u)[4], int i) { return __uint_as_float(u[i]); }
    static __device__ __forceinline__ uint32_t load(const void* row, long e) { return static_cast<const uint32_t*>(row)[e]; }
    static __device__ __forceinline__ void put(uint32_t (&u)[4], int i, uint32_t v) { u[i] = v; }
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        float m;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
        return __float_as_uint(m);
    }
    static __device__ __forceinline__ float top(uint32_t m) { return __uint_as_float(m); }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int E = 8, kLowBit = 16;
    static constexpr uint32_t kLeast = 0xff80ff80u;
    static __device__ __forceinline__ float get(const uint32_t (&u)[4], int i) { return __uint_as_float(i & 1 ? u[i >> 1] & 0xffff0000u : u[i >> 1] << 16); }
    static __device__ __forceinline__ uint32_t load(const void* row, long e) { return static_cast<const uint16_t*>(row)[e]; }
    static __device__ __forceinline__ void put(uint32_t (&u)[4], int i, uint32_t v) { u[i >> 1] = i & 1 ? (u[i >> 1] & 0xffffu) | v << 16 : (u[i >> 1] & 0xffff0000u) | v; }
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t m;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
        return m;
    }
    static __device__ __forceinline__ float top(uint32_t m) {
        const uint32_t v = max2(m, m >> 16 | m << 16);
        return __uint_as_float(v << 16);
    }
};
template <> struct Vec<__half> {
    static constexpr int E = 8, kLowBit = 13;
    static constexpr uint32_t kLeast = 0xfc00fc00u;
    static __device__ __forceinline__ float get(const uint32_t (&u)[4], int i) {
        return __half2float(__ushort_as_half(uint16_t(i & 1 ? u[i >> 1] >> 16 : u[i >> 1] & 0xffffu)));
    }
    static __device__ __forceinline__ uint32_t load(const void* row, long e) { return static_cast<const uint16_t*>(row)[e]; }
    static __device__ __forceinline__ void put(uint32_t (&u)[4], int i, uint32_t v) { u[i >> 1] = i & 1 ? (u[i >> 1] & 0xffffu) | v << 16 : (u[i >> 1] & 0xffff0000u) | v; }
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t m;
        asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
        return m;
    }
    static __device__ __forceinline__ float top(uint32_t m) {
        const uint32_t v = max2(m, m >> 16 | m << 16);
        return __half2float(__ushort_as_half(uint16_t(v & 0xffffu)));
    }
};

// A row, in vectors that are aligned in memory: vector c holds the elements c * E - shift ...; what of the first and the last
// one is not the row's reads as -inf.
template <class T>
struct Row {
    static constexpr int E = Vec<T>::E;
    const T* base;                           // the row's first element
    int K, shift, vectors;
    __device__ __forceinline__ Row(const void* logits, size_t row, int k) : base(static_cast<const T*>(logits) + row * k), K(k) {
        shift = int(row * k % E);
        vectors = (K + shift + E - 1) / E;
    }
    __device__ __forceinline__ long first(int c) const { return long(c) * E - shift; }
    __device__ __forceinline__ void load(int c, uint32_t (&u)[4]) const {
        const long e = first(c);
        if (e >= 0 && e + E <= K) {
            const uint4 q = __ldg(reinterpret_cast<const uint4*>(base + e));
            u[0] = q.x; u[1] = q.y; u[2] = q.z; u[3] = q.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = Vec<T>::kLeast;
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (e + i >= 0 && e + i < K) Vec<T>::put(u, i, Vec<T>::load(base, e + i));
        }
    }
    // f(vector, its index) for every vector, the block's threads side by side; kMany vectors are loaded before the first is used
    template <int kMany, class F>
    __device__ __forceinline__ void each(F&& f) const {
        for (int c = threadIdx.x; c < vectors; c += kMany * int(blockDim.x)) {
            uint32_t u[kMany][4];
#pragma unroll
            for (int m = 0; m < kMany; ++m)
                if (c + m * int(blockDim.x) < vectors) load(c + m * int(blockDim.x), u[m]);
#pragma unroll
            for (int m = 0; m < kMany; ++m)
                if (c + m * int(blockDim.x) < vectors) f(u[m], c + m * int(blockDim.x));
        }
    }
};

// Bits that order like the values.
__device__ __forceinline__ uint32_t order(float z) {
    const uint32_t b = __float_as_uint(z);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unorder(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// exp((z - max) / temperature) as a whole number of 2^-bits.  Table-driven (after Tang, 1989): 2^(i/16) for the whole part of
// x = 16 log2 of it, and a polynomial for the rest, |r| <= 1/2, through (2^(r/16) - 1) / r at the five Chebyshev nodes (relative error 9e-15).
// Numbers become whole by adding 3 * 2^51 or 2^52 to them.
struct Scale {
    double top, inv, per16;                  // the row's maximum, 1 / temperature, 16 log2(e) / temperature
    double unit;                             // 2^bits
    double least;                            // smallest x that has a weight
    const double* table;                     // 2^(i/16) * unit
    bool infinite;                           // the maximum is +inf: only such logits have weight
    __device__ __forceinline__ double x(float z) const {
        if (infinite) return z == INFINITY ? 0.0 : -INFINITY;
        return (double(z) - top) * per16;
    }
    __device__ __forceinline__ u64 weight(float z, double from) const {
        const double v = x(z);
        if (!(v >= from)) return 0ull;       // (NaN: -inf at an infinite temperature)
        const double t = v + 6755399441055744.0;
        const int i = __double2loint(t);
        const double r = v - (t - 6755399441055744.0);
        double p = fma(r, 0x1.5d893e58acc63p-30, 0x1.3b2c4ac7da565p-23);
        p = fma(r, p, 0x1.c6b08d6faa1bep-17);
        p = fma(r, p, 0x1.ebfbdff6988c8p-11);
        p = fma(r, p, 0x1.62e42fefa39efp-5) * r;
        double s = table[i & 15];
        s = __hiloint2double(__double2hiint(s) + (i >> 4 << 20), __double2loint(s));
        const double w = fma(s, p, s) + 4503599627370496.0;
        return u64(__double_as_longlong(w)) & 0xfffffffffffffull;
    }
    __device__ __forceinline__ u64 weight(float z) const { return weight(z, least); }
};
constexpr double kLeastX = -16.0 * kWeightBits;

struct Shared {
    uint32_t lo[kBins], hi[kBins];           // histogram: weights in two words, or counts in the first
    u64 key[kList], weight[kList];           // list: order of the value above, ~id below
    u64 piece[kPieces];
    uint32_t ties[kPieces];
    double table[16];
    u64 warp_sum[32];
    uint32_t warp_word[32];
    float warp_z[32];
    int bin, count;
    u64 above;
    uint32_t key_lo, key_hi;
    float border_z;
    uint32_t border_ties;
    int found;
    u64 found_weight;
    uint32_t found_ties;
};

__device__ __forceinline__ void add_weight(uint32_t* lo, uint32_t* hi, u64 w) {
    const uint32_t l = uint32_t(w), old = atomicAdd(lo, l);
    const uint32_t up = uint32_t(w >> 32) + (old + l < old ? 1u : 0u);
    if (up) atomicAdd(hi, up);
}

// Inclusive sums over the block's threads (in order) of two numbers; every thread also gets the totals.
template <int kThreads>
__device__ __forceinline__ void block_scan(Shared& s, u64& a, uint32_t& c, u64& all_a, uint32_t& all_c) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 x = __shfl_up_sync(0xffffffffu, a, o);
        const uint32_t y = __shfl_up_sync(0xffffffffu, c, o);
        if (lane >= o) { a += x; c += y; }
    }
    __syncthreads();
    if (lane == 31) { s.warp_sum[warp] = a; s.warp_word[warp] = c; }
    __syncthreads();
    u64 before = 0;
    uint32_t before_c = 0;
    all_a = 0; all_c = 0;
#pragma unroll 4
    for (int i = 0; i < kThreads / 32; ++i) {
        if (i == warp) { before = all_a; before_c = all_c; }
        all_a += s.warp_sum[i];
        all_c += s.warp_word[i];
    }
    a += before;
    c += before_c;
}
__device__ __forceinline__ u64 warp_sum(u64 a) {
#pragma unroll
    for (int o = 16; o; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
    return a;
}
template <int kThreads>
__device__ __forceinline__ u64 block_sum(Shared& s, u64 a) {
    a = warp_sum(a);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s.warp_sum[threadIdx.x >> 5] = a;
    __syncthreads();
    a = (threadIdx.x & 31) < kThreads / 32 ? s.warp_sum[threadIdx.x & 31] : 0ull;
    return warp_sum(a);
}

// The first bin up to which the histogram holds `want`: its index and what lies in front of it go to s.bin (-1: there is none) and s.above.
template <int kThreads>
__device__ __forceinline__ void find_bin(Shared& s, u64 want) {
    constexpr int kEach = kBins / kThreads;
    __syncthreads();
    if (threadIdx.x == 0) s.bin = -1;
    u64 w[kEach], a = 0, all;
    uint32_t none = 0, none_all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        w[i] = u64(s.hi[kEach * threadIdx.x + i]) << 32 | s.lo[kEach * threadIdx.x + i];
        a += w[i];
    }
    u64 before = a;
    block_scan<kThreads>(s, a, none, all, none_all);
    before = a - before;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (before < want && before + w[i] >= want) { s.bin = kEach * threadIdx.x + i; s.above = before; }
        before += w[i];
    }
    __syncthreads();
}

// Where the part kept ends: tokens above `z` are kept, and of those equal to it the first `ties` by id.
struct Border { float z; uint32_t ties; };

// The value at which the tokens in falling order, down to `from`, reach `want` of weight, or of their number; false: they do not.
template <int kThreads, bool kByWeight, class T>
__device__ __noinline__ bool select(Shared& s, const Row<T>& row, const Scale& sc, float top, float from, u64 want, Border& border) {
    constexpr int E = Vec<T>::E;
    const float scale = float(kBins) / (top - from);          // (top == from: infinite or NaN, and every value then is in bin 0)
    auto bin_of = [&](float z) { const float b = (top - z) * scale; return b < float(kBins - 1) ? int(b) : b >= float(kBins - 1) ? kBins - 1 : 0; };
    uint32_t lo = 0, hi = 0, step = 0;                        // after the first histogram: bins of `step` keys from hi down to lo
    u64 above = 0;
    for (;;) {
        for (int i = threadIdx.x; i < kBins; i += kThreads) { s.lo[i] = 0; s.hi[i] = 0; }
        __syncthreads();
        auto bin_or_none = [&](float z) {
            if (step == 0) return z >= from && z > -INFINITY ? bin_of(z) : -1;
            const uint32_t k = order(z);
            return k >= lo && k <= hi ? int((hi - k) / step) : -1;
        };
        row.template each<2>([&](uint32_t (&u)[4], int) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float z = Vec<T>::get(u, i) + 0.f;
                const int b = bin_or_none(z);
                if (b < 0) continue;
                if (kByWeight) add_weight(&s.lo[b], &s.hi[b], sc.weight(z));
                else atomicAdd(&s.lo[b], 1u);
            }
        });
        find_bin<kThreads>(s, want - above);
        if (s.bin < 0) return false;                          // (only of the first histogram)
        const int bin = s.bin;
        above += s.above;
        __syncthreads();
        if (threadIdx.x == 0) { s.count = 0; s.key_lo = 0xffffffffu; s.key_hi = 0u; }
        __syncthreads();
        uint32_t least = 0xffffffffu, most = 0u;
        row.template each<2>([&](uint32_t (&u)[4], int) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float z = Vec<T>::get(u, i) + 0.f;
                if (bin_or_none(z) != bin) continue;
                const uint32_t k = order(z);
                least = min(least, k);
                most = max(most, k);
                const int at = atomicAdd(&s.count, 1);
                if (at < kList) { s.key[at] = k; s.weight[at] = kByWeight ? sc.weight(z) : 1ull; }
            }
        });
        least = __reduce_min_sync(0xffffffffu, least);
        most = __reduce_max_sync(0xffffffffu, most);
        if ((threadIdx.x & 31) == 0) { atomicMin(&s.key_lo, least); atomicMax(&s.key_hi, most); }
        __syncthreads();
        lo = s.key_lo; hi = s.key_hi;
        const int n = s.count;
        if (n <= kList || lo == hi) {
            // all pairs; a bin of one value is one pair
            for (int i = threadIdx.x; i < (lo == hi ? 1 : n); i += kThreads) {
                const u64 mine = s.key[i];
                u64 before = above, equal = 0;
                if (lo == hi) equal = s.weight[0] * u64(n);
                else
                    for (int j = 0; j < n; ++j) {
                        const u64 other = s.key[j], w = s.weight[j];
                        before += other > mine ? w : 0ull;
                        equal += other == mine ? w : 0ull;
                    }
                if (before < want && before + equal >= want) {        // (all tokens of that value write the same)
                    s.border_z = unorder(uint32_t(mine));
                    s.border_ties = uint32_t((want - before + s.weight[i] - 1) / s.weight[i]);
                }
            }
            __syncthreads();
            border = {s.border_z, s.border_ties};
            return true;
        }
        step = (hi - lo) / kBins + 1;
        __syncthreads();
    }
}

template <class T, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) sample_kernel(const SampleParams p) {
    constexpr int E = Vec<T>::E, kWarps = kThreads / 32;
    __shared__ Shared s;
    const int n = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Row<T> row(p.logits, n, p.K);
    grid_dependency_wait();
    grid_dependents_launch();
    const float temperature = p.temperature ? p.temperature[n] : 1.f;
    int k = p.top_k ? p.top_k[n] : 0;
    const float top_p = p.top_p ? p.top_p[n] : 1.f, min_p = p.min_p ? p.min_p[n] : 0.f;
    if (k < 0 || k >= p.K) k = 0;
    if (threadIdx.x < 16) s.table[threadIdx.x] = exp2(double(threadIdx.x) / 16.0) * double(1ull << p.bits);
    auto answer = [&](int token, float logprob) {
        p.token[n] = token;
        if (p.logprob) p.logprob[n] = logprob;
    };

    // ---- the maximum (NaN if there is one)
    uint32_t m = Vec<T>::kLeast;
    row.template each<4>([&](uint32_t (&u)[4], int) { m = Vec<T>::max2(m, Vec<T>::max2(Vec<T>::max2(u[0], u[1]), Vec<T>::max2(u[2], u[3]))); });
    const float mine = Vec<T>::top(m) + 0.f;                  // (of this thread's tokens)
    float top = mine;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = __uint_as_float(Vec<float>::max2(__float_as_uint(top), __float_as_uint(__shfl_xor_sync(0xffffffffu, top, o))));
    if (lane == 0) s.warp_z[warp] = top;
    __syncthreads();
    for (int i = 0; i < kWarps; ++i) top = __uint_as_float(Vec<float>::max2(__float_as_uint(top), __float_as_uint(s.warp_z[i])));
    if (top != top || top == -INFINITY || temperature != temperature) {
        if (threadIdx.x == 0) answer(-1, NAN);
        return;
    }
    if (temperature <= 0.f || k == 1 || top_p <= 0.f) {       // the first token that has the maximum
        uint32_t at = 0xffffffffu;
        if (mine == top)
            row.template each<2>([&](uint32_t (&u)[4], int c) {
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if (Vec<T>::get(u, i) == top) at = min(at, uint32_t(row.first(c) + i));
            });
        at = __reduce_min_sync(0xffffffffu, at);
        if (lane == 0) s.warp_word[warp] = at;
        __syncthreads();
        for (int i = 0; i < kWarps; ++i) at = min(at, s.warp_word[i]);
        if (threadIdx.x == 0) answer(int(at), 0.f);
        return;
    }
    const double inv = 1.0 / double(temperature);
    const double min_x = min_p > 0.f ? 16.0 * log2(fmin(double(min_p), 1.0)) : -INFINITY;                   // (NaN: no filter)
    const Scale sc{double(top), inv, inv * (16.0 * 1.4426950408889634074), double(1ull << p.bits), kLeastX, s.table, top == INFINITY};
    const double kept_x = fmax(kLeastX, min_x);               // of what the last filter keeps
    const bool by_p = top_p < 1.f;
    const float u = p.uniform[n];
    auto target_of = [&](u64 total) -> u64 {
        const u64 t = u > 0.f ? u64(double(fminf(u, 1.f - 0x1p-24f)) * double(total)) : 0ull;
        return t < total ? t : total - 1;
    };
    auto part_of = [&](u64 total) -> u64 {                     // the weight that top-p wants
        const double part = ceil(double(top_p) * double(total));
        return part < 1.0 ? 1ull : u64(part) < total ? u64(part) : total;
    };
    auto logprob_of = [&](float z, u64 total) {
        return float(sc.x(z) * (0.69314718055994530942 / 16.0) - log(double(total) / sc.unit));
    };

    // ---- small top-k
    if (k > 0 && k <= kThreads / 2) {
        // the k-th largest of the threads' maxima, from its highest bit down (0: fewer than k threads have a finite one)
        const uint32_t key = mine == -INFINITY ? 0u : order(mine);
        uint32_t bound = 0;
        for (int b = 31; b >= Vec<T>::kLowBit; --b) {
            const uint32_t next = bound | 1u << b;
            if (__syncthreads_count(key >= next) >= k) bound = next;
        }
        // (the bits of a negative value's key below kLowBit are ones: the bound may be a little low, which is as good)
        if (threadIdx.x == 0) s.count = 0;
        __syncthreads();
        if (key >= bound && mine > -INFINITY)
            row.template each<4>([&](uint32_t (&u4)[4], int c) {
                if (order(Vec<T>::top(Vec<T>::max2(Vec<T>::max2(u4[0], u4[1]), Vec<T>::max2(u4[2], u4[3]))) + 0.f) < bound) return;
#pragma unroll 1
                for (int i = 0; i < E; ++i) {
                    const float z = Vec<T>::get(u4, i) + 0.f;
                    if (z == -INFINITY || order(z) < bound) continue;
                    const int at = atomicAdd(&s.count, 1);
                    if (at < kList) { s.key[at] = u64(order(z)) << 32 | uint32_t(~uint32_t(row.first(c) + i)); s.weight[at] = sc.weight(z); }
                }
            });
        __syncthreads();
        const int count = s.count;
        if (count <= kList) {
            constexpr int kEach = kList / kThreads;
            u64 before[kEach], sum = 0;
            bool in[kEach];
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int i = threadIdx.x + e * kThreads;
                before[e] = 0;
                in[e] = false;
                if (i >= count) continue;
                const u64 me = s.key[i];
                int rank = 0;
                for (int j = 0; j < count; ++j)
                    if (s.key[j] > me) { ++rank; before[e] += s.weight[j]; }
                in[e] = rank < k;
                if (in[e]) sum += s.weight[i];
            }
            const u64 want = by_p ? part_of(block_sum<kThreads>(s, sum)) : ~0ull;
            sum = 0;
            u64 kept[kEach];
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int i = threadIdx.x + e * kThreads;
                kept[e] = 0;
                if (i >= count) continue;
                if (in[e] && before[e] < want) kept[e] = sc.weight(unorder(uint32_t(s.key[i] >> 32)), kept_x);
                s.weight[i] = kept[e];
                sum += kept[e];
            }
            const u64 total = block_sum<kThreads>(s, sum), target = target_of(total);
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int i = threadIdx.x + e * kThreads;
                if (i >= count || kept[e] == 0) continue;
                const uint32_t id = uint32_t(s.key[i]);        // (inverted: a larger one is an earlier token)
                u64 front = 0;
                for (int j = 0; j < count; ++j) front += uint32_t(s.key[j]) > id ? s.weight[j] : 0ull;
                if (front <= target && front + kept[e] > target) answer(int(~id), logprob_of(unorder(uint32_t(s.key[i] >> 32)), total));
            }
            return;
        }
        __syncthreads();
    }

    // ---- where the part kept ends
    Border border{-INFINITY, 0xffffffffu};
    const float floor_z = float(fmax(double(top) - 31.0 * double(temperature), -3.4028234663852886e38));        // (what has any weight lies above)
    if (k > 0) select<kThreads, false>(s, row, sc, top, sc.infinite ? INFINITY : floor_z, u64(k), border);     // (false: fewer have any weight)
    if (by_p) {
        u64 sum = 0;
        row.template each<2>([&](uint32_t (&u4)[4], int) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float z = Vec<T>::get(u4, i) + 0.f;
                if (z > border.z) sum += sc.weight(z);
            }
        });
        sum = block_sum<kThreads>(s, sum);
        if (border.ties != 0xffffffffu) sum += u64(border.ties) * sc.weight(border.z);
        const double share = (1.0 - double(top_p)) * double(sum) / sc.unit / double(p.K);
        // (a little lower, so that roundings exclude nothing)
        const double low = double(top) + double(temperature) * (log(share) - 1e-3) - 1e-6 * fabs(double(top));
        const float from = sc.infinite ? INFINITY : float(fmax(low, double(floor_z)));
        Border nucleus{-INFINITY, 0u};
        if (select<kThreads, true>(s, row, sc, top, from, part_of(sum), nucleus) ||
            select<kThreads, true>(s, row, sc, top, sc.infinite ? INFINITY : floor_z, part_of(sum), nucleus))      // (top_p next to 1)
            border = nucleus;
    }

    // ---- sums of what is kept, by pieces of consecutive ids: a warp takes a piece
    const int each = (row.vectors + 32 * kPieces / 2 - 1) / (32 * kPieces / 2);                // vectors of a piece per lane
    const int pieces = (row.vectors + 32 * each - 1) / (32 * each);
    __syncthreads();
    for (int q = warp; q < pieces; q += kWarps) {
        u64 sum = 0;
        uint32_t ties = 0;
        for (int o = 0; o < each; ++o) {
            const int c = (q * each + o) * 32 + lane;
            if (c >= row.vectors) break;
            uint32_t u4[4];
            row.load(c, u4);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float z = Vec<T>::get(u4, i) + 0.f;
                if (z > border.z) sum += sc.weight(z, kept_x);
                else if (z == border.z) ++ties;
            }
        }
        sum = warp_sum(sum);
        ties = __reduce_add_sync(0xffffffffu, ties);
        if (lane == 0) { s.piece[q] = sum; s.ties[q] = ties; }
    }
    __syncthreads();
    const u64 tie_weight = border.z > -INFINITY ? sc.weight(border.z, kept_x) : 0ull;
    const bool has = int(threadIdx.x) < pieces;
    const uint32_t my_ties = has ? s.ties[threadIdx.x] : 0u;
    uint32_t ties = my_ties, all_ties;
    u64 none = 0, none_all;
    block_scan<kThreads>(s, none, ties, none_all, all_ties);
    const uint32_t before_ties = ties - my_ties;               // in front of this thread's piece
    const uint32_t kept_ties = before_ties >= border.ties ? 0u : min(my_ties, border.ties - before_ties);
    const u64 here = has ? s.piece[threadIdx.x] + u64(kept_ties) * tie_weight : 0ull;
    u64 sum = here, total;
    uint32_t no_ties = 0, no_all;
    block_scan<kThreads>(s, sum, no_ties, total, no_all);
    const u64 target = target_of(total);
    if (here > 0 && sum > target && sum - here <= target) {
        s.found = threadIdx.x;
        s.found_weight = sum - here;                           // in front of the piece
        s.found_ties = before_ties;
    }
    __syncthreads();

    // ---- within the piece: a vector to a thread
    u64 done = s.found_weight;
    uint32_t done_ties = s.found_ties;
    const int c0 = s.found * each * 32, c1 = min(c0 + each * 32, row.vectors);
    for (int o = c0; o < c1; o += kThreads) {
        const int c = o + int(threadIdx.x);
        uint32_t u4[4] = {Vec<T>::kLeast, Vec<T>::kLeast, Vec<T>::kLeast, Vec<T>::kLeast};
        if (c < c1) row.load(c, u4);
        uint32_t own = 0, all_t;
#pragma unroll
        for (int i = 0; i < E; ++i) own += Vec<T>::get(u4, i) + 0.f == border.z ? 1u : 0u;
        uint32_t t = own;
        u64 nothing = 0, nothing_all;
        block_scan<kThreads>(s, nothing, t, nothing_all, all_t);
        t = done_ties + t - own;                               // ties in front of this vector
        u64 w[E], a = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float z = Vec<T>::get(u4, i) + 0.f;
            const bool tie = z == border.z;
            w[i] = z > border.z ? sc.weight(z, kept_x) : tie && t < border.ties ? tie_weight : 0ull;
            t += tie ? 1u : 0u;
            a += w[i];
        }
        u64 at = a, all;
        uint32_t x = 0, all_x;
        block_scan<kThreads>(s, at, x, all, all_x);
        at += done - a;                                        // in front of this vector
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (w[i] > 0 && at <= target && at + w[i] > target) answer(int(row.first(c) + i), logprob_of(Vec<T>::get(u4, i) + 0.f, total));
            at += w[i];
        }
        done += all;
        done_ties += all_t;
        if (done > target) break;
    }
}

template <class T>
int launch_sample(const SampleParams& p, cudaStream_t st) {
    // two blocks an SM overlap one's loads with the other's arithmetic; up to one row an SM, all threads go to it
    if (p.N <= device_sm_count()) return launch_chained(sample_kernel<T, 1024>, dim3(p.N), dim3(1024), 0, st, 1, p);
    return launch_chained(sample_kernel<T, 512>, dim3(p.N), dim3(512), 0, st, 1, p);
}

}  // namespace

size_t sample_tokens_workspace_bytes(int, int) { return 0; }

int launch_sample_tokens(const SampleArgs& a, void*, cudaStream_t st) {
    int log_k = 0;
    while ((1ll << log_k) < a.K) ++log_k;
    const SampleParams p{a.N, a.K, log_k > 18 ? 62 - log_k : kWeightBits, a.logits, a.uniform, a.temperature, a.top_p, a.min_p, a.top_k, a.token, a.logprob};
    LaunchScope scope(KID_SAMPLE, double(a.N) * a.K * dtype_bytes(a.type), st);
    switch (a.type) {
        case DT_F32: return launch_sample<float>(p, st);
        case DT_BF16: return launch_sample<__nv_bfloat16>(p, st);
        default: return launch_sample<__half>(p, st);
    }
}

}  // namespace pcl

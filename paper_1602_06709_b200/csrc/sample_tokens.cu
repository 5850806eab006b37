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
// A block takes a row (a cluster of blocks, where there are few rows and long ones); what it reads once it finds in L2 the next time.
//   Every row: the maximum, two 16-bit logits to an instruction.
//   Small top-k: the k-th largest of the threads' maxima is a bound that k tokens reach and few others; those go to a list in shared memory,
//     and everything else happens there, by comparing all pairs.
//   Top-p alone: a histogram over z says in which few bins the part kept ends, one pass takes the exact weights, and those bins' tokens go to the
//     list, where the exact border is found.
//   Whatever does not fit in the list: the value at the border is found by histograms of weights or counts, finer each time.
//   What is kept is summed by pieces of consecutive ids, and the piece in which the random number falls is searched.
// The cost is the weights', and the chains of dependent operations that they are: without a filter the 64-bit pipe is active for 38 % of the time and
// the issue slots are used for 59 %, top-p 18 and 60 %, so neither is the limit by itself; warps wait for fixed latencies, for each other at barriers
// and for loads.  Measured, 512 rows of 131072 bf16 logits (20.5 us to read): top-k 51 us, no filter 109, min-p 117, top-p 258-280, mixed 175 (about 160
// with masked tokens); one row of 32003: 9.5, 13, 14, 27 us; one of 131072: 13.5, 14, 15, 33.  Dear forms: top-k of 5000 in the 512 rows 340, top-p
// where few different values fill a bin (steps of 2: 727; all equal: 1230).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "pcl_internal.h"
#include "pcl_ptx.cuh"

namespace pcl {

namespace {

constexpr int kBins = 2048;
constexpr int kList = 4096;                  // tokens of the list
constexpr int kMostSmall = 1024;             // of them, at most, where all of them are compared with all
constexpr int kPairs = 512;                  // up to here they are compared pair by pair
constexpr int kPieces = 256;                 // pieces of consecutive ids, at most
constexpr int kWeightBits = 44;

struct SampleParams {
    int N, K, bits;                          // bits: a weight of 1 is 2^bits
    int ordered;                             // rows are taken in the order of falling cost
    int ranks;                               // blocks that share a row
    double reach;                            // how many temperatures below the largest a weight is 0
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
template <class T, bool kPart>
struct Row {
    static constexpr int E = Vec<T>::E;
    const T* base;                           // the row's first element
    const uint4* aligned;                    // vector 0
    int K, shift, vectors, first_whole;
    int from, to;                            // kPart: the vectors that this block works on
    unsigned whole;                          // vectors that are the row's altogether, from first_whole on
    __device__ __forceinline__ Row(const void* logits, size_t row, int k) : base(static_cast<const T*>(logits) + row * k), K(k) {
        shift = int(row * k % E);
        vectors = (K + shift + E - 1) / E;
        aligned = reinterpret_cast<const uint4*>(base - shift);
        first_whole = shift ? 1 : 0;
        const int last = (K + shift) % E ? vectors - 1 : vectors;
        whole = last > first_whole ? unsigned(last - first_whole) : 0u;
        from = 0;
        to = vectors;
    }
    __device__ __forceinline__ void part(int rank, int ranks) {
        const int each = (vectors + ranks - 1) / ranks;
        from = min(rank * each, vectors);
        to = min(from + each, vectors);
    }
    __device__ __forceinline__ int lo() const { return kPart ? from : 0; }
    __device__ __forceinline__ int hi() const { return kPart ? to : vectors; }
    __device__ __forceinline__ float value(int id) const {
        const uint32_t u[4] = {Vec<T>::load(base, id), 0u, 0u, 0u};
        return Vec<T>::get(u, 0);
    }
    __device__ __forceinline__ long first(int c) const { return long(c) * E - shift; }
    __device__ __forceinline__ void load(int c, uint32_t (&u)[4]) const {
        if (unsigned(c - first_whole) < whole) {
            const uint4 q = __ldg(aligned + c);
            u[0] = q.x; u[1] = q.y; u[2] = q.z; u[3] = q.w;
        } else {
            const long e = first(c);
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = Vec<T>::kLeast;
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (e + i >= 0 && e + i < K) Vec<T>::put(u, i, Vec<T>::load(base, e + i));
        }
    }
    __device__ __forceinline__ void load_whole(int c, uint32_t (&u)[4]) const {
        const uint4 q = __ldg(aligned + c);
        u[0] = q.x; u[1] = q.y; u[2] = q.z; u[3] = q.w;
    }
    // f(vector, its index) for every vector of the block, its threads side by side; kMany vectors are loaded before the first is used
    template <int kMany, class F>
    __device__ __forceinline__ void each(F&& f) const {
        const int n = int(blockDim.x), end = kPart ? min(first_whole + int(whole), to) : first_whole + int(whole);
        int c = (kPart ? max(first_whole, from) : first_whole) + int(threadIdx.x);
        uint32_t u[kMany][4];
        for (; c + (kMany - 1) * n < end; c += kMany * n) {
#pragma unroll
            for (int m = 0; m < kMany; ++m) load_whole(c + m * n, u[m]);
#pragma unroll
            for (int m = 0; m < kMany; ++m) f(u[m], c + m * n);
        }
#pragma unroll
        for (int m = 0; m < kMany - 1; ++m)
            if (c + m * n < end) load_whole(c + m * n, u[m]);
#pragma unroll
        for (int m = 0; m < kMany - 1; ++m)
            if (c + m * n < end) f(u[m], c + m * n);
        // the row's first and last vector, where they are not whole
        if (threadIdx.x < 2) {
            c = threadIdx.x ? vectors - 1 : 0;
            if (unsigned(c - first_whole) >= whole && c >= lo() && c < hi() && (threadIdx.x == 0 || vectors > 1)) {
                load(c, u[0]);
                f(u[0], c);
            }
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
    double top, per16;                       // the row's maximum, 16 log2(e) / temperature
    unsigned lowest;                         // first word of -768 / per16: 2^-48, which is 0 in the result
    uint32_t table;                          // (shared memory) 2^(i/16) * 2^bits, its exponent less by i/16 of a power of two
    __device__ __forceinline__ double root(int i) const {
        double v;
        asm("ld.shared.f64 %0, [%1];" : "=d"(v) : "r"(table + (i & 15) * 8));
        return v;
    }
    __device__ __forceinline__ double x(float z) const { return (double(z) - top) * per16; }
    // keep = false: 0.  (Not of +inf; what is not kept may be -inf or NaN.)
    __device__ __forceinline__ u64 weight(float z, bool keep = true) const {
        const double raw = double(z) - top;
        // (of negative numbers the one with the larger first word is the lower)
        const double d = __hiloint2double(int(keep ? min(unsigned(__double2hiint(raw)), lowest) : lowest), __double2loint(raw));
        const double t = fma(d, per16, 6755399441055744.0);
        const int i = __double2loint(t);
        const double r = fma(d, per16, 6755399441055744.0 - t);
        double p = fma(r, 0x1.5d893e58acc63p-30, 0x1.3b2c4ac7da565p-23);
        p = fma(r, p, 0x1.c6b08d6faa1bep-17);
        p = fma(r, p, 0x1.ebfbdff6988c8p-11);
        p = fma(r, p, 0x1.62e42fefa39efp-5);
        p = fma(r, p, 1.0);
        const double s = root(i);
        const double w = fma(__hiloint2double(__double2hiint(s) + (i << 16), __double2loint(s)), p, 4503599627370496.0);
        return u64(__double_as_longlong(w)) - 0x4330000000000000ull;
    }
    // The weights of N values (kAll: of all of them, -inf among them; else of those not below `from`), step by step for all of them: their chains of
    // dependent operations run side by side.  Each is 0x433 << 52 too large.
    template <int N, bool kAll>
    __device__ __forceinline__ void raw_weights(const float (&z)[N], float from, u64 (&w)[N]) const {
        double d[N], r[N], p[N];
        int i[N];
#pragma unroll
        for (int n = 0; n < N; ++n) d[n] = double(z[n]) - top;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const unsigned hi = min(unsigned(__double2hiint(d[n])), lowest);
            d[n] = __hiloint2double(int(kAll || z[n] >= from ? hi : lowest), __double2loint(d[n]));
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const double t = fma(d[n], per16, 6755399441055744.0);
            i[n] = __double2loint(t);
            r[n] = 6755399441055744.0 - t;
        }
#pragma unroll
        for (int n = 0; n < N; ++n) r[n] = fma(d[n], per16, r[n]);
#pragma unroll
        for (int n = 0; n < N; ++n) p[n] = fma(r[n], 0x1.5d893e58acc63p-30, 0x1.3b2c4ac7da565p-23);
#pragma unroll
        for (int n = 0; n < N; ++n) p[n] = fma(r[n], p[n], 0x1.c6b08d6faa1bep-17);
#pragma unroll
        for (int n = 0; n < N; ++n) p[n] = fma(r[n], p[n], 0x1.ebfbdff6988c8p-11);
#pragma unroll
        for (int n = 0; n < N; ++n) p[n] = fma(r[n], p[n], 0x1.62e42fefa39efp-5);
#pragma unroll
        for (int n = 0; n < N; ++n) p[n] = fma(r[n], p[n], 1.0);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const double s = root(i[n]);
            w[n] = u64(__double_as_longlong(fma(__hiloint2double(__double2hiint(s) + (i[n] << 16), __double2loint(s)), p[n], 4503599627370496.0)));
        }
    }
    static constexpr u64 kRaw = 0x4330000000000000ull;
};

struct Shared {
    uint32_t count[kBins], high[kBins];      // histogram: counts, or weights in two words
    u64 key[kList], weight[kList];           // list: order of the value above, ~id below
    u64 piece[kPieces];
    double table[16];
    u64 warp_sum[32];
    uint32_t warp_word[32];
    float warp_z[32];
    double warp_low[32], warp_high[32];
    uint32_t warp_count[32];
    int bin, last_bin, listed, found, token, border_id;
    u64 above, found_front;
    uint32_t key_lo, key_hi, ties;
    float border_z;
    u64 swap[2];                             // what this block tells the others of its cluster
};

// The blocks that share a row (one, or a cluster): what they tell each other.  Every block makes the same calls.
__device__ __forceinline__ u64 load_of(const u64* p, uint32_t rank) {
    u64 v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(map_to_cta(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t load_of(const uint32_t* p, uint32_t rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(map_to_cta(p, rank)) : "memory");
    return v;
}
template <bool kMany>
struct Team {
    Shared& s;
    uint32_t rank, ranks;
    int turn = 0;                            // (two words in turn: one barrier each is enough)
    __device__ __forceinline__ Team(Shared& shared, uint32_t r) : s(shared), rank(kMany ? cluster_ctarank() : 0u), ranks(kMany ? r : 1u) {}
    __device__ __forceinline__ void sync() const {
        if constexpr (kMany) cluster_sync_all();
        else __syncthreads();
    }
    // Before the first block that others do without, and before any block ends: what they read from each other has been read.
    __device__ __forceinline__ void part() const {
        if constexpr (kMany) cluster_sync_all();
    }
    __device__ __forceinline__ bool first() const { return !kMany || rank == 0; }
    // f over the blocks' values, in the blocks' order; before: over those of the blocks in front of this one
    template <class F>
    __device__ __forceinline__ u64 all(u64 mine, F&& f, u64* before = nullptr) {
        if (before) *before = 0;
        if constexpr (!kMany) return mine;
        if (threadIdx.x == 0) s.swap[turn] = mine;
        cluster_sync_all();
        u64 v = load_of(&s.swap[turn], 0);
        for (uint32_t r = 1; r < ranks; ++r) {
            if (before && r == rank) *before = v;
            v = f(v, load_of(&s.swap[turn], r));
        }
        turn ^= 1;
        return v;
    }
    __device__ __forceinline__ u64 sum(u64 mine, u64* before = nullptr) { return all(mine, [](u64 a, u64 b) { return a + b; }, before); }
    // A token to the first block's list.
    __device__ __forceinline__ void push(u64 key, u64 weight, int most) const {
        if constexpr (kMany) {
            uint32_t at;
            asm volatile("atom.shared::cluster.add.u32 %0, [%1], 1;" : "=r"(at) : "r"(map_to_cta(&s.listed, 0)) : "memory");
            if (int(at) >= most) return;
            asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(map_to_cta(&s.key[at], 0)), "l"(key) : "memory");
            asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(map_to_cta(&s.weight[at], 0)), "l"(weight) : "memory");
        } else {
            const int at = atomicAdd(&s.listed, 1);
            if (at < most) { s.key[at] = key; s.weight[at] = weight; }
        }
    }
    // a word of the first block, or of any
    template <class W>
    __device__ __forceinline__ W of(const W& word, uint32_t r = 0) const {
        if constexpr (kMany) return load_of(&word, r);
        else return word;
    }
    __device__ __forceinline__ int of(const int& word) const { return int(of(reinterpret_cast<const uint32_t&>(word))); }
    __device__ __forceinline__ float of(const float& word) const { return __uint_as_float(of(reinterpret_cast<const uint32_t&>(word))); }
};

// Where the part kept ends: tokens above `z` are kept, and of those equal to it the ones up to `id` (kAllIds: all of them).
constexpr int kAllIds = 0x7fffffff;
constexpr float kLowest = -3.4028234663852886e38f;
struct Border {
    float z;
    int id;
    __device__ __forceinline__ bool keeps(float v, int token) const { return v > z || (v == z && token <= id); }
};

__device__ __forceinline__ void add_weight(uint32_t* lo, uint32_t* hi, u64 w) {
    const uint32_t l = uint32_t(w), old = atomicAdd(lo, l);
    const uint32_t up = uint32_t(w >> 32) + (old + l < old ? 1u : 0u);
    if (up) atomicAdd(hi, up);
}

__device__ __forceinline__ u64 warp_sum(u64 a) {              // (of up to 2^63 in all)
    const uint32_t x = __reduce_add_sync(0xffffffffu, uint32_t(a) & 0xffffffu), y = __reduce_add_sync(0xffffffffu, uint32_t(a >> 24) & 0xffffffu),
                   z = __reduce_add_sync(0xffffffffu, uint32_t(a >> 48));
    return x + (u64(y) << 24) + (u64(z) << 48);
}
template <class V>
__device__ __forceinline__ V warp_scan(V a) {                 // inclusive
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V x = __shfl_up_sync(0xffffffffu, a, o);
        if (int(threadIdx.x & 31) >= o) a += x;
    }
    return a;
}
template <int kThreads>
__device__ __forceinline__ u64 block_sum(Shared& s, u64 a) {
    a = warp_sum(a);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s.warp_sum[threadIdx.x >> 5] = a;
    __syncthreads();
    return warp_sum((threadIdx.x & 31) < kThreads / 32 ? s.warp_sum[threadIdx.x & 31] : 0ull);
}
// Inclusive sums over the block's threads, in order; `words` of the block's warps.
template <int kThreads, class V>
__device__ __forceinline__ V block_scan(V* words, V a, V& all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    a = warp_scan(a);
    __syncthreads();
    if (lane == 31) words[warp] = a;
    __syncthreads();
    const V w = warp_scan(lane < kThreads / 32 ? words[lane] : V(0));
    all = __shfl_sync(0xffffffffu, w, 31);
    const V before = __shfl_sync(0xffffffffu, w, warp ? warp - 1 : 0);
    return warp ? a + before : a;
}

// The first bin up to which the histogram holds `want`: its index and what lies in front of it go to s.bin (-1: there is none) and s.above.
template <int kThreads>
__device__ __forceinline__ void find_bin(Shared& s, u64 want) {
    constexpr int kEach = kBins / kThreads;
    __syncthreads();
    if (threadIdx.x == 0) s.bin = -1;
    u64 w[kEach], a = 0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        w[i] = u64(s.high[kEach * threadIdx.x + i]) << 32 | s.count[kEach * threadIdx.x + i];
        a += w[i];
    }
    u64 before = block_scan<kThreads>(s.warp_sum, a, all) - a;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (before < want && before + w[i] >= want) { s.bin = kEach * threadIdx.x + i; s.above = before; }
        before += w[i];
    }
    __syncthreads();
}

// Sums of f(vector, its index) over pieces of consecutive ids: the vectors [c0, c1) in pieces of 32 * each, a warp to a piece at a time, to s.piece
// (kAdd: added to it).  The next vector is on its way while one is worked on.
template <int kThreads, bool kAdd = false, class T, bool kPart, class F>
__device__ __forceinline__ void sum_pieces(Shared& s, const Row<T, kPart>& row, int c0, int c1, int each, F&& f) {
    const int lane = threadIdx.x & 31, pieces = (c1 - c0 + 32 * each - 1) / (32 * each);
    int q = threadIdx.x >> 5, o = 0, c = c0 + q * each * 32 + lane;
    u64 sum = 0;
    uint32_t u[4], next[4];
    if (c < c1) row.load(c, next);
    while (q < pieces) {
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = next[i];
        const int at = c;
        const bool last = ++o == each;
        const int done = q;
        if (last) {
            o = 0;
            q += kThreads / 32;
            c = c0 + q * each * 32 + lane;
        } else {
            c += 32;
        }
        if (c < c1) row.load(c, next);
        if (at < c1) sum += f(u, at);
        if (last) {
            __syncwarp();
            sum = warp_sum(sum);
            if (lane == 0) s.piece[done] = kAdd ? s.piece[done] + sum : sum;
            sum = 0;
        }
    }
    __syncthreads();
}
// f of values and ids, one by one, as a function of a vector.
template <class T, bool kPart, class F>
__device__ __forceinline__ auto by_value(const Row<T, kPart>& row, F&& f) {
    return [&row, f](const uint32_t (&u)[4], int c) mutable -> u64 {
        const int id = int(row.first(c));
        u64 sum = 0;
#pragma unroll
        for (int i = 0; i < Vec<T>::E; ++i) sum += f(Vec<T>::get(u, i), id + i);
        return sum;
    };
}
// The weights of the values not below `from` (kAll: of all).
template <bool kAll, class T>
__device__ __forceinline__ u64 vector_weight(const Scale& sc, const uint32_t (&u)[4], float from) {
    u64 sum = 0;
#pragma unroll
    for (int i = 0; i < Vec<T>::E; i += 4) {
        float z[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = Vec<T>::get(u, i + j);
        u64 w[4];
        sc.template raw_weights<4, kAll>(z, from, w);
        sum += (w[0] + w[1]) + (w[2] + w[3]);
    }
    return sum - Vec<T>::E * Scale::kRaw;
}
// The id at which the sum of f over rising ids first exceeds `target`, given s.piece of the block's vectors.
template <int kThreads, class T, bool kPart, class F>
__device__ __forceinline__ int locate(Shared& s, const Row<T, kPart>& row, int each, u64 target, F&& f) {
    constexpr int E = Vec<T>::E;
    int c0 = row.lo(), c1 = row.hi();
    u64 front = 0;
    for (;;) {
        const int pieces = (c1 - c0 + 32 * each - 1) / (32 * each);
        const u64 mine = int(threadIdx.x) < pieces ? s.piece[threadIdx.x] : 0ull;
        u64 all;
        const u64 upto = front + block_scan<kThreads>(s.warp_sum, mine, all);
        if (mine > 0 && upto > target && upto - mine <= target) { s.found = threadIdx.x; s.found_front = upto - mine; }
        __syncthreads();
        c0 += s.found * each * 32;
        c1 = min(c0 + each * 32, c1);
        front = s.found_front;
        if (each <= 8) break;
        each = (each + kPieces - 1) / kPieces;                 // (long rows: the piece in pieces)
        sum_pieces<kThreads>(s, row, c0, c1, each, by_value(row, f));
    }
    if (threadIdx.x < 32) {                                    // a warp, 32 vectors at a time
        for (int c = c0 + threadIdx.x; c - int(threadIdx.x) < c1; c += 32) {
            uint32_t u[4] = {Vec<T>::kLeast, Vec<T>::kLeast, Vec<T>::kLeast, Vec<T>::kLeast};
            if (c < c1) row.load(c, u);
            const int id = int(row.first(c));
            u64 w[E], a = 0;
#pragma unroll
            for (int i = 0; i < E; ++i) { w[i] = c < c1 ? f(Vec<T>::get(u, i), id + i) : 0ull; a += w[i]; }
            const u64 upto = front + warp_scan(a);
            u64 at = upto - a;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                if (w[i] > 0 && at <= target && at + w[i] > target) s.token = id + i;
                at += w[i];
            }
            front = __shfl_sync(0xffffffffu, upto, 31);
            if (front > target) break;
        }
    }
    __syncthreads();
    return s.token;
}

// The value at which the tokens in falling order, down to `from`, reach `want` of weight, or of their number, and how many tokens of that
// value that takes; false: they do not.  For whatever does not fit in the list.
template <int kThreads, bool kByWeight, class T, bool kPart>
__device__ __noinline__ bool select(Shared& s, const Row<T, kPart>& row, const Scale& sc, float top, float from, u64 want, float& border, uint32_t& ties) {
    constexpr int E = Vec<T>::E;
    const float scale = float(kBins) / (top - from);          // (top == from: infinite, and every value then is in bin 0)
    auto bin_of = [&](float z) { const float b = (top - z) * scale; return b < float(kBins - 1) ? int(b) : b >= float(kBins - 1) ? kBins - 1 : 0; };
    uint32_t lo = 0, hi = 0, step = 0;                        // after the first histogram: bins of `step` keys from hi down to lo
    u64 above = 0;
    for (;;) {
        for (int i = threadIdx.x; i < kBins; i += kThreads) { s.count[i] = 0; s.high[i] = 0; }
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
                if (kByWeight) add_weight(&s.count[b], &s.high[b], sc.weight(z));
                else atomicAdd(&s.count[b], 1u);
            }
        });
        find_bin<kThreads>(s, want - above);
        if (s.bin < 0) return false;                          // (only of the first histogram)
        const int bin = s.bin;
        above += s.above;
        __syncthreads();
        if (threadIdx.x == 0) { s.listed = 0; s.key_lo = 0xffffffffu; s.key_hi = 0u; }
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
                const int at = atomicAdd(&s.listed, 1);
                if (at < kList) { s.key[at] = k; s.weight[at] = kByWeight ? sc.weight(z) : 1ull; }
            }
        });
        least = __reduce_min_sync(0xffffffffu, least);
        most = __reduce_max_sync(0xffffffffu, most);
        if ((threadIdx.x & 31) == 0) { atomicMin(&s.key_lo, least); atomicMax(&s.key_hi, most); }
        __syncthreads();
        lo = s.key_lo; hi = s.key_hi;
        const int n = s.listed;
        if (n <= kMostSmall || lo == hi) {
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
                    s.ties = uint32_t((want - before + s.weight[i] - 1) / s.weight[i]);
                }
            }
            __syncthreads();
            border = s.border_z;
            ties = s.ties;
            return true;
        }
        step = (hi - lo) / kBins + 1;
        __syncthreads();
    }
}

// The lowest finite value, not above `top`, for which f holds; f holds for `top` and for whatever lies above a value for which it does.  From a guess
// by steps that double, then halve.
template <class F>
__device__ __forceinline__ float lowest_with(float guess, float top, F&& f) {
    const uint32_t bottom = order(kLowest), most = order(top);
    const uint32_t at = min(max(order(guess), bottom), most);
    uint32_t lo = bottom - 1, hi = most;                      // the highest key without and the lowest with, from outside
    if (f(unorder(at))) {
        hi = at;
        for (uint32_t step = 1; hi > bottom && hi - bottom >= step; step *= 2) {
            if (!f(unorder(hi - step))) { lo = hi - step; break; }
            hi -= step;
        }
    } else {
        lo = at;
        for (uint32_t step = 1; hi - lo > step; step *= 2) {
            if (f(unorder(lo + step))) { hi = lo + step; break; }
            lo += step;
        }
    }
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (f(unorder(mid))) hi = mid;
        else lo = mid;
    }
    return unorder(hi);
}

// What top-p keeps of a row without top-k: the border, or false where the tokens near it do not fit in the list, or min-p keeps less (the border then
// is min-p's).  Leaves the sums of what is
// kept (and not below `least`) in s.piece, and the weight of the whole row in `total`.
//   A histogram over z from the top down to `from` counts tokens and adds up their places in the bins (to a 64th of a bin), which gives the weight
//   of each bin to 1 part in 4000; the border lies in the bins, one or two as a rule, where the weight up to there can be top_p of all.  One pass then
//   takes the exact weights: of all tokens, of those above these bins, and those in them go to the list, where the exact border is found.
constexpr int kCountBits = 13;               // of a bin's word; the rest holds the places
template <int kThreads, bool kMany, class T, bool kPart, class Part>
__device__ __forceinline__ bool nucleus(Shared& s, Team<kMany>& team, const Row<T, kPart>& row, const Scale& sc, float top, float from, double unit, float top_p, float least, int each,
                                        const Part& part_of, u64& total, Border& border) {
    constexpr int E = Vec<T>::E, kEach = kBins / kThreads;
    const float scale = float(kBins) / (top - from);
    const bool usable = scale > 0.f && scale < 1e30f;
    for (int i = threadIdx.x; i < kBins; i += kThreads) s.count[i] = 0;
    if (threadIdx.x == 0) { s.bin = kBins; s.last_bin = kBins - 1; }
    __syncthreads();
    uint32_t inside = 0;
    if (usable)
        row.template each<4>([&](uint32_t (&u)[4], int) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float z = Vec<T>::get(u, i);
                if (z >= from) {
                    const int place = min(int((top - z) * (scale * 64.f)), kBins * 64 - 1);       // in 64ths of a bin
                    atomicAdd(&s.count[place >> 6], 1u | uint32_t(place & 63) << kCountBits);
                    ++inside;
                }
            }
        });
    team.sync();
    // bounds of the weight up to each bin and of all of it: a token's place is known to 1/64 of a bin (and a rounding of 1/1000), and within a bin
    // exp(-f * width) lies between 1 - f width and that plus (f width)^2 / 2
    const double width = double(top - from) / kBins * sc.per16 * (0.69314718055994530942 / 16.0);       // of a bin, in nats
    double low = 0.0, high = 0.0, lows[kEach], highs[kEach], all_low, all_high;
    uint32_t counted = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int b = kEach * threadIdx.x + i;
        uint32_t n = 0, place = 0;
        for (uint32_t r = 0; r < team.ranks; ++r) {
            const uint32_t word = team.of(s.count[b], r);
            n += word & ((1u << kCountBits) - 1);
            place += word >> kCountBits;
        }
        counted += n;
        const double at = n ? unit * exp(-double(b) * width) : 0.0, places = double(place) * (1.0 / 64.0) * width;
        lows[i] = fmax(at * (double(n) - places - double(n) * width * (1.0 / 64.0 + 1e-3)) - double(n), 0.0);
        highs[i] = at * (double(n) - places + double(n) * (width * 1e-3 + 0.5 * width * width)) + double(n);      // (weights are whole numbers)
        if (b == kBins - 1) { lows[i] = 0.0; highs[i] = double(n) * (at * (1.0 + 1e-3 * width) + 1.0); }           // (the last bin may reach further down)
        low += lows[i];
        high += highs[i];
    }
    low = block_scan<kThreads>(s.warp_low, low, all_low) - low;
    high = block_scan<kThreads>(s.warp_high, high, all_high) - high;
    uint32_t all_counted, all_inside;
    block_scan<kThreads>(s.warp_word, counted, all_counted);
    block_scan<kThreads>(s.warp_count, inside, all_inside);
    all_inside = uint32_t(team.sum(all_inside));
    if (!usable || all_counted != all_inside) return false;    // (a bin's count has overflown)
    const double want_low = double(top_p) * all_low * (1.0 - 1e-9), want_high = double(top_p) * all_high * (1.0 + 1e-9) + 1.0;
    int first = kBins, last = kBins - 1;
    bool early = false, late = false;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        high += highs[i];
        low += lows[i];
        if (!early && high * (1.0 + 1e-9) >= want_low) { first = kEach * threadIdx.x + i; early = true; }
        if (!late && low * (1.0 - 1e-9) >= want_high) { last = kEach * threadIdx.x + i; late = true; }
    }
    first = __reduce_min_sync(0xffffffffu, first);
    last = __reduce_min_sync(0xffffffffu, last);
    if ((threadIdx.x & 31) == 0) { atomicMin(&s.bin, first); atomicMin(&s.last_bin, last); }
    __syncthreads();
    first = s.bin;
    last = s.last_bin;
    if (first > last) return false;                            // (not met: the bounds hold)
    // as bounds on the values: those from `over` on lie above the bins, those from `in` on above them or in them
    const float places = scale * 64.f, begin = float(first) * 64.f, end = float(last + 1) * 64.f;
    const float over = first == 0 ? INFINITY : lowest_with(top - begin / places, top, [&](float z) { return (top - z) * places < begin; });
    const float in = last == kBins - 1 ? from : fmaxf(from, lowest_with(top - end / places, top, [&](float z) { return (top - z) * places < end; }));
    if (least >= over) {                                       // min-p keeps less than what top-p keeps in any case
        border = {least, kAllIds};
        return false;
    }
    u64 above = 0, sum = 0;
    sum_pieces<kThreads>(s, row, row.lo(), row.hi(), each, [&](const uint32_t (&u)[4], int c) -> u64 {
        u64 kept = 0;
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            float z[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) z[j] = Vec<T>::get(u, i + j);
            u64 w[4];
            sc.template raw_weights<4, true>(z, 0.f, w);
            bool listed = false;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[j] -= Scale::kRaw;
                sum += w[j];
                kept += z[j] >= over ? w[j] : 0ull;
                listed |= z[j] >= in && z[j] < over;
            }
            if (listed) {
                const int id = int(row.first(c)) + i;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (z[j] >= in && z[j] < over) team.push(u64(order(z[j] + 0.f)) << 32 | uint32_t(~uint32_t(id + j)), w[j], kList);
            }
        }
        above += kept;
        return kept;
    });
    total = team.sum(block_sum<kThreads>(s, sum));
    above = team.sum(block_sum<kThreads>(s, above));
    const int n = team.of(s.listed);
    const u64 want = part_of(total);
    if (n > kList || above >= want) return false;              // (the second is not met)
    // the border: the key at which `want` is reached, for the first block to find
    if (!team.first()) {
    } else if (n <= kPairs) {
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const u64 mine = s.key[i];
            u64 before = above;
#pragma unroll 4
            for (int j = 0; j < n; ++j) before += s.key[j] > mine ? s.weight[j] : 0ull;
            if (before < want && before + s.weight[i] >= want) { s.border_z = unorder(uint32_t(mine >> 32)); s.border_id = int(~uint32_t(mine)); }
        }
    } else {                                                   // bit by bit: the highest key from which on, upwards, there is enough
        u64 key = 0;
        for (int b = 63; b >= 0; --b) {
            const u64 next = key | 1ull << b;
            u64 upto = 0;
            for (int i = threadIdx.x; i < n; i += kThreads) upto += s.key[i] >= next ? s.weight[i] : 0ull;
            if (above + block_sum<kThreads>(s, upto) >= want) key = next;
        }
        if (threadIdx.x == 0 && key) { s.border_z = unorder(uint32_t(key >> 32)); s.border_id = int(~uint32_t(key)); }
    }
    team.sync();
    border = {team.of(s.border_z), team.of(s.border_id)};
    if (border.id < 0) return false;                           // (not met)
    const u64 last_key = u64(order(border.z)) << 32 | uint32_t(~uint32_t(border.id));
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const u64 key = team.of(s.key[i]);
        const int c = (int(~uint32_t(key)) + row.shift) / E;
        if (key >= last_key && unorder(uint32_t(key >> 32)) >= least && c >= row.lo() && c < row.hi())
            atomicAdd(&s.piece[(c - row.lo()) / (32 * each)], team.of(s.weight[i]));
    }
    __syncthreads();
    return true;
}

// The row of this block where the costly rows come first (rows of one kind in their order): those with top-p and no small top-k, then those that
// need the weights of all tokens, then the others; a late costly row would leave the other SMs idle (512 x 131072, mixed settings: bf16 183 us in the
// order of the rows, 175 so, fp32 205 and 183; rows that all cost the same lose 2 us by it, 108 to 110).  Every block reads the settings of all rows for
// it, so that it is done only where a row is long next to their number: mixed bf16, 600 x 32000 68 us without and 61 with, 2000 x 131072 393 and 342, but
// 2000 x 32000 152 and 156, 8192 x 1000 with a temperature 203 and 463.
constexpr int kMostOrdered = 8192;           // (16 bits count the rows of a kind)
constexpr int kOrderedPerRow = 32;           // tokens of a row for each row of the call
template <int kThreads>
__device__ __forceinline__ int costly_first(Shared& s, const SampleParams& p) {
    const int each = (p.N + kThreads - 1) / kThreads, first = threadIdx.x * each, last = min(first + each, p.N);
    auto kind = [&](int n) {                                   // as a word of which 16 bits count the rows of a kind
        const int k = p.top_k ? p.top_k[n] : 0;
        const float q = p.top_p ? p.top_p[n] : 1.f;
        if ((p.temperature && !(p.temperature[n] > 0.f)) || q <= 0.f || (k > 0 && k <= kThreads / 2)) return 32;
        return (k > 0 && k < p.K) || q < 1.f ? 0 : 16;
    };
    u64 mine = 0, all;
    for (int n = first; n < last; ++n) mine += 1ull << kind(n);
    u64 before = block_scan<kThreads>(s.warp_sum, mine, all) - mine;
    const int kinds[3] = {0, int(all & 0xffff), int(all & 0xffff) + int(all >> 16 & 0xffff)};
    for (int n = first; n < last; ++n) {
        const int b = kind(n);
        if (kinds[b >> 4] + int(before >> b & 0xffff) == int(blockIdx.x)) s.found = n;
        before += 1ull << b;
    }
    __syncthreads();
    return s.found;
}

template <class T, int kThreads, bool kMany>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) sample_kernel(const SampleParams p) {
    constexpr int E = Vec<T>::E, kWarps = kThreads / 32;
    extern __shared__ __align__(16) uint8_t smem[];
    Shared& s = *reinterpret_cast<Shared*>(smem);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_dependency_wait();
    grid_dependents_launch();
    Team<kMany> team(s, uint32_t(p.ranks));
    const int n = p.ordered ? costly_first<kThreads>(s, p) : int(blockIdx.x / team.ranks);
    Row<T, kMany> row(p.logits, n, p.K);
    if constexpr (kMany) row.part(int(team.rank), int(team.ranks));
    if (threadIdx.x == 0) { s.listed = 0; s.border_id = -1; }
    const float temperature = p.temperature ? p.temperature[n] : 1.f;
    int k = p.top_k ? p.top_k[n] : 0;
    const float top_p = p.top_p ? p.top_p[n] : 1.f, min_p = p.min_p ? p.min_p[n] : 0.f, u = p.uniform[n];
    if (k < 0 || k >= p.K) k = 0;
    const u64 one = 1ull << p.bits;
    const double unit = double(one);
    if (threadIdx.x < 16) {
        const double v = exp2(double(threadIdx.x) / 16.0) * unit;
        s.table[threadIdx.x] = __hiloint2double(__double2hiint(v) - (int(threadIdx.x) << 16), __double2loint(v));
    }
    auto answer = [&](int token, float logprob) {
        p.token[n] = token;
        if (p.logprob) p.logprob[n] = logprob;
    };

    // ---- the maximum (NaN if there is one)
    uint32_t m = Vec<T>::kLeast;
    row.template each<4>([&](uint32_t (&q)[4], int) { m = Vec<T>::max2(m, Vec<T>::max2(Vec<T>::max2(q[0], q[1]), Vec<T>::max2(q[2], q[3]))); });
    const float mine = Vec<T>::top(m) + 0.f;                  // (of this thread's tokens)
    float top = mine;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = __uint_as_float(Vec<float>::max2(__float_as_uint(top), __float_as_uint(__shfl_xor_sync(0xffffffffu, top, o))));
    if (lane == 0) s.warp_z[warp] = top;
    __syncthreads();
    for (int i = 0; i < kWarps; ++i) top = __uint_as_float(Vec<float>::max2(__float_as_uint(top), __float_as_uint(s.warp_z[i])));
    top = __uint_as_float(uint32_t(team.all(__float_as_uint(top), [](u64 a, u64 b) { return u64(Vec<float>::max2(uint32_t(a), uint32_t(b))); })));
    if (top != top || top == -INFINITY || temperature != temperature) {
        if (threadIdx.x == 0 && team.first()) answer(-1, NAN);
        team.part();
        return;
    }
    if (temperature <= 0.f || k == 1 || top_p <= 0.f) {       // the first token that has the maximum
        uint32_t at = 0xffffffffu;
        if (mine == top)
            row.template each<4>([&](uint32_t (&q)[4], int c) {
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if (Vec<T>::get(q, i) == top) at = min(at, uint32_t(row.first(c) + i));
            });
        at = __reduce_min_sync(0xffffffffu, at);
        if (lane == 0) s.warp_word[warp] = at;
        __syncthreads();
        for (int i = 0; i < kWarps; ++i) at = min(at, s.warp_word[i]);
        at = uint32_t(team.all(at, [](u64 a, u64 b) { return a < b ? a : b; }));
        if (threadIdx.x == 0 && team.first()) answer(int(at), 0.f);
        team.part();
        return;
    }
    const double per16 = fmax(16.0 * 1.4426950408889634074 / double(temperature), 1e-290);         // (an infinite temperature: all weights 1)
    const Scale sc{double(top), per16, unsigned(__double2hiint(-768.0 / per16)), smem_u32(s.table)};
    const bool infinite = top == INFINITY, by_p = top_p < 1.f;
    auto target_of = [&](u64 total) -> u64 {
        const u64 t = u > 0.f ? u64(double(fminf(u, 1.f - 0x1p-24f)) * double(total)) : 0ull;
        return t < total ? t : total - 1;
    };
    auto part_of = [&](u64 total) -> u64 {                     // the weight that top-p wants
        const double part = ceil(double(top_p) * double(total));
        return part < 1.0 ? 1ull : u64(part) < total ? u64(part) : total;
    };
    auto logprob_of = [&](float z, u64 total) {
        return float((infinite ? 0.0 : sc.x(z) * (0.69314718055994530942 / 16.0)) - log(double(total) / unit));
    };
    // the lowest value that min-p keeps: x(z) >= 16 log2(min_p) (NaN: no filter)
    float least = kLowest;
    if (min_p > 0.f && !infinite) {
        const double min_x = 16.0 * log2(fmin(double(min_p), 1.0));
        least = lowest_with(float(fmax(double(top) + min_x / per16, double(kLowest))), top, [&](float v) { return sc.x(v) >= min_x; });
    }

    // ---- small top-k
    if (k > 0 && k <= kThreads / 2 && !infinite) {
        // the q-th largest of the threads' maxima, from its highest bit down, or a bound that few more reach (0: fewer than q are finite).  Of several
        // blocks: their share of k each, and the lowest of their bounds; where one has too few, k each and the highest.
        const uint32_t key = mine == -INFINITY ? 0u : order(mine);
        auto bound_of = [&](int q) {
            uint32_t found = 0;
            for (int b = 31; b >= Vec<T>::kLowBit; --b) {
                const uint32_t next = found | 1u << b;
                const int reach = __syncthreads_count(key >= next);
                if (reach >= q) found = next;
                if (reach >= q && reach <= q + 16) break;
            }
            return found;
        };
        uint32_t bound = bound_of((k + int(team.ranks) - 1) / int(team.ranks));
        if constexpr (kMany) {
            bound = uint32_t(team.all(bound, [](u64 a, u64 b) { return a < b ? a : b; }));
            if (bound == 0) bound = uint32_t(team.all(bound_of(k), [](u64 a, u64 b) { return a > b ? a : b; }));
        }
        // (the bits of a negative value's key below kLowBit are ones: the bound may be a little low, which is as good)
        __syncthreads();
        const float bound_z = bound > order(-INFINITY) ? unorder(bound) : kLowest;
        if (key >= bound && mine > -INFINITY)
            row.template each<4>([&](uint32_t (&q)[4], int c) {
                if (!(Vec<T>::top(Vec<T>::max2(Vec<T>::max2(q[0], q[1]), Vec<T>::max2(q[2], q[3]))) >= bound_z)) return;
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float z = Vec<T>::get(q, i);
                    if (z >= bound_z) team.push(u64(order(z + 0.f)) << 32 | uint32_t(~uint32_t(row.first(c) + i)), 0ull, kMostSmall);
                }
            });
        team.sync();
        const int count = team.of(s.listed);
        if (count <= kMostSmall) {
            team.part();
            if (!team.first()) return;
            constexpr int kEach = kMostSmall / kThreads;
            u64 before[kEach], sum = 0, kept[kEach];
            for (int i = threadIdx.x; i < count; i += kThreads) s.weight[i] = sc.weight(unorder(uint32_t(s.key[i] >> 32)));
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int i = threadIdx.x + e * kThreads;
                before[e] = kept[e] = 0;
                if (i >= count) continue;
                const u64 me = s.key[i];
                int rank = 0;
#pragma unroll 4
                for (int j = 0; j < count; ++j)
                    if (s.key[j] > me) { ++rank; before[e] += s.weight[j]; }
                if (rank < k) kept[e] = s.weight[i];
                sum += kept[e];
            }
            const u64 want = by_p ? part_of(block_sum<kThreads>(s, sum)) : ~0ull;
            sum = 0;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int i = threadIdx.x + e * kThreads;
                if (i >= count) continue;
                if (before[e] >= want || unorder(uint32_t(s.key[i] >> 32)) < least) kept[e] = 0;
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
#pragma unroll 4
                for (int j = 0; j < count; ++j) front += uint32_t(s.key[j]) > id ? s.weight[j] : 0ull;
                if (front <= target && front + kept[e] > target) answer(int(~id), logprob_of(unorder(uint32_t(s.key[i] >> 32)), total));
            }
            return;
        }
        __syncthreads();
    }

    // ---- where the part kept ends
    Border border{kLowest, kAllIds};
    bool summed = false;                                       // the pieces' sums are there
    const float floor_z = float(fmax(double(top) - p.reach * double(temperature), double(kLowest)));       // (what has any weight lies above)
    auto pieces_each = [&] { return (row.hi() - row.lo() + 32 * kPieces - 1) / (32 * kPieces); };        // vectors of a piece per lane
    u64 whole = 0;
    if (by_p && k == 0 && !infinite) summed = nucleus<kThreads>(s, team, row, sc, top, floor_z, unit, top_p, least, pieces_each(), part_of, whole, border);
    const bool by_least = least > kLowest && border.z == least;                                      // (min-p keeps less than top-p in any case)
    const bool alone = kMany && (infinite || k > 0 || (by_p && !summed && !by_least));               // what is rare or needs several passes is the first
    if (alone) {                                                                                     // block's
        team.part();
        if (!team.first()) return;
        row.part(0, 1);
    }
    const int each = pieces_each();
    auto nth_of = [&](float z, uint32_t ties) {                // the border at that many tokens of value z
        sum_pieces<kThreads>(s, row, row.lo(), row.hi(), each, by_value(row, [&](float v, int) -> u64 { return v == z ? 1ull : 0ull; }));
        const int id = locate<kThreads>(s, row, each, u64(ties) - 1, [&](float v, int) -> u64 { return v == z ? 1ull : 0ull; });
        __syncthreads();
        return Border{z, id};
    };
    if (infinite) {                                            // the tokens of +inf share everything
        u64 count = 0;
        row.template each<2>([&](uint32_t (&q)[4], int) {
#pragma unroll
            for (int i = 0; i < E; ++i) count += Vec<T>::get(q, i) == INFINITY ? 1 : 0;
        });
        count = block_sum<kThreads>(s, count);
        if (k > 0 && u64(k) < count) count = u64(k);
        if (by_p) count = (part_of(count * one) + one - 1) / one;
        border = nth_of(INFINITY, uint32_t(count));
    } else {
        float z = 0.f;
        uint32_t ties = 0;
        if (k > 0 && select<kThreads, false>(s, row, sc, top, floor_z, u64(k), z, ties)) border = nth_of(z, ties);     // (else fewer have any weight)
        if (by_p && !summed && !by_least) {
            __syncthreads();
            u64 sum = 0;
            row.template each<2>([&](uint32_t (&q)[4], int c) {
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float v = Vec<T>::get(q, i);
                    sum += sc.weight(v, border.keeps(v, int(row.first(c)) + i));
                }
            });
            sum = block_sum<kThreads>(s, sum);
            // what top-p can keep: not what weighs less than (1 - top_p) / K of the total, a little lower so that roundings exclude nothing
            const double share = (1.0 - double(top_p)) * double(sum) / unit / double(p.K);
            const double low = double(top) + double(temperature) * (log(share) - 1e-3) - 1e-6 * fabs(double(top));
            const float from = float(fmax(low, double(floor_z)));
            const u64 want = part_of(sum);
            if (select<kThreads, true>(s, row, sc, top, from, want, z, ties) || select<kThreads, true>(s, row, sc, top, floor_z, want, z, ties))
                border = nth_of(z, ties);                      // (the second: top_p next to 1)
        }
        if (least > border.z) border = {least, kAllIds};
    }

    // ---- the token
    auto kept_weight = [&](float v, int id) -> u64 { return infinite ? border.keeps(v, id) ? one : 0ull : sc.weight(v, border.keeps(v, id)); };
    if (!summed) {
        __syncthreads();
        if (infinite || border.id != kAllIds)
            sum_pieces<kThreads>(s, row, row.lo(), row.hi(), each, by_value(row, kept_weight));
        else if (border.z > kLowest)
            sum_pieces<kThreads>(s, row, row.lo(), row.hi(), each, [&](const uint32_t (&q)[4], int) { return vector_weight<false, T>(sc, q, border.z); });
        else
            sum_pieces<kThreads>(s, row, row.lo(), row.hi(), each, [&](const uint32_t (&q)[4], int) { return vector_weight<true, T>(sc, q, 0.f); });
    }
    const u64 own = block_sum<kThreads>(s, int(threadIdx.x) < (row.hi() - row.lo() + 32 * each - 1) / (32 * each) ? s.piece[threadIdx.x] : 0ull);
    u64 front = 0;
    const u64 total = alone ? own : team.sum(own, &front), target = target_of(total);
    if (target >= front && target - front < own) {
        const int token = locate<kThreads>(s, row, each, target - front, kept_weight);
        if (threadIdx.x == 0) answer(token, logprob_of(row.value(token), total));
    }
    if (!alone) team.part();
}

template <class T, int kThreads, bool kMany>
int launch_threads(const SampleParams& p, cudaStream_t st) {
    static PerDeviceOnce once;
    auto kernel = sample_kernel<T, kThreads, kMany>;
    const int rc = once.run([&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(sizeof(Shared))) == cudaSuccess ? PCL_OK : PCL_ERR_CUDA;
    });
    return rc != PCL_OK ? rc : launch_chained(kernel, dim3(unsigned(p.N) * p.ranks), dim3(kThreads), sizeof(Shared), st, unsigned(p.ranks), p);
}
template <class T>
int launch_sample(const SampleParams& p, cudaStream_t st) {
    // Two blocks an SM overlap one's loads with the other's arithmetic.  Up to one row an SM, all threads go to it; with fewer and long rows a cluster of
    // up to 8 SMs does, each with 16384 tokens or more (below that what the blocks tell each other costs more than it saves: 1 x 32003 by top-k
    // 9.5 us on one SM, 12.5 on four; 1 x 131072 without a filter 28.7 on one, 14.1 on eight).  Clusters of 8 fill half of the SMs at most: more do not
    // find their 8 next to each other at once (16 x 131072: 27 us on clusters of 8, 17 on 30 clusters of 4).
    const int sms = device_sm_count();
    SampleParams q = p;
    q.ranks = 1;
    if (p.N <= sms) {
        while (q.ranks < 8 && p.N * q.ranks * 2 <= (q.ranks < 4 ? sms : sms / 2) && p.K / (q.ranks * 2) >= 16384) q.ranks *= 2;
        return q.ranks > 1 ? launch_threads<T, 1024, true>(q, st) : launch_threads<T, 1024, false>(q, st);
    }
    q.ordered = p.N > 2 * sms && p.N <= kMostOrdered && long(p.K) >= long(kOrderedPerRow) * p.N && (p.top_k || p.top_p || p.temperature);
    return launch_threads<T, 512, false>(q, st);
}

}  // namespace

size_t sample_tokens_workspace_bytes(int, int) { return 0; }

int launch_sample_tokens(const SampleArgs& a, void*, cudaStream_t st) {
    int log_k = 0;
    while ((1ll << log_k) < a.K) ++log_k;
    const int bits = log_k > 18 ? 62 - log_k : kWeightBits;
    // weights are rounded to the nearest 2^-bits, so they end (bits + 1) ln 2 below the largest (and a margin for roundings on the way)
    const SampleParams p{a.N, a.K, bits, 0, 1, 0.69314718055994530942 * (bits + 1) + 0.05, a.logits, a.uniform, a.temperature, a.top_p, a.min_p, a.top_k, a.token, a.logprob};
    LaunchScope scope(KID_SAMPLE, double(a.N) * a.K * dtype_bytes(a.type), st);
    switch (a.type) {
        case DT_F32: return launch_sample<float>(p, st);
        case DT_BF16: return launch_sample<__nv_bfloat16>(p, st);
        default: return launch_sample<__half>(p, st);
    }
}

}  // namespace pcl

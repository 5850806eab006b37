// One token of each row of logits: temperature, top-k, top-p and min-p, from a given random number.
//
//   d = (z - max z) / temperature,  weight = exp(d).  In the order of falling z (equal ones: rising id) the filters keep a first part of the
//   row: top_k tokens; of them those in front of which lies less than top_p of their weight; those with d >= log(min_p).
//   Among the kept, in the order of their ids, the first whose cumulated weight exceeds uniform times the total.
//
// Which token that is depends on sums over up to all tokens, next to which one token's weight can be tiny: weights are taken
// in 64 bits and held as whole numbers of 2^-44 (less for rows of more than 2^18), so that sums do not depend on the order of
// additions and the histograms can be built with atomics.
//
// A block takes a row.  A first pass finds the maximum.  With top-k or top-p a histogram over d, of counts and of weights, says in
// which bin the part kept ends; the bin is divided again, by the bits of its values, until one value is left; then counts say how many
// tokens of that value are kept.  The last pass sums what is kept by pieces of consecutive ids, and the piece in which the random
// number falls is searched.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "pcl_internal.h"
#include "pcl_ptx.cuh"

namespace pcl {

namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 2048;
constexpr int kWeightBits = 44;
constexpr double kFloor = -30.5;             // log(2^-44): what lies lower has weight 0

struct SampleParams {
    int N, K, bits;                          // bits: a weight of 1 is 2^bits
    const void* logits;
    const float *uniform, *temperature, *top_p, *min_p;
    const int* top_k;
    int* token;
    float* logprob;
};

using u64 = unsigned long long;

template <class T> __device__ __forceinline__ float logit(const T* p);
template <> __device__ __forceinline__ float logit(const float* p) { return *p + 0.f; }                 // (-0 is 0)
template <> __device__ __forceinline__ float logit(const __nv_bfloat16* p) { return __bfloat162float(*p) + 0.f; }
template <> __device__ __forceinline__ float logit(const __half* p) { return __half2float(*p) + 0.f; }

// Bits that order like the values.
__device__ __forceinline__ uint32_t order(float z) {
    const uint32_t b = __float_as_uint(z);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unorder(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

struct Scale {
    double top, inv;                         // the row's maximum, 1 / temperature
    double unit;                             // 2^bits
    __device__ __forceinline__ double d(float z) const {
        return double(z) == top ? 0.0 : z == -INFINITY ? -INFINITY : (double(z) - top) * inv;        // (infinite maxima and temperatures)
    }
    __device__ __forceinline__ u64 weight(double dv) const { return dv >= kFloor ? __double2ull_rn(exp(dv) * unit) : 0ull; }      // (NaN: 0)
};
__device__ __forceinline__ int bin_of(double dv) {           // 0 at the maximum; monotone in z
    const int b = int(float(-dv) * float(kBins / 30.5));
    return b < kBins ? b : kBins - 1;
}

struct Shared {
    uint32_t count[kBins], lo[kBins], hi[kBins];             // histogram: tokens, and their weights in two words
    u64 sum[kThreads];                                       // scan of bins or pieces
    uint32_t ties[kThreads];
    u64 warp_sum[kWarps];
    uint32_t warp_word[kWarps];
    float warp_z[kWarps];
    int bin;
    u64 above_weight, bin_weight;
    uint32_t above_count, bin_count;
    uint32_t key_lo, key_hi;
    int found;
    u64 found_weight;
    int found_at;
};

__device__ __forceinline__ u64 shfl_up64(u64 v, int o) { return __shfl_up_sync(0xffffffffu, v, o); }
// Inclusive sums over the block's threads (in order) of two numbers; every thread also gets the totals.
__device__ __forceinline__ void block_scan(Shared& s, u64& a, uint32_t& c, u64& all_a, uint32_t& all_c) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 x = shfl_up64(a, o);
        const uint32_t y = __shfl_up_sync(0xffffffffu, c, o);
        if (lane >= o) { a += x; c += y; }
    }
    __syncthreads();
    if (lane == 31) { s.warp_sum[warp] = a; s.warp_word[warp] = c; }
    __syncthreads();
    u64 before = 0;
    uint32_t before_c = 0;
    all_a = 0; all_c = 0;
    for (int i = 0; i < kWarps; ++i) {
        if (i == warp) { before = all_a; before_c = all_c; }
        all_a += s.warp_sum[i];
        all_c += s.warp_word[i];
    }
    a += before;
    c += before_c;
}

__device__ __forceinline__ void add_to_bin(Shared& s, int b, u64 w) {
    atomicAdd(&s.count[b], 1u);
    const uint32_t lo = uint32_t(w), old = atomicAdd(&s.lo[b], lo);
    const uint32_t up = uint32_t(w >> 32) + (old + lo < old ? 1u : 0u);
    if (up) atomicAdd(&s.hi[b], up);
}
__device__ __forceinline__ void clear_bins(Shared& s) {
    for (int i = threadIdx.x; i < kBins; i += kThreads) { s.count[i] = 0; s.lo[i] = 0; s.hi[i] = 0; }
    __syncthreads();
}
// The first bin up to which there are `want_count` tokens, or (by_weight) weights of `want_weight`; -1: there is none.  Leaves what lies in
// front of it and in it in s.
__device__ __forceinline__ void find_bin(Shared& s, bool by_weight, uint32_t want_count, u64 want_weight) {
    __syncthreads();
    if (threadIdx.x == 0) s.bin = -1;
    const int b0 = 2 * threadIdx.x;
    u64 w[2];
    uint32_t c[2];
    for (int i = 0; i < 2; ++i) { w[i] = u64(s.hi[b0 + i]) << 32 | s.lo[b0 + i]; c[i] = s.count[b0 + i]; }
    u64 a = w[0] + w[1], all_a;
    uint32_t n = c[0] + c[1], all_n;
    block_scan(s, a, n, all_a, all_n);
    a -= w[0] + w[1];
    n -= c[0] + c[1];
    for (int i = 0; i < 2; ++i) {
        const bool before = by_weight ? a < want_weight : n < want_count;
        const bool reached = by_weight ? a + w[i] >= want_weight : n + c[i] >= want_count;
        if (before && reached) { s.bin = b0 + i; s.above_weight = a; s.above_count = n; s.bin_weight = w[i]; s.bin_count = c[i]; }
        a += w[i];
        n += c[i];
    }
    __syncthreads();
}

// Where the part kept ends: tokens above `z` are kept, and of those equal to it the first `ties` by id.
struct Border { float z; uint32_t ties; };

// The value at which the count or the weight is reached, within the first histogram's bin in s (found by find_bin); weight: what is kept up
// to the border.
template <class T>
__device__ __forceinline__ Border descend(Shared& s, const SampleParams& p, const T* z, const Scale& sc, bool by_weight, uint32_t want_count,
                                          u64 want_weight, u64& weight) {
    const int first_bin = s.bin;
    u64 above = s.above_weight;
    uint32_t above_n = s.above_count;
    // the range of the bin's values
    __syncthreads();
    if (threadIdx.x == 0) { s.key_lo = 0xffffffffu; s.key_hi = 0u; }
    __syncthreads();
    uint32_t lo = 0xffffffffu, hi = 0u;
    for (int i = threadIdx.x; i < p.K; i += kThreads) {
        const float v = logit(z + i);
        const double dv = sc.d(v);
        if (dv >= kFloor && bin_of(dv) == first_bin) { lo = min(lo, order(v)); hi = max(hi, order(v)); }
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if ((threadIdx.x & 31) == 0) { atomicMin(&s.key_lo, lo); atomicMax(&s.key_hi, hi); }
    __syncthreads();
    lo = s.key_lo; hi = s.key_hi;
    for (;;) {
        const uint32_t step = (hi - lo) / kBins + 1;
        clear_bins(s);
        for (int i = threadIdx.x; i < p.K; i += kThreads) {
            const float v = logit(z + i);
            const uint32_t k = order(v);
            if (k >= lo && k <= hi) add_to_bin(s, int((hi - k) / step), sc.weight(sc.d(v)));
        }
        find_bin(s, by_weight, want_count - above_n, want_weight - above);
        above += s.above_weight;
        above_n += s.above_count;
        hi -= uint32_t(s.bin) * step;
        if (step == 1) {
            const float v = unorder(hi);
            const u64 one = sc.weight(sc.d(v));
            const uint32_t ties = by_weight ? (one ? uint32_t((want_weight - above + one - 1) / one) : s.bin_count) : want_count - above_n;
            weight = above + u64(ties) * one;
            __syncthreads();
            return {v, ties};
        }
        lo = hi - lo < step ? lo : hi - (step - 1);
        __syncthreads();
    }
}

template <class T>
__global__ void __launch_bounds__(kThreads, 1) sample_kernel(const SampleParams p) {
    __shared__ Shared s;
    const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_dependency_wait();
    grid_dependents_launch();
    const T* z = static_cast<const T*>(p.logits) + size_t(row) * p.K;
    const float temperature = p.temperature ? p.temperature[row] : 1.f;
    int k = p.top_k ? p.top_k[row] : 0;
    const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
    if (k < 0 || k > p.K) k = 0;

    // ---- the maximum, and the first token that has it
    float top = -INFINITY;
    int at = 0x7fffffff;
    bool bad = temperature != temperature;
    for (int i = threadIdx.x; i < p.K; i += kThreads) {
        const float v = logit(z + i);
        bad |= v != v;
        if (v > top) { top = v; at = i; }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const float v = __shfl_xor_sync(0xffffffffu, top, o);
        const int i = __shfl_xor_sync(0xffffffffu, at, o);
        if (v > top || (v == top && i < at)) { top = v; at = i; }
    }
    if (lane == 0) { s.warp_z[warp] = top; s.warp_word[warp] = uint32_t(at); }
    bad = __syncthreads_or(bad);
    for (int i = 0; i < kWarps; ++i)
        if (s.warp_z[i] > top || (s.warp_z[i] == top && int(s.warp_word[i]) < at)) { top = s.warp_z[i]; at = int(s.warp_word[i]); }
    if (bad || top == -INFINITY) {
        if (threadIdx.x == 0) {
            p.token[row] = -1;
            if (p.logprob) p.logprob[row] = NAN;
        }
        return;
    }
    if (temperature <= 0.f || k == 1 || top_p <= 0.f) {
        if (threadIdx.x == 0) {
            p.token[row] = at;
            if (p.logprob) p.logprob[row] = 0.f;
        }
        return;
    }
    const Scale sc{double(top), 1.0 / double(temperature), double(1ull << p.bits)};

    // ---- where the part kept ends
    Border border{-INFINITY, 0xffffffffu};
    const bool by_k = k > 0 && k < p.K, by_p = top_p < 1.f;
    if (by_k || by_p) {
        clear_bins(s);
        for (int i = threadIdx.x; i < p.K; i += kThreads) {
            const double dv = sc.d(logit(z + i));
            if (dv >= kFloor) add_to_bin(s, bin_of(dv), sc.weight(dv));
        }
        __syncthreads();
        u64 total = 0;
        {
            const int b0 = 2 * threadIdx.x;
            u64 a = (u64(s.hi[b0]) << 32 | s.lo[b0]) + (u64(s.hi[b0 + 1]) << 32 | s.lo[b0 + 1]);
            uint32_t none = 0, n;
            block_scan(s, a, none, total, n);
        }
        bool rebuilt = false;
        if (by_k) {
            find_bin(s, false, uint32_t(k), 0);
            if (s.bin >= 0) {                                  // (else fewer than k have any weight)
                border = descend(s, p, z, sc, false, uint32_t(k), 0, total);
                rebuilt = true;
            }
        }
        if (by_p) {
            const double part = ceil(double(top_p) * double(total));
            const u64 want = part < 1.0 ? 1ull : u64(part) < total ? u64(part) : total;
            if (rebuilt) {
                clear_bins(s);
                for (int i = threadIdx.x; i < p.K; i += kThreads) {
                    const double dv = sc.d(logit(z + i));
                    if (dv >= kFloor) add_to_bin(s, bin_of(dv), sc.weight(dv));
                }
            }
            find_bin(s, true, 0, want);
            border = descend(s, p, z, sc, true, 0, want, total);
        }
    }
    const double least = min_p > 0.f ? log(fmin(double(min_p), 1.0)) : -INFINITY;         // (NaN: no filter)
    auto weight_of = [&](float v) {
        const double dv = sc.d(v);
        return dv >= least ? sc.weight(dv) : 0ull;
    };

    // ---- sums of what is kept, by pieces of consecutive ids: a warp takes a piece
    const int piece = (p.K + kThreads * 32 - 1) / (kThreads * 32) * 32;
    __syncthreads();
    s.sum[threadIdx.x] = 0;
    s.ties[threadIdx.x] = 0;
    __syncthreads();
    for (int q = warp; q < kThreads && size_t(q) * piece < size_t(p.K); q += kWarps) {
        u64 sum = 0;
        uint32_t ties = 0;
        for (int i = lane; i < piece; i += 32) {
            const size_t e = size_t(q) * piece + i;
            if (e >= size_t(p.K)) break;
            const float v = logit(z + e);
            if (v > border.z) sum += weight_of(v);
            else if (v == border.z) ++ties;
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        ties = __reduce_add_sync(0xffffffffu, ties);
        if (lane == 0) { s.sum[q] = sum; s.ties[q] = ties; }
    }
    __syncthreads();
    const u64 tie_weight = weight_of(border.z);
    uint32_t mine = s.ties[threadIdx.x], ties = mine, all_ties;
    u64 none = 0, none_all;
    block_scan(s, none, ties, none_all, all_ties);
    const uint32_t before_ties = ties - mine;                  // in front of this thread's piece
    const uint32_t kept = before_ties >= border.ties ? 0u : min(mine, border.ties - before_ties);
    const u64 here = s.sum[threadIdx.x] + u64(kept) * tie_weight;
    u64 sum = here, total;
    uint32_t no_ties = 0, no_all;
    block_scan(s, sum, no_ties, total, no_all);
    const float u = p.uniform[row];
    u64 target = u > 0.f ? u64(double(fminf(u, 1.f - 0x1p-24f)) * double(total)) : 0ull;
    if (target >= total) target = total - 1;
    if (here > 0 && sum > target && sum - here <= target) {
        s.found = threadIdx.x;
        s.found_weight = sum - here;                           // in front of the piece
        s.above_count = before_ties;
    }
    __syncthreads();

    // ---- within the piece
    const size_t base = size_t(s.found) * piece;
    u64 done = s.found_weight;
    uint32_t done_ties = s.above_count;
    for (int o = 0; o < piece; o += kThreads) {
        const size_t e = base + o + threadIdx.x;
        const bool in = o + int(threadIdx.x) < piece && e < size_t(p.K);
        const float v = in ? logit(z + e) : -INFINITY;
        const bool tie = in && v == border.z;
        uint32_t t = tie ? 1u : 0u, all_t;
        u64 nothing = 0, nothing_all;
        block_scan(s, nothing, t, nothing_all, all_t);
        const bool keep = in && (v > border.z || (tie && done_ties + t <= border.ties));
        const u64 w = keep ? weight_of(v) : 0ull;
        u64 a = w, all;
        uint32_t x = 0, all_x;
        block_scan(s, a, x, all, all_x);
        if (w > 0 && done + a > target && done + a - w <= target) {
            p.token[row] = int(e);
            if (p.logprob) p.logprob[row] = float(sc.d(v) - log(double(total) / sc.unit));
        }
        done += all;
        done_ties += all_t;
        if (done > target) break;
    }
}

}  // namespace

size_t sample_tokens_workspace_bytes(int, int) { return 0; }

int launch_sample_tokens(const SampleArgs& a, void*, cudaStream_t st) {
    int log_k = 0;
    while ((1ll << log_k) < a.K) ++log_k;
    SampleParams p{a.N, a.K, log_k > 18 ? 62 - log_k : kWeightBits, a.logits, a.uniform, a.temperature, a.top_p, a.min_p, a.top_k, a.token, a.logprob};
    LaunchScope scope(KID_SAMPLE, double(a.N) * a.K * dtype_bytes(a.type), st);
    switch (a.type) {
        case DT_F32: return launch_chained(sample_kernel<float>, dim3(a.N), dim3(kThreads), 0, st, 1, p);
        case DT_BF16: return launch_chained(sample_kernel<__nv_bfloat16>, dim3(a.N), dim3(kThreads), 0, st, 1, p);
        default: return launch_chained(sample_kernel<__half>, dim3(a.N), dim3(kThreads), 0, st, 1, p);
    }
}

}  // namespace pcl

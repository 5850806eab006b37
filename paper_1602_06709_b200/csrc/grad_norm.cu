// Norm of many tensors as one vector, and what training does with it: clipped copies of them, or the clipped SGD step.
//
//   norm = sqrt(sum g^2),  f = min(1, max_norm / (norm + 1e-6));   out = f g   or   w <- w - lr f g
//
// Bound by memory: one launch reads the tensors, a second one reads them again and writes.  The work is cut into items of 16 KB that do not
// cross tensors; the blocks take them in turn, the second launch from the end, as the first one read that last (clipped copies of 20M fp32 elements
// 46 us from the front and 42 from the end, of 34M 75 and 71; nothing to be had for 133M, where L2 holds too small a part).  The tensors'
// addresses and sizes are kernel parameters, so a call needs no copy and can be captured.
//
// Every 64 bytes or so are squared and summed in fp32 and added up in 64 bits, in a fixed order; where an fp32 sum leaves the range in which it
// loses nothing, the same squares are taken in 64 bits.
//
// Measured, over several cards and runs: norm of 500M bf16 elements 145 us (6.9 TB/s), with clipped copies 487-496 (3 GB, 6.0-6.2 TB/s); clipped step of
// VGG-A's 133M fp32 parameters 333-340 us (2.1 GB, 6.3-6.4 TB/s); clipped copies of the DNN's 34M fp32 gradients 70.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "pcl_internal.h"
#include "pcl_ptx.cuh"

namespace pcl {

namespace {

constexpr int kBlock = 256;
constexpr int kVectors = 4;                                  // 16-byte vectors of an item per thread
constexpr unsigned kItemBytes = kBlock * kVectors * 16;
// Blocks of an SM, which the registers are shared out to: the sums and the step hold 32 registers of loads a thread, the clipped copy half of that
// (500M bf16: 3 blocks 487 us, 4 492, 5 486, 6 487; gradients of the DNN 72, 71, 70, 70; stores marked as streaming 495, items in the order of
// the sums 494).
constexpr int kBlocksPerSm = 4, kCopyBlocksPerSm = 5;
constexpr int kMostTensors = 640;                            // of a launch: its parameters are limited to 32 KB

// Tensors of a launch.  lead: elements between the 16-byte boundary below a gradient and its start; first: its first item.
template <int kMost> struct Tensors {
    int count;
    unsigned items;
    const void* g[kMost];
    void* out[kMost];
    unsigned long long n[kMost];
    unsigned first[kMost];
    unsigned char type[kMost], lead[kMost];
};

struct ApplyParams {
    const double* partial;
    int partials;
    float max_norm, lr;
    float* norm;
};

// Elements of a vector of type kType.
template <int kType> constexpr int kPer = kType == DT_F32 ? 4 : 8;
template <int kType>
__device__ __forceinline__ void unpack(const uint4& q, float (&v)[kPer<kType>]) {
    const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (kType == DT_F32) {
            v[i] = __uint_as_float(u[i]);
        } else if constexpr (kType == DT_BF16) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        } else {
            const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
            v[2 * i] = h.x;
            v[2 * i + 1] = h.y;
        }
    }
}
template <int kType>
__device__ __forceinline__ uint4 pack(const float (&v)[kPer<kType>]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (kType == DT_F32) {
            u[i] = __float_as_uint(v[i]);
        } else if constexpr (kType == DT_BF16) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            u[i] = *reinterpret_cast<const uint32_t*>(&h);
        } else {
            const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
            u[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}
// Element i of a vector as bits, and a vector of which only the elements [lo, hi) exist.
template <class P>
__device__ __forceinline__ uint4 load_some(const P* base, int type, int lo, int hi) {
    uint32_t u[4] = {0u, 0u, 0u, 0u};
    if (type == DT_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i >= lo && i < hi) u[i] = reinterpret_cast<const uint32_t*>(base)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= lo && i < hi) u[i / 2] |= uint32_t(reinterpret_cast<const uint16_t*>(base)[i]) << (16 * (i % 2));
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}
__device__ __forceinline__ void store_some(void* base, int type, const uint4& q, int lo, int hi) {
    const uint32_t u[4] = {q.x, q.y, q.z, q.w};
    if (type == DT_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i >= lo && i < hi) static_cast<uint32_t*>(base)[i] = u[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= lo && i < hi) static_cast<uint16_t*>(base)[i] = uint16_t(u[i / 2] >> (16 * (i % 2)));
    }
}

// Sum over the block, in a fixed order; every thread gets it.
__device__ __forceinline__ double block_sum(double s, double* words) {
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) words[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.0;
    for (int i = 0; i < kBlock / 32; ++i) s += words[i];
    return s;
}
__device__ __forceinline__ double sum_partials(const double* partial, int n, double* words) {
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += kBlock) s += __ldcg(partial + i);
    return block_sum(s, words);
}

template <int kMost>
__device__ __forceinline__ void find_tensor(const Tensors<kMost>& p, unsigned item, int& t) {      // (empty tensors have no items)
    while (t + 1 < p.count && item >= p.first[t + 1]) ++t;
    while (item < p.first[t]) --t;
}

// An item as a thread sees it: its vectors are first, first + kBlock, ... of the tensor, counted from the 16-byte boundary below its start.
struct Item {
    int type, lead, per;
    bool whole;                                               // every vector of the item is the tensor's altogether
    unsigned long long first, end;                            // end: the tensor's elements and those in front of it
};
template <int kMost>
__device__ __forceinline__ Item item_of(const Tensors<kMost>& p, unsigned item, int t) {
    Item v;
    v.type = p.type[t];
    v.lead = p.lead[t];
    v.per = v.type == DT_F32 ? 4 : 8;
    v.end = p.n[t] + v.lead;
    const unsigned long long vec = (unsigned long long)(item - p.first[t]) * (kBlock * kVectors);
    v.first = vec + threadIdx.x;
    v.whole = (vec > 0 || v.lead == 0) && (vec + kBlock * kVectors) * v.per <= v.end;
    return v;
}
// Which elements of a vector are the tensor's: [lo, hi).
struct Part { int lo, hi; };
__device__ __forceinline__ Part part_of(const Item& v, unsigned long long vec) {
    const unsigned long long e = vec * v.per;
    return {e < unsigned(v.lead) ? int(v.lead - e) : 0, e + v.per <= v.end ? v.per : e < v.end ? int(v.end - e) : 0};
}
// The item's vectors from `base` (a gradient, or what lies in the same way; aligned: on 16 bytes).
__device__ __forceinline__ void load_item(const Item& v, const char* base, bool aligned, uint4 (&q)[kVectors]) {
    if (v.whole && aligned) {
        const uint4* s = reinterpret_cast<const uint4*>(base) + v.first;
#pragma unroll
        for (int i = 0; i < kVectors; ++i) q[i] = s[i * kBlock];
    } else {
#pragma unroll
        for (int i = 0; i < kVectors; ++i) {
            const unsigned long long vec = v.first + i * kBlock;
            const Part e = part_of(v, vec);
            q[i] = e.lo == 0 && e.hi == v.per && aligned ? *reinterpret_cast<const uint4*>(base + vec * 16)
                                                         : load_some(base + vec * 16, v.type, e.lo, e.hi);
        }
    }
}
template <int kType>
__device__ __forceinline__ void add_squares(const uint4 (&q)[kVectors], double& total) {
    constexpr int E = kPer<kType>;
    float s[kVectors];
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
        float v[E];
        unpack<kType>(q[i], v);
        any |= q[i].x | q[i].y | q[i].z | q[i].w;
        s[i] = 0.f;
#pragma unroll
        for (int j = 0; j < E; ++j) s[i] = fmaf(v[j], v[j], s[i]);
    }
    const float sum = (s[0] + s[1]) + (s[2] + s[3]);
    static_assert(kVectors == 4, "four sums");
    if ((sum > 1e-28f && sum < 1e36f) || any == 0) {
        total += double(sum);
    } else {                                                  // squares that fp32 does not hold (or an infinity, or NaN)
#pragma unroll
        for (int i = 0; i < kVectors; ++i) {
            float v[E];
            unpack<kType>(q[i], v);
#pragma unroll 1
            for (int j = 0; j < E; ++j) total = fma(double(v[j]), double(v[j]), total);
        }
    }
}
template <int kMost>
__device__ __forceinline__ const char* base_of(const Tensors<kMost>& p, int t, const Item& v) { return static_cast<const char*>(p.g[t]) - v.lead * (16 / v.per); }

// The next item is on its way while one is worked on.
template <int kMost>
__global__ void __launch_bounds__(kBlock, kBlocksPerSm) sum_squares_kernel(const __grid_constant__ Tensors<kMost> p, double* partial) {
    __shared__ double words[kBlock / 32];
    grid_dependency_wait();
    grid_dependents_launch();
    double total = 0.0;
    int t = 0, type = 0;
    uint4 q[kVectors], next[kVectors];
    auto fetch = [&](unsigned item) {
        find_tensor(p, item, t);
        const Item v = item_of(p, item, t);
        type = v.type;
        load_item(v, base_of(p, t, v), true, next);
    };
    unsigned item = blockIdx.x;
    if (item < p.items) fetch(item);
    for (; item < p.items; item += gridDim.x) {
        const int now = type;
#pragma unroll
        for (int i = 0; i < kVectors; ++i) q[i] = next[i];
        if (p.items - item > gridDim.x) fetch(item + gridDim.x);
        if (now == DT_F32) add_squares<DT_F32>(q, total);
        else if (now == DT_BF16) add_squares<DT_BF16>(q, total);
        else add_squares<DT_F16>(q, total);
    }
    total = block_sum(total, words);
    if (threadIdx.x == 0) partial[blockIdx.x] = total;
}

__global__ void __launch_bounds__(kBlock) norm_kernel(const double* partial, int n, float* norm) {
    __shared__ double words[kBlock / 32];
    grid_dependency_wait();
    grid_dependents_launch();
    const double s = sum_partials(partial, n, words);
    if (threadIdx.x == 0) *norm = float(sqrt(s));
}

// out = factor g (the clipping factor), or w + factor g (-lr times it).
template <int kType, bool kSgd>
__device__ __forceinline__ void apply_item(const Item& v, char* out, bool aligned, const uint4 (&q)[kVectors], const uint4 (&w)[kVectors], float factor) {
    constexpr int E = kPer<kType>;
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
        float g[E], x[E];
        unpack<kType>(q[i], g);
        if (kSgd) unpack<kType>(w[i], x);
#pragma unroll
        for (int j = 0; j < E; ++j) g[j] = kSgd ? fmaf(factor, g[j], x[j]) : factor * g[j];
        const uint4 r = pack<kType>(g);
        const unsigned long long vec = v.first + i * kBlock;
        if (v.whole && aligned) {
            reinterpret_cast<uint4*>(out)[vec] = r;
        } else {
            const Part e = part_of(v, vec);
            if (e.lo == 0 && e.hi == E && aligned) reinterpret_cast<uint4*>(out)[vec] = r;
            else store_some(out + vec * 16, kType, r, e.lo, e.hi);
        }
    }
}
// kSgd: out are the weights, stepped in place; else out = f g.
template <int kMost, bool kSgd>
__global__ void __launch_bounds__(kBlock, kSgd ? kBlocksPerSm : kCopyBlocksPerSm) apply_kernel(const __grid_constant__ Tensors<kMost> p, const ApplyParams a) {
    __shared__ double words[kBlock / 32];
    grid_dependency_wait();
    grid_dependents_launch();
    const double norm = sqrt(sum_partials(a.partial, a.partials, words));
    const double ratio = double(a.max_norm) / (norm + 1e-6);
    const float f = ratio >= 1.0 ? 1.f : float(ratio);       // (a NaN stays one)
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = float(norm);
    const float factor = kSgd ? -a.lr * f : f;
    int t = p.count - 1;
    for (unsigned i0 = blockIdx.x; i0 < p.items; i0 += gridDim.x) {
        const unsigned item = p.items - 1 - i0;
        find_tensor(p, item, t);
        const Item v = item_of(p, item, t);
        char* out = static_cast<char*>(p.out[t]) - v.lead * (16 / v.per);
        const bool aligned = (reinterpret_cast<uintptr_t>(out) & 15) == 0;      // out lies like g: whole vectors there too
        uint4 q[kVectors], w[kVectors];
        load_item(v, base_of(p, t, v), true, q);
        if (kSgd) load_item(v, out, aligned, w);
        if (v.type == DT_F32) apply_item<DT_F32, kSgd>(v, out, aligned, q, w, factor);
        else if (v.type == DT_BF16) apply_item<DT_BF16, kSgd>(v, out, aligned, q, w, factor);
        else apply_item<DT_F16, kSgd>(v, out, aligned, q, w, factor);
    }
}

int most_partials() { return device_sm_count() * kBlocksPerSm; }         // of a launch

// Tensors [from, to) of the call.
template <int kMost>
void fill(Tensors<kMost>& p, const TensorListArgs& a, int from, int to) {
    p.count = 0;
    p.items = 0;
    for (int i = from; i < to; ++i) {
        if (a.sizes[i] == 0) continue;
        const int k = p.count++;
        const size_t es = dtype_bytes(a.types[i]);
        p.g[k] = a.grads[i];
        p.out[k] = a.out ? a.out[i] : nullptr;
        p.n[k] = a.sizes[i];
        p.type[k] = (unsigned char)a.types[i];
        p.lead[k] = (unsigned char)((reinterpret_cast<uintptr_t>(a.grads[i]) & 15) / es);
        p.first[k] = p.items;
        p.items += unsigned(((p.n[k] + p.lead[k]) * es + kItemBytes - 1) / kItemBytes);
    }
}

template <int kMost>
int launch_one(const TensorListArgs& a, int from, int to, bool apply, double* partial, int partials, int& blocks, cudaStream_t st) {
    Tensors<kMost> p;
    fill(p, a, from, to);
    const int most = device_sm_count() * (apply && !a.sgd ? kCopyBlocksPerSm : kBlocksPerSm);
    blocks = p.items < unsigned(most) ? int(p.items) : most;
    if (blocks == 0) {
        if (!apply || from > 0) return PCL_OK;
        blocks = 1;                                           // (the norm is written all the same)
    }
    if (!apply) return launch_chained(sum_squares_kernel<kMost>, dim3(blocks), dim3(kBlock), 0, st, 1, p, partial);
    const ApplyParams ap{partial, partials, a.max_norm, a.lr, a.norm};
    return a.sgd ? launch_chained(apply_kernel<kMost, true>, dim3(blocks), dim3(kBlock), 0, st, 1, p, ap)
                 : launch_chained(apply_kernel<kMost, false>, dim3(blocks), dim3(kBlock), 0, st, 1, p, ap);
}
// (a short list is a short parameter block: what a launch costs grows with it)
int launch_some(const TensorListArgs& a, int from, int to, bool apply, double* partial, int partials, int& blocks, cudaStream_t st) {
    if (to - from <= 32) return launch_one<32>(a, from, to, apply, partial, partials, blocks, st);
    if (to - from <= 128) return launch_one<128>(a, from, to, apply, partial, partials, blocks, st);
    return launch_one<kMostTensors>(a, from, to, apply, partial, partials, blocks, st);
}

}  // namespace

size_t grad_norm_workspace_bytes(int count) {
    return align_up(size_t((count + kMostTensors - 1) / kMostTensors) * most_partials() * sizeof(double), 256);
}

int launch_grad_norm(const TensorListArgs& a, void* ws, cudaStream_t st) {
    double* partial = static_cast<double*>(ws);
    double bytes = 0.0;
    for (int i = 0; i < a.count; ++i) bytes += double(a.sizes[i]) * dtype_bytes(a.types[i]);
    int partials = 0, blocks = 0;
    for (int from = 0; from < a.count; from += kMostTensors) {
        const int to = a.count - from < kMostTensors ? a.count : from + kMostTensors;
        LaunchScope scope(KID_GRAD_NORM, bytes, st);
        const int rc = launch_some(a, from, to, false, partial + partials, 0, blocks, st);
        if (rc != PCL_OK) return rc;
        partials += blocks;
    }
    if (!a.out) {
        LaunchScope scope(KID_GRAD_NORM, 0.0, st);
        return launch_chained(norm_kernel, dim3(1), dim3(kBlock), 0, st, 1, static_cast<const double*>(partial), partials, a.norm);
    }
    for (int from = 0; from < a.count; from += kMostTensors) {
        const int to = a.count - from < kMostTensors ? a.count : from + kMostTensors;
        LaunchScope scope(KID_GRAD_NORM, bytes * (a.sgd ? 3 : 2), st);
        const int rc = launch_some(a, from, to, true, partial, partials, blocks, st);
        if (rc != PCL_OK) return rc;
    }
    return PCL_OK;
}

}  // namespace pcl

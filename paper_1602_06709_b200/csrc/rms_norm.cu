// RMS norm of rows with the residual's addition, its 8-bit form and its gradient; 8-bit rows of a matrix.
//
//   h = x + residual,  y[c] = h[c] * r * w[c],  r = 1 / sqrt(mean(h^2) + eps)
//   dx = dh + r * (g - n * mean(g n)),  dw[c] = sum over the rows of dy[c] n[c],      g = dy w,  n = h r
//
// All of it is bound by memory.  A row is read once and stays in the registers of a group of threads: a group of 32 to 1024
// threads takes a row, in chunks of 16 bytes, up to kMaxChunks a thread; a block holds several groups, each group walks over rows, and
// the weights of its chunks stay in registers.  Chunks are counted in the flat tensor, not in the row, so that they are
// aligned whatever the row length: a row of odd length starts and ends inside a chunk, and those two are read and written
// element by element.  The distance between a group's rows is a multiple of a chunk's elements, so all of its rows start
// at the same place of a chunk and the weights (and the sums of dw) in its registers keep their columns.
// Rows too long for that (more than 32768 16-bit or 16384 fp32 elements; gradient: half of it) are walked over twice.
//
// Sums over a row are fp32 in a fixed tree.  h is rounded when it is stored, but the norm is that of the sum before rounding.  A row whose
// sum of squares leaves fp32's range is scaled by a power of two first.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <math.h>

#include "pcl_internal.h"
#include "pcl_ptx.cuh"

namespace pcl {

namespace {

constexpr float kLargestE4m3 = 448.f;
constexpr float kLeastScale = 1.17549435e-38f;      // 2^-126: the scale of a row of zeros (its inverse is finite)

template <class T> struct Elem;
template <> struct Elem<float> {
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
template <> struct Elem<__nv_bfloat16> {
    static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Elem<__half> {
    static __device__ __forceinline__ float get(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half put(float v) { return __float2half_rn(v); }
};

// 16 bytes of a tensor.
template <class T> struct alignas(16) Chunk {
    static constexpr int E = 16 / int(sizeof(T));
    T e[E];
    __device__ __forceinline__ void values(float (&v)[E]) const {
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = Elem<T>::get(e[i]);
    }
};
template <class T>
__device__ __forceinline__ Chunk<T> load_chunk(const T* p) {
    Chunk<T> c;
    *reinterpret_cast<uint4*>(&c) = *reinterpret_cast<const uint4*>(p);
    return c;
}
// Which elements of a chunk belong to the row: [lo, hi).
struct Span { int lo, hi; };
template <class T>
__device__ __forceinline__ Chunk<T> load_span(const T* p, Span s) {
    constexpr int E = Chunk<T>::E;
    if (s.lo == 0 && s.hi == E) return load_chunk(p);
    Chunk<T> c;
#pragma unroll
    for (int i = 0; i < E; ++i) c.e[i] = i >= s.lo && i < s.hi ? p[i] : Elem<T>::put(0.f);
    return c;
}
// The weights of a chunk that starts at column c (aligned only where rows start on chunks).
template <class T>
__device__ __forceinline__ Chunk<T> load_weights(const T* w, int c, Span s, int shift) {
    constexpr int E = Chunk<T>::E;
    if (shift == 0) return load_span(w + c, s);
    Chunk<T> v;
#pragma unroll
    for (int i = 0; i < E; ++i) v.e[i] = i >= s.lo && i < s.hi ? w[c + i] : Elem<T>::put(0.f);
    return v;
}
template <class T>
__device__ __forceinline__ void store_span(T* p, Span s, const float (&v)[Chunk<T>::E]) {
    constexpr int E = Chunk<T>::E;
    Chunk<T> c;
#pragma unroll
    for (int i = 0; i < E; ++i) c.e[i] = Elem<T>::put(v[i]);
    if (s.lo == 0 && s.hi == E) {
        *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&c);
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i >= s.lo && i < s.hi) p[i] = c.e[i];
    }
}
// E values as e4m3 bytes.
template <int E>
__device__ __forceinline__ void store_span_q8(uint8_t* p, Span s, const float (&v)[E]) {
    uint32_t q[E / 4];
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i], v[4 * i + 1]), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i + 2], v[4 * i + 3]), __NV_SATFINITE, __NV_E4M3);
        q[i] = lo | hi << 16;
    }
    if (s.lo == 0 && s.hi == E) {
        if constexpr (E == 8) *reinterpret_cast<uint2*>(p) = make_uint2(q[0], q[1]);
        else *reinterpret_cast<uint32_t*>(p) = q[0];
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i >= s.lo && i < s.hi) p[i] = uint8_t(q[i / 4] >> (8 * (i % 4)));
    }
}

// |v| as an integer that orders like it; NaN is above everything, so it survives a maximum.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// A group of threads that shares a row: whole warps, several groups to a block.  Reductions alternate between two sets of words, so that
// one barrier each is enough.
struct Group {
    int size, rank, index;       // threads, this thread's place, which group of the block
    float2* words;               // [2][32 warps] of the block
    int turn = 0;
    __device__ __forceinline__ void sync() const {
        if (size == int(blockDim.x)) __syncthreads();
        else named_barrier_sync(1 + index, size);
    }
    // The group's sum of a and maximum of m (in the same order for every thread).
    __device__ __forceinline__ void sum_and_max(float& a, uint32_t& m) {
#pragma unroll
        for (int o = 16; o; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
        m = __reduce_max_sync(0xffffffffu, m);
        if (size == 32) return;
        float2* slot = words + turn * 32 + index * (size >> 5);
        turn ^= 1;
        if ((rank & 31) == 0) slot[rank >> 5] = make_float2(a, __uint_as_float(m));
        sync();
        a = 0.f; m = 0;
        for (int i = 0; i < size >> 5; ++i) { a += slot[i].x; m = max(m, __float_as_uint(slot[i].y)); }
    }
    __device__ __forceinline__ float sum(float a) {
        uint32_t none = 0;
        sum_and_max(a, none);
        return a;
    }
};

enum RowMode { ROW_NORM = 0, ROW_NORM_Q8, ROW_QUANTIZE };

struct RowParams {
    int N, C, group;             // group: threads that share a row
    float eps;
    const void *x, *residual, *w;
    void *h, *y;
    float *scale, *rstd;
};

// The sum of squares left fp32's range, or lost all of its bits: the row times a power of two, with the values near 1, but no
// further up than eps times its square stays in range.
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((min(max(e, -126), 126) + 127) << 23); }
__device__ __forceinline__ int exponent(float v) { return (__float_as_int(v) >> 23) - 127; }      // of a positive number; -127: subnormal
__device__ __forceinline__ float row_rescale(uint32_t top, float eps) {
    const float t = __uint_as_float(top);
    if (!(t > 0.f) || t == INFINITY) return 1.f;              // (zeros, infinities and NaN stay what they are)
    const int up = -exponent(t);
    return power_of_two(eps > 0.f ? min(up, (100 - exponent(eps)) / 2) : up);
}
__device__ __forceinline__ bool out_of_range(float ss, float eps) { return !(ss < 1e38f) || (ss < 1e-24f && eps < 1e-20f); }

template <class T, int V, RowMode kMode>
__global__ void __launch_bounds__(1024) row_kernel(const RowParams p) {
    constexpr int E = Chunk<T>::E;
    __shared__ float2 words[64];
    Group g{p.group, int(threadIdx.x) % p.group, int(threadIdx.x) / p.group, words};
    const int groups = blockDim.x / p.group, total = groups * gridDim.x;
    int row = blockIdx.x * groups + g.index;
    const T* x = static_cast<const T*>(p.x);
    const T* res = static_cast<const T*>(p.residual);
    const T* w = static_cast<const T*>(p.w);
    const int shift = int((size_t(row) * p.C) % E);           // (of all of this group's rows)
    Span span[V];
    Chunk<T> weight[V];
    grid_dependency_wait();
    grid_dependents_launch();
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (g.rank + i * p.group) * E - shift;     // the chunk's first column
        span[i] = {c < 0 ? -c : 0, p.C - c < E ? (p.C - c > 0 ? p.C - c : 0) : E};
        if (kMode != ROW_QUANTIZE && row < p.N && span[i].hi > span[i].lo) weight[i] = load_weights(w, c, span[i], shift);
    }
    const float mean = 1.f / float(p.C);
    for (; row < p.N; row += total) {
        const size_t at = size_t(row) * p.C - shift;
        float v[V][E];
        float ss = 0.f;
        uint32_t top = 0;
        Chunk<T> a[V], b[V];
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (span[i].hi > span[i].lo) {
                const size_t o = at + size_t(g.rank + i * p.group) * E;
                a[i] = load_span(x + o, span[i]);
                if (kMode != ROW_QUANTIZE && res) b[i] = load_span(res + o, span[i]);
            }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (span[i].hi <= span[i].lo) continue;
            a[i].values(v[i]);
            if (kMode != ROW_QUANTIZE && res) {
                float r[E];
                b[i].values(r);
#pragma unroll
                for (int j = 0; j < E; ++j) v[i][j] += r[j];
                if (p.h) store_span(static_cast<T*>(p.h) + at + size_t(g.rank + i * p.group) * E, span[i], v[i]);
            }
            float wf[E];
            if (kMode == ROW_NORM_Q8) weight[i].values(wf);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                if (kMode != ROW_QUANTIZE) ss = fmaf(v[i][j], v[i][j], ss);
                if (kMode == ROW_NORM_Q8) top = max(top, magnitude(v[i][j] * wf[j]));
                if (kMode == ROW_QUANTIZE) top = max(top, magnitude(v[i][j]));
            }
        }
        g.sum_and_max(ss, top);
        float r = 1.f;
        if (kMode != ROW_QUANTIZE) {
            if (out_of_range(ss, p.eps) || (kMode == ROW_NORM_Q8 && top >= 0x7f800000u)) {
                // (rare; every thread of the group takes it)
                uint32_t big = 0;
                float none = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (span[i].hi > span[i].lo)
#pragma unroll
                        for (int j = 0; j < E; ++j) big = max(big, magnitude(v[i][j]));
                g.sum_and_max(none, big);
                const float s = row_rescale(big, p.eps);
                ss = 0.f; top = 0;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if (span[i].hi <= span[i].lo) continue;
                    float wf[E];
                    if (kMode == ROW_NORM_Q8) weight[i].values(wf);
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        v[i][j] *= s;
                        ss = fmaf(v[i][j], v[i][j], ss);
                        if (kMode == ROW_NORM_Q8) top = max(top, magnitude(v[i][j] * wf[j]));
                    }
                }
                g.sum_and_max(ss, top);
                r = __frsqrt_rn(fmaf(ss, mean, (p.eps * s) * s));
                if (g.rank == 0 && p.rstd) p.rstd[row] = r * s;
            } else {
                r = __frsqrt_rn(fmaf(ss, mean, p.eps));
                if (g.rank == 0 && p.rstd) p.rstd[row] = r;
            }
        }
        float inv = 1.f;
        if (kMode != ROW_NORM) {
            const float most = __uint_as_float(top) * r / kLargestE4m3;
            const float scale = most < kLeastScale ? kLeastScale : most;
            if (g.rank == 0) p.scale[row] = scale;
            inv = 1.f / scale;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (span[i].hi <= span[i].lo) continue;
            const size_t o = at + size_t(g.rank + i * p.group) * E;
            float wf[E];
            if (kMode != ROW_QUANTIZE) weight[i].values(wf);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                if (kMode != ROW_QUANTIZE) v[i][j] = v[i][j] * r * wf[j];
                if (kMode != ROW_NORM) v[i][j] *= inv;
            }
            if (kMode == ROW_NORM) store_span(static_cast<T*>(p.y) + o, span[i], v[i]);
            else store_span_q8<E>(static_cast<uint8_t*>(p.y) + o, span[i], v[i]);
        }
    }
}

// Rows that do not fit in a block's registers: the row is walked over twice (the second time it comes from L2), element by
// element.
template <class T, RowMode kMode>
__global__ void __launch_bounds__(1024) long_row_kernel(const RowParams p) {
    __shared__ float2 words[64];
    Group g{int(blockDim.x), int(threadIdx.x), 0, words};
    const T* x = static_cast<const T*>(p.x);
    const T* res = static_cast<const T*>(p.residual);
    const T* w = static_cast<const T*>(p.w);
    grid_dependency_wait();
    grid_dependents_launch();
    for (int row = blockIdx.x; row < p.N; row += gridDim.x) {
        const size_t at = size_t(row) * p.C;
        auto value = [&](int c) {
            const float v = Elem<T>::get(x[at + c]);
            return kMode != ROW_QUANTIZE && res ? v + Elem<T>::get(res[at + c]) : v;
        };
        float ss = 0.f, s = 1.f;
        uint32_t top = 0;
        auto measure = [&] {
            ss = 0.f; top = 0;
            for (int c = g.rank; c < p.C; c += g.size) {
                const float v = value(c) * s;
                ss = fmaf(v, v, ss);
                top = max(top, magnitude(kMode == ROW_NORM_Q8 ? v * Elem<T>::get(w[c]) : v));
            }
            g.sum_and_max(ss, top);
        };
        measure();
        float r = 1.f;
        if (kMode != ROW_QUANTIZE) {
            if (out_of_range(ss, p.eps) || (kMode == ROW_NORM_Q8 && top >= 0x7f800000u)) {
                uint32_t big = 0;
                float none = 0.f;
                for (int c = g.rank; c < p.C; c += g.size) big = max(big, magnitude(value(c)));
                g.sum_and_max(none, big);
                s = row_rescale(big, p.eps);
                measure();
            }
            r = __frsqrt_rn(fmaf(ss, 1.f / float(p.C), (p.eps * s) * s));
            if (g.rank == 0 && p.rstd) p.rstd[row] = r * s;
        }
        float inv = 1.f;
        if (kMode != ROW_NORM) {
            const float most = __uint_as_float(top) * r / kLargestE4m3;
            const float scale = most < kLeastScale ? kLeastScale : most;
            if (g.rank == 0) p.scale[row] = scale;
            inv = 1.f / scale;
        }
        for (int c = g.rank; c < p.C; c += g.size) {
            float v = value(c);
            if (kMode != ROW_QUANTIZE && res && p.h) static_cast<T*>(p.h)[at + c] = Elem<T>::put(v);
            if (kMode != ROW_QUANTIZE) v = v * s * r * Elem<T>::get(w[c]);
            if (kMode == ROW_NORM) static_cast<T*>(p.y)[at + c] = Elem<T>::put(v);
            else static_cast<uint8_t*>(p.y)[at + c] = uint8_t(__nv_cvt_float_to_fp8(v * inv, __NV_SATFINITE, __NV_E4M3));
        }
    }
}

// ---- gradient
struct GradParams {
    int N, C, group;
    const void *h, *w;
    const float* rstd;
    const void *dy, *dh;
    void *dx;
    float* parts;                // [blocks][C]: sums of dw over each block's rows, or null
};

template <class T, int V>
__global__ void __launch_bounds__(512) row_grad_kernel(const GradParams p) {
    constexpr int E = Chunk<T>::E;
    extern __shared__ float merged[];                          // [C], where a block has several groups
    __shared__ float2 words[64];
    Group g{p.group, int(threadIdx.x) % p.group, int(threadIdx.x) / p.group, words};
    const int groups = blockDim.x / p.group, total = groups * gridDim.x;
    int row = blockIdx.x * groups + g.index;
    const T* h = static_cast<const T*>(p.h);
    const T* w = static_cast<const T*>(p.w);
    const T* dy = static_cast<const T*>(p.dy);
    const T* dh = static_cast<const T*>(p.dh);
    const int shift = int((size_t(row) * p.C) % E);
    Span span[V];
    Chunk<T> weight[V];
    float dw[V][E];
    grid_dependency_wait();
    grid_dependents_launch();
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (g.rank + i * p.group) * E - shift;
        span[i] = {c < 0 ? -c : 0, p.C - c < E ? (p.C - c > 0 ? p.C - c : 0) : E};
#pragma unroll
        for (int j = 0; j < E; ++j) dw[i][j] = 0.f;
        if (row < p.N && span[i].hi > span[i].lo) weight[i] = load_weights(w, c, span[i], shift);
    }
    const float mean = 1.f / float(p.C);
    for (; row < p.N; row += total) {
        const size_t at = size_t(row) * p.C - shift;
        const float r = p.rstd[row];
        Chunk<T> a[V], b[V], d[V];
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (span[i].hi > span[i].lo) {
                const size_t o = at + size_t(g.rank + i * p.group) * E;
                a[i] = load_span(h + o, span[i]);
                b[i] = load_span(dy + o, span[i]);
                if (dh) d[i] = load_span(dh + o, span[i]);
            }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (span[i].hi <= span[i].lo) continue;
            float n[E], y[E], wf[E];
            a[i].values(n); b[i].values(y); weight[i].values(wf);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float t = n[j] * r * y[j];               // dy n
                dw[i][j] += t;
                dot = fmaf(t, wf[j], dot);
            }
        }
        dot = g.sum(dot) * mean;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (span[i].hi <= span[i].lo) continue;
            float n[E], y[E], wf[E], o[E];
            a[i].values(n); b[i].values(y); weight[i].values(wf);
            if (dh) d[i].values(o);
#pragma unroll
            for (int j = 0; j < E; ++j) o[j] = fmaf(r, fmaf(n[j] * r, -dot, y[j] * wf[j]), dh ? o[j] : 0.f);
            store_span(static_cast<T*>(p.dx) + at + size_t(g.rank + i * p.group) * E, span[i], o);
        }
    }
    if (!p.parts) return;
    // the groups' sums in the groups' order, then the block's to its row of the parts
    float* part = p.parts + size_t(blockIdx.x) * p.C;
    for (int q = 0; q < groups; ++q) {
        if (q == g.index) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (g.rank + i * p.group) * E - shift;
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (j >= span[i].lo && j < span[i].hi) {
                        if (groups == 1) part[c + j] = dw[i][j];
                        else merged[c + j] = q == 0 ? dw[i][j] : merged[c + j] + dw[i][j];
                    }
            }
        }
        if (groups > 1) __syncthreads();
    }
    if (groups > 1)
        for (int c = threadIdx.x; c < p.C; c += blockDim.x) part[c] = merged[c];
}

template <class T>
__global__ void __launch_bounds__(1024) long_row_grad_kernel(const GradParams p) {
    __shared__ float2 words[64];
    Group g{int(blockDim.x), int(threadIdx.x), 0, words};
    const T* h = static_cast<const T*>(p.h);
    const T* w = static_cast<const T*>(p.w);
    const T* dy = static_cast<const T*>(p.dy);
    const T* dh = static_cast<const T*>(p.dh);
    float* part = p.parts ? p.parts + size_t(blockIdx.x) * p.C : nullptr;
    grid_dependency_wait();
    grid_dependents_launch();
    bool first = true;
    for (int row = blockIdx.x; row < p.N; row += gridDim.x, first = false) {
        const size_t at = size_t(row) * p.C;
        const float r = p.rstd[row];
        float dot = 0.f;
        for (int c = g.rank; c < p.C; c += g.size) {
            const float t = Elem<T>::get(h[at + c]) * r * Elem<T>::get(dy[at + c]);
            if (part) part[c] = first ? t : part[c] + t;
            dot = fmaf(t, Elem<T>::get(w[c]), dot);
        }
        dot = g.sum(dot) / float(p.C);
        for (int c = g.rank; c < p.C; c += g.size) {
            const float n = Elem<T>::get(h[at + c]) * r, y = Elem<T>::get(dy[at + c]);
            const float o = dh ? Elem<T>::get(dh[at + c]) : 0.f;
            static_cast<T*>(p.dx)[at + c] = Elem<T>::put(fmaf(r, fmaf(n, -dot, y * Elem<T>::get(w[c])), o));
        }
    }
}

// dw[c] = the sum of the parts' column c, in their order: a warp's lanes take 32 columns, its block's warps every 16th part.
constexpr int kSumWarps = 16;
template <class T>
__global__ void __launch_bounds__(kSumWarps * 32) sum_parts_kernel(const float* parts, int rows, int C, T* dw) {
    __shared__ float sums[kSumWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    grid_dependency_wait();
    grid_dependents_launch();
    float s = 0.f;
    if (c < C)
#pragma unroll 8
        for (int r = warp; r < rows; r += kSumWarps) s += parts[size_t(r) * C + c];
    sums[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < C) {
        for (int i = 1; i < kSumWarps; ++i) s += sums[i][lane];
        dw[c] = Elem<T>::put(s);
    }
}

constexpr int kMaxChunks = 4;
constexpr int kBlock = 512;                  // threads of a block of small groups
constexpr int kMostParts = 296;              // blocks of the gradient

// Threads that share a row of `chunks` chunks (a row that starts inside a chunk may have one more): as many as keep `v` chunks each.
int group_size(int chunks, int v) {
    int g = 32;
    while (g * v < chunks) g *= 2;
    return g;
}
int row_chunks(int C, int E) { return (C + E - 1) / E + (C % E != 0); }

template <class T, RowMode kMode>
int launch_rows(RowParams p, cudaStream_t st) {
    constexpr int E = Chunk<T>::E;
    const int chunks = row_chunks(p.C, E), sms = device_sm_count();
    if (chunks > 1024 * kMaxChunks) {
        const int grid = p.N < 2 * sms ? p.N : 2 * sms;
        return launch_chained(long_row_kernel<T, kMode>, dim3(grid), dim3(1024), 0, st, 1, p);
    }
    // few rows: one chunk a thread, for the shortest way from the first load to the last store
    const int v = chunks <= 1024 && p.N <= 2 * sms ? 1 : chunks <= 2048 ? 2 : 4;
    p.group = group_size(chunks, v);
    const int block = p.group > kBlock || p.N <= sms ? p.group : kBlock, groups = block / p.group;
    int grid = sms * (2048 / block);
    const int unit = groups < E ? E / groups : 1;              // (a group's rows are a multiple of E apart)
    grid = grid / unit * unit;
    const int need = (p.N + groups - 1) / groups;
    if (grid > need) grid = need;                              // (every group then has one row)
    if (v == 1) return launch_chained(row_kernel<T, 1, kMode>, dim3(grid), dim3(block), 0, st, 1, p);
    if (v == 2) return launch_chained(row_kernel<T, 2, kMode>, dim3(grid), dim3(block), 0, st, 1, p);
    return launch_chained(row_kernel<T, 4, kMode>, dim3(grid), dim3(block), 0, st, 1, p);
}

template <RowMode kMode>
int launch_rows_of(int type, const RowParams& p, cudaStream_t st) {
    switch (type) {
        case DT_F32: return launch_rows<float, kMode>(p, st);
        case DT_BF16: return launch_rows<__nv_bfloat16, kMode>(p, st);
        default: return launch_rows<__half, kMode>(p, st);
    }
}

template <class T>
int launch_grad(GradParams p, void* dw, cudaStream_t st) {
    constexpr int E = Chunk<T>::E;
    const int chunks = row_chunks(p.C, E), sms = device_sm_count();
    int grid, rc;
    if (chunks > 512 * kMaxChunks) {
        grid = p.N < kMostParts ? p.N : kMostParts;
        rc = launch_chained(long_row_grad_kernel<T>, dim3(grid), dim3(1024), 0, st, 1, p);
    } else {
        const int v = chunks <= 1024 ? 2 : 4;
        p.group = group_size(chunks, v);
        const int block = kBlock, groups = block / p.group;
        grid = 2 * sms < kMostParts ? 2 * sms : kMostParts;
        const int unit = groups < E ? E / groups : 1;
        grid = grid / unit * unit;
        const int need = (p.N + groups - 1) / groups;
        if (grid > need) grid = need;
        const size_t smem = groups > 1 && p.parts ? size_t(p.C) * 4 : 0;      // (groups of up to 256 threads: 16 KB)
        rc = v == 2 ? launch_chained(row_grad_kernel<T, 2>, dim3(grid), dim3(block), smem, st, 1, p)
                    : launch_chained(row_grad_kernel<T, 4>, dim3(grid), dim3(block), smem, st, 1, p);
    }
    if (rc != PCL_OK || !dw) return rc;
    return launch_chained(sum_parts_kernel<T>, dim3((p.C + 31) / 32), dim3(kSumWarps * 32), 0, st, 1, static_cast<const float*>(p.parts), grid, p.C,
                          static_cast<T*>(dw));
}

}  // namespace

size_t rms_norm_workspace_bytes(int N, int C) { return align_up(size_t(N < kMostParts ? N : kMostParts) * C * 4, 256); }

int launch_rms_norm_fwd(int N, int C, int type, const void* x, const void* residual, const void* w, float eps, void* h, void* y,
                        float* scale, float* rstd, cudaStream_t st) {
    const RowParams p{N, C, 0, eps, x, residual, w, h, y, scale, rstd};
    LaunchScope scope(KID_RMS_NORM, double(N) * C * (dtype_bytes(type) * (residual ? 3 : 1) + (scale ? 1 : dtype_bytes(type))), st);
    return scale ? launch_rows_of<ROW_NORM_Q8>(type, p, st) : launch_rows_of<ROW_NORM>(type, p, st);
}

int launch_quantize_rows(int N, int C, int type, const void* x, void* q, float* scale, cudaStream_t st) {
    const RowParams p{N, C, 0, 0.f, x, nullptr, nullptr, nullptr, q, scale, nullptr};
    LaunchScope scope(KID_RMS_NORM, double(N) * C * (dtype_bytes(type) + 1), st);
    return launch_rows_of<ROW_QUANTIZE>(type, p, st);
}

int launch_rms_norm_bwd(int N, int C, int type, const void* h, const void* w, const float* rstd, const void* dy, const void* dh,
                        void* dx, void* dw, void* ws, cudaStream_t st) {
    const GradParams p{N, C, 0, h, w, rstd, dy, dh, dx, dw ? static_cast<float*>(ws) : nullptr};
    LaunchScope scope(KID_RMS_NORM, double(N) * C * dtype_bytes(type) * (dh ? 4 : 3), st);
    switch (type) {
        case DT_F32: return launch_grad<float>(p, dw, st);
        case DT_BF16: return launch_grad<__nv_bfloat16>(p, dw, st);
        default: return launch_grad<__half>(p, dw, st);
    }
}

}  // namespace pcl

// RMS norm of rows with the residual's addition, its 8-bit form and its gradient; 8-bit rows of a matrix.
//
//   h = x + residual,  y[c] = h[c] * r * w[c],  r = 1 / sqrt(mean(h^2) + eps)
//   dx = dh + r * (g - n * mean(g n)),  dw[c] = sum over the rows of dy[c] n[c],      g = dy w,  n = h r
//
// All of it is bound by memory: a row is read once, its values stay in the registers of a group of 4 to 512 threads (up to 32 each) until
// its sum is known, or, in the gradient, in shared memory.
//   Many rows: persistent blocks of several groups.  One warp copies sets of consecutive rows into a ring in shared memory (cp.async.bulk), so
//   that what is in flight does not depend on registers; weights, and the sums of dw, stay in registers.
//   Few rows (at most kFewRows per SM): a block takes a row, straight to registers, in one step.
//   Rows of more than 16384 elements are walked over twice.
// Threads take chunks of 16 bytes that are counted in the flat tensor, not in the row, and so are aligned whatever the row length: what a row
// of odd length has in front of its first whole chunk and behind its last are edges, an element each to the group's first threads.  The
// distance between a group's rows is a multiple of a chunk's elements, so that all of them start at the same place of a chunk and registers keep
// their columns.
//
// Sums over a row are fp32 in a fixed tree.  h is rounded when it is stored, but the norm is that of the sum before rounding.  A row whose
// sum of squares leaves fp32's range is scaled by a power of two first.
//
// Measured, over several cards and runs: 32768 x 4096 bf16 with a residual 170-177 us (1.07 GB, 6.1-6.3 TB/s), its gradient 165-177 (6.1-6.5 TB/s);
// 3001 x 1037 fp16 to 8 bits 7.4; gradient of 5000 x 1001 fp32 18.2 (a third of it the second launch and edges); one row of 2048 bf16 3.3-3.8, nearly
// all of it launch and call.  Rows of more than 16384 elements are far from that: 2048 x 32768 bf16 with a residual 375, its gradient 564 (by bytes: 82).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

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

// Two fp32 operations in one instruction: the kernels of ordinary row lengths are bound by instructions before they are bound by memory.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 o;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(o.x), "=f"(o.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return o;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 o;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(o.x), "=f"(o.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return o;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 o;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
        "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(o.x), "=f"(o.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return o;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// 16 bytes of a tensor, and its values in pairs.
template <class T> struct Chunk {
    static constexpr int E = 16 / int(sizeof(T)), P = E / 2;
    uint32_t u[4];
    __device__ __forceinline__ void values(float2 (&v)[P]) const {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if constexpr (sizeof(T) == 4) v[i] = make_float2(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]));
            else if constexpr (std::is_same_v<T, __half>) v[i] = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
            else v[i] = make_float2(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xffff0000u));
        }
    }
    __device__ __forceinline__ void pack(const float2 (&v)[P]) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if constexpr (sizeof(T) == 4) {
                u[2 * i] = __float_as_uint(v[i].x);
                u[2 * i + 1] = __float_as_uint(v[i].y);
            } else if constexpr (std::is_same_v<T, __half>) {
                const __half2 h = __floats2half2_rn(v[i].x, v[i].y);
                u[i] = *reinterpret_cast<const uint32_t*>(&h);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[i].x, v[i].y);
                u[i] = *reinterpret_cast<const uint32_t*>(&h);
            }
        }
    }
};
template <class T>
__device__ __forceinline__ Chunk<T> load_chunk(const void* p) {
    const uint4 q = *static_cast<const uint4*>(p);
    return {{q.x, q.y, q.z, q.w}};
}
template <class T>
__device__ __forceinline__ void store_chunk(T* p, const float2 (&v)[Chunk<T>::P]) {
    Chunk<T> c;
    c.pack(v);
    *reinterpret_cast<uint4*>(p) = make_uint4(c.u[0], c.u[1], c.u[2], c.u[3]);
}
// Values as e4m3 bytes.
template <int P>
__device__ __forceinline__ void store_q8(uint8_t* p, const float2 (&v)[P]) {
    uint32_t q[P / 2];
#pragma unroll
    for (int i = 0; i < P / 2; ++i) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(v[2 * i], __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(v[2 * i + 1], __NV_SATFINITE, __NV_E4M3);
        q[i] = lo | hi << 16;
    }
    if constexpr (P == 4) *reinterpret_cast<uint2*>(p) = make_uint2(q[0], q[1]);
    else *reinterpret_cast<uint32_t*>(p) = q[0];
}

// |v| as an integer that orders like it; NaN is above everything, so it survives a maximum.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// A group of threads that shares a row: 4, 8 or 16 lanes of a warp, or whole warps; several groups to a block.  Reductions over several warps
// alternate between two sets of words, so that one barrier each is enough.
struct Group {
    int size, rank, index;       // threads, this thread's place, which group of the block
    float* words;                // [2][2][32] of the block: sums and maxima of its warps
    uint32_t mask;               // the group's lanes of this warp
    int turn = 0;
    __device__ __forceinline__ Group(int size_, float* words_)
        : size(size_), rank(int(threadIdx.x) % size_), index(int(threadIdx.x) / size_), words(words_),
          mask(size_ < 32 ? ((1u << size_) - 1) << (threadIdx.x & 31 & ~unsigned(size_ - 1)) : 0xffffffffu) {}
    __device__ __forceinline__ void sync() const {
        __syncwarp();                        // (a warp's first lane has just stored its sums alone, and the barrier wants whole warps)
        if (size == int(blockDim.x)) __syncthreads();
        else named_barrier_sync(1 + index, size);
    }
    // The group's sum of a and (kMax) maximum of m, in the same order for every thread.
    template <bool kMax>
    __device__ __forceinline__ void sum_and_max(float& a, uint32_t& m) {
        if (size < 32) {
            for (int o = size >> 1; o; o >>= 1) {
                a += __shfl_xor_sync(mask, a, o);
                if (kMax) m = max(m, __shfl_xor_sync(mask, m, o));
            }
            return;
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
        if (kMax) m = __reduce_max_sync(0xffffffffu, m);
        if (size == 32) return;
        float* sums = words + turn * 64;
        const int warps = size >> 5, first = index * warps;
        turn ^= 1;
        if ((rank & 31) == 0) {
            sums[first + (rank >> 5)] = a;
            if (kMax) sums[32 + first + (rank >> 5)] = __uint_as_float(m);
        }
        sync();
        a = 0.f;
        if (kMax) m = 0;
#pragma unroll 4
        for (int i = first; i < first + warps; ++i) {
            a += sums[i];
            if (kMax) m = max(m, __float_as_uint(sums[32 + i]));
        }
    }
    __device__ __forceinline__ float sum(float a) {
        uint32_t none;
        sum_and_max<false>(a, none);
        return a;
    }
    // of one row or two at once
    __device__ __forceinline__ void sums(float (&a)[1]) { a[0] = sum(a[0]); }
    __device__ __forceinline__ void sums(float (&a)[2]) {
        for (int o = (size < 32 ? size : 32) >> 1; o; o >>= 1) {
            a[0] += __shfl_xor_sync(mask, a[0], o);
            a[1] += __shfl_xor_sync(mask, a[1], o);
        }
        if (size <= 32) return;
        float* sums = words + turn * 64;
        const int warps = size >> 5, first = index * warps;
        turn ^= 1;
        if ((rank & 31) == 0) {
            sums[first + (rank >> 5)] = a[0];
            sums[32 + first + (rank >> 5)] = a[1];
        }
        sync();
        a[0] = a[1] = 0.f;
#pragma unroll 4
        for (int i = first; i < first + warps; ++i) {
            a[0] += sums[i];
            a[1] += sums[32 + i];
        }
    }
};

constexpr int kPipeMost = 512;               // threads of a group, at most

enum RowMode { ROW_NORM = 0, ROW_NORM_Q8, ROW_QUANTIZE };

struct RowParams {
    int N, C;
    float eps;
    const void *x, *residual, *w;
    void *h, *y;
    float *scale, *rstd;
};

// The sum of squares left fp32's range, or lost all of its bits: the row times a power of two, with the largest value between 1/2 and 1, but no
// further up than eps times its square stays in range.
__device__ __forceinline__ float power_of_two(int e) { return e < -126 ? __int_as_float(0x00800000 >> (-126 - e)) : __int_as_float((min(e, 126) + 127) << 23); }
__device__ __forceinline__ int exponent(float v) { return (__float_as_int(v) >> 23) - 127; }      // of a positive number; -127: subnormal
__device__ __forceinline__ float row_rescale(uint32_t top, float eps) {
    const float t = __uint_as_float(top);
    if (!(t > 0.f) || t == INFINITY) return 1.f;              // (zeros, infinities and NaN stay what they are)
    const int up = -exponent(t) - 1;
    return power_of_two(eps > 0.f ? min(up, (100 - exponent(eps)) / 2) : up);
}
__device__ __forceinline__ bool out_of_range(float ss, float eps) { return !(ss < 1e38f) || (ss < 1e-24f && eps < 1e-20f); }
// The same of the products of values and weights, whose largest is top and which 1 / sqrt(mean) takes to y: above fp32's range, or so small that
// their roundings (half of 2^-149) reach a scale above its least.
__device__ __forceinline__ bool products_out_of_range(uint32_t top, float mean) {
    if (top - 0x00800000u < 0x7f000000u) return false;        // (an ordinary number)
    return top >= 0x7f800000u || (__uint_as_float(top) + 0x1p-149f) * __frsqrt_rn(mean) > kLargestE4m3 * kLeastScale;
}

// What a thread has of a row: up to V chunks, `group` apart, and, where the row is not just those (kWhole = false), maybe an element at the edges:
// in front of the first whole chunk, or behind the last one that has a thread.
template <class T, int V, bool kWhole>
struct Place {
    static constexpr int E = Chunk<T>::E;
    int group, rank, head, chunks;           // head: elements in front of the first whole chunk
    int edge;                                // the column of this thread's edge element, or -1
    __device__ __forceinline__ Place(int C, int group_, int rank_, size_t row) : group(group_), rank(rank_), head(0), chunks(C / E), edge(-1) {
        if (kWhole) return;
        head = min(int((E - row * C % E) % E), C);
        chunks = min((C - head) / E, V * group);
        const int tail = C - head - chunks * E;
        if (rank < head) edge = rank;
        else if (rank < head + tail) edge = C - tail + rank - head;
    }
    __device__ __forceinline__ int column(int i) const { return head + (rank + i * group) * E; }
    __device__ __forceinline__ bool live(int i) const { return rank + i * group < chunks; }
    __device__ __forceinline__ bool has_edge() const { return !kWhole && edge >= 0; }
    __device__ __forceinline__ Chunk<T> weights(const T* w, int i) const {
        if (kWhole) return load_chunk<T>(w + column(i));
        float2 v[E / 2];
#pragma unroll
        for (int j = 0; j < E / 2; ++j) v[j] = make_float2(Elem<T>::get(w[column(i) + 2 * j]), Elem<T>::get(w[column(i) + 2 * j + 1]));
        Chunk<T> c;
        c.pack(v);                           // (exact)
        return c;
    }
};

// The norm of a row whose values are in v and ve (h in fp32; 0 where the thread has none): its factor r, after the row was scaled where it had to
// be, and, of the 8-bit forms, the inverse of y's scale.
template <class T, int V, RowMode kMode, bool kWhole>
__device__ __forceinline__ void row_factors(Group& g, const RowParams& p, int row, bool store, const Place<T, V, kWhole>& at, float2 (&v)[V][Chunk<T>::P], float& ve,
                                            const Chunk<T> (&weight)[V], float we, float& r, float& inv) {
    constexpr int P = Chunk<T>::P;
    auto measure = [&](float& ss, uint32_t& top) {
        float2 sum = make_float2(kWhole || kMode == ROW_QUANTIZE ? 0.f : ve * ve, 0.f);
        top = kWhole || kMode == ROW_NORM ? 0u : magnitude(kMode == ROW_NORM_Q8 ? ve * we : ve);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!at.live(i)) continue;
            float2 wf[P];
            if (kMode == ROW_NORM_Q8) weight[i].values(wf);
#pragma unroll
            for (int j = 0; j < P; ++j) {
                if (kMode != ROW_QUANTIZE) sum = fma2(v[i][j], v[i][j], sum);
                if (kMode != ROW_NORM) {
                    const float2 y = kMode == ROW_NORM_Q8 ? mul2(v[i][j], wf[j]) : v[i][j];
                    top = max(top, max(magnitude(y.x), magnitude(y.y)));
                }
            }
        }
        ss = sum.x + sum.y;
        g.sum_and_max<kMode != ROW_NORM>(ss, top);
    };
    const float mean = 1.f / float(p.C);
    float ss;
    uint32_t top;
    measure(ss, top);
    r = 1.f;
    if (kMode != ROW_QUANTIZE) {
        float s = 1.f;
        if (out_of_range(ss, p.eps) || (kMode == ROW_NORM_Q8 && products_out_of_range(top, fmaf(ss, mean, p.eps)))) {       // (rare; every thread of the group takes it)
            uint32_t big = magnitude(ve);
            float none = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (at.live(i))
#pragma unroll
                    for (int j = 0; j < P; ++j) big = max(big, max(magnitude(v[i][j].x), magnitude(v[i][j].y)));
            g.sum_and_max<true>(none, big);
            s = row_rescale(big, p.eps);
            ve *= s;
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < P; ++j) v[i][j] = mul2(v[i][j], both(s));
            measure(ss, top);
        }
        r = __frsqrt_rn(fmaf(ss, mean, (p.eps * s) * s));
        if (store && g.rank == 0 && p.rstd) p.rstd[row] = r * s;
    }
    inv = 1.f;
    if (kMode != ROW_NORM) {
        const float most = __uint_as_float(top) * r / kLargestE4m3;
        const float scale = most < kLeastScale ? kLeastScale : most;
        if (store && g.rank == 0) p.scale[row] = scale;
        inv = 1.f / scale;
    }
}
template <class T, int V, RowMode kMode, bool kWhole>
__device__ __forceinline__ void row_store(const RowParams& p, size_t first, const Place<T, V, kWhole>& at, float2 (&v)[V][Chunk<T>::P], float ve,
                                          const Chunk<T> (&weight)[V], float we, float r, float inv) {
    constexpr int P = Chunk<T>::P;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (!at.live(i)) continue;
        float2 wf[P];
        if (kMode != ROW_QUANTIZE) weight[i].values(wf);
#pragma unroll
        for (int j = 0; j < P; ++j) {
            if (kMode != ROW_QUANTIZE) v[i][j] = mul2(mul2(v[i][j], both(r)), wf[j]);
            if (kMode != ROW_NORM) v[i][j] = mul2(v[i][j], both(inv));
        }
        if (kMode == ROW_NORM) store_chunk(static_cast<T*>(p.y) + (first + at.column(i)), v[i]);
        else store_q8<P>(static_cast<uint8_t*>(p.y) + (first + at.column(i)), v[i]);
    }
    if (at.has_edge()) {
        if (kMode != ROW_QUANTIZE) ve = ve * r * we;
        if (kMode == ROW_NORM) static_cast<T*>(p.y)[first + at.edge] = Elem<T>::put(ve);
        else static_cast<uint8_t*>(p.y)[first + at.edge] = uint8_t(__nv_cvt_float_to_fp8(ve * inv, __NV_SATFINITE, __NV_E4M3));
    }
}
template <class T, int V, bool kWhole>
__device__ __forceinline__ void store_h(T* h, size_t first, const Place<T, V, kWhole>& at, const float2 (&v)[V][Chunk<T>::P], float ve) {
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (at.live(i)) store_chunk(h + (first + at.column(i)), v[i]);
    if (at.has_edge()) h[first + at.edge] = Elem<T>::put(ve);
}

// ---- few rows: one to a block
template <class T, int V, RowMode kMode, bool kWhole>
__global__ void __launch_bounds__(1024) row_kernel(const RowParams p) {
    constexpr int P = Chunk<T>::P;
    __shared__ float words[128];
    Group g(int(blockDim.x), words);
    const int row = blockIdx.x;
    const T* x = static_cast<const T*>(p.x);
    const T* res = static_cast<const T*>(p.residual);
    const Place<T, V, kWhole> at(p.C, int(blockDim.x), int(threadIdx.x), row);
    Chunk<T> weight[V];
    float2 v[V][P];
    float ve = 0.f, we = 0.f;
    grid_dependency_wait();
    grid_dependents_launch();
    const size_t first = size_t(row) * p.C;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (at.live(i)) {
            const Chunk<T> a = load_chunk<T>(x + (first + at.column(i)));
            Chunk<T> b;
            if (kMode != ROW_QUANTIZE && res) b = load_chunk<T>(res + (first + at.column(i)));
            if (kMode != ROW_QUANTIZE) weight[i] = at.weights(static_cast<const T*>(p.w), i);
            a.values(v[i]);
            if (kMode != ROW_QUANTIZE && res) {
                float2 u[P];
                b.values(u);
#pragma unroll
                for (int j = 0; j < P; ++j) v[i][j] = add2(v[i][j], u[j]);
            }
        }
    if (at.has_edge()) {
        ve = Elem<T>::get(x[first + at.edge]);
        if (kMode != ROW_QUANTIZE && res) ve += Elem<T>::get(res[first + at.edge]);
        if (kMode != ROW_QUANTIZE) we = Elem<T>::get(static_cast<const T*>(p.w)[at.edge]);
    }
    if (kMode != ROW_QUANTIZE && p.h) store_h<T, V>(static_cast<T*>(p.h), first, at, v, ve);
    float r, inv;
    row_factors<T, V, kMode>(g, p, row, true, at, v, ve, weight, we, r, inv);
    row_store<T, V, kMode>(p, first, at, v, ve, weight, we, r, inv);
}

// ---- many rows
// A ring of `stages` slots in shared memory; a slot holds a set of rows (`per_group` to a group, `groups` apart) of each tensor.
struct Pipe {
    int group, per_group, sets, stages, slot;      // threads that share a row; bytes of one tensor's rows in a slot
    unsigned int* status;
};
constexpr int kMostStages = 8;
struct PipeShared {
    uint64_t full[kMostStages], empty[kMostStages];
    float words[128];
    uint32_t abort_flag;
};
// The rows of a set: the bytes that are copied start and end on multiples of 16, and end inside the tensor (where it ends inside a chunk, the
// rest is read from memory).
struct Set { int first, rows; size_t from; uint32_t bytes; };
template <class T>
__device__ __forceinline__ Set rows_of(int s, int rows_per_set, int N, int C) {
    Set o;
    o.first = s * rows_per_set;
    o.rows = min(rows_per_set, N - o.first);
    const size_t total = size_t(N) * C * sizeof(T), end = (size_t(o.first) + o.rows) * C * sizeof(T);
    o.from = size_t(o.first) * C * sizeof(T) & ~size_t(15);
    const size_t up = (end + 15) & ~size_t(15);
    o.bytes = uint32_t((up < total ? up : total & ~size_t(15)) - o.from);
    return o;
}
__device__ __forceinline__ void pipe_begin(PipeShared& sh, int stages, int consumer_warps) {
    if (threadIdx.x == 0) {
        for (int i = 0; i < stages; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], consumer_warps); }
        sh.abort_flag = 0;
        mbar_fence_init();
    }
    __syncthreads();
}
// The copying thread.
template <class T, int kTensors>
__device__ __forceinline__ void pipe_produce(PipeShared& sh, const Pipe& q, uint8_t* ring, int groups, int N, int C, const void* const (&src)[kTensors]) {
    int n = 0;
    uint32_t tensors = 0;
#pragma unroll
    for (int t = 0; t < kTensors; ++t) tensors += src[t] != nullptr;
    const int slots = tensors * q.slot;
    bool ok = true;
    for (int s = blockIdx.x; s < q.sets; s += gridDim.x, ++n) {
        const int stage = n % q.stages;
        if (n >= q.stages && !bounded_wait(&sh.empty[stage], (n / q.stages - 1) & 1, &sh.abort_flag, q.status, WAIT_PRODUCER_EMPTY)) { ok = false; break; }
        const Set o = rows_of<T>(s, q.per_group * groups, N, C);
        mbar_expect_tx_one(&sh.full[stage], o.bytes * tensors);
        uint8_t* dst = ring + size_t(stage) * slots;
#pragma unroll
        for (int t = 0; t < kTensors; ++t)
            if (src[t]) {
                if (o.bytes) bulk_load(dst, static_cast<const uint8_t*>(src[t]) + o.from, o.bytes, &sh.full[stage]);
                dst += q.slot;
            }
    }
    if (!ok)          // given up: copies already under way still land in this block's shared memory; wait (bounded) for them
        for (int i = max(0, n - q.stages); i < n; ++i)
            for (int spin = 0; spin < 1 << 20 && !mbar_try_wait(&sh.full[i % q.stages], (i / q.stages) & 1); ++spin) {}
}
// Byte at which row `first + n` of a set starts in a slot.
template <class T, bool kWhole>
__device__ __forceinline__ uint32_t row_start(int s, int rows_per_set, int n, int C) {
    const uint32_t lead = kWhole ? 0u : uint32_t(size_t(s) * rows_per_set * C * sizeof(T)) & 15u;
    return lead + uint32_t(n) * C * uint32_t(sizeof(T));
}
// An element of a slot, or, behind the copied bytes (the end of a tensor that ends inside 16 bytes), of the tensor.
template <class T>
__device__ __forceinline__ float slot_element(const uint8_t* slot, uint32_t at, size_t size, const T* tensor, size_t element) {
    return Elem<T>::get(element * sizeof(T) < (size & ~size_t(15)) ? *reinterpret_cast<const T*>(slot + at) : tensor[element]);
}

template <class T, int V, RowMode kMode, bool kWhole, int kConsumers>
__global__ void __launch_bounds__(kConsumers + 32, V * Chunk<T>::E > 16 ? 1 : kConsumers == 256 ? 3 : 2) row_pipe_kernel(const RowParams p, const Pipe q) {
    constexpr int P = Chunk<T>::P;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ PipeShared sh;
    const int consumers = int(blockDim.x) - 32, groups = consumers / q.group;
    pipe_begin(sh, q.stages, consumers / 32);
    grid_dependency_wait();
    grid_dependents_launch();
    const T* x = static_cast<const T*>(p.x);
    const T* res = static_cast<const T*>(p.residual);
    if (int(threadIdx.x) >= consumers) {
        if (int(threadIdx.x) == consumers) {
            const void* const src[2] = {x, kMode != ROW_QUANTIZE ? res : nullptr};
            pipe_produce<T, 2>(sh, q, ring, groups, p.N, p.C, src);
        }
        return;
    }
    Group g(q.group, sh.words);
    const Place<T, V, kWhole> at(p.C, q.group, g.rank, size_t(blockIdx.x) * q.per_group * groups + g.index);
    Chunk<T> weight[V];
    float we = 0.f;
    if (kMode != ROW_QUANTIZE) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (at.live(i)) weight[i] = at.weights(static_cast<const T*>(p.w), i);
        if (at.has_edge()) we = Elem<T>::get(static_cast<const T*>(p.w)[at.edge]);
    }
    const int slots = (kMode != ROW_QUANTIZE && res ? 2 : 1) * q.slot, rows_per_set = q.per_group * groups;
    const size_t size = size_t(p.N) * p.C * sizeof(T);
    bool ok = true;                                            // (a wait ran out: the rest of the loop keeps its barriers, but stores nothing)
    int stage = 0;
    uint32_t phase = 0;
    for (int s = blockIdx.x; s < q.sets; s += gridDim.x) {
        ok = ok && bounded_wait(&sh.full[stage], phase, &sh.abort_flag, q.status, WAIT_EPI_TMEM_FULL);
        const uint8_t* slot = ring + size_t(stage) * slots;
        for (int k = 0; k < q.per_group; ++k) {
            const int n = k * groups + g.index, row = s * rows_per_set + n;
            const bool mine = row < p.N;                       // (of the whole group)
            const uint8_t* from = slot + row_start<T, kWhole>(s, rows_per_set, n, p.C);
            const size_t begin = size_t(row) * p.C;
            float2 v[V][P];
            float ve = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (!at.live(i) || !mine) continue;
                load_chunk<T>(from + at.column(i) * int(sizeof(T))).values(v[i]);
                if (kMode != ROW_QUANTIZE && res) {
                    float2 u[P];
                    load_chunk<T>(from + q.slot + at.column(i) * int(sizeof(T))).values(u);
#pragma unroll
                    for (int j = 0; j < P; ++j) v[i][j] = add2(v[i][j], u[j]);
                }
            }
            if (at.has_edge() && mine) {
                ve = slot_element(from, at.edge * sizeof(T), size, x, begin + at.edge);
                if (kMode != ROW_QUANTIZE && res) ve += slot_element(from + q.slot, at.edge * sizeof(T), size, res, begin + at.edge);
            }
            if (k + 1 == q.per_group) {                        // the slot is read
                __syncwarp();
                if ((threadIdx.x & 31) == 0) mbar_arrive(&sh.empty[stage]);
            }
            if (!mine) continue;                               // (the lanes of a warp may part here: reductions are the group's own)
            if (kMode != ROW_QUANTIZE && p.h && ok) store_h<T, V>(static_cast<T*>(p.h), begin, at, v, ve);
            float r, inv;
            row_factors<T, V, kMode>(g, p, row, ok, at, v, ve, weight, we, r, inv);
            if (ok) row_store<T, V, kMode>(p, begin, at, v, ve, weight, we, r, inv);
        }
        if (++stage == q.stages) { stage = 0; phase ^= 1u; }
    }
}

// Rows that do not fit in a block's registers: the row is walked over twice (the second time it comes from L2), element by
// element.
template <class T, RowMode kMode>
__global__ void __launch_bounds__(1024) long_row_kernel(const RowParams p) {
    __shared__ float words[128];
    Group g(int(blockDim.x), words);
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
            g.sum_and_max<true>(ss, top);
        };
        measure();
        float r = 1.f;
        if (kMode != ROW_QUANTIZE) {
            if (out_of_range(ss, p.eps) || (kMode == ROW_NORM_Q8 && products_out_of_range(top, fmaf(ss, 1.f / float(p.C), p.eps)))) {
                uint32_t big = 0;
                float none = 0.f;
                for (int c = g.rank; c < p.C; c += g.size) big = max(big, magnitude(value(c)));
                g.sum_and_max<true>(none, big);
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
    int N, C;
    const void *h, *w;
    const float* rstd;
    const void *dy, *dh;
    void *dx;
    float* parts;                // [blocks][C]: sums of dw over each block's rows, or null
};

template <class T, int V, bool kWhole, int kConsumers, bool kPairs>
__global__ void __launch_bounds__(kConsumers + 32, kConsumers == 256 ? 2 : 1) row_grad_kernel(const GradParams p, const Pipe q) {
    constexpr int P = Chunk<T>::P;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ PipeShared sh;
    const int consumers = int(blockDim.x) - 32, groups = consumers / q.group;
    pipe_begin(sh, q.stages, consumers / 32);
    grid_dependency_wait();
    grid_dependents_launch();
    const T* h = static_cast<const T*>(p.h);
    const T* dy = static_cast<const T*>(p.dy);
    const T* dh = static_cast<const T*>(p.dh);
    if (int(threadIdx.x) >= consumers) {
        if (int(threadIdx.x) == consumers) {
            const void* const src[3] = {h, dy, dh};
            pipe_produce<T, 3>(sh, q, ring, groups, p.N, p.C, src);
        }
        return;
    }
    Group g(q.group, sh.words);
    const Place<T, V, kWhole> at(p.C, q.group, g.rank, size_t(blockIdx.x) * q.per_group * groups + g.index);
    Chunk<T> weight[V];
    float2 dw[V][P];
    float we = 0.f, dwe = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int j = 0; j < P; ++j) dw[i][j] = both(0.f);
        if (at.live(i)) weight[i] = at.weights(static_cast<const T*>(p.w), i);
    }
    if (at.has_edge()) we = Elem<T>::get(static_cast<const T*>(p.w)[at.edge]);
    const float mean = 1.f / float(p.C);
    const int slots = (dh ? 3 : 2) * q.slot, rows_per_set = q.per_group * groups;
    const size_t size = size_t(p.N) * p.C * sizeof(T);
    bool ok = true;
    int stage = 0;
    uint32_t phase = 0;
    // rows are taken kRows at a time: one reduction (and barrier) for both
    constexpr int kRows = kPairs ? 2 : 1;
    // (one row: known here, which saves 16-bit types registers, 10000 x 3333 bf16 83 -> 62 us; fp32 code is slower by it, 8000 x 2501 52 -> 56)
    const int per_group = kPairs || sizeof(T) == 4 ? q.per_group : 1;
    auto factors = [&](int s, int k, float (&r)[kRows]) {
#pragma unroll
        for (int b = 0; b < kRows; ++b) {
            const int row = s * rows_per_set + (k + b) * groups + g.index;
            r[b] = s < q.sets && k + b < per_group && row < p.N ? p.rstd[row] : 0.f;
        }
    };
    float next[kRows];
    factors(blockIdx.x, 0, next);
    for (int s = blockIdx.x; s < q.sets; s += gridDim.x) {
        ok = ok && bounded_wait(&sh.full[stage], phase, &sh.abort_flag, q.status, WAIT_EPI_TMEM_FULL);
        const uint8_t* slot = ring + size_t(stage) * slots;
        for (int k = 0; k < per_group; k += kRows) {
            float r[kRows], xe[kRows], ye[kRows], dot[kRows];
#pragma unroll
            for (int b = 0; b < kRows; ++b) { r[b] = next[b]; xe[b] = ye[b] = dot[b] = 0.f; }
            if (k + kRows < per_group) factors(s, k + kRows, next);
            else factors(s + gridDim.x, 0, next);
            const int n = k * groups + g.index, row = s * rows_per_set + n;
            if (row >= p.N) break;                             // (of the whole group)
            const bool second = kPairs && k + 1 < per_group && row + groups < p.N;
            // dot = sum of g h = sum of dy w h;  dw += r dy h
#pragma unroll
            for (int b = 0; b < kRows; ++b) {
                if (b > 0 && !second) break;
                const uint8_t* from = slot + row_start<T, kWhole>(s, rows_per_set, n + b * groups, p.C);
                float2 sum = both(0.f);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if (!at.live(i)) continue;
                    float2 x[P], y[P], wf[P];
                    load_chunk<T>(from + at.column(i) * int(sizeof(T))).values(x);
                    load_chunk<T>(from + q.slot + at.column(i) * int(sizeof(T))).values(y);
                    weight[i].values(wf);
#pragma unroll
                    for (int j = 0; j < P; ++j) {
                        const float2 t = mul2(mul2(x[j], both(r[b])), y[j]);
                        dw[i][j] = add2(dw[i][j], t);
                        sum = fma2(t, wf[j], sum);
                    }
                }
                dot[b] = sum.x + sum.y;
                if (at.has_edge()) {
                    const size_t element = size_t(row + b * groups) * p.C + at.edge;
                    xe[b] = slot_element(from, at.edge * sizeof(T), size, h, element) * r[b];
                    ye[b] = slot_element(from + q.slot, at.edge * sizeof(T), size, dy, element);
                    dwe += xe[b] * ye[b];
                    dot[b] = fmaf(xe[b] * ye[b], we, dot[b]);
                    ye[b] *= we;
                }
            }
            g.sums(dot);
#pragma unroll
            for (int b = 0; b < kRows; ++b) {
                if (b > 0 && !second) break;
                const uint8_t* from = slot + row_start<T, kWhole>(s, rows_per_set, n + b * groups, p.C);
                const size_t begin = size_t(row + b * groups) * p.C;
                const float2 rr = both(r[b]), minus = both(-dot[b] * mean);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if (!at.live(i)) continue;
                    float2 x[P], y[P], wf[P], d[P];
                    load_chunk<T>(from + at.column(i) * int(sizeof(T))).values(x);
                    load_chunk<T>(from + q.slot + at.column(i) * int(sizeof(T))).values(y);
                    if (dh) load_chunk<T>(from + 2 * q.slot + at.column(i) * int(sizeof(T))).values(d);
                    weight[i].values(wf);
#pragma unroll
                    for (int j = 0; j < P; ++j) {
                        const float2 t = fma2(mul2(x[j], rr), minus, mul2(y[j], wf[j]));
                        d[j] = fma2(rr, t, dh ? d[j] : both(0.f));
                    }
                    if (ok) store_chunk(static_cast<T*>(p.dx) + (begin + at.column(i)), d);
                }
                if (at.has_edge() && ok) {
                    const float d = dh ? slot_element(from + 2 * q.slot, at.edge * sizeof(T), size, dh, begin + at.edge) : 0.f;
                    static_cast<T*>(p.dx)[begin + at.edge] = Elem<T>::put(fmaf(r[b], fmaf(xe[b], minus.x, ye[b]), d));
                }
            }
        }
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(&sh.empty[stage]);          // the slot is read
        if (++stage == q.stages) { stage = 0; phase ^= 1u; }
    }
    if (!p.parts) return;
    // the sums of a warp's groups (rows of whole chunks, so all have the same columns), then those of the block's warps or groups in their order
    // (in the ring, which is free now), then the block's to its row of the parts
    __syncwarp();
    int turns = groups, my_turn = g.index;
    if (kWhole && q.group < 32) {
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < P; ++j)
                for (int o = q.group; o < 32; o <<= 1) {
                    dw[i][j].x += __shfl_xor_sync(0xffffffffu, dw[i][j].x, o);
                    dw[i][j].y += __shfl_xor_sync(0xffffffffu, dw[i][j].y, o);
                }
        turns = consumers / 32;
        my_turn = int(threadIdx.x & 31) < q.group ? int(threadIdx.x) >> 5 : -1;
    }
    float* part = p.parts + size_t(blockIdx.x) * p.C;
    float* merged = reinterpret_cast<float*>(ring);
    for (int t = 0; t < turns; ++t) {
        __syncwarp();                        // (lanes of a warp part at `continue`, and the barrier wants whole warps)
        if (turns > 1) named_barrier_sync(15, consumers);
        if (t != my_turn) continue;
        float* to = turns == 1 ? part : merged;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!at.live(i)) continue;
            if (kWhole) {                                      // (16 bytes at a time: single stores a chunk apart write each sector eight times)
#pragma unroll
                for (int j = 0; j < P; j += 2) {
                    float4* f = reinterpret_cast<float4*>(to + at.column(i) + 2 * j);
                    float4 v = make_float4(dw[i][j].x, dw[i][j].y, dw[i][j + 1].x, dw[i][j + 1].y);
                    if (t > 0) { const float4 u = *f; v = make_float4(u.x + v.x, u.y + v.y, u.z + v.z, u.w + v.w); }
                    *f = v;
                }
            } else {
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    float* f = to + at.column(i) + 2 * j;
                    f[0] = t == 0 ? dw[i][j].x : f[0] + dw[i][j].x;
                    f[1] = t == 0 ? dw[i][j].y : f[1] + dw[i][j].y;
                }
            }
        }
        if (at.has_edge()) to[at.edge] = t == 0 ? dwe : to[at.edge] + dwe;
    }
    __syncwarp();
    if (turns > 1) {
        named_barrier_sync(15, consumers);
        for (int c = threadIdx.x; c < p.C; c += consumers) part[c] = merged[c];
    }
}

template <class T>
__global__ void __launch_bounds__(1024) long_row_grad_kernel(const GradParams p) {
    __shared__ float words[128];
    Group g(int(blockDim.x), words);
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

// dw[c] = the sum of the parts' column c: a warp's lanes take 32 columns, its block's warps every 32nd part.
constexpr int kSumWarps = 32;
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

// Blocks of the gradient: each leaves a row of sums, which costs a short call more than half of the SMs' second block gains (512 x 4096: 13.9 us
// with two, 9.4 with one).
int grad_blocks(int N) { const int sms = device_sm_count(); return N < sms ? N : N < 8 * sms ? sms : 2 * sms; }
constexpr int kFewRows = 2;
constexpr int kMostRing = 216 * 1024;        // of all blocks of an SM

// (of whole chunks; a row shorter than one has one all the same)
int row_chunks(int C, int E) { return C < E ? 1 : C / E; }

// A thread takes 16 elements of a row, 32 in rows that 512 threads would not cover; a chunk in rows that 32 lanes cover then.  Groups follow from
// that: whole warps, or, for short rows of whole chunks, 4, 8 or 16 lanes (32768 x 64 bf16 with a residual, 8 lanes: 11.0 -> 4.8 us).
template <class T> constexpr int kMostV = 32 / Chunk<T>::E;
template <class T> bool too_long(int C) { return row_chunks(C, Chunk<T>::E) > kPipeMost * kMostV<T>; }
template <class T>
struct PipeShape { Pipe q; int v, groups, consumers, grid; bool whole; size_t smem; };
template <class T>
int pipe_shape(PipeShape<T>& o, int N, int C, int tensors, int threads, int blocks_per_sm, int wide_threads, bool pairs) {
    constexpr int E = Chunk<T>::E;
    const int chunks = row_chunks(C, E), sms = device_sm_count();
    o.v = chunks <= 32 ? 1 : chunks <= 64 ? 2 : chunks <= kPipeMost * kMostV<T> / 2 ? kMostV<T> / 2 : kMostV<T>;
    o.q.group = ((chunks + o.v - 1) / o.v + 31) / 32 * 32;
    // a warp less, where it leaves no more than an element for each thread (3001 x 1037 fp16 to 8 bits, 64 threads instead of 96: 11.6 -> 7.9 us)
    const int less = o.q.group - 32;
    if (less >= 32 && (chunks - o.v * less) * E + (C % E ? 2 * (E - 1) : 0) <= less) o.q.group = less;
    o.whole = C % E == 0 && o.v * o.q.group >= chunks;
    if (C % E == 0)
        while (o.q.group <= 32 && o.q.group > 4 && o.q.group / 2 >= chunks) o.q.group /= 2;
    o.groups = o.q.group > threads ? 1 : threads / o.q.group;
    o.consumers = o.groups * o.q.group;
    const size_t row = size_t(C) * sizeof(T);
    // several rows to a group where they are short (and where a group's rows still start alike), and two where they are worked on in pairs: 32768 x 4096
    // bf16 gradient 185 -> 160 us, 20000 x 5120 206 -> 151
    int m = 1;
    auto more = [&](int to) {                                  // (the rows are there, and two stages of them fit an SM)
        return long(N) / (to * o.groups) >= 8L * sms && 2 * (align_up(size_t(to) * o.groups * row + 32, 128) * tensors) <= size_t(kMostRing);
    };
    if (o.groups % E == 0 || C % E == 0)
        while (m < 16 && (m * o.groups * row < 4096 || (pairs && m == 1)) && more(2 * m)) m *= 2;
    o.q.per_group = m;
    const int rows = m * o.groups;
    o.q.sets = (N + rows - 1) / rows;
    o.q.slot = int(align_up(rows * row + 32, 128));
    const size_t stage = size_t(o.q.slot) * tensors;
    // (blocks of more than 256 threads: as many as their registers and three stages each leave room for)
    if (o.consumers > 256) blocks_per_sm = std::min(blocks_per_sm, wide_threads / (o.consumers + 32));
    while (o.consumers > 256 && blocks_per_sm > 1 && 3 * stage * blocks_per_sm > size_t(kMostRing)) --blocks_per_sm;
    const size_t ring = kMostRing / blocks_per_sm / 128 * 128;
    const size_t room = 2 * stage > ring ? kMostRing : ring;
    const size_t stages = room / stage;
    if (stages < 1) return PCL_ERR_UNSUPPORTED_SHAPE;
    o.q.stages = int(stages < size_t(kMostStages) ? stages : kMostStages);
    o.smem = stage * o.q.stages;
    o.grid = sms * (room == kMostRing ? 1 : blocks_per_sm);
    int unit = 1;
    while (C % E != 0 && rows * unit % E != 0) unit *= 2;       // (a group's rows are a multiple of E apart)
    o.grid = o.grid / unit * unit;
    if (o.grid > o.q.sets) o.grid = o.q.sets;
    o.q.status = device_status_ptr();
    return o.q.status ? PCL_OK : PCL_ERR_CUDA;
}
template <class K>
int allow_smem(PerDeviceOnce& once, K kernel) {
    return once.run([&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostRing) == cudaSuccess ? PCL_OK : PCL_ERR_CUDA;
    });
}

template <class T, int V, RowMode kMode, bool kWhole>
int launch_pipe(const RowParams& p, const PipeShape<T>& o, cudaStream_t st) {
    auto launch = [&](PerDeviceOnce& once, auto kernel) {
        const int rc = allow_smem(once, kernel);
        return rc != PCL_OK ? rc : launch_chained(kernel, dim3(o.grid), dim3(o.consumers + 32), o.smem, st, 1, p, o.q);
    };
    static PerDeviceOnce once256, once512;
    if constexpr (V * Chunk<T>::E <= 16)
        if (o.consumers <= 256) return launch(once256, row_pipe_kernel<T, V, kMode, kWhole, 256>);
    if constexpr (V * Chunk<T>::E >= 16) return launch(once512, row_pipe_kernel<T, V, kMode, kWhole, 512>);
    return PCL_ERR_UNSUPPORTED_SHAPE;                          // (not reached: fewer than 16 elements a thread are groups of 32)
}
template <class T, int V, RowMode kMode>
int launch_few(const RowParams& p, int block, cudaStream_t st) {
    if (p.C % Chunk<T>::E == 0) return launch_chained(row_kernel<T, V, kMode, true>, dim3(p.N), dim3(block), 0, st, 1, p);
    return launch_chained(row_kernel<T, V, kMode, false>, dim3(p.N), dim3(block), 0, st, 1, p);
}
template <class T, RowMode kMode>
int launch_rows(const RowParams& p, cudaStream_t st) {
    constexpr int E = Chunk<T>::E;
    const int chunks = row_chunks(p.C, E), sms = device_sm_count();
    if (too_long<T>(p.C)) {
        const int grid = p.N < 2 * sms ? p.N : 2 * sms;
        return launch_chained(long_row_kernel<T, kMode>, dim3(grid), dim3(1024), 0, st, 1, p);
    }
    if (p.N <= kFewRows * sms) {
        const int v = chunks <= 1024 ? 1 : chunks <= 2048 ? 2 : 4, block = (((chunks + v - 1) / v) + 31) / 32 * 32;
        if (v == 1) return launch_few<T, 1, kMode>(p, block, st);
        if (v == 2) return launch_few<T, 2, kMode>(p, block, st);
        if constexpr (E == 4) return launch_few<T, 4, kMode>(p, block, st);
        return PCL_ERR_UNSUPPORTED_SHAPE;                      // (not reached: longer 16-bit rows are walked over twice)
    }
    PipeShape<T> o;
    // Long streams of 16-bit rows: two blocks of 512 threads (32768 x 4096 with a residual 194 -> 168 us, 65536 x 2048 191 -> 182); else three of 256
    // (without a residual 114 -> 100, fp32 16384 x 4096 192 -> 176, to 8 bits 32768 x 4096 176 -> 152, 1500 x 4096 12.8 -> 10.5).
    const bool wide = kMode == ROW_NORM && E == 8 && p.residual && p.C % E == 0 && chunks >= 256 && long(p.N) * chunks >= 256L * 48 * sms;
    const int rc = pipe_shape(o, p.N, p.C, kMode != ROW_QUANTIZE && p.residual ? 2 : 1, wide ? 512 : 256, 3, 2 * (512 + 32), false);
    if (rc != PCL_OK) return rc;
#define PCL_ROWS(V_) return o.whole ? launch_pipe<T, V_, kMode, true>(p, o, st) : launch_pipe<T, V_, kMode, false>(p, o, st)
    if (o.v == 1) PCL_ROWS(1);
    if (o.v == 2) PCL_ROWS(2);
    if (o.v == 4) PCL_ROWS(4);
    PCL_ROWS(kMostV<T>);
#undef PCL_ROWS
}

template <RowMode kMode>
int launch_rows_of(int type, const RowParams& p, cudaStream_t st) {
    switch (type) {
        case DT_F32: return launch_rows<float, kMode>(p, st);
        case DT_BF16: return launch_rows<__nv_bfloat16, kMode>(p, st);
        default: return launch_rows<__half, kMode>(p, st);
    }
}

template <class T, int V, bool kWhole>
int launch_grad_pipe(const GradParams& p, const PipeShape<T>& o, cudaStream_t st) {
    const size_t merged = o.consumers / 32 > 1 ? size_t(p.C) * 4 : 0, smem = o.smem > merged ? o.smem : merged;
    auto launch = [&](PerDeviceOnce& once, auto kernel) {
        const int rc = allow_smem(once, kernel);
        return rc != PCL_OK ? rc : launch_chained(kernel, dim3(o.grid), dim3(o.consumers + 32), smem, st, 1, p, o.q);
    };
    static PerDeviceOnce once256, once512, pairs256, pairs512;
    const bool pairs = o.q.per_group > 1 || V * Chunk<T>::E > 16;      // (4096 x 16384 bf16, a row at a time: 152 us against 133)
    if constexpr (V * Chunk<T>::E <= 16)
        if (o.consumers <= 256) return pairs ? launch(pairs256, row_grad_kernel<T, V, kWhole, 256, true>) : launch(once256, row_grad_kernel<T, V, kWhole, 256, false>);
    if constexpr (V * Chunk<T>::E >= 16)
        return pairs ? launch(pairs512, row_grad_kernel<T, V, kWhole, 512, true>) : launch(once512, row_grad_kernel<T, V, kWhole, 512, false>);
    return PCL_ERR_UNSUPPORTED_SHAPE;
}
template <class T>
int launch_grad(const GradParams& p, void* dw, cudaStream_t st) {
    constexpr int E = Chunk<T>::E;
    const int sms = device_sm_count();
    int grid, rc;
    if (too_long<T>(p.C)) {
        grid = grad_blocks(p.N);
        rc = launch_chained(long_row_grad_kernel<T>, dim3(grid), dim3(1024), 0, st, 1, p);
    } else {
        PipeShape<T> o;
        const bool few = grad_blocks(p.N) <= sms && row_chunks(p.C, E) > 64;
        rc = pipe_shape(o, p.N, p.C, p.dh ? 3 : 2, few ? 512 : 256, few ? 1 : 2, 512 + 32, true);
        if (rc != PCL_OK) return rc;
        int unit = 1;
        while (p.C % E != 0 && o.q.per_group * o.groups * unit % E != 0) unit *= 2;
        grid = grad_blocks(p.N) / unit * unit;
        if (o.grid > grid && grid > 0) o.grid = grid;
        grid = o.grid;
        const bool whole = o.whole;
        if (o.v == 1) rc = whole ? launch_grad_pipe<T, 1, true>(p, o, st) : launch_grad_pipe<T, 1, false>(p, o, st);
        else if (o.v == 2) rc = whole ? launch_grad_pipe<T, 2, true>(p, o, st) : launch_grad_pipe<T, 2, false>(p, o, st);
        else if (o.v == 4) rc = whole ? launch_grad_pipe<T, 4, true>(p, o, st) : launch_grad_pipe<T, 4, false>(p, o, st);
        else rc = whole ? launch_grad_pipe<T, kMostV<T>, true>(p, o, st) : launch_grad_pipe<T, kMostV<T>, false>(p, o, st);
    }
    if (rc != PCL_OK || !dw) return rc;
    return launch_chained(sum_parts_kernel<T>, dim3((p.C + 31) / 32), dim3(kSumWarps * 32), 0, st, 1, static_cast<const float*>(p.parts), grid, p.C,
                          static_cast<T*>(dw));
}

}  // namespace

size_t rms_norm_workspace_bytes(int N, int C) { return align_up(size_t(grad_blocks(N)) * align_up(C, 4) * 4, 256); }

int launch_rms_norm_fwd(int N, int C, int type, const void* x, const void* residual, const void* w, float eps, void* h, void* y,
                        float* scale, float* rstd, cudaStream_t st) {
    const RowParams p{N, C, eps, x, residual, w, h, y, scale, rstd};
    LaunchScope scope(KID_RMS_NORM, double(N) * C * (dtype_bytes(type) * (residual ? 3 : 1) + (scale ? 1 : dtype_bytes(type))), st);
    return scale ? launch_rows_of<ROW_NORM_Q8>(type, p, st) : launch_rows_of<ROW_NORM>(type, p, st);
}

int launch_quantize_rows(int N, int C, int type, const void* x, void* q, float* scale, cudaStream_t st) {
    const RowParams p{N, C, 0.f, x, nullptr, nullptr, nullptr, q, scale, nullptr};
    LaunchScope scope(KID_RMS_NORM, double(N) * C * (dtype_bytes(type) + 1), st);
    return launch_rows_of<ROW_QUANTIZE>(type, p, st);
}

int launch_rms_norm_bwd(int N, int C, int type, const void* h, const void* w, const float* rstd, const void* dy, const void* dh,
                        void* dx, void* dw, void* ws, cudaStream_t st) {
    const GradParams p{N, C, h, w, rstd, dy, dh, dx, dw ? static_cast<float*>(ws) : nullptr};
    LaunchScope scope(KID_RMS_NORM, double(N) * C * dtype_bytes(type) * (dh ? 4 : 3), st);
    switch (type) {
        case DT_F32: return launch_grad<float>(p, dw, st);
        case DT_BF16: return launch_grad<__nv_bfloat16>(p, dw, st);
        default: return launch_grad<__half>(p, dw, st);
    }
}

}  // namespace pcl

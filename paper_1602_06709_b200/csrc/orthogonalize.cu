// Orthogonalised update: five (or `steps`) Newton-Schulz steps on X0 = U / (|U|_F + 1e-7),
//   A = X X^T,  B = b A + c A A,  X <- a X + B X          (X^T X, X B for a matrix with more rows than columns)
// bring the singular values of U close to 1 and keep its singular vectors.
//
// Every product runs on the 16-bit tensor cores with fp16 operands scaled by powers of two: all values are bounded (|X|, |A|
// <= 1.5, |B| <= 2.9 by the polynomial), so fp16 has the three mantissa bits that bf16 lacks at no loss of range.  X
// itself keeps 22 bits until the last step, in two fp16 planes of which the products see the first; the last step takes the rounded X in its linear term too, so that the
// rounding is passed on by the polynomial's derivative (which is small at 1) instead of by B alone.  Relative error of the
// result (2-norm) 3e-4 .. 1.6e-3 on random, decaying and nearly low-rank spectra, where bf16 iterates give 1e-2 .. 2e-1.
// A and A A are symmetric: the tiles below the diagonal are copies of those above it.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "pcl_internal.h"
#include "pcl_ptx.cuh"

namespace pcl {

namespace {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr double kNsEps = 1e-7;
constexpr float kScaleX = 16384.f, kScaleB = 8192.f;        // of X and A, and of B
constexpr int kMaxNormBlocks = 1024;                        // partial sums per matrix

// kVec consecutive elements as fp32
template <int kVec>
__device__ __forceinline__ void load_vec(const void* p, int type, size_t i, float (&o)[kVec]) {
    if constexpr (kVec == 1) {
        o[0] = type == DT_F32 ? static_cast<const float*>(p)[i]
             : type == DT_BF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]) : __half2float(static_cast<const __half*>(p)[i]);
    } else {
        static_assert(kVec == 4, "");
        if (type == DT_F32) {
            const float4 v = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
            o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
        } else {
            const uint2 v = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + i);
            if (type == DT_BF16) {
                o[0] = __uint_as_float(v.x << 16); o[1] = __uint_as_float(v.x & 0xffff0000u);
                o[2] = __uint_as_float(v.y << 16); o[3] = __uint_as_float(v.y & 0xffff0000u);
            } else {
                const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&v.x)), b = __half22float2(*reinterpret_cast<const __half2*>(&v.y));
                o[0] = a.x; o[1] = a.y; o[2] = b.x; o[3] = b.y;
            }
        }
    }
}
template <int kVec>
__device__ __forceinline__ void store_vec(float* p, size_t i, const float (&v)[kVec]) {
    if constexpr (kVec == 1) p[i] = v[0];
    else *reinterpret_cast<float4*>(p + i) = make_float4(v[0], v[1], v[2], v[3]);
}

struct StageArgs {
    const void* g; int type;
    float* momentum; float mu; int nesterov;
    double* part;               // [count][kMaxNormBlocks]
    int parts;
    __half* xh;                 // [count][M][ld] X0 * kScaleX
    __half* xl;                 // what rounding left, times 2^11 (null: not needed)
    int M, N, ld;
    int* counters;              // of the products' split workspace, to be zeroed (null: none)
};

// Sum of squares of U (64-bit: the squares of a gradient leave the range of fp32), and the momentum update.
template <int kVec>
__global__ void __launch_bounds__(256) ortho_norm_kernel(StageArgs a) {
    __shared__ double red[8];
    grid_dependency_wait();
    grid_dependents_launch();
    const size_t n = size_t(a.M) * a.N, off = n * blockIdx.y;
    double sum = 0.0;
#pragma unroll 2
    for (size_t i = (size_t(blockIdx.x) * 256 + threadIdx.x) * kVec; i < n; i += size_t(gridDim.x) * 256 * kVec) {
        float u[kVec];
        load_vec<kVec>(a.g, a.type, off + i, u);
        if (a.momentum) {
            float m[kVec];
            load_vec<kVec>(a.momentum, DT_F32, off + i, m);
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                m[j] = fmaf(a.mu, m[j], u[j]);
                u[j] = a.nesterov ? fmaf(a.mu, m[j], u[j]) : m[j];
            }
            store_vec<kVec>(a.momentum, off + i, m);
        }
#pragma unroll
        for (int j = 0; j < kVec; ++j) sum += double(u[j]) * double(u[j]);
    }
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) sum += red[i];
        a.part[size_t(blockIdx.y) * kMaxNormBlocks + blockIdx.x] = sum;
    }
}

// X0 in two fp16 planes.
template <int kVec>
__global__ void __launch_bounds__(256) ortho_stage_kernel(StageArgs a) {
    __shared__ double red[8];
    double sum = 0.0;
    grid_dependency_wait();
    grid_dependents_launch();
    for (int i = threadIdx.x; i < a.parts; i += 256) sum += a.part[size_t(blockIdx.y) * kMaxNormBlocks + i];
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (a.counters && blockIdx.x == 0 && blockIdx.y == 0)
        for (int i = threadIdx.x; i < int(kGemm16CounterBytes / 4); i += 256) a.counters[i] = 0;
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = sum;
    __syncthreads();
    sum = 0.0;
    for (int i = 0; i < 8; ++i) sum += red[i];
    const float inv = float(1.0 / (sqrt(sum) + kNsEps));
    const size_t off = size_t(a.M) * a.N * blockIdx.y, off_x = size_t(a.M) * a.ld * blockIdx.y;
    for (int r = blockIdx.x; r < a.M; r += gridDim.x)
#pragma unroll 2
        for (int c = threadIdx.x * kVec; c < a.N; c += 256 * kVec) {
            const size_t i = off + size_t(r) * a.N + c, o = off_x + size_t(r) * a.ld + c;
            float u[kVec];
            if (a.momentum) {
                float m[kVec];
                load_vec<kVec>(a.momentum, DT_F32, i, m);
                if (a.nesterov) {
                    load_vec<kVec>(a.g, a.type, i, u);
#pragma unroll
                    for (int j = 0; j < kVec; ++j) u[j] = fmaf(a.mu, m[j], u[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < kVec; ++j) u[j] = m[j];
                }
            } else {
                load_vec<kVec>(a.g, a.type, i, u);
            }
#pragma unroll
            for (int j = 0; j < kVec; ++j) u[j] *= inv * kScaleX;
            alignas(8) __half h[kVec], l[kVec];
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                h[j] = __float2half_rn(u[j]);
                l[j] = __float2half_rn((u[j] - __half2float(h[j])) * 2048.f);
            }
            if constexpr (kVec == 1) {
                a.xh[o] = h[0];
                if (a.xl) a.xl[o] = l[0];
            } else {
                *reinterpret_cast<uint2*>(a.xh + o) = *reinterpret_cast<const uint2*>(h);
                if (a.xl) *reinterpret_cast<uint2*>(a.xl + o) = *reinterpret_cast<const uint2*>(l);
            }
        }
}

// The three products of a step, with everything their tiling depends on.
Gemm16Args gram_args(int count, int M, int N) {
    const int d = M < N ? M : N;
    Gemm16Args a{d, d, M < N ? N : M, count, false, {}, {}, GEMM16_SYM};
    a.split_ws = reinterpret_cast<void*>(256);               // (until the workspace is known)
    return a;
}
Gemm16Args square_args(int count, int M, int N) {
    const int d = M < N ? M : N;
    return gram_args(count, d, d);
}
Gemm16Args apply_args(int count, int M, int N) {
    Gemm16Args a{M, N, M < N ? M : N, count, false, {}, {}, GEMM16_STEP};
    a.split_ws = reinterpret_cast<void*>(256);
    return a;
}

struct OrthoLayout { size_t part, xl, xh[2], a, b, split, split_bytes, total; int ld, d, ldd; };
OrthoLayout ortho_layout(int count, int M, int N) {
    OrthoLayout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
    l.ld = int(align_up(N, 8));
    l.d = M < N ? M : N;
    l.ldd = int(align_up(l.d, 8));
    l.part = take(size_t(count) * kMaxNormBlocks * 8);
    l.xl = take(size_t(count) * M * l.ld * 2);
    for (size_t& o : l.xh) o = take(size_t(count) * M * l.ld * 2);
    l.a = take(size_t(count) * l.d * l.ldd * 2);
    l.b = take(size_t(count) * l.d * l.ldd * 2);
    for (const Gemm16Args& a : {gram_args(count, M, N), square_args(count, M, N), apply_args(count, M, N)}) {
        const size_t b = gemm16_split_ws_bytes(a);
        if (b > l.split_bytes) l.split_bytes = b;
    }
    l.split = take(l.split_bytes);
    l.total = at;
    return l;
}

}  // namespace

size_t orthogonalize_workspace_bytes(int count, int M, int N) { return ortho_layout(count, M, N).total; }

int launch_orthogonalize(const OrthoArgs& o, void* ws, cudaStream_t st) {
    const OrthoLayout l = ortho_layout(o.count, o.M, o.N);
    char* base = static_cast<char*>(ws);
    __half* xl = reinterpret_cast<__half*>(base + l.xl);
    __half* xh[2] = {reinterpret_cast<__half*>(base + l.xh[0]), reinterpret_cast<__half*>(base + l.xh[1])};
    void *A = base + l.a, *B = base + l.b;
    const bool wide = o.M <= o.N;
    const long xb = long(o.M) * l.ld, db = long(l.d) * l.ldd;
    StageArgs s{o.g, o.type, o.momentum, o.mu, o.nesterov, reinterpret_cast<double*>(base + l.part), 0, xh[0],
                o.steps > 1 ? xl : nullptr, o.M, o.N, l.ld, l.split_bytes ? reinterpret_cast<int*>(base + l.split) : nullptr};
    // four elements at a time where every row starts on a multiple of four (16 bytes of fp32, 8 bytes of the 16-bit types)
    const bool vec = o.N % 4 == 0;
    const double elems = double(o.count) * o.M * o.N;
    const size_t per_block = 256 * 4 * 4, want = (size_t(o.M) * o.N + per_block - 1) / per_block;
    const size_t cap = size_t(device_sm_count()) * 8 / o.count + 1;
    s.parts = int(want < cap ? want : cap);
    if (s.parts > kMaxNormBlocks) s.parts = kMaxNormBlocks;
    {
        LaunchScope scope(KID_ORTHO, elems * (o.momentum ? 8.0 + dtype_bytes(o.type) : double(dtype_bytes(o.type))), st);
        const int rc = launch_chained(vec ? ortho_norm_kernel<4> : ortho_norm_kernel<1>, dim3(s.parts, o.count), dim3(256), 0, st, 1, s);
        if (rc != PCL_OK) return rc;
    }
    {
        LaunchScope scope(KID_ORTHO, elems * (4.0 + dtype_bytes(o.type) + (o.momentum ? 4.0 : 0.0)), st);
        const int rc = launch_chained(vec ? ortho_stage_kernel<4> : ortho_stage_kernel<1>, dim3(o.M < 2048 ? o.M : 2048, o.count),
                                      dim3(256), 0, st, 1, s);
        if (rc != PCL_OK) return rc;
    }
    int cur = 0;
    for (int it = 0; it < o.steps; ++it) {
        const bool last = it + 1 == o.steps;
        const Gemm16Operand gram{xh[cur], l.ld, xb, !wide};
        Gemm16Args g1 = gram_args(o.count, o.M, o.N);
        g1.a = g1.b = gram;
        g1.split_ws = base + l.split;
        g1.alpha = 1.f / kScaleX;                             // kScaleX^2 A -> kScaleX A
        g1.out = A; g1.out_type = DT_F16; g1.out_ld = l.ldd; g1.out_batch = db;
        int rc = launch_gemm16(g1, st);
        if (rc != PCL_OK) return rc;
        const Gemm16Operand am{A, l.ldd, db, false}, bm{B, l.ldd, db, false};
        Gemm16Args g2 = square_args(o.count, o.M, o.N);
        g2.a = g2.b = am;
        g2.split_ws = base + l.split;
        g2.alpha = kNsC * kScaleB / (kScaleX * kScaleX);
        g2.src = A; g2.src_type = DT_F16; g2.src_ld = l.ldd; g2.src_batch = db; g2.beta = kNsB * kScaleB / kScaleX;
        g2.out = B; g2.out_type = DT_F16; g2.out_ld = l.ldd; g2.out_batch = db;
        rc = launch_gemm16(g2, st);
        if (rc != PCL_OK) return rc;
        Gemm16Args g3 = apply_args(o.count, o.M, o.N);
        g3.a = wide ? bm : Gemm16Operand{xh[cur], l.ld, xb, false};
        g3.b = wide ? Gemm16Operand{xh[cur], l.ld, xb, true} : bm;
        g3.split_ws = base + l.split;
        g3.src = xh[cur]; g3.src_type = DT_F16; g3.src_ld = l.ld; g3.src_batch = xb;
        if (last) {                                           // to the caller's matrix
            g3.epi = GEMM16_GENERAL;
            g3.alpha = 1.f / (kScaleX * kScaleB); g3.beta = kNsA / kScaleX;
            g3.out = o.out; g3.out_type = o.type; g3.out_ld = o.N; g3.out_batch = long(o.M) * o.N;
            if (o.momentum) {
                g3.update = true;
                g3.keep = 1.f - o.lr * o.weight_decay;
                g3.step = o.lr * sqrtf(o.M > o.N ? float(o.M) / float(o.N) : 1.f);
            }
        } else {                                              // kScaleX X, in two planes (the second in place)
            g3.alpha = 1.f / kScaleB; g3.beta = kNsA;
            g3.src_lo = xl;
            g3.out = xh[cur ^ 1]; g3.out_ld = l.ld; g3.out_batch = xb;
            if (it + 2 < o.steps) g3.out_lo = xl;
        }
        rc = launch_gemm16(g3, st);
        if (rc != PCL_OK) return rc;
        cur ^= 1;
    }
    return PCL_OK;
}

}  // namespace pcl

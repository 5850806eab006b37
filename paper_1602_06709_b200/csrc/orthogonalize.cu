// Orthogonalised update: five (or `steps`) Newton-Schulz steps on X0 = U / (|U|_F + 1e-7),
//   A = X X^T,  B = b A + c A A,  X <- a X + B X          (X^T X, X B for a matrix with more rows than columns)
// bring the singular values of U close to 1 and keep its singular vectors.
//
// Every product runs on the 16-bit tensor cores with fp16 operands scaled by powers of two: all values are bounded (|X|, |A|
// <= 1.5, |B| <= 2.9 by the polynomial), so fp16 has the three mantissa bits that bf16 lacks at no loss of range.  X
// itself stays in fp32 until the last step; the last step takes the rounded X in its linear term too, so that the
// rounding is passed on by the polynomial's derivative (which is small at 1) instead of by B alone.  Relative error of the
// result (2-norm) 3e-4 .. 1.6e-3 on random, decaying and nearly low-rank spectra, where bf16 iterates give 1e-2 .. 2e-1.
// A and A A are symmetric: the tiles below the diagonal are copies of those above it.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "pcl_internal.h"

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
    float* x;                   // [count][M][ld] fp32 (null: not needed)
    __half* xh;                 // [count][M][ld]
    int M, N, ld;
};

// Sum of squares of U (64-bit: the squares of a gradient leave the range of fp32), and the momentum update.
template <int kVec>
__global__ void __launch_bounds__(256) ortho_norm_kernel(StageArgs a) {
    __shared__ double red[8];
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

// X0 in fp32 and as the first product's fp16 operand.
template <int kVec>
__global__ void __launch_bounds__(256) ortho_stage_kernel(StageArgs a) {
    __shared__ double red[8];
    double sum = 0.0;
    for (int i = threadIdx.x; i < a.parts; i += 256) sum += a.part[size_t(blockIdx.y) * kMaxNormBlocks + i];
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
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
            for (int j = 0; j < kVec; ++j) u[j] *= inv;
            if (a.x) store_vec<kVec>(a.x, o, u);
            if constexpr (kVec == 1) {
                a.xh[o] = __float2half_rn(u[0] * kScaleX);
            } else {
                const __half2 lo = __floats2half2_rn(u[0] * kScaleX, u[1] * kScaleX), hi = __floats2half2_rn(u[2] * kScaleX, u[3] * kScaleX);
                *reinterpret_cast<uint2*>(a.xh + o) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
            }
        }
}

struct OrthoLayout { size_t part, x, xh[2], a, b, total; int ld, d, ldd; };
OrthoLayout ortho_layout(int count, int M, int N) {
    OrthoLayout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
    l.ld = int(align_up(N, 8));
    l.d = M < N ? M : N;
    l.ldd = int(align_up(l.d, 8));
    l.part = take(size_t(count) * kMaxNormBlocks * 8);
    l.x = take(size_t(count) * M * l.ld * 4);
    for (size_t& o : l.xh) o = take(size_t(count) * M * l.ld * 2);
    l.a = take(size_t(count) * l.d * l.ldd * 2);
    l.b = take(size_t(count) * l.d * l.ldd * 2);
    l.total = at;
    return l;
}

}  // namespace

size_t orthogonalize_workspace_bytes(int count, int M, int N) { return ortho_layout(count, M, N).total; }

int launch_orthogonalize(const OrthoArgs& o, void* ws, cudaStream_t st) {
    const OrthoLayout l = ortho_layout(o.count, o.M, o.N);
    char* base = static_cast<char*>(ws);
    float* x = reinterpret_cast<float*>(base + l.x);
    __half* xh[2] = {reinterpret_cast<__half*>(base + l.xh[0]), reinterpret_cast<__half*>(base + l.xh[1])};
    void *A = base + l.a, *B = base + l.b;
    const bool wide = o.M <= o.N;
    const long xb = long(o.M) * l.ld, db = long(l.d) * l.ldd;
    StageArgs s{o.g, o.type, o.momentum, o.mu, o.nesterov, reinterpret_cast<double*>(base + l.part), 0, o.steps > 1 ? x : nullptr,
                xh[0], o.M, o.N, l.ld};
    // four elements at a time where every row starts on a multiple of four (16 bytes of fp32, 8 bytes of the 16-bit types)
    const bool vec = o.N % 4 == 0;
    const double elems = double(o.count) * o.M * o.N;
    const size_t per_block = 256 * 4 * 4, want = (size_t(o.M) * o.N + per_block - 1) / per_block;
    const size_t cap = size_t(device_sm_count()) * 8 / o.count + 1;
    s.parts = int(want < cap ? want : cap);
    if (s.parts > kMaxNormBlocks) s.parts = kMaxNormBlocks;
    {
        LaunchScope scope(KID_ORTHO, elems * (o.momentum ? 8.0 + dtype_bytes(o.type) : double(dtype_bytes(o.type))), st);
        if (vec) ortho_norm_kernel<4><<<dim3(s.parts, o.count), 256, 0, st>>>(s);
        else ortho_norm_kernel<1><<<dim3(s.parts, o.count), 256, 0, st>>>(s);
    }
    if (cudaGetLastError() != cudaSuccess) return PCL_ERR_CUDA;
    {
        LaunchScope scope(KID_ORTHO, elems * (6.0 + dtype_bytes(o.type) + (o.momentum ? 4.0 : 0.0)), st);
        const dim3 grid(o.M < 2048 ? o.M : 2048, o.count);
        if (vec) ortho_stage_kernel<4><<<grid, 256, 0, st>>>(s);
        else ortho_stage_kernel<1><<<grid, 256, 0, st>>>(s);
    }
    if (cudaGetLastError() != cudaSuccess) return PCL_ERR_CUDA;
    int cur = 0;
    for (int it = 0; it < o.steps; ++it) {
        const bool last = it + 1 == o.steps;
        const Gemm16Operand gram{xh[cur], l.ld, xb, !wide};
        Gemm16Args g1{l.d, l.d, wide ? o.N : o.M, o.count, false, gram, gram, GEMM16_LINEAR};
        g1.symmetric = true;
        g1.alpha = 1.f / kScaleX;                             // kScaleX^2 A -> kScaleX A
        g1.out = A; g1.out_type = DT_F16; g1.out_ld = l.ldd; g1.out_batch = db;
        int rc = launch_gemm16(g1, st);
        if (rc != PCL_OK) return rc;
        const Gemm16Operand am{A, l.ldd, db, false}, bm{B, l.ldd, db, false};
        Gemm16Args g2{l.d, l.d, l.d, o.count, false, am, am, GEMM16_LINEAR};
        g2.symmetric = true;
        g2.alpha = kNsC * kScaleB / (kScaleX * kScaleX);
        g2.src = A; g2.src_type = DT_F16; g2.src_ld = l.ldd; g2.src_batch = db; g2.beta = kNsB * kScaleB / kScaleX;
        g2.out = B; g2.out_type = DT_F16; g2.out_ld = l.ldd; g2.out_batch = db;
        rc = launch_gemm16(g2, st);
        if (rc != PCL_OK) return rc;
        Gemm16Args g3{o.M, o.N, l.d, o.count, false, wide ? bm : Gemm16Operand{xh[cur], l.ld, xb, false},
                      wide ? Gemm16Operand{xh[cur], l.ld, xb, true} : bm, GEMM16_LINEAR};
        g3.alpha = 1.f / (kScaleX * kScaleB);
        if (last) {
            g3.src = xh[cur]; g3.src_type = DT_F16; g3.beta = kNsA / kScaleX;
            g3.out = o.out; g3.out_type = o.type; g3.out_ld = o.N; g3.out_batch = long(o.M) * o.N;
            if (o.momentum) {
                g3.update = true;
                g3.keep = 1.f - o.lr * o.weight_decay;
                g3.step = o.lr * sqrtf(o.M > o.N ? float(o.M) / float(o.N) : 1.f);
            }
        } else {
            g3.src = x; g3.src_type = DT_F32; g3.beta = kNsA;
            if (it + 2 < o.steps) { g3.out = x; g3.out_type = DT_F32; g3.out_ld = l.ld; g3.out_batch = xb; }
            g3.out2 = xh[cur ^ 1]; g3.out2_ld = l.ld; g3.out2_batch = xb; g3.scale2 = kScaleX;
        }
        g3.src_ld = l.ld; g3.src_batch = xb;
        rc = launch_gemm16(g3, st);
        if (rc != PCL_OK) return rc;
        cur ^= 1;
    }
    return PCL_OK;
}

}  // namespace pcl

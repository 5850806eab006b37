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
constexpr int kNormBlocks = 64;                             // partial sums per matrix

__device__ __forceinline__ float elem(const void* p, int type, size_t i) {
    if (type == DT_F32) return static_cast<const float*>(p)[i];
    if (type == DT_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}

struct StageArgs {
    const void* g; int type;
    float* momentum; float mu; int nesterov;
    double* part;               // [count][kNormBlocks]
    float* x;                   // [count][M][ld] fp32 (null: not needed)
    __half* xh;                 // [count][M][ld]
    int M, N, ld;
};

// Sum of squares of U (64-bit: the squares of a gradient leave the range of fp32), and the momentum update.
__global__ void __launch_bounds__(256) ortho_norm_kernel(StageArgs a) {
    __shared__ double red[8];
    const size_t n = size_t(a.M) * a.N, off = n * blockIdx.y;
    double sum = 0.0;
    for (size_t i = size_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += size_t(gridDim.x) * 256) {
        float u = elem(a.g, a.type, off + i);
        if (a.momentum) {
            const float m = fmaf(a.mu, a.momentum[off + i], u);
            a.momentum[off + i] = m;
            u = a.nesterov ? fmaf(a.mu, m, u) : m;
        }
        sum += double(u) * double(u);
    }
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) sum += red[i];
        a.part[size_t(blockIdx.y) * kNormBlocks + blockIdx.x] = sum;
    }
}

// X0 in fp32 and as the first product's fp16 operand.
__global__ void __launch_bounds__(256) ortho_stage_kernel(StageArgs a) {
    __shared__ float inv_s;
    if (threadIdx.x == 0) {
        double sum = 0.0;
        for (int i = 0; i < kNormBlocks; ++i) sum += a.part[size_t(blockIdx.y) * kNormBlocks + i];
        inv_s = float(1.0 / (sqrt(sum) + kNsEps));
    }
    __syncthreads();
    const float inv = inv_s;
    const size_t off = size_t(a.M) * a.N * blockIdx.y, off_x = size_t(a.M) * a.ld * blockIdx.y;
    for (int r = blockIdx.x; r < a.M; r += gridDim.x)
        for (int c = threadIdx.x; c < a.N; c += 256) {
            const size_t i = off + size_t(r) * a.N + c;
            float u = elem(a.g, a.type, i);
            if (a.momentum) {
                const float m = a.momentum[i];
                u = a.nesterov ? fmaf(a.mu, m, u) : m;
            }
            const float v = u * inv;
            const size_t o = off_x + size_t(r) * a.ld + c;
            if (a.x) a.x[o] = v;
            a.xh[o] = __float2half_rn(v * kScaleX);
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
    l.part = take(size_t(count) * kNormBlocks * 8);
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
    StageArgs s{o.g, o.type, o.momentum, o.mu, o.nesterov, reinterpret_cast<double*>(base + l.part), o.steps > 1 ? x : nullptr,
                xh[0], o.M, o.N, l.ld};
    const double elems = double(o.count) * o.M * o.N;
    {
        LaunchScope scope(KID_ORTHO, elems * (o.momentum ? 8.0 + dtype_bytes(o.type) : double(dtype_bytes(o.type))), st);
        ortho_norm_kernel<<<dim3(kNormBlocks, o.count), 256, 0, st>>>(s);
    }
    if (cudaGetLastError() != cudaSuccess) return PCL_ERR_CUDA;
    {
        LaunchScope scope(KID_ORTHO, elems * (6.0 + dtype_bytes(o.type) + (o.momentum ? 4.0 : 0.0)), st);
        ortho_stage_kernel<<<dim3(o.M < 2048 ? o.M : 2048, o.count), 256, 0, st>>>(s);
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

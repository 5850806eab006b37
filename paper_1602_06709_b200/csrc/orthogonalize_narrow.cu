// Orthogonalised update of narrow matrices (at most 64 rows or columns; d of them, k the long side).  A step multiplies X by a
// polynomial of its d x d Gram matrix, X <- Q X with Q = a + b A + c A^2, so A <- Q A Q, and `steps` of them make
//   A_0 = X0 X0^T,   P = Q_{steps-1} .. Q_1 Q_0,   X <- P X0:
// one pass over the matrix for A_0 and one for the result, whatever the number of steps, and the steps themselves on d x d matrices
// in shared memory.  Small singular values grow 3.4445-fold a step, their squares in A and what rounding adds to them
// 12-fold (2e4 times in four steps): A and Q are held in 64 bits, which leaves 1e-11 of that.
//
// Three launches: products of 64-element pieces of the long side, a block or so each (d^2 k multiply-adds, 64 per cycle and SM in 64
// bits); the steps; and the result, from P in fp32.  The steps (four products of d^3 multiply-adds each, on the 64-bit matrix
// instructions) are latency: a cluster of eight CTAs per matrix, an eighth of the rows each, whose new rows are written into all eight,
// with two cluster barriers a step of about 1 us.  More than kFewMatrices clusters wait for one another: then a CTA per matrix (48
// of 32 x 256: 42 us; 64 rows: 98 instead of 108 us, 32 of them 93 instead of 75).
// Against the tensor-core form, where a matrix of 16 rows fills 6 % of a tile and the 15 products' latencies are all of the time:
// 16 x 172 57 -> 16 us, 64 x 4096 140 -> 48 us, 1000 of 32 x 64 220 -> 149 us; many matrices of 64 rows are its side's
// (1000 of 64 x 64: 291 instead of 548 us).  Its error, 2.0e-3 with 16 .. 40 rows against 1.6e-3 with 256, is 1e-7 here.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "pcl_internal.h"
#include "pcl_ptx.cuh"

namespace pcl {

namespace {

constexpr double kNsA = 3.4445, kNsB = -4.7750, kNsC = 2.0315, kNsEps = 1e-7;
constexpr int kMostChunks = 64;                  // partial Gram matrices (a block per SM where that is a quarter of the pieces)
constexpr int kStepCtas = 8, kStepThreads = 256;
constexpr int kDim = 64;
constexpr int kLd = 68;                          // row length in shared memory: fragments of 4 x 8 elements touch every bank once
constexpr int kPiece = 64;                       // of the long side
// of a CTA that has `blocks` eights of rows
constexpr size_t step_smem(int side, int blocks) { return size_t(2 * side + 3 * 8 * blocks) * kLd * 8; }
constexpr int kFewMatrices = 32;

struct NarrowArgs {
    const void* g; int type;
    float* momentum; float mu; int nesterov;
    int d, k, wide, pieces, chunks, steps;       // wide: the matrix is d x k, else k x d
    unsigned by_d;                               // e / d = e * by_d >> 20 for e < 4096
    double* part;                                // [count][chunks][dim][dim], dim = d rounded up to 16, 32 or 64
    float* p; float2* inv;                       // [count][kDim][kDim]; [count]: X0 = (U * x) * y, x a power of two
    void* out; float keep, step;
};

template <class T> __device__ __forceinline__ float value(T v);
template <> __device__ __forceinline__ float value(float v) { return v; }
template <> __device__ __forceinline__ float value(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float value(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T rounded(float v);
template <> __device__ __forceinline__ float rounded(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 rounded(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half rounded(float v) { return __float2half_rn(v); }

// The elements of a piece as a thread of 256 takes them: number e = thread + 256 i of the piece's elements in the order of memory (a
// wide matrix: rows of kPiece).  Short side j, long side l.  Behind the end ok is false and `at` the piece's first element, so that
// all loads can be issued without a branch between them.
struct Place { int j, l; bool ok; size_t at; };
__device__ __forceinline__ Place place(const NarrowArgs& a, int e, int l0, int length) {
    Place p;
    if (a.wide) {
        p.j = e / kPiece; p.l = e % kPiece;
        p.ok = p.j < a.d && p.l < length;
        p.at = size_t(l0) + (p.ok ? size_t(p.j) * a.k + p.l : 0);
    } else {
        p.l = int(unsigned(e) * a.by_d >> 20); p.j = e - p.l * a.d;
        p.ok = p.l < length;
        p.at = size_t(l0) * a.d + (p.ok ? e : 0);
    }
    return p;
}

// Partial Gram matrices of U in 64 bits, and the momentum update.  16 x 16 threads, kB x kB results each, of which the ones below the
// diagonal of 16 x 16 squares are copies.
template <class T, int kB>
__global__ void __launch_bounds__(256) narrow_gram_kernel(NarrowArgs a) {
    constexpr int kSide = 16 * kB;
    __shared__ double tile[kPiece][kSide + 1];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int i = threadIdx.x; i < kPiece * (kSide + 1); i += 256) (&tile[0][0])[i] = 0.0;
    double acc[kB][kB] = {};
    grid_dependency_wait();
    grid_dependents_launch();
    const size_t base = size_t(blockIdx.y) * a.d * a.k;
    for (int piece = blockIdx.x; piece < a.pieces; piece += gridDim.x) {
        const int l0 = piece * kPiece, length = a.k - l0 < kPiece ? a.k - l0 : kPiece;
        const T* g = static_cast<const T*>(a.g) + base;
        float* momentum = a.momentum + base;
        T u[4 * kB];
        float m[4 * kB];
        Place at[4 * kB];
#pragma unroll
        for (int i = 0; i < 4 * kB; ++i) {
            at[i] = place(a, threadIdx.x + 256 * i, l0, length);
            u[i] = g[at[i].at];
        }
        if (a.momentum) {
#pragma unroll
            for (int i = 0; i < 4 * kB; ++i) m[i] = momentum[at[i].at];
        }
        __syncthreads();                         // (the tile's zeros, or the products of the piece before)
#pragma unroll
        for (int i = 0; i < 4 * kB; ++i) {
            float v = value(u[i]);
            if (a.momentum) {
                m[i] = fmaf(a.mu, m[i], v);
                v = a.nesterov ? fmaf(a.mu, m[i], v) : m[i];
                if (at[i].ok) momentum[at[i].at] = m[i];
            }
            if (at[i].ok) tile[at[i].l][at[i].j] = double(v);
        }
        __syncthreads();
#pragma unroll 2
        for (int l = 0; l < length; ++l) {
            double x[kB], y[kB];
#pragma unroll
            for (int i = 0; i < kB; ++i) { x[i] = tile[l][ty + 16 * i]; y[i] = tile[l][tx + 16 * i]; }
#pragma unroll
            for (int i = 0; i < kB; ++i)
#pragma unroll
                for (int j = i; j < kB; ++j) acc[i][j] = fma(x[i], y[j], acc[i][j]);
        }
    }
    double* part = a.part + (size_t(blockIdx.y) * a.chunks + blockIdx.x) * (kSide * kSide);
#pragma unroll
    for (int i = 0; i < kB; ++i)
#pragma unroll
        for (int j = i; j < kB; ++j) {
            part[(ty + 16 * i) * kSide + tx + 16 * j] = acc[i][j];
            if (j > i) part[(tx + 16 * j) * kSide + ty + 16 * i] = acc[i][j];
        }
}

// Eight rows times the matrix y: columns 8 * warp .. of the result, a lane's two (column 8 * warp + 2 * (lane % 4), row lane / 4).
// x: that row; n: the depth in fours.
__device__ __forceinline__ double2 times(const double* x, const double* y, int warp, int lane, int n) {
    const double *xa = x + (lane & 3), *yb = y + (lane & 3) * kLd + 8 * warp + (lane >> 2);
    double c[2][2] = {};
#pragma unroll
    for (int k = 0; k < kDim / 4; ++k)
        if (k < n)
            asm("mma.sync.aligned.m8n8k4.row.col.f64.f64.f64.f64 {%0, %1}, {%2}, {%3}, {%0, %1};"
                         : "+d"(c[k & 1][0]), "+d"(c[k & 1][1]) : "d"(xa[4 * k]), "d"(yb[4 * k * kLd]));
    return make_double2(c[0][0] + c[1][0], c[0][1] + c[1][1]);
}
// Two elements of this CTA's rows to the same place in all CTAs of the cluster.
template <int kCtas>
__device__ __forceinline__ void to_all(double* at, double2 v) {
    if constexpr (kCtas == 1) { *reinterpret_cast<double2*>(at) = v; return; }
#pragma unroll
    for (uint32_t r = 0; r < kCtas; ++r)
        asm volatile("st.shared::cluster.v2.f64 [%0], {%1, %2};" ::"r"(map_to_cta(at, r)), "d"(v.x), "d"(v.y) : "memory");
}
template <int kCtas>
__device__ __forceinline__ void step_barrier() {
    if constexpr (kCtas == 1) __syncthreads();
    else cluster_sync_all();
}

// The steps: A and Q in the shared memory of every CTA, of P and A Q its own rows (in eights: `blocks`), eight columns a warp.  Q is
// written when every CTA is past the products with the Q before (the barrier behind A), A when every CTA is past A A (the
// barrier behind Q) and the CTA itself past its rows of A Q.
template <int kCtas>
__global__ void __launch_bounds__(kStepThreads) narrow_steps_kernel(NarrowArgs a, int side) {
    extern __shared__ __align__(16) double shared[];
    const int rows = (a.d + kCtas - 1) / kCtas, blocks = (rows + 7) / 8, n = (a.d + 3) / 4;
    double *A = shared, *Q = A + side * kLd, *own_t = Q + side * kLd, *own_p = own_t + 8 * blocks * kLd;     // own_p: two, in turn
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = kCtas == 1 ? 0 : int(cluster_ctarank());
    const int matrix = int(blockIdx.x) / kCtas, first = rank * rows, col = 8 * warp + 2 * (lane & 3);
    for (int i = threadIdx.x; i < (2 * side + 24 * blocks) * kLd; i += kStepThreads) shared[i] = 0.0;
    // f(own row, row of A, whether there is one at this column) for the lane's rows
    auto each = [&](auto f) {
        if (8 * warp < a.d)
            for (int own = lane >> 2; own < 8 * blocks; own += 8) f(own, first + own, own < rows && first + own < a.d && col < a.d);
    };
    auto row_a = [&](int own) { return own < rows ? A + (first + own) * kLd : own_t + own * kLd; };       // (no row: zeros)
    grid_dependency_wait();
    grid_dependents_launch();
    step_barrier<kCtas>();                       // (zeros before anything is written into them)
    each([&](int own, int row, bool has) {
        if (!has) return;
        double2 sum = make_double2(0.0, 0.0);
        const double* part = a.part + size_t(matrix) * a.chunks * side * side + row * side + col;
#pragma unroll 16
        for (int c = 0; c < a.chunks; ++c) {
            const double2 v = __ldcg(reinterpret_cast<const double2*>(part + size_t(c) * side * side));
            sum.x += v.x; sum.y += v.y;
        }
        to_all<kCtas>(A + row * kLd + col, sum);
        if (col == (row & ~1)) own_p[own * kLd + row] = 1.0;
    });
    step_barrier<kCtas>();
    double squares = 0.0;                        // (zeros behind d)
    for (int i = lane; i < side; i += 32) squares += A[i * (kLd + 1)];
    for (int o = 16; o > 0; o >>= 1) squares += __shfl_xor_sync(0xffffffffu, squares, o);
    const double inv = 1.0 / (sqrt(squares) + kNsEps);
    __syncthreads();
    for (int i = threadIdx.x; i < side * kLd; i += kStepThreads) A[i] *= inv * inv;
    __syncthreads();
    // (norms from 2^100: their reciprocal times 2^64, because fp32 has fewer bits below 2^-126)
    if (rank == 0 && threadIdx.x == 0) a.inv[matrix] = inv < 0x1p-100 ? make_float2(0x1p-64f, float(inv * 0x1p64)) : make_float2(1.f, float(inv));
    for (int s = 0; s < a.steps; ++s) {
        const bool last = s + 1 == a.steps;
        each([&](int own, int row, bool has) {
            const double2 x = times(row_a(own), A, warp, lane, n);
            if (!has) return;
            const double2 v = *reinterpret_cast<const double2*>(A + row * kLd + col);
            to_all<kCtas>(Q + row * kLd + col, make_double2(kNsB * v.x + kNsC * x.x + (col == row ? kNsA : 0.0),
                                                            kNsB * v.y + kNsC * x.y + (col + 1 == row ? kNsA : 0.0)));
        });
        step_barrier<kCtas>();
        const double* p = own_p + (s & 1) * 8 * blocks * kLd;
        double* new_p = own_p + (~s & 1) * 8 * blocks * kLd;
        each([&](int own, int row, bool has) {
            const double2 x = times(p + own * kLd, Q, warp, lane, n);
            if (last) {
                if (has) *reinterpret_cast<float2*>(a.p + (size_t(matrix) * kDim + row) * kDim + col) = make_float2(float(x.x), float(x.y));
                return;
            }
            *reinterpret_cast<double2*>(new_p + own * kLd + col) = x;
            *reinterpret_cast<double2*>(own_t + own * kLd + col) = times(row_a(own), Q, warp, lane, n);
        });
        if (last) break;
        __syncthreads();                         // (own_t is whole; and the warps have read the CTA's rows of A)
        each([&](int own, int row, bool has) {
            const double2 x = times(own_t + own * kLd, Q, warp, lane, n);
            if (has) to_all<kCtas>(A + row * kLd + col, x);
        });
        step_barrier<kCtas>();
    }
}

// X = P X0 and what is made of it.  16 x 16 threads: kB rows of P (its columns: P is symmetric) and four positions each.
template <class T, int kB>
__global__ void __launch_bounds__(256, 2) narrow_apply_kernel(NarrowArgs a) {
    __shared__ __align__(16) float p[kDim * kDim];
    __shared__ __align__(16) float x[kDim * (kPiece + 4)];       // [j][l], then the piece's results in the order of memory
    const int tl = threadIdx.x & 15, ti = threadIdx.x >> 4;
    grid_dependency_wait();
    grid_dependents_launch();
    const size_t base = size_t(blockIdx.y) * a.d * a.k;
    const float4* src = reinterpret_cast<const float4*>(a.p + size_t(blockIdx.y) * kDim * kDim);
    for (int i = threadIdx.x; i < a.d * (kDim / 4); i += 256) reinterpret_cast<float4*>(p)[i] = __ldcg(src + i);
    const float2 inv = __ldcg(a.inv + blockIdx.y);
    for (int piece = blockIdx.x; piece < a.pieces; piece += gridDim.x) {
        const int l0 = piece * kPiece, length = a.k - l0 < kPiece ? a.k - l0 : kPiece;
        const T* g = static_cast<const T*>(a.g) + base;
        T *out = static_cast<T*>(a.out) + base, u[4 * kB], w[4 * kB];
        const float* momentum = a.momentum + base;
        float m[4 * kB];
        auto at = [&](int i) { return place(a, threadIdx.x + 256 * i, l0, length); };
        if (!a.momentum || a.nesterov) {
#pragma unroll
            for (int i = 0; i < 4 * kB; ++i) u[i] = g[at(i).at];
        }
        if (a.momentum) {                        // (and the update: out is read)
#pragma unroll
            for (int i = 0; i < 4 * kB; ++i) { const size_t e = at(i).at; m[i] = momentum[e]; w[i] = out[e]; }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4 * kB; ++i)
            if (const Place p = at(i); p.ok) {
                const float v = !a.momentum ? value(u[i]) : a.nesterov ? fmaf(a.mu, m[i], value(u[i])) : m[i];
                x[p.j * (kPiece + 4) + p.l] = v * inv.x * inv.y;
            }
        __syncthreads();
        float acc[kB][4] = {};
#pragma unroll 4
        for (int j = 0; j < a.d; ++j) {
            const float4 v = *reinterpret_cast<const float4*>(x + j * (kPiece + 4) + 4 * tl);
            float q[kB];
            if constexpr (kB == 4) {
                const float4 f = *reinterpret_cast<const float4*>(p + j * kDim + 4 * ti);
                q[0] = f.x; q[1] = f.y; q[2] = f.z; q[3] = f.w;
            } else {
#pragma unroll
                for (int i = 0; i < kB; ++i) q[i] = p[j * kDim + kB * ti + i];
            }
#pragma unroll
            for (int i = 0; i < kB; ++i) {
                acc[i][0] = fmaf(q[i], v.x, acc[i][0]); acc[i][1] = fmaf(q[i], v.y, acc[i][1]);
                acc[i][2] = fmaf(q[i], v.z, acc[i][2]); acc[i][3] = fmaf(q[i], v.w, acc[i][3]);
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kB; ++i) {
            const int r = kB * ti + i;
            if (r < a.d)
#pragma unroll
                for (int c = 0; c < 4; ++c) x[a.wide ? r * kPiece + 4 * tl + c : (4 * tl + c) * a.d + r] = acc[i][c];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4 * kB; ++i) {
            float v = x[threadIdx.x + 256 * i];
            if (a.momentum) v = fmaf(a.keep, value(w[i]), -a.step * v);
            if (const Place p = at(i); p.ok) out[p.at] = rounded<T>(v);
        }
    }
}

template <class T> auto gram_kernel(int side) { return side == 16 ? narrow_gram_kernel<T, 1> : side == 32 ? narrow_gram_kernel<T, 2> : narrow_gram_kernel<T, 4>; }
template <class T> auto apply_kernel(int side) { return side == 16 ? narrow_apply_kernel<T, 1> : side == 32 ? narrow_apply_kernel<T, 2> : narrow_apply_kernel<T, 4>; }
auto gram_kernel(int type, int side) { return type == DT_F32 ? gram_kernel<float>(side) : type == DT_BF16 ? gram_kernel<__nv_bfloat16>(side) : gram_kernel<__half>(side); }
auto apply_kernel(int type, int side) { return type == DT_F32 ? apply_kernel<float>(side) : type == DT_BF16 ? apply_kernel<__nv_bfloat16>(side) : apply_kernel<__half>(side); }

struct NarrowLayout { size_t part, p, inv, total; int side, chunks, pieces; };
NarrowLayout narrow_layout(int count, int M, int N) {
    NarrowLayout l{};
    const int d = M < N ? M : N, k = M < N ? N : M;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
    l.side = d <= 16 ? 16 : d <= 32 ? 32 : 64;
    l.pieces = (k + kPiece - 1) / kPiece;
    const int share = device_sm_count() * 2 / count + 1;
    l.chunks = l.pieces < share ? l.pieces : share;
    const int most = l.pieces >= 4 * kMostChunks ? device_sm_count() : kMostChunks;
    if (l.chunks > most) l.chunks = most;
    l.part = take(size_t(count) * l.chunks * l.side * l.side * 8);
    l.p = take(size_t(count) * kDim * kDim * 4);
    l.inv = take(size_t(count) * 8);
    l.total = at;
    return l;
}

}  // namespace

bool orthogonalize_is_narrow(int count, int M, int N) {
    const int d = M < N ? M : N;
    return d <= kDim / 2 || (d <= kDim && count <= kFewMatrices);
}

size_t orthogonalize_narrow_workspace_bytes(int count, int M, int N) { return narrow_layout(count, M, N).total; }

int launch_orthogonalize_narrow(const OrthoArgs& o, void* ws, cudaStream_t st) {
    static PerDeviceOnce once;
    int rc = once.run([] {
        const bool ok = cudaFuncSetAttribute(narrow_steps_kernel<1>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(step_smem(kDim, 8))) == cudaSuccess &&
                        cudaFuncSetAttribute(narrow_steps_kernel<kStepCtas>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(step_smem(kDim, 1))) == cudaSuccess;
        return ok ? int(PCL_OK) : int(PCL_ERR_CUDA);
    });
    if (rc != PCL_OK) return rc;
    const NarrowLayout l = narrow_layout(o.count, o.M, o.N);
    char* base = static_cast<char*>(ws);
    const bool wide = o.M <= o.N;
    const int d = wide ? o.M : o.N, k = wide ? o.N : o.M;
    NarrowArgs a{o.g, o.type, o.momentum, o.mu, o.nesterov, d, k, wide, l.pieces, l.chunks, o.steps, unsigned((1u << 20) / unsigned(d) + 1),
                 reinterpret_cast<double*>(base + l.part), reinterpret_cast<float*>(base + l.p), reinterpret_cast<float2*>(base + l.inv),
                 o.out, 1.f - o.lr * o.weight_decay, o.lr * sqrtf(o.M > o.N ? float(o.M) / float(o.N) : 1.f)};
    const double elems = double(o.count) * o.M * o.N, eb = double(dtype_bytes(o.type));
    {
        LaunchScope scope(KID_ORTHO, elems * (eb + (o.momentum ? 8.0 : 0.0)), st);
        rc = launch_chained(gram_kernel(o.type, l.side), dim3(l.chunks, o.count), dim3(256), 0, st, 1, a);
        if (rc != PCL_OK) return rc;
    }
    {
        LaunchScope scope(KID_ORTHO, 8.0 * o.count * o.steps * double(d) * d * d, st);
        rc = o.count <= kFewMatrices
                 ? launch_chained(narrow_steps_kernel<kStepCtas>, dim3(unsigned(o.count) * kStepCtas), dim3(kStepThreads), step_smem(l.side, 1), st, kStepCtas, a, l.side)
                 : launch_chained(narrow_steps_kernel<1>, dim3(unsigned(o.count)), dim3(kStepThreads), step_smem(l.side, (d + 7) / 8), st, 1, a, l.side);
        if (rc != PCL_OK) return rc;
    }
    LaunchScope scope(KID_ORTHO, elems * (2.0 * eb + (o.momentum ? 4.0 + eb : 0.0)), st);
    const int share = device_sm_count() * 4 / o.count + 1;
    return launch_chained(apply_kernel(o.type, l.side), dim3(l.pieces < share ? l.pieces : share, o.count), dim3(256), 0, st, 1, a);
}

}  // namespace pcl

// Softmax cross-entropy of a fully-connected layer over many classes, in pieces of the classes: the logits
//   z[n][k] = bias[k] + sum_c x[n][c] * w[k][c]
// exist only as accumulators (16-bit operands) or as one piece in the workspace (fp32 operands).
//   forward    lse[n] = log sum_k exp z[n][k];  row_loss[n] = lse[n] - z[n][label]
//   backward   z again, piece by piece;  dz = g[n] (exp(z - lse[n]) - onehot);  dx = dz w,  dw = dz^T x,  db = sum_n dz
// so the forward call is one product of 2 N C K flops and the backward call three of them.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "pcl_internal.h"
#include "pcl_ptx.cuh"

namespace pcl {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// A piece of dz (or, with fp32 operands, of the logits) takes at most this much workspace.  (Smaller pieces, which would stay in L2,
// cost more launches and waves than they save: 1024 rows, 1024 -> 100000 backward 571 us with 64 MB, 486 with 256.)
constexpr size_t kPieceBytes = size_t(256) << 20;
// dx sums over no more classes than this in one accumulator: the tensor core's additions truncate.  What goes beyond is added in
// fp32, rounded: the parts of a split product where there are few enough tiles (39 rows, 304 -> 123078: 107 us, 255 in
// pieces), else pieces of so many classes.  dw's sums over the rows are not cut: where all products have the same sign they are 3e-5 to
// 2e-4 low with 65536 rows and 4e-4 with 10^6, less than half a step of fp16 (4.9e-4).
constexpr int kMostClasses = 16384;

__device__ __forceinline__ float elem16(const void* p, int type, size_t i) {
    if (type == DT_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}

// Where C is no multiple of 8, x and w are copied to padded rows (TMA needs strides of 16 bytes): a warp per row, 16 bytes per
// store, in the longest loads that every row starts on a multiple of (950 rows, 3358 -> 77338, forward: 740 us with single
// elements, 553 with two; 3357: 672).  Rows of whole 128-byte lines, where TMA reads a row
// of a tile from one line instead of two, are not worth a copy by themselves (3001 rows, 1032 -> 50021: forward 275 -> 266 us,
// backward 914 -> 876, but 1024 rows 97 -> 116 and 377 -> 394).
struct PadSource { const uint16_t* src; uint16_t* dst; long rows; };
template <int kVec>      // elements per load: every row starts on a multiple of so many
__global__ void __launch_bounds__(256) pad_rows_kernel(PadSource first, PadSource second, int C, int ldc) {
    grid_dependency_wait();
    grid_dependents_launch();
    for (long n = blockIdx.x * 8l + (threadIdx.x >> 5); n < first.rows + second.rows; n += gridDim.x * 8l) {
        const bool one = n < first.rows;
        const long r = one ? n : n - first.rows;
        const uint16_t* row = (one ? first.src : second.src) + r * C;
        uint16_t* dst = (one ? first.dst : second.dst) + r * ldc;
#pragma unroll 2
        for (int c = (threadIdx.x & 31) * 8; c < ldc; c += 256) {
            alignas(16) uint16_t e[8] = {};
#pragma unroll
            for (int i = 0; i < 8; i += kVec)
                if (c + i < C) {
                    if constexpr (kVec == 4) *reinterpret_cast<uint2*>(e + i) = __ldg(reinterpret_cast<const uint2*>(row + c + i));
                    else if constexpr (kVec == 2) *reinterpret_cast<uint32_t*>(e + i) = __ldg(reinterpret_cast<const uint32_t*>(row + c + i));
                    else e[i] = __ldg(row + c + i);
                }
            *reinterpret_cast<uint4*>(dst + c) = *reinterpret_cast<const uint4*>(e);
        }
    }
}
PadSource pad_source(const void* src, void* dst, long rows) { return {static_cast<const uint16_t*>(src), static_cast<uint16_t*>(dst), rows}; }
int launch_pad_rows(const PadSource& first, const PadSource& second, int C, int ldc, cudaStream_t st) {
    const long rows = first.rows + second.rows;
    LaunchScope scope(KID_VOCAB_LOSS, 4.0 * double(rows) * C, st);
    const long cap = long(device_sm_count()) * 8, blocks = (rows + 7) / 8;
    return launch_chained(C % 4 == 0 ? pad_rows_kernel<4> : C % 2 == 0 ? pad_rows_kernel<2> : pad_rows_kernel<1>, dim3(unsigned(blocks < cap ? blocks : cap)), dim3(256), 0, st, 1, first, second, C, ldc);
}

// (max, sum of exp(z - max)) pairs of disjoint sets of classes, joined.  A set without a finite logit is (-inf, 0).
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
    const float nm = fmaxf(m, m2);
    const float ref = nm == -INFINITY ? 0.f : nm;
    s = s * exp2f((m - ref) * kLog2e) + s2 * exp2f((m2 - ref) * kLog2e);
    m = nm;
}
__device__ __forceinline__ void join_warp(float& m, float& s) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
        join(m, s, m2, s2);
    }
}
__device__ __forceinline__ void finish_row(int n, float m, float s, const int* labels, int ignore_label, int K,
                                           const float* label_z, float* row_loss, float* lse, unsigned int* status) {
    const float l = s == 0.f ? -INFINITY : m + logf(s);          // (no finite logit: -inf)
    lse[n] = l;
    const int label = labels[n];
    float loss = 0.f;
    if (!is_special(label, ignore_label)) {
        if (label < 0 || label >= K) atomicCAS(status, 0u, static_cast<unsigned int>(kStatusBadLabel));
        else loss = label_z[n] == -INFINITY && l == -INFINITY ? INFINITY : l - label_z[n];      // (NaN where l is)
    }
    row_loss[n] = loss;
}

// Mean over the rows that count, by the last block of the grid to end (`ended` counts them; the launch in front of it set it to
// 0): fixed order, 0 if no row counts.
__device__ __forceinline__ void mean_by_last_block(unsigned* ended, const float* row_loss, const int* labels, int ignore_label, int N,
                                                   float* loss) {
    __shared__ double sums[8];
    __shared__ int counts[8];
    __shared__ bool last;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(ended, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    double sum = 0.0;
    int count = 0;
#pragma unroll 4
    for (int n = threadIdx.x; n < N; n += 256) {
        sum += __ldcg(row_loss + n);
        count += !is_special(labels[n], ignore_label);
    }
    for (int o = 16; o > 0; o >>= 1) { sum += __shfl_xor_sync(0xffffffffu, sum, o); count += __shfl_xor_sync(0xffffffffu, count, o); }
    if ((threadIdx.x & 31) == 0) { sums[threadIdx.x >> 5] = sum; counts[threadIdx.x >> 5] = count; }
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0; count = 0;
        for (int i = 0; i < 8; ++i) { sum += sums[i]; count += counts[i]; }
        loss[0] = count ? float(sum / count) : 0.f;
    }
}

// One warp per row: joins the parts that the product's epilogue left.
__global__ void __launch_bounds__(256) loss_rows_kernel(const float2* __restrict__ part, int part_ld, int parts,
                                                        const float* __restrict__ label_z, const int* __restrict__ labels,
                                                        int ignore_label, int N, int K, float* __restrict__ row_loss,
                                                        float* __restrict__ lse, float* __restrict__ loss, unsigned* ended,
                                                        unsigned int* status) {
    grid_dependency_wait();
    grid_dependents_launch();
    const int lane = threadIdx.x & 31;
    for (int n = blockIdx.x * 8 + (threadIdx.x >> 5); n < N; n += gridDim.x * 8) {
        float m = -INFINITY, s = 0.f;
        for (int i = lane; i < parts; i += 32) {
            const float2 v = part[size_t(n) * part_ld + i];
            join(m, s, v.x, v.y);
        }
        join_warp(m, s);
        if (lane == 0) finish_row(n, m, s, labels, ignore_label, K, label_z, row_loss, lse, status);
    }
    mean_by_last_block(ended, row_loss, labels, ignore_label, N, loss);
}

// The same from the parts of the products themselves (reductions that are cut to fill the GPU): one block per row adds them up,
// with the bias, to the logits.
__device__ __forceinline__ float2 block_join(float m, float s) {
    __shared__ float ms[8], ss[8];
    join_warp(m, s);
    if ((threadIdx.x & 31) == 0) { ms[threadIdx.x >> 5] = m; ss[threadIdx.x >> 5] = s; }
    __syncthreads();
    m = ms[0]; s = ss[0];
    for (int i = 1; i < 8; ++i) join(m, s, ms[i], ss[i]);
    __syncthreads();
    return make_float2(m, s);
}
__global__ void __launch_bounds__(256) loss_parts_kernel(const float* __restrict__ z, int parts, size_t part_step, int ld,
                                                         const void* __restrict__ bias, int type, const int* __restrict__ labels,
                                                         int ignore_label, int N, int K, float* __restrict__ label_z,
                                                         float* __restrict__ row_loss, float* __restrict__ lse, float* __restrict__ loss,
                                                         unsigned* ended, unsigned int* status) {
    grid_dependency_wait();
    grid_dependents_launch();
    for (int n = blockIdx.x; n < N; n += gridDim.x) {
        const int label = labels[n];
        float m = -INFINITY, s = 0.f;
        for (int k = threadIdx.x; k < K; k += 256) {
            const float* src = z + size_t(n) * ld + k;
            float v = 0.f;
#pragma unroll 4
            for (int p = 0; p < parts; ++p) v += src[p * part_step];
            if (bias) v += elem16(bias, type, k);
            if (k == label) label_z[n] = v;
            join(m, s, v, v == -INFINITY ? 0.f : 1.f);
        }
        const float2 r = block_join(m, s);
        if (threadIdx.x == 0) finish_row(n, r.x, r.y, labels, ignore_label, K, label_z, row_loss, lse, status);
    }
    mean_by_last_block(ended, row_loss, labels, ignore_label, N, loss);
}

// What a row's dz is multiplied with, and what the products are multiplied with afterwards.  16-bit dz is kept in range by a
// power of two: fp16 has no normal numbers below 2^-14, and a probability over 100 000 classes divided by the number
// of rows lies far below; bf16 has the exponents of fp32.  The largest row gradient goes into the products' factor whole: where all
// are the same, as in a mean, its rounding would otherwise be in every element of dz in the same direction.
__global__ void __launch_bounds__(1024) grad_rows_kernel(const int* __restrict__ labels, int ignore_label,
                                                         const float* __restrict__ row_grad, int N, int type,
                                                         float* __restrict__ row_scale, float* __restrict__ alpha, int* counters) {
    __shared__ int counts[32];
    __shared__ float tops[32];
    grid_dependency_wait();
    grid_dependents_launch();
    if (counters)                                         // of the products' split workspace
        for (int i = threadIdx.x; i < int(kGemm16CounterBytes / 4); i += 1024) counters[i] = 0;
    int count = 0;
    float top = 0.f;
    for (int n = threadIdx.x; n < N; n += 1024)
        if (!is_special(labels[n], ignore_label)) {
            ++count;
            if (row_grad) top = fmaxf(top, fabsf(row_grad[n]));
        }
    for (int o = 16; o > 0; o >>= 1) {
        count += __shfl_xor_sync(0xffffffffu, count, o);
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    if ((threadIdx.x & 31) == 0) { counts[threadIdx.x >> 5] = count; tops[threadIdx.x >> 5] = top; }
    __syncthreads();
    count = 0; top = 0.f;
    for (int i = 0; i < 32; ++i) { count += counts[i]; top = fmaxf(top, tops[i]); }
    if (!row_grad) top = 1.f;
    const float up = type == DT_F16 ? 16384.f : 1.f;      // |dz| <= 2^14
    const bool whole = !row_grad || (type != DT_F32 && top > 1e-30f && top < 1e30f);
    for (int n = threadIdx.x; n < N; n += 1024) {
        float g = is_special(labels[n], ignore_label) ? 0.f : row_grad ? row_grad[n] : 1.f;
        if (whole) g = g / top * up;
        row_scale[n] = g;
    }
    if (threadIdx.x == 0) alpha[0] = !whole ? 1.f : row_grad ? top / up : 1.f / (up * float(count > 0 ? count : 1));
}

// db[k] = alpha * sum_n dz[n][k].  A block takes 64 columns, eight at a time per thread (rows of dz are padded to 64), and 32 rows
// at once; the 32 sums of a column are added in order.
__global__ void __launch_bounds__(256) dz_colsum_kernel(const uint16_t* __restrict__ dz, int N, int P, int ld, int type, const float* alpha,
                                                        void* __restrict__ db) {
    __shared__ float sums[32][65];
    grid_dependency_wait();
    grid_dependents_launch();
    const int c8 = (threadIdx.x & 7) * 8, r0 = threadIdx.x >> 3;
    const uint16_t* src = dz + blockIdx.x * 64 + c8;
    float s[8] = {};
#pragma unroll 4
    for (int n = r0; n < N; n += 32) {
        const uint4 v = *reinterpret_cast<const uint4*>(src + size_t(n) * ld);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            s[2 * i] += type == DT_BF16 ? __uint_as_float(w[i] << 16) : f.x;
            s[2 * i + 1] += type == DT_BF16 ? __uint_as_float(w[i] & 0xffff0000u) : f.y;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[r0][c8 + i] = s[i];
    __syncthreads();
    const int k = blockIdx.x * 64 + threadIdx.x;
    if (threadIdx.x < 64 && k < P) {
        float total = 0.f;
        for (int i = 0; i < 32; ++i) total += sums[i][threadIdx.x];
        total *= alpha[0];
        if (type == DT_BF16) static_cast<__nv_bfloat16*>(db)[k] = __float2bfloat16_rn(total);
        else static_cast<__half*>(db)[k] = __float2half_rn(total);
    }
}

// ---- fp32 operands: a piece of the logits is in the workspace
// one block per row; state[n] = (max, sum) over the pieces so far
__global__ void __launch_bounds__(256) piece_stats_kernel(const float* __restrict__ z, int N, int P, int col0,
                                                          const int* __restrict__ labels, float2* __restrict__ state,
                                                          float* __restrict__ label_z, unsigned* ended) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *ended = 0u;
    for (int n = blockIdx.x; n < N; n += gridDim.x) {
        const float* row = z + size_t(n) * P;
        float m = -INFINITY, s = 0.f;
        for (int k = threadIdx.x; k < P; k += 256) m = fmaxf(m, row[k]);
        const float ref = m == -INFINITY ? 0.f : m;
        for (int k = threadIdx.x; k < P; k += 256) s += exp2f((row[k] - ref) * kLog2e);
        const float2 v = block_join(m, s);
        if (threadIdx.x == 0) {
            float m0 = v.x, s0 = v.y;
            if (col0 > 0) { const float2 o = state[n]; m0 = o.x; s0 = o.y; join(m0, s0, v.x, v.y); }
            state[n] = make_float2(m0, s0);
            const int rel = max(labels[n], -1) - col0;
            if (rel >= 0 && rel < P) label_z[n] = row[rel];
        }
    }
}
__global__ void __launch_bounds__(256) piece_dz_kernel(float* __restrict__ z, int N, int P, int col0, const int* __restrict__ labels,
                                                       const float* __restrict__ lse, const float* __restrict__ row_scale,
                                                       const float* __restrict__ alpha) {
    for (int n = blockIdx.x; n < N; n += gridDim.x) {
        float* row = z + size_t(n) * P;
        const float l = lse[n], g = l == -INFINITY ? 0.f : row_scale[n] * alpha[0];     // (no finite logit: no gradient)
        const int rel = max(labels[n], -1) - col0;
        for (int k = threadIdx.x; k < P; k += 256) {
            const float q = exp2f((row[k] - l) * kLog2e) - (k == rel ? 1.f : 0.f);
            row[k] = g == 0.f ? 0.f : g * q;
        }
    }
}
__global__ void __launch_bounds__(256) add_kernel(float* __restrict__ out, const float* __restrict__ v, size_t n) {
    for (size_t i = size_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += size_t(gridDim.x) * 256) out[i] += v[i];
}

int row_blocks(int N) { const int cap = device_sm_count() * 8; return N < cap ? N : cap; }
int launched() { return cudaGetLastError() == cudaSuccess ? PCL_OK : PCL_ERR_CUDA; }

// Classes per piece: as many as the piece's budget allows, in multiples of 256.
int piece_classes(int N, int K, size_t elem_bytes) {
    size_t p = kPieceBytes / (size_t(N) * elem_bytes) / 256 * 256;
    if (p < 256) p = 256;
    return p < size_t(K) ? int(p) : K;
}
// Row length of the padded copies: whole 128-byte lines, unless that more than doubles a row.
int staged_ld(int C) { return int(align_up(C, C >= 64 ? 64 : 8)); }
// Rows of w that are staged at a time where C is no multiple of 8.
int stage_classes(int C, int K) {
    size_t p = kPieceBytes / (size_t(staged_ld(C)) * 2) / 256 * 256;
    if (p < 256) p = 256;
    return p < size_t(K) ? int(p) : K;
}

// The products, with everything their tiling depends on; P classes of a piece.
Gemm16Args stats_args(int N, int C, int P, bool bf16) {
    Gemm16Args a{N, P, C, 1, bf16, {}, {}, GEMM16_STATS};
    a.split_ws = reinterpret_cast<void*>(256);               // (until the workspace is known)
    return a;
}
Gemm16Args dz_args(int N, int C, int P, bool bf16) {
    Gemm16Args a = stats_args(N, C, P, bf16);
    a.epi = GEMM16_DZ;
    return a;
}
Gemm16Args dx_args(int N, int C, int P, bool bf16) {
    Gemm16Args a{N, C, P, 1, bf16, {}, {}, GEMM16_GENERAL};
    a.most_blocks = kMostClasses / 64;
    a.split_ws = reinterpret_cast<void*>(256);
    return a;
}
Gemm16Args dw_args(int N, int C, int P, bool bf16) {
    Gemm16Args a{P, C, N, 1, bf16, {}, {}, GEMM16_GENERAL};
    a.split_ws = reinterpret_cast<void*>(256);
    return a;
}

struct Layout { size_t part, label_z, row_scale, alpha, xs, wst, dz, dx, fc, split, split_bytes, total; int piece, parts, k_parts, ldc, ldp; bool stage; };
Layout layout(int N, int C, int K, int type, bool backward) {
    Layout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
    const bool stage = l.stage = type != DT_F32 && C % 8 != 0;
    const bool bf16 = type == DT_BF16;
    l.ldc = stage ? staged_ld(C) : C;
    l.alpha = take(4);
    auto split = [&](const Gemm16Args& a) {
        const size_t b = gemm16_split_ws_bytes(a);
        if (b > l.split_bytes) l.split_bytes = b;
    };
    if (type == DT_F32) {
        l.piece = piece_classes(N, K, 4);
        if (backward) l.row_scale = take(size_t(N) * 4);
        else { l.label_z = take(size_t(N) * 4); l.part = take(size_t(N) * 8); }
        l.dz = take(size_t(N) * l.piece * 4);
        const int last = K - (K - 1) / l.piece * l.piece;
        size_t fc = 0;
        for (int p : {l.piece, last})
            for (int pass : {int(PCL_PASS_FWD), int(PCL_PASS_BWD_DATA)}) {
                const size_t b = pcl_fc_workspace_bytes(N, C, p, pass);
                fc = b > fc ? b : fc;
            }
        l.fc = take(fc);
        if (backward && l.piece < K) l.dx = take(size_t(N) * C * 4);
    } else if (!backward) {
        l.piece = stage ? stage_classes(C, K) : K;
        l.label_z = take(size_t(N) * 4);
        if (l.piece == K) l.k_parts = gemm16_parts(stats_args(N, C, K, bf16));
        if (l.k_parts > 1) {
            l.ldp = int(align_up(K, 32));
            l.dz = take(size_t(l.k_parts) * N * l.ldp * 4);
        }
        const int last = K - (K - 1) / l.piece * l.piece;
        l.parts = (K - 1) / l.piece * gemm16_stats_parts(stats_args(N, C, l.piece, bf16)) + gemm16_stats_parts(stats_args(N, C, last, bf16));
        l.part = take(size_t(N) * l.parts * 8);
        if (stage) { l.xs = take(size_t(N) * l.ldc * 2); l.wst = take(size_t(l.piece) * l.ldc * 2); }
    } else {
        l.piece = piece_classes(N, K, 2);
        if (stage && l.piece > stage_classes(C, K)) l.piece = stage_classes(C, K);
        if (l.piece > kMostClasses && !gemm16_possible(dx_args(N, C, l.piece, bf16))) l.piece = kMostClasses;
        l.ldp = int(align_up(l.piece, 64));
        l.row_scale = take(size_t(N) * 4);
        l.dz = take(size_t(N) * l.ldp * 2);
        if (l.piece < K) l.dx = take(size_t(N) * C * 4);
        if (stage) { l.xs = take(size_t(N) * l.ldc * 2); l.wst = take(size_t(l.piece) * l.ldc * 2); }
        const int last = K - (K - 1) / l.piece * l.piece;
        for (int p : {l.piece, last}) { split(dz_args(N, C, p, bf16)); split(dx_args(N, C, p, bf16)); split(dw_args(N, C, p, bf16)); }
    }
    l.split = take(l.split_bytes);
    l.total = at;
    return l;
}

}  // namespace

size_t vocab_loss_workspace_bytes(int N, int C, int K, int type, bool backward) { return layout(N, C, K, type, backward).total; }

int launch_vocab_loss_fwd(int N, int C, int K, int type, const void* x, const void* w, const void* bias, const int* labels,
                          int ignore_label, float* loss, float* row_loss, float* lse, void* ws, cudaStream_t st) {
    const Layout l = layout(N, C, K, type, false);
    char* base = static_cast<char*>(ws);
    float2* part = reinterpret_cast<float2*>(base + l.part);
    float* label_z = reinterpret_cast<float*>(base + l.label_z);
    unsigned int* status = device_status_ptr();
    if (!status) return PCL_ERR_CUDA;
    int rc = PCL_OK, parts = 0, part_ld = l.parts;
    unsigned* ended = reinterpret_cast<unsigned*>(base + l.alpha);
    if (type == DT_F32) {
        float* z = reinterpret_cast<float*>(base + l.dz);
        const size_t fc_bytes = l.split - l.fc;
        for (int p0 = 0; p0 < K; p0 += l.piece) {
            const int P = K - p0 < l.piece ? K - p0 : l.piece;
            rc = pcl_fc_fwd(N, C, P, static_cast<const float*>(x), static_cast<const float*>(w) + size_t(p0) * C,
                            bias ? static_cast<const float*>(bias) + p0 : nullptr, z, PCL_ACT_NONE, base + l.fc, fc_bytes, st);
            if (rc != PCL_OK) return rc;
            LaunchScope scope(KID_VOCAB_LOSS, 4.0 * double(N) * P, st);
            piece_stats_kernel<<<row_blocks(N), 256, 0, st>>>(z, N, P, p0, labels, part, label_z, ended);
            if ((rc = launched()) != PCL_OK) return rc;
        }
        parts = part_ld = 1;
    } else {
        const bool stage = l.stage;
        const void* xs = x;
        if (stage) xs = base + l.xs;
        for (int p0 = 0; p0 < K; p0 += l.piece) {
            const int P = K - p0 < l.piece ? K - p0 : l.piece;
            const void* wp = static_cast<const uint16_t*>(w) + size_t(p0) * C;
            if (stage) {                     // (x with the first piece of w)
                rc = launch_pad_rows(pad_source(x, base + l.xs, p0 == 0 ? N : 0), pad_source(wp, base + l.wst, P), C, l.ldc, st);
                if (rc != PCL_OK) return rc;
                wp = base + l.wst;
            }
            Gemm16Args a = stats_args(N, C, P, type == DT_BF16);
            a.a = {xs, l.ldc, 0, false}; a.b = {wp, l.ldc, 0, false};
            a.split_ws = nullptr;
            a.clear = ended;
            if (l.k_parts > 1) {
                a.epi = GEMM16_PARTS; a.k_parts = l.k_parts;
                a.out = base + l.dz; a.out_ld = l.ldp; a.out_batch = long(N) * l.ldp;
                rc = launch_gemm16(a, st);
                if (rc != PCL_OK) return rc;
                LaunchScope scope(KID_VOCAB_LOSS, 4.0 * double(N) * K * l.k_parts, st);
                return launch_chained(loss_parts_kernel, dim3(row_blocks(N)), dim3(256), 0, st, 1, reinterpret_cast<const float*>(base + l.dz),
                                    l.k_parts, size_t(N) * l.ldp, l.ldp, bias, type, labels, ignore_label, N, K, label_z, row_loss, lse,
                                    loss, ended, status);
            }
            a.bias = bias ? static_cast<const uint16_t*>(bias) + p0 : nullptr;
            a.labels = labels; a.col0 = p0; a.part = part + parts; a.part_ld = part_ld; a.label_z = label_z;
            rc = launch_gemm16(a, st);
            if (rc != PCL_OK) return rc;
            parts += gemm16_stats_parts(a);
        }
    }
    LaunchScope scope(KID_VOCAB_LOSS, 8.0 * double(N) * parts, st);
    const int blocks = (N + 7) / 8, cap = device_sm_count() * 8;
    return launch_chained(loss_rows_kernel, dim3(blocks < cap ? blocks : cap), dim3(256), 0, st, 1, part, part_ld, parts, label_z, labels,
                          ignore_label, N, K, row_loss, lse, loss, ended, status);
}

int launch_vocab_loss_bwd(int N, int C, int K, int type, const void* x, const void* w, const void* bias, const int* labels,
                          int ignore_label, const float* lse, const float* row_grad, void* dx, void* dw, void* dbias, void* ws,
                          cudaStream_t st) {
    const Layout l = layout(N, C, K, type, true);
    char* base = static_cast<char*>(ws);
    float* row_scale = reinterpret_cast<float*>(base + l.row_scale);
    float* alpha = reinterpret_cast<float*>(base + l.alpha);
    int rc = PCL_OK;
    {
        LaunchScope scope(KID_VOCAB_LOSS, 12.0 * double(N), st);
        rc = launch_chained(grad_rows_kernel, dim3(1), dim3(1024), 0, st, 1, labels, ignore_label, row_grad, N, type, row_scale,
                            alpha, l.split_bytes ? reinterpret_cast<int*>(base + l.split) : nullptr);
    }
    if (rc != PCL_OK) return rc;
    if (type == DT_F32) {
        float* z = reinterpret_cast<float*>(base + l.dz);
        const size_t fc_bytes = (l.piece < K ? l.dx : l.split) - l.fc;
        for (int p0 = 0; p0 < K; p0 += l.piece) {
            const int P = K - p0 < l.piece ? K - p0 : l.piece;
            const float* wp = static_cast<const float*>(w) + size_t(p0) * C;
            rc = pcl_fc_fwd(N, C, P, static_cast<const float*>(x), wp, bias ? static_cast<const float*>(bias) + p0 : nullptr, z,
                            PCL_ACT_NONE, base + l.fc, fc_bytes, st);
            if (rc != PCL_OK) return rc;
            {
                LaunchScope scope(KID_VOCAB_LOSS, 8.0 * double(N) * P, st);
                piece_dz_kernel<<<row_blocks(N), 256, 0, st>>>(z, N, P, p0, labels, lse, row_scale, alpha);
            }
            if ((rc = launched()) != PCL_OK) return rc;
            float* dxp = !dx || p0 == 0 ? static_cast<float*>(dx) : reinterpret_cast<float*>(base + l.dx);
            rc = pcl_fc_bwd(N, C, P, static_cast<const float*>(x), wp, nullptr, PCL_ACT_NONE, z, dxp,
                            static_cast<float*>(dw) + size_t(p0) * C, dbias ? static_cast<float*>(dbias) + p0 : nullptr,
                            base + l.fc, fc_bytes, st);
            if (rc != PCL_OK) return rc;
            if (dx && p0 > 0) {
                LaunchScope scope(KID_VOCAB_LOSS, 12.0 * double(N) * C, st);
                add_kernel<<<device_sm_count() * 8, 256, 0, st>>>(static_cast<float*>(dx), dxp, size_t(N) * C);
                if ((rc = launched()) != PCL_OK) return rc;
            }
        }
        return PCL_OK;
    }
    const bool stage = l.stage, bf16 = type == DT_BF16;
    uint16_t* dz = reinterpret_cast<uint16_t*>(base + l.dz);
    float* dx_acc = reinterpret_cast<float*>(base + l.dx);
    const void* xs = x;
    if (stage) xs = base + l.xs;
    for (int p0 = 0; p0 < K; p0 += l.piece) {
        const int P = K - p0 < l.piece ? K - p0 : l.piece;
        const void* wp = static_cast<const uint16_t*>(w) + size_t(p0) * C;
        if (stage) {                     // (x with the first piece of w)
            rc = launch_pad_rows(pad_source(x, base + l.xs, p0 == 0 ? N : 0), pad_source(wp, base + l.wst, P), C, l.ldc, st);
            if (rc != PCL_OK) return rc;
            wp = base + l.wst;
        }
        Gemm16Args z = dz_args(N, C, P, bf16);
        z.a = {xs, l.ldc, 0, false}; z.b = {wp, l.ldc, 0, false};
        z.split_ws = base + l.split;
        z.bias = bias ? static_cast<const uint16_t*>(bias) + p0 : nullptr;
        z.labels = labels; z.col0 = p0; z.lse = lse; z.row_scale = row_scale;
        z.out = dz; z.out_type = type; z.out_ld = l.ldp;
        rc = launch_gemm16(z, st);
        if (rc != PCL_OK) return rc;
        if (dbias) {
            LaunchScope scope(KID_VOCAB_LOSS, 2.0 * double(N) * P, st);
            rc = launch_chained(dz_colsum_kernel, dim3((P + 63) / 64), dim3(256), 0, st, 1, dz, N, P, l.ldp, type, alpha,
                                static_cast<uint16_t*>(dbias) + p0);
            if (rc != PCL_OK) return rc;
        }
        if (dx) {
            Gemm16Args g = dx_args(N, C, P, bf16);
            g.a = {dz, l.ldp, 0, false}; g.b = {wp, l.ldc, 0, true};
            g.split_ws = base + l.split;
            const bool last = p0 + l.piece >= K;
            g.alpha_dev = alpha;
            if (p0 > 0) { g.src = dx_acc; g.src_type = DT_F32; g.src_ld = C; g.beta = 1.f; }
            g.out = last ? dx : dx_acc; g.out_type = last ? type : int(DT_F32); g.out_ld = C;
            rc = launch_gemm16(g, st);
            if (rc != PCL_OK) return rc;
        }
        Gemm16Args g = dw_args(N, C, P, bf16);
        g.a = {dz, l.ldp, 0, true}; g.b = {xs, l.ldc, 0, true};
        g.split_ws = base + l.split;
        g.alpha_dev = alpha;
        g.out = static_cast<uint16_t*>(dw) + size_t(p0) * C; g.out_type = type; g.out_ld = C;
        rc = launch_gemm16(g, st);
        if (rc != PCL_OK) return rc;
    }
    return PCL_OK;
}

}  // namespace pcl

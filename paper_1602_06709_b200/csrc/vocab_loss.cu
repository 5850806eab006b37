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

namespace pcl {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// A piece of dz (or, with fp32 operands, of the logits) takes at most this much workspace.
constexpr size_t kPieceBytes = size_t(256) << 20;

__device__ __forceinline__ float elem(const void* p, int type, size_t i) {
    if (type == DT_F32) return static_cast<const float*>(p)[i];
    if (type == DT_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}

// Rows whose length is no multiple of 8 elements cannot be read by TMA (16-byte strides): they are copied to padded rows.
__global__ void __launch_bounds__(256) pad_rows_kernel(const uint16_t* __restrict__ src, uint16_t* __restrict__ dst, long rows,
                                                       int C, int ldc) {
    for (long r = blockIdx.x; r < rows; r += gridDim.x)
        for (int c = threadIdx.x; c < ldc; c += blockDim.x) dst[r * ldc + c] = c < C ? src[r * C + c] : uint16_t(0);
}
int launch_pad_rows(const void* src, void* dst, long rows, int C, int ldc, cudaStream_t st) {
    LaunchScope scope(KID_VOCAB_LOSS, 4.0 * double(rows) * C, st);
    const long cap = long(device_sm_count()) * 16;
    pad_rows_kernel<<<int(rows < cap ? rows : cap), 256, 0, st>>>(static_cast<const uint16_t*>(src), static_cast<uint16_t*>(dst),
                                                                  rows, C, ldc);
    return cudaGetLastError() == cudaSuccess ? PCL_OK : PCL_ERR_CUDA;
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
    if (label != ignore_label) {
        if (label < 0 || label >= K) atomicCAS(status, 0u, static_cast<unsigned int>(kStatusBadLabel));
        else loss = label_z[n] == -INFINITY ? INFINITY : l - label_z[n];
    }
    row_loss[n] = loss;
}

// One warp per row: joins the parts that the product's epilogue left.
__global__ void __launch_bounds__(256) loss_rows_kernel(const float2* __restrict__ part, int part_ld, int parts,
                                                        const float* __restrict__ label_z, const int* __restrict__ labels,
                                                        int ignore_label, int N, int K, float* __restrict__ row_loss,
                                                        float* __restrict__ lse, unsigned int* status) {
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
}

// Mean over the rows that count (fixed order; 0 if none does).
__global__ void __launch_bounds__(1024) loss_mean_kernel(const float* __restrict__ row_loss, const int* __restrict__ labels,
                                                         int ignore_label, int N, float* __restrict__ loss) {
    __shared__ double sums[32];
    __shared__ int counts[32];
    double sum = 0.0;
    int count = 0;
    for (int n = threadIdx.x; n < N; n += 1024) {
        sum += row_loss[n];
        count += labels[n] != ignore_label;
    }
    for (int o = 16; o > 0; o >>= 1) { sum += __shfl_xor_sync(0xffffffffu, sum, o); count += __shfl_xor_sync(0xffffffffu, count, o); }
    if ((threadIdx.x & 31) == 0) { sums[threadIdx.x >> 5] = sum; counts[threadIdx.x >> 5] = count; }
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0; count = 0;
        for (int i = 0; i < 32; ++i) { sum += sums[i]; count += counts[i]; }
        loss[0] = count ? float(sum / count) : 0.f;
    }
}

// What a row's dz is multiplied with, and what the products are multiplied with afterwards.  16-bit dz is kept in range by a
// power of two: fp16 has no normal numbers below 2^-14, and a probability over 100 000 classes divided by the number
// of rows lies far below; bf16 has the exponents of fp32.
__global__ void __launch_bounds__(1024) grad_rows_kernel(const int* __restrict__ labels, int ignore_label,
                                                         const float* __restrict__ row_grad, int N, int f16,
                                                         float* __restrict__ row_scale, float* __restrict__ alpha) {
    __shared__ int counts[32];
    __shared__ float tops[32];
    int count = 0;
    float top = 0.f;
    for (int n = threadIdx.x; n < N; n += 1024)
        if (labels[n] != ignore_label) {
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
    float up = 1.f;
    if (f16 && top > 0.f && top < 1e30f) {
        int e;
        frexpf(top, &e);                                  // top = f * 2^e, f in [0.5, 1)
        const int shift = 14 - e < 100 ? 14 - e : 100;    // |dz| <= 2 * 2^14
        up = ldexpf(1.f, shift);
    }
    for (int n = threadIdx.x; n < N; n += 1024)
        row_scale[n] = labels[n] == ignore_label ? 0.f : (row_grad ? row_grad[n] * up : up);
    if (threadIdx.x == 0) alpha[0] = row_grad ? 1.f / up : 1.f / (up * float(count > 0 ? count : 1));
}

// db[k] = alpha * sum_n dz[n][k].  32 columns x 8 row lanes per block, rows in a fixed order.
template <class T>
__global__ void __launch_bounds__(256) dz_colsum_kernel(const T* __restrict__ dz, int N, int P, int ld, const float* alpha,
                                                        T* __restrict__ db) {
    __shared__ float sums[8][33];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int k = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (k < P)
        for (int n = w; n < N; n += 8) s += float(dz[size_t(n) * ld + k]);
    sums[w][lane] = s;
    __syncthreads();
    if (w == 0 && k < P) {
        s = 0.f;
        for (int i = 0; i < 8; ++i) s += sums[i][lane];
        db[k] = T(s * alpha[0]);
    }
}

// ---- fp32 operands: a piece of the logits is in the workspace
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
// one block per row; state[n] = (max, sum) over the pieces so far
__global__ void __launch_bounds__(256) piece_stats_kernel(const float* __restrict__ z, int N, int P, int col0,
                                                          const int* __restrict__ labels, float2* __restrict__ state,
                                                          float* __restrict__ label_z) {
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
            const int rel = labels[n] - col0;
            if (rel >= 0 && rel < P) label_z[n] = row[rel];
        }
    }
}
__global__ void __launch_bounds__(256) piece_dz_kernel(float* __restrict__ z, int N, int P, int col0, const int* __restrict__ labels,
                                                       const float* __restrict__ lse, const float* __restrict__ row_scale,
                                                       const float* __restrict__ alpha) {
    for (int n = blockIdx.x; n < N; n += gridDim.x) {
        float* row = z + size_t(n) * P;
        const float g = row_scale[n] * alpha[0], l = lse[n], ref = l == -INFINITY ? 0.f : l;
        const int rel = labels[n] - col0;
        for (int k = threadIdx.x; k < P; k += 256) {
            const float q = exp2f((row[k] - ref) * kLog2e) - (k == rel ? 1.f : 0.f);
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
// Rows of w that are staged at a time where C is no multiple of 8.
int stage_classes(int C, int K) {
    size_t p = kPieceBytes / (align_up(C, 8) * 2) / 256 * 256;
    if (p < 256) p = 256;
    return p < size_t(K) ? int(p) : K;
}

struct Layout { size_t part, label_z, row_scale, alpha, xs, wst, dz, dx, fc, total; int piece, parts, ldc, ldp; };
Layout layout(int N, int C, int K, int type, bool backward) {
    Layout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
    l.ldc = int(align_up(C, 8));
    const bool stage = type != DT_F32 && C % 8 != 0;
    l.alpha = take(4);
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
        const int last = K - (K - 1) / l.piece * l.piece;
        l.parts = (K - 1) / l.piece * gemm16_stats_parts(N, l.piece) + gemm16_stats_parts(N, last);
        l.part = take(size_t(N) * l.parts * 8);
        if (stage) { l.xs = take(size_t(N) * l.ldc * 2); l.wst = take(size_t(l.piece) * l.ldc * 2); }
    } else {
        l.piece = piece_classes(N, K, 2);
        if (stage && l.piece > stage_classes(C, K)) l.piece = stage_classes(C, K);
        l.ldp = int(align_up(l.piece, 64));
        l.row_scale = take(size_t(N) * 4);
        l.dz = take(size_t(N) * l.ldp * 2);
        if (l.piece < K) l.dx = take(size_t(N) * C * 4);
        if (stage) { l.xs = take(size_t(N) * l.ldc * 2); l.wst = take(size_t(l.piece) * l.ldc * 2); }
    }
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
    if (type == DT_F32) {
        float* z = reinterpret_cast<float*>(base + l.dz);
        const size_t fc_bytes = l.total - l.fc;
        for (int p0 = 0; p0 < K; p0 += l.piece) {
            const int P = K - p0 < l.piece ? K - p0 : l.piece;
            rc = pcl_fc_fwd(N, C, P, static_cast<const float*>(x), static_cast<const float*>(w) + size_t(p0) * C,
                            bias ? static_cast<const float*>(bias) + p0 : nullptr, z, PCL_ACT_NONE, base + l.fc, fc_bytes, st);
            if (rc != PCL_OK) return rc;
            LaunchScope scope(KID_VOCAB_LOSS, 4.0 * double(N) * P, st);
            piece_stats_kernel<<<row_blocks(N), 256, 0, st>>>(z, N, P, p0, labels, part, label_z);
            if ((rc = launched()) != PCL_OK) return rc;
        }
        parts = part_ld = 1;
    } else {
        const bool stage = C % 8 != 0;
        const void* xs = x;
        if (stage) {
            rc = launch_pad_rows(x, base + l.xs, N, C, l.ldc, st);
            if (rc != PCL_OK) return rc;
            xs = base + l.xs;
        }
        for (int p0 = 0; p0 < K; p0 += l.piece) {
            const int P = K - p0 < l.piece ? K - p0 : l.piece;
            const void* wp = static_cast<const uint16_t*>(w) + size_t(p0) * C;
            if (stage) {
                rc = launch_pad_rows(wp, base + l.wst, P, C, l.ldc, st);
                if (rc != PCL_OK) return rc;
                wp = base + l.wst;
            }
            Gemm16Args a{N, P, C, 1, type == DT_BF16, {xs, l.ldc, 0, false}, {wp, l.ldc, 0, false}, GEMM16_STATS};
            a.bias = bias ? static_cast<const uint16_t*>(bias) + p0 : nullptr;
            a.labels = labels; a.col0 = p0; a.part = part + parts; a.part_ld = part_ld; a.label_z = label_z;
            rc = launch_gemm16(a, st);
            if (rc != PCL_OK) return rc;
            parts += gemm16_stats_parts(N, P);
        }
    }
    {
        LaunchScope scope(KID_VOCAB_LOSS, 8.0 * double(N) * parts, st);
        const int blocks = (N + 7) / 8, cap = device_sm_count() * 8;
        loss_rows_kernel<<<blocks < cap ? blocks : cap, 256, 0, st>>>(part, part_ld, parts, label_z, labels, ignore_label, N, K,
                                                                      row_loss, lse, status);
    }
    if ((rc = launched()) != PCL_OK) return rc;
    {
        LaunchScope scope(KID_VOCAB_LOSS, 8.0 * double(N), st);
        loss_mean_kernel<<<1, 1024, 0, st>>>(row_loss, labels, ignore_label, N, loss);
    }
    return launched();
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
        grad_rows_kernel<<<1, 1024, 0, st>>>(labels, ignore_label, row_grad, N, type == DT_F16, row_scale, alpha);
    }
    if ((rc = launched()) != PCL_OK) return rc;
    if (type == DT_F32) {
        float* z = reinterpret_cast<float*>(base + l.dz);
        const size_t fc_bytes = (l.piece < K ? l.dx : l.total) - l.fc;
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
    const bool stage = C % 8 != 0, bf16 = type == DT_BF16;
    uint16_t* dz = reinterpret_cast<uint16_t*>(base + l.dz);
    float* dx_acc = reinterpret_cast<float*>(base + l.dx);
    const void* xs = x;
    if (stage) {
        rc = launch_pad_rows(x, base + l.xs, N, C, l.ldc, st);
        if (rc != PCL_OK) return rc;
        xs = base + l.xs;
    }
    for (int p0 = 0; p0 < K; p0 += l.piece) {
        const int P = K - p0 < l.piece ? K - p0 : l.piece;
        const void* wp = static_cast<const uint16_t*>(w) + size_t(p0) * C;
        if (stage) {
            rc = launch_pad_rows(wp, base + l.wst, P, C, l.ldc, st);
            if (rc != PCL_OK) return rc;
            wp = base + l.wst;
        }
        Gemm16Args z{N, P, C, 1, bf16, {xs, l.ldc, 0, false}, {wp, l.ldc, 0, false}, GEMM16_DZ};
        z.bias = bias ? static_cast<const uint16_t*>(bias) + p0 : nullptr;
        z.labels = labels; z.col0 = p0; z.lse = lse; z.row_scale = row_scale;
        z.out = dz; z.out_type = type; z.out_ld = l.ldp;
        rc = launch_gemm16(z, st);
        if (rc != PCL_OK) return rc;
        if (dbias) {
            LaunchScope scope(KID_VOCAB_LOSS, 2.0 * double(N) * P, st);
            if (bf16)
                dz_colsum_kernel<__nv_bfloat16><<<(P + 31) / 32, 256, 0, st>>>(reinterpret_cast<const __nv_bfloat16*>(dz), N, P, l.ldp, alpha,
                                                                               static_cast<__nv_bfloat16*>(dbias) + p0);
            else
                dz_colsum_kernel<__half><<<(P + 31) / 32, 256, 0, st>>>(reinterpret_cast<const __half*>(dz), N, P, l.ldp, alpha,
                                                                        static_cast<__half*>(dbias) + p0);
            if ((rc = launched()) != PCL_OK) return rc;
        }
        if (dx) {
            Gemm16Args g{N, C, P, 1, bf16, {dz, l.ldp, 0, false}, {wp, l.ldc, 0, true}, GEMM16_LINEAR};
            const bool last = p0 + l.piece >= K;
            g.alpha_dev = alpha;
            if (p0 > 0) { g.src = dx_acc; g.src_type = DT_F32; g.src_ld = C; g.beta = 1.f; }
            g.out = last ? dx : dx_acc; g.out_type = last ? type : int(DT_F32); g.out_ld = C;
            rc = launch_gemm16(g, st);
            if (rc != PCL_OK) return rc;
        }
        Gemm16Args g{P, C, N, 1, bf16, {dz, l.ldp, 0, true}, {xs, l.ldc, 0, true}, GEMM16_LINEAR};
        g.alpha_dev = alpha;
        g.out = static_cast<uint16_t*>(dw) + size_t(p0) * C; g.out_type = type; g.out_ld = C;
        rc = launch_gemm16(g, st);
        if (rc != PCL_OK) return rc;
    }
    return PCL_OK;
}

}  // namespace pcl

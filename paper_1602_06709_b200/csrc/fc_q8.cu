// FC layer with e4m3 operands, a scale for each row of x (rms_norm.cu writes such rows) and for each output (row of w):
//   y[n][k] = act(x_scale[n] * w_scale[k] * sum_c x[n][c] w[k][c] + bias[k])
// The products are exact and summed in fp32 by the tensor core; scales, bias and activation are the GEMM's epilogue (tc_gemm16.cu).
//
// Bound by the tensor cores for many rows, by the reading of w for few.  Measured: 8192 rows, 4096 -> 16384 bf16 390 us by itself (2.8 PFLOP/s, the
// tensor pipe active for 93 % of the time), 434-450 in a long run under the power cap; 16 rows of it 15.1-15.9 us (67 MB, 4.3-4.5 TB/s).
//
// TMA wants rows that start on multiples of 16 bytes: with C % 16 != 0 both operands are copied to padded rows first.
#include "pcl_internal.h"
#include "pcl_ptx.cuh"

namespace pcl {

namespace {

// The counters of the GEMM's split tiles; the GEMM sets itself up meanwhile.
__global__ void __launch_bounds__(256) clear_kernel(uint4* p, int n) {
    grid_dependency_wait();
    grid_dependents_launch();
    for (int i = threadIdx.x; i < n; i += 256) p[i] = make_uint4(0u, 0u, 0u, 0u);
}

struct Rows8 { const uint8_t* src; uint8_t* dst; long rows; };

// Rows of C bytes to rows of ldc (a multiple of 16), zeros behind.  A warp takes a row, a lane 16 bytes of it, from five aligned words.
__global__ void __launch_bounds__(256) pad_rows8_kernel(Rows8 first, Rows8 second, int C, int ldc) {
    grid_dependency_wait();
    grid_dependents_launch();
    for (long n = blockIdx.x * 8l + (threadIdx.x >> 5); n < first.rows + second.rows; n += gridDim.x * 8l) {
        const bool one = n < first.rows;
        const long r = one ? n : n - first.rows, size = (one ? first.rows : second.rows) * C;
        const uint8_t* src = one ? first.src : second.src;
        uint8_t* dst = (one ? first.dst : second.dst) + r * ldc;
        for (int c = (threadIdx.x & 31) * 16; c < ldc; c += 512) {
            const long at = r * C + c, word = at & ~3l;
            uint32_t v[4];
            if (c + 16 <= C && word + 20 <= size) {
                const uint32_t* s = reinterpret_cast<const uint32_t*>(src + word);
                uint32_t u[5];
#pragma unroll
                for (int i = 0; i < 5; ++i) u[i] = __ldg(s + i);
                const unsigned shift = unsigned(at - word) * 8;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = __funnelshift_r(u[i], u[i + 1], shift);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (c + 4 * i + j < C) v[i] |= uint32_t(src[at + 4 * i + j]) << (8 * j);
                }
            }
            *reinterpret_cast<uint4*>(dst + c) = make_uint4(v[0], v[1], v[2], v[3]);
        }
    }
}

Gemm16Args args(int N, int C, int K, int out_type) {
    Gemm16Args a{};
    a.M = N; a.N = K; a.K = int(align_up(C, 16) / 2); a.batch = 1;
    a.bf16 = out_type == DT_BF16;
    a.epi = GEMM16_Q8;
    a.split_ws = reinterpret_cast<void*>(256);            // (until the workspace is known)
    return a;
}

}  // namespace

size_t fc_q8_workspace_bytes(int N, int C, int K) {
    const size_t padded = C % 16 ? align_up(size_t(N) * align_up(C, 16), 256) + align_up(size_t(K) * align_up(C, 16), 256) : 0;
    return align_up(gemm16_split_ws_bytes(args(N, C, K, DT_F32)), 256) + padded;
}

int launch_fc_q8(int N, int C, int K, int out_type, const void* x, const float* x_scale, const void* w, const float* w_scale,
                 const void* bias, void* y, int act, void* ws, cudaStream_t st) {
    Gemm16Args a = args(N, C, K, out_type);
    const size_t split = gemm16_split_ws_bytes(a);
    const int ldc = int(align_up(C, 16));
    if (!gemm16_possible(a)) return PCL_ERR_UNSUPPORTED_SHAPE;
    a.split_ws = split ? ws : nullptr;
    if (split) {
        LaunchScope scope(KID_ZERO, double(kGemm16CounterBytes), st);
        const int rc = launch_chained(clear_kernel, dim3(1), dim3(256), 0, st, 1, static_cast<uint4*>(ws), int(kGemm16CounterBytes / 16));
        if (rc != PCL_OK) return rc;
    }
    if (C % 16) {
        uint8_t* xs = static_cast<uint8_t*>(ws) + align_up(split, 256);
        uint8_t* wp = xs + align_up(size_t(N) * ldc, 256);
        LaunchScope scope(KID_PAD_ROWS8, 2.0 * (double(N) + K) * C, st);
        const long blocks = (long(N) + K + 7) / 8, cap = long(device_sm_count()) * 8;
        const int rc = launch_chained(pad_rows8_kernel, dim3(unsigned(blocks < cap ? blocks : cap)), dim3(256), 0, st, 1,
                                      Rows8{static_cast<const uint8_t*>(x), xs, N}, Rows8{static_cast<const uint8_t*>(w), wp, K}, C, ldc);
        if (rc != PCL_OK) return rc;
        x = xs;
        w = wp;
    }
    a.a = {x, ldc / 2, 0, false};
    a.b = {w, ldc / 2, 0, false};
    a.out = y; a.out_type = out_type; a.out_ld = K;
    a.bias = bias; a.row_scale = x_scale; a.col_scale = w_scale; a.act = act;
    return launch_gemm16(a, st);
}

}  // namespace pcl

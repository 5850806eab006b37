// Orthogonalised update: five (or `steps`) Newton-Schulz steps on X0 = U / (|U|_F + 1e-7),
//   A = X X^T,  B = b A + c A A,  X <- a X + B X          (X^T X, X B for a matrix with more rows than columns)
// bring the singular values of U close to 1 and keep its singular vectors.
//
// Every product runs on the 16-bit tensor cores with fp16 operands scaled by powers of two: all values are bounded (|X|, |A|
// <= 1.5, |B| <= 2.9 by the polynomial), so fp16 has the three mantissa bits that bf16 lacks at no loss of range.  X
// itself keeps 22 bits until the last step, in two fp16 planes of which the products see the first; the last step takes the
// rounded X in its linear term too, so that the rounding is passed on by the polynomial's derivative (which is small at 1)
// instead of by B alone.  Relative error of the result (2-norm) 3e-4 .. 2e-3 on random, decaying and nearly low-rank
// spectra (up to 2.8e-3 where all singular values are alike; batches of 33 .. 64 rows 2.5e-3 and 4.1e-3), where bf16 iterates
// give 1e-2 .. 2e-1.  The Gram product's sums are not cut: 2.0e-3 with 2^20 columns too.  (Narrow matrices: orthogonalize_narrow.cu.)
// A and A A are symmetric: the tiles below the diagonal are copies of those above it.
//
// All 3 * steps products run in ONE cooperative launch (the roles of the 16-bit GEMM, see tc_gemm16.cu, one product after
// another) with a barrier of all CTAs between them: a launch of its own costs every product its set-up and the fetching
// of its code, together as much as a product of 512 x 512 matrices takes (8 x 256 x 512: 122 -> 102 us; now 90).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "gemm16_device.cuh"

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
    int* counters;              // of the products, to be zeroed
    unsigned* barrier;          // of all CTAs, to be zeroed
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
    if (blockIdx.x == 0 && blockIdx.y == 0)
    {
        for (int i = threadIdx.x; i < int(kGemm16CounterBytes / 4); i += 256) a.counters[i] = 0;
        if (threadIdx.x == 0) *a.barrier = 0u;
    }
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = sum;
    __syncthreads();
    sum = 0.0;
    for (int i = 0; i < 8; ++i) sum += red[i];
    const float inv = float(kScaleX / (sqrt(sum) + kNsEps));       // (1 / norm by itself may lie below the range of fp32)
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
Gemm16Args gram_args(int count, int M, int N, int form) {
    const int d = M < N ? M : N;
    Gemm16Args a{d, d, M < N ? N : M, count, false, {}, {}, GEMM16_SYM};
    a.form = form;
    a.split_ws = reinterpret_cast<void*>(256);               // (until the workspace is known)
    return a;
}
Gemm16Args square_args(int count, int M, int N, int form) {
    const int d = M < N ? M : N;
    return gram_args(count, d, d, form);
}
Gemm16Args apply_args(int count, int M, int N, int form) {
    Gemm16Args a{M, N, M < N ? M : N, count, false, {}, {}, GEMM16_STEP};
    a.form = form;
    a.split_ws = reinterpret_cast<void*>(256);
    return a;
}
// CTA pairs or single CTAs for all three.
int ortho_form(int count, int M, int N) {
    double time[2];
    for (int f = 0; f < 2; ++f) {
        const int form = f == 0 ? GEMM16_FORM_PAIR : GEMM16_FORM_SINGLE;
        time[f] = plan16(gram_args(count, M, N, form)).time + plan16(square_args(count, M, N, form)).time + plan16(apply_args(count, M, N, form)).time;
    }
    return time[0] <= time[1] ? GEMM16_FORM_PAIR : GEMM16_FORM_SINGLE;
}

struct OrthoLayout { size_t part, xl, xh[2], a, b, barrier, counters, total; int ld, d, ldd, form; };
OrthoLayout ortho_layout(int count, int M, int N) {
    OrthoLayout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
    // rows of whole 128-byte lines: TMA writes a row of a tile into other rows' sectors otherwise (8200 x 4100: a sixth of the time)
    l.ld = int(align_up(N, 64));
    l.d = M < N ? M : N;
    l.ldd = int(align_up(l.d, 64));
    l.form = ortho_form(count, M, N);
    l.part = take(size_t(count) * kMaxNormBlocks * 8);
    l.xl = take(size_t(count) * M * l.ld * 2);
    for (size_t& o : l.xh) o = take(size_t(count) * M * l.ld * 2);
    l.a = take(size_t(count) * l.d * l.ldd * 2);
    l.b = take(size_t(count) * l.d * l.ldd * 2);
    l.barrier = take(4);                                     // (all words of the counters may be in use: 128 tiles of pairs in two parts)
    size_t split = kGemm16CounterBytes;
    for (const Gemm16Args& a : {gram_args(count, M, N, l.form), square_args(count, M, N, l.form), apply_args(count, M, N, l.form)}) {
        const size_t b = gemm16_split_ws_bytes(a);
        if (b > split) split = b;
    }
    l.counters = take(split);
    l.total = at;
    return l;
}

struct OrthoParams {
    CUtensorMap xk[2], xmn[2], a, b;             // operands: X K-major and MN-major, A, B
    CUtensorMap x_out[2], a_out, b_out, lo_out;  // results, and what is added to them
    Gemm16Params gram, square, step, final;
    const void* x[2];
    void* out;
    int steps, wide;
    unsigned* barrier;                           // CTAs that have ended a product, summed over the products
};

// All CTAs have ended product `done` (0-based): called by the producing warp of each when it has issued its own copies.  Its
// epilogue warps have completed their stores (phase_end_bar); the counter is waited for no longer than the library's wait
// limit.  Then this CTA's epilogue warps may go on (phase_go_bar).
__device__ __forceinline__ bool ortho_barrier(Gemm16Ctx& c, const OrthoParams& o, int done) {
    if (!bounded_wait_addr_warp(smem_u32(&c.sh->phase_end_bar), done & 1, &c.sh->abort_flag, c.status, WAIT_GRID)) return false;
    int ok = 1;
    if (c.lane == 0) {
        __threadfence();
        atomicAdd(o.barrier, 1u);
        const unsigned want = gridDim.x * unsigned(done + 1);
        unsigned long long t0 = 0, limit = 0;
        for (unsigned spin = 0;; ++spin) {
            unsigned v;
            asm volatile("ld.acquire.gpu.u32 %0, [%1];" : "=r"(v) : "l"(o.barrier) : "memory");
            if (int(v - want) >= 0) break;
            if ((spin & 63u) == 63u) {
                const unsigned long long now = global_nanos();
                if (t0 == 0) { t0 = now; limit = wait_limit_nanos(c.status); }
                else if (now - t0 > limit) {
                    ok = 0;
                    *static_cast<volatile uint32_t*>(&c.sh->abort_flag) = 1u;
                    atomicCAS(c.status, 0u, unsigned(WAIT_GRID));
                    break;
                }
            }
        }
        // (the products' results are read through TMA: by this warp, whose lanes have a fence below, and by the epilogue warps, which
        // the arrival lets go, so that one has to stand before it)
        asm volatile("fence.proxy.async.global;" ::: "memory");
        if (ok) mbar_arrive(&c.sh->phase_go_bar);
    }
    ok = __shfl_sync(0xffffffffu, ok, 0);
    asm volatile("fence.proxy.async.global;" ::: "memory");
    return ok != 0;
}

template <bool kPair>
__global__ void __launch_bounds__(kThreads16, 1) orthogonalize_kernel(const __grid_constant__ OrthoParams o) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ Gemm16Shared sh;
    Gemm16Ctx c = gemm16_begin<kPair>(&sh, smem_raw, o.gram.status, kStages16 - 1);
    const int products = 3 * o.steps;
    if (c.warp == 0) {
        bool ok = true;
        for (int i = 0; i < products && ok; ++i) {
            const int step = i / 3, kind = i - 3 * step, cur = step & 1;
            const Gemm16Params& p = kind == 0 ? o.gram : kind == 1 ? o.square : o.step;
            const Item16 tile = decode_item(p, c.first < p.items ? c.first : 0);
            if (i > 0) ok = ortho_barrier(c, o, i - 1);
            if (!ok) break;
            if (kind == 2 && o.wide) ok = produce_items<kPair, false, true>(c, p, tile, &o.b, &o.xmn[cur]);
            else if (kind == 0 && !o.wide) ok = produce_items<kPair, true, true>(c, p, tile, &o.xmn[cur], &o.xmn[cur]);
            else
                ok = produce_items<kPair, false, false>(c, p, tile, kind == 1 ? &o.a : &o.xk[cur],
                                                        kind == 1 ? &o.a : kind == 0 ? &o.xk[cur] : &o.b);
        }
        if (!ok) drain_producer(c);
    } else if (c.warp == 1) {
        if (c.pair_rank == 0) {
            bool ok = true;
            for (int i = 0; i < products && ok; ++i) {
                const int kind = i % 3;
                if (kind == 2 && o.wide) ok = issue_items<kPair, false, true, false>(c, o.step);
                else if (kind == 0 && !o.wide) ok = issue_items<kPair, true, true, false>(c, o.gram);
                else ok = issue_items<kPair, false, false, false>(c, kind == 0 ? o.gram : kind == 1 ? o.square : o.step);
            }
        }
        __syncwarp();
    } else {
        bool ok = true;
        for (int i = 0; i < products && ok; ++i) {
            const int step = i / 3, kind = i - 3 * step, cur = step & 1;
            if (i > 0)      // (what is added to the product comes from the products before)
                ok = bounded_wait_warp(&sh.phase_go_bar, (i - 1) & 1, &sh.abort_flag, c.status, WAIT_GRID);
            if (!ok) break;
            if (kind < 2)
                ok = finish_items<kPair, GEMM16_SYM, false>(c, kind == 0 ? o.gram : o.square, kind == 0 ? &o.a_out : &o.b_out, nullptr,
                                                            nullptr, nullptr, kind == 0 ? nullptr : &o.a_out);
            else if (step + 1 < o.steps)
                ok = finish_items<kPair, GEMM16_STEP, false>(c, o.step, &o.x_out[cur ^ 1], step + 2 < o.steps ? &o.lo_out : nullptr, nullptr, nullptr,
                                                             &o.x_out[cur], &o.lo_out);
            else
                ok = finish_items<kPair, GEMM16_FINAL, false>(c, o.final, nullptr, nullptr, o.x[cur], o.out);
            __syncwarp();
            if (c.lane == 0) {
                bulk_wait_group0();      // (their completion includes the proxy fence on this side; a full one took 0.6 us a product)
                mbar_arrive(&sh.phase_end_bar);
            }
        }
        if (!ok) drain_fetch(c);
        __syncwarp();
    }
    gemm16_end<kPair>(c);
}

template <bool kPair>
int launch_ortho_kernel(const OrthoParams& o, cudaStream_t st) {
    static PerDeviceOnce once;
    static std::atomic<int> resident[64];        // CTAs (pairs) that run at the same time, per device
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return PCL_ERR_CUDA;
    cudaLaunchConfig_t lc = {};
    lc.blockDim = dim3(kThreads16);
    lc.dynamicSmemBytes = kSmem16Fetch;
    lc.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kPair ? 2 : 1; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeCooperative;
    attr[1].val.cooperative = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    const int rc = once.run([&] {
        if (cudaFuncSetAttribute(orthogonalize_kernel<kPair>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem16Fetch) != cudaSuccess) return int(PCL_ERR_CUDA);
        int n = 0;
        lc.gridDim = dim3(kPair ? 2 : 1);
        if (cudaOccupancyMaxActiveClusters(&n, orthogonalize_kernel<kPair>, &lc) != cudaSuccess || n < 1) return int(PCL_ERR_CUDA);
        resident[dev].store(n);
        return int(PCL_OK);
    });
    if (rc != PCL_OK) return rc;
    int most = o.gram.items > o.square.items ? o.gram.items : o.square.items;
    if (o.step.items > most) most = o.step.items;
    const int n = resident[dev].load();
    lc.gridDim = dim3(unsigned(most < n ? most : n) * (kPair ? 2 : 1));
    lc.numAttrs = 2;
    return cudaLaunchKernelEx(&lc, orthogonalize_kernel<kPair>, o) == cudaSuccess ? PCL_OK : PCL_ERR_CUDA;
}

}  // namespace

size_t orthogonalize_workspace_bytes(int count, int M, int N) {
    return orthogonalize_is_narrow(count, M, N) ? orthogonalize_narrow_workspace_bytes(count, M, N) : ortho_layout(count, M, N).total;
}

int launch_orthogonalize(const OrthoArgs& o, void* ws, cudaStream_t st) {
    if (orthogonalize_is_narrow(o.count, o.M, o.N)) return launch_orthogonalize_narrow(o, ws, st);
    const OrthoLayout l = ortho_layout(o.count, o.M, o.N);
    char* base = static_cast<char*>(ws);
    __half* xl = reinterpret_cast<__half*>(base + l.xl);
    __half* xh[2] = {reinterpret_cast<__half*>(base + l.xh[0]), reinterpret_cast<__half*>(base + l.xh[1])};
    void *A = base + l.a, *B = base + l.b;
    const bool wide = o.M <= o.N;
    const long xb = long(o.M) * l.ld, db = long(l.d) * l.ldd;
    StageArgs s{o.g, o.type, o.momentum, o.mu, o.nesterov, reinterpret_cast<double*>(base + l.part), 0, xh[0],
                o.steps > 1 ? xl : nullptr, o.M, o.N, l.ld, reinterpret_cast<int*>(base + l.counters),
                reinterpret_cast<unsigned*>(base + l.barrier)};
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
    // the products
    OrthoParams op;
    const Gemm16Operand xk[2] = {{xh[0], l.ld, xb, false}, {xh[1], l.ld, xb, false}}, xmn[2] = {{xh[0], l.ld, xb, true}, {xh[1], l.ld, xb, true}};
    const Gemm16Operand am{A, l.ldd, db, false}, bm{B, l.ldd, db, false};
    Gemm16Args g1 = gram_args(o.count, o.M, o.N, l.form), g2 = square_args(o.count, o.M, o.N, l.form), g3 = apply_args(o.count, o.M, o.N, l.form);
    g1.alpha = 1.f / kScaleX;                                 // kScaleX^2 A -> kScaleX A
    g2.alpha = kNsC * kScaleB / (kScaleX * kScaleX);
    g2.beta = kNsB * kScaleB / kScaleX;
    g3.alpha = 1.f / kScaleB; g3.beta = kNsA;                 // kScaleX X, in two planes (the second in place)
    Gemm16Args g4 = g3;                                       // the last step's: to the caller's matrix
    g4.epi = GEMM16_FINAL;
    g4.src = xh[0]; g4.src_type = DT_F16; g4.src_ld = l.ld; g4.src_batch = xb;
    g4.alpha = 1.f / (kScaleX * kScaleB); g4.beta = kNsA / kScaleX;
    g4.out = o.out; g4.out_type = o.type; g4.out_ld = o.N; g4.out_batch = long(o.M) * o.N;
    if (o.momentum) {
        g4.update = true;
        g4.keep = 1.f - o.lr * o.weight_decay;
        g4.step = o.lr * sqrtf(o.M > o.N ? float(o.M) / float(o.N) : 1.f);
    }
    int rc = PCL_OK;
    auto fill = [&](Gemm16Params& p, Gemm16Args& a, const Plan16& pl) {
        a.split_ws = base + l.counters;
        if (rc == PCL_OK) rc = fill_params16(p, a, pl);
    };
    const Plan16 pl1 = plan16(g1), pl2 = plan16(g2), pl3 = plan16(g3);
    fill(op.gram, g1, pl1); fill(op.square, g2, pl2); fill(op.step, g3, pl3); fill(op.final, g4, pl3);
    auto operand = [&](CUtensorMap* m, const Gemm16Operand& a, int rows, int K) { if (rc == PCL_OK) rc = operand_tmap(m, a, rows, K, o.count, false); };
    for (int i = 0; i < 2; ++i) {
        operand(&op.xk[i], xk[i], o.M, o.N);
        operand(&op.xmn[i], xmn[i], o.N, o.M);
        if (rc == PCL_OK) rc = make_tmap16(&op.x_out[i], xh[i], DT_F16, o.N, o.M, o.count, l.ld, xb, 32, 32);
        op.x[i] = xh[i];
    }
    operand(&op.a, am, l.d, l.d);
    operand(&op.b, bm, l.d, l.d);
    if (rc == PCL_OK) rc = make_tmap16(&op.lo_out, xl, DT_F16, o.N, o.M, o.count, l.ld, xb, 32, 32);
    if (rc == PCL_OK) rc = make_tmap16(&op.a_out, A, DT_F16, l.d, l.d, o.count, l.ldd, db, 32, 32);
    if (rc == PCL_OK) rc = make_tmap16(&op.b_out, B, DT_F16, l.d, l.d, o.count, l.ldd, db, 32, 32);
    if (rc != PCL_OK) return rc;
    op.out = o.out; op.steps = o.steps; op.wide = wide;
    op.barrier = reinterpret_cast<unsigned*>(base + l.barrier);
    const double m = l.d, k = o.M < o.N ? o.N : o.M;
    LaunchScope scope(KID_ORTHO, o.steps * o.count * (3.0 * m * m * k + m * m * m), st);
    return l.form == GEMM16_FORM_PAIR ? launch_ortho_kernel<true>(op, st) : launch_ortho_kernel<false>(op, st);
}

}  // namespace pcl

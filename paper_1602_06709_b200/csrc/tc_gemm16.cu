// 16-bit GEMM on tcgen05 (kind::f16: bf16 or fp16 operands, fp32 accumulators in TMEM), the contraction behind the
// vocabulary loss and the orthogonalised update:  acc[r][c] = sum_k A(r, k) * B(c, k), either operand K-major or MN-major.
//
// Persistent, warp-specialised: warp 0 TMA producer, warp 1 MMA issuer, warps 2-9 epilogue (two per TMEM lane quarter).
// Two accumulator sets: the epilogue of a tile overlaps the main loop of the next one.  A slot of the ring is one
// 64-element reduction block: 128 rows of A and 128 of B, 16 KB each (128-byte swizzle).
//   kPair = true   two CTAs of a cluster compute a 256 x 256 tile (M = 256, N = 256 MMAs): each loads its own 128 rows of
//                  A and half of the rows of B, i.e. 32 KB per 512 tensor cycles and SM (64 B/clk).
//   kPair = false  one CTA, a 128 x 128 tile: 32 KB per 256 tensor cycles, which is more than L2 delivers (~60 B/clk and
//                  SM with all SMs pulling), so it is for results with too few tiles to fill the GPU with pairs.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "pcl_internal.h"
#include "pcl_ptx.cuh"

namespace pcl {

namespace {

constexpr int kThreads16 = 320;
constexpr int kStages16 = 6;
constexpr int kSlotBytes = 32768;
constexpr int kStagingBytes = 8 * 4096;                       // one 32-row x 128-byte tile per epilogue warp
constexpr int kSmem16 = kStages16 * kSlotBytes + kStagingBytes + 1024;
constexpr int kGroupM = 8;                                    // m tiles that share a sweep over n (L2 reuse)
constexpr float kLog2e = 1.4426950408889634f;
// Up to here a logit times log2(e) stays in range, so that exp(z - ref) is one multiply-add and one ex2; beyond (classes masked
// with the type's lowest value) the difference is taken first.
constexpr float kScaledLimit = 1e38f;

struct Gemm16Params {
    int M, N, k_blocks, batch;
    int m_tiles, n_tiles, tiles_per_matrix, total_tiles;
    int symmetric, bf16;
    int epi;
    float alpha, beta, scale2, keep, step;
    const float* alpha_dev;
    const void* src; int src_type, src_vec; long src_ld, src_batch;
    void* out; int out_type, out_tma, out_vec; long out_ld, out_batch;
    int has_out2, update;
    const void* bias;
    const int* labels;
    int col0;
    float2* part; int part_ld;
    float* label_z;
    const float* lse;
    const float* row_scale;
    unsigned int* status;
};

// 32 consecutive elements of a row as fp32; `valid` of them exist.  vec: 16-byte aligned.
__device__ __forceinline__ void load_chunk(const void* base, int type, size_t off, int valid, bool vec, float (&o)[32]) {
    if (type == DT_F32) {
        const float* s = static_cast<const float*>(base) + off;
        if (vec && valid >= 32) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float4 v = reinterpret_cast<const float4*>(s)[j];
                o[4 * j] = v.x; o[4 * j + 1] = v.y; o[4 * j + 2] = v.z; o[4 * j + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = j < valid ? s[j] : 0.f;
        }
        return;
    }
    const uint16_t* s = static_cast<const uint16_t*>(base) + off;
    if (vec && valid >= 32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint4 v = reinterpret_cast<const uint4*>(s)[j];
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (type == DT_BF16) {
                    o[8 * j + 2 * i] = __uint_as_float(w[i] << 16);
                    o[8 * j + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
                } else {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                    o[8 * j + 2 * i] = f.x; o[8 * j + 2 * i + 1] = f.y;
                }
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            float f = 0.f;
            if (j < valid) {
                const uint16_t u = s[j];
                f = type == DT_BF16 ? __uint_as_float(uint32_t(u) << 16) : __half2float(__ushort_as_half(u));
            }
            o[j] = f;
        }
    }
}
__device__ __forceinline__ uint32_t pack16(float lo, float hi, bool bf16) {
    if (bf16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void store_elem(void* base, int type, size_t off, float v) {
    if (type == DT_F32) static_cast<float*>(base)[off] = v;
    else if (type == DT_BF16) static_cast<__nv_bfloat16*>(base)[off] = __float2bfloat16_rn(v);
    else static_cast<__half*>(base)[off] = __float2half_rn(v);
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void st_shared_u4(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

struct Tile16 { int b, m, n; };
__device__ __forceinline__ Tile16 decode_tile(const Gemm16Params& p, int t) {
    Tile16 o;
    o.b = t / p.tiles_per_matrix;
    int r = t - o.b * p.tiles_per_matrix;
    if (p.symmetric) {                       // tiles (m, n >= m), row by row
        int m = 0;
        while (r >= p.n_tiles - m) { r -= p.n_tiles - m; ++m; }
        o.m = m; o.n = m + r;
        return o;
    }
    const int per_group = kGroupM * p.n_tiles;
    const int g = r / per_group;
    r -= g * per_group;
    const int left = p.m_tiles - g * kGroupM;
    const int gm = left < kGroupM ? left : kGroupM;
    o.n = r / gm;
    o.m = g * kGroupM + (r - o.n * gm);
    return o;
}

// One 32-row x 128-byte tile of a warp to global memory: the staging buffer is free once the previous store has read it.
__device__ __forceinline__ void staging_wait(int lane) {
    if (lane == 0) bulk_wait_group_read0();
    __syncwarp();
}
__device__ __forceinline__ void staging_store(const CUtensorMap* tm, uint32_t stg, int lane, int col, int row, int b) {
    fence_proxy_async_shared();
    __syncwarp();
    if (lane == 0) {
        tma_store_3d(tm, stg, col, row, b);
        bulk_commit_group();
    }
}

template <bool kPair, bool kAMn, bool kBMn, int kEpi>
__global__ void __launch_bounds__(kThreads16, 1)
tc_gemm16_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                 const __grid_constant__ CUtensorMap tmOut, const __grid_constant__ CUtensorMap tmOut2, Gemm16Params p) {
    constexpr int kTileM = kPair ? 256 : 128;
    constexpr int kBN = kPair ? 256 : 128;
    constexpr int kHalf = kBN / 2;                   // columns per epilogue warp
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full_bar[kStages16];
    __shared__ uint64_t empty_bar[kStages16];
    __shared__ uint64_t acc_full_bar[2];
    __shared__ uint64_t acc_empty_bar[2];
    __shared__ uint32_t tmem_base_slot;
    __shared__ uint32_t abort_flag;

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t pair_rank = kPair ? cluster_ctarank() : 0u;
    const int first = kPair ? int(cluster_id_x()) : int(blockIdx.x);
    const int stride = kPair ? int(nclusters_x()) : int(gridDim.x);

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages16; ++s) { mbar_init(&full_bar[s], 1); mbar_init(&empty_bar[s], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&acc_full_bar[i], 1); mbar_init(&acc_empty_bar[i], kPair ? 16 : 8); }
        abort_flag = 0;
        mbar_fence_init();
        prefetch_tmap(&tmA);
        prefetch_tmap(&tmB);
    }
    if (warp == 1) {
        if constexpr (kPair) { tmem_alloc_pair(&tmem_base_slot, 2 * kBN); tmem_relinquish_pair(); }
        else { tmem_alloc(&tmem_base_slot, 2 * kBN); tmem_relinquish(); }
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (kPair) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = tmem_base_slot;

    if (warp == 0) {
        // ---------------------------------------------------------------- producer (whole warp, an elected lane issues)
        const uint32_t full0 = smem_u32(&full_bar[0]), empty0 = smem_u32(&empty_bar[0]), ring0 = smem_u32(smem);
        const uint32_t full_dst0 = kPair ? map_to_cta(&full_bar[0], 0) : full0;
        int stage = 0;
        uint32_t phase = 0;
        long issued = 0;
        bool ok = true;
        for (int t = first; t < p.total_tiles && ok; t += stride) {
            const Tile16 tile = decode_tile(p, t);
            const int ra = tile.m * kTileM + int(pair_rank) * 128, rb = tile.n * kBN + int(pair_rank) * (kBN / 2);
            for (int kb = 0; kb < p.k_blocks; ++kb) {
                if (!bounded_wait_addr_warp(empty0 + 8 * stage, phase ^ 1u, &abort_flag, p.status, WAIT_PRODUCER_EMPTY)) { ok = false; break; }
                if (pair_rank == 0) mbar_expect_tx_addr(full0 + 8 * stage, kPair ? 2 * kSlotBytes : kSlotBytes);
                const uint32_t dst = ring0 + stage * kSlotBytes, bar = full_dst0 + 8 * stage;
                if constexpr (kAMn) {
                    tma_load_3d_addr<kPair>(dst, &tmA, bar, ra, kb * 64, tile.b);
                    tma_load_3d_addr<kPair>(dst + 8192, &tmA, bar, ra + 64, kb * 64, tile.b);
                } else {
                    tma_load_3d_addr<kPair>(dst, &tmA, bar, kb * 64, ra, tile.b);
                }
                if constexpr (kBMn) {
                    tma_load_3d_addr<kPair>(dst + 16384, &tmB, bar, rb, kb * 64, tile.b);
                    tma_load_3d_addr<kPair>(dst + 24576, &tmB, bar, rb + 64, kb * 64, tile.b);
                } else {
                    tma_load_3d_addr<kPair>(dst + 16384, &tmB, bar, kb * 64, rb, tile.b);
                }
                ++issued;
                if (++stage == kStages16) { stage = 0; phase ^= 1u; }
            }
        }
        if (!ok) {
            // Gave up: copies already issued still land in this CTA's shared memory; wait (bounded) for them.
            const int pending = issued < kStages16 ? int(issued) : kStages16;
            for (int j = 0; j < pending; ++j) {
                if (--stage < 0) { stage = kStages16 - 1; phase ^= 1u; }
                for (uint32_t spin = 0; spin < (1u << 20); ++spin)
                    if (mbar_try_wait(&full_bar[stage], phase)) break;
            }
        }
    } else if (warp == 1) {
        // ---------------------------------------------------------------- MMA issuer
        if (pair_rank == 0) {
            const uint32_t idesc = make_idesc_f16(kBN, p.bf16 != 0, kAMn, kBMn, kTileM);
            const uint32_t ring0 = smem_u32(smem);
            // K-major: 8-row groups 1 KB apart.  MN-major: 64-row groups 8 KB apart, 8-deep reduction groups 1 KB apart.
            const uint64_t da = make_smem_desc(ring0, kAMn ? 8192 : 0, 1024, kSwizzle128B);
            const uint64_t db = make_smem_desc(ring0 + 16384, kBMn ? 8192 : 0, 1024, kSwizzle128B);
            const uint32_t a_hi = uint32_t(da >> 32), b_hi = uint32_t(db >> 32), a_lo0 = uint32_t(da), b_lo0 = uint32_t(db);
            const uint32_t full0 = smem_u32(&full_bar[0]), empty0 = smem_u32(&empty_bar[0]);
            const uint32_t af0 = smem_u32(&acc_full_bar[0]), ae0 = smem_u32(&acc_empty_bar[0]);
            int stage = 0;
            uint32_t phase = 0;
            int it = 0;
            bool ok = true;
            for (int t = first; t < p.total_tiles && ok; t += stride, ++it) {
                const uint32_t buf = it & 1;
                if (!bounded_wait_addr_warp(ae0 + 8 * buf, ((it >> 1) & 1) ^ 1u, &abort_flag, p.status, WAIT_MMA_TMEM_EMPTY)) { ok = false; break; }
                tc_fence_after();
                const uint32_t d = tmem_base + buf * kBN;
                uint32_t accum = 0;
                for (int kb = 0; kb < p.k_blocks; ++kb) {
                    if (!bounded_wait_addr_warp(full0 + 8 * stage, phase, &abort_flag, p.status, WAIT_MMA_FULL)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t off = uint32_t(stage) * (kSlotBytes / 16);
                    umma_kstep_f16<kPair, kAMn ? 128 : 2, kBMn ? 128 : 2>(d, a_lo0 + off, b_lo0 + off, a_hi, b_hi, idesc, accum);
                    accum = 1;
                    umma_commit_addr<kPair>(empty0 + 8 * stage);
                    if (++stage == kStages16) { stage = 0; phase ^= 1u; }
                }
                if (ok) umma_commit_addr<kPair>(af0 + 8 * buf);
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- epilogue
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const uint32_t stg = smem_u32(smem) + kStages16 * kSlotBytes + (warp - 2) * 4096;
        const uint32_t stg_row = stg + lane * 128;
        const uint32_t sw = lane & 7;
        const uint32_t ae0 = smem_u32(&acc_empty_bar[0]);
        const uint32_t ae_dst0 = kPair ? map_to_cta(&acc_empty_bar[0], 0) : ae0;
        const float alpha = kEpi == GEMM16_LINEAR ? p.alpha * (p.alpha_dev ? __ldg(p.alpha_dev) : 1.f) : 1.f;
        int it = 0;
        for (int t = first; t < p.total_tiles; t += stride, ++it) {
            const Tile16 tile = decode_tile(p, t);
            const uint32_t buf = it & 1;
            const int row0 = tile.m * kTileM + int(pair_rank) * 128 + quarter * 32, row = row0 + lane;
            const int cbase = tile.n * kBN + half * kHalf;
            const bool row_ok = row < p.M;
            int label = -1;
            float lse = 0.f, g = 0.f;
            if constexpr (kEpi != GEMM16_LINEAR) {
                if (row_ok) label = p.labels[row] - p.col0;
                if constexpr (kEpi == GEMM16_DZ) {
                    if (row_ok) { lse = p.lse[row]; g = p.row_scale[row]; }
                }
            }
            if (!bounded_wait_warp_relaxed(&acc_full_bar[buf], (it >> 1) & 1, &abort_flag, p.status, WAIT_EPI_TMEM_FULL)) break;
            tc_fence_after();
            const uint32_t taddr = tmem_base + buf * kBN + half * kHalf + (uint32_t(quarter * 32) << 16);
            float mx = -INFINITY, sum = 0.f;            // STATS: running maximum and sum of this thread's half row
            for (int c = 0; c < kHalf; c += 32) {
                const int col = cbase + c;
                if (col >= p.N) break;
                const int valid = p.N - col < 32 ? p.N - col : 32;
                uint32_t u[32];
                tmem_ld_32x32(taddr + c, u);
                float s[32];
                if constexpr (kEpi == GEMM16_LINEAR) {
                    if (p.src) load_chunk(p.src, p.src_type, size_t(tile.b) * p.src_batch + size_t(row_ok ? row : 0) * p.src_ld + col,
                                          row_ok ? valid : 0, p.src_vec != 0, s);
                } else {
                    if (p.bias) load_chunk(p.bias, p.bf16 ? DT_BF16 : DT_F16, size_t(col), valid, true, s);
                }
                tmem_ld_wait();
                float v[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(u[j]);
                if constexpr (kEpi == GEMM16_STATS) {
                    if (p.bias)
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] += s[j];
                    if (valid < 32)
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = j < valid ? v[j] : -INFINITY;
                    const int rel = label - col;
                    if (rel >= 0 && rel < valid) {
                        float z = 0.f;
#pragma unroll
                        for (int j = 0; j < 32; ++j) z = j == rel ? v[j] : z;
                        p.label_z[row] = z;
                    }
                    float cm = v[0];
#pragma unroll
                    for (int j = 1; j < 32; ++j) cm = fmaxf(cm, v[j]);
                    const float nm = fmaxf(mx, cm);
                    const float ref = nm == -INFINITY ? 0.f : nm;                 // (an empty chunk adds exp(-inf) = 0)
                    float add = 0.f;
                    if (fabsf(ref) < kScaledLimit) {
                        const float ref2 = ref * kLog2e;
#pragma unroll
                        for (int j = 0; j < 32; ++j) add += ex2(fmaf(v[j], kLog2e, -ref2));
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) add += ex2((v[j] - ref) * kLog2e);
                    }
                    sum = sum * ex2((mx - ref) * kLog2e) + add;
                    mx = nm;
                } else if constexpr (kEpi == GEMM16_DZ) {
                    if (p.bias)
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] += s[j];
                    const int rel = label - col;
                    const float ref = lse == -INFINITY ? 0.f : lse;               // a row without any finite logit has p = 0
                    const float ref2 = ref * kLog2e;
                    if (fabsf(ref) < kScaledLimit) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = ex2(fmaf(v[j], kLog2e, -ref2));
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = ex2((v[j] - ref) * kLog2e);
                    }
                    if (rel >= 0 && rel < 32)
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] -= j == rel ? 1.f : 0.f;
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = g == 0.f ? 0.f : g * v[j];      // (rows left out: exactly 0, whatever z is)
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] *= alpha;
                    if (p.src)
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = fmaf(p.beta, s[j], v[j]);
                    if (p.update) {
                        load_chunk(p.out, p.out_type, size_t(tile.b) * p.out_batch + size_t(row_ok ? row : 0) * p.out_ld + col,
                                   row_ok ? valid : 0, p.out_vec != 0, s);
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = fmaf(p.keep, s[j], -p.step * v[j]);
                    }
                }
                if constexpr (kEpi != GEMM16_STATS) {
                    const bool odd = (c & 32) != 0;
                    if (!p.out_tma) {
                        if (row_ok && p.out) {
                            const size_t off = size_t(tile.b) * p.out_batch + size_t(row) * p.out_ld + col;
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (j < valid) store_elem(p.out, p.out_type, off + j, v[j]);
                        }
                    } else if (kEpi == GEMM16_LINEAR && p.out_type == DT_F32) {
                        staging_wait(lane);
#pragma unroll
                        for (uint32_t j = 0; j < 8; ++j)
                            st_shared_v4(stg_row + ((j ^ sw) << 4), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                        if (row0 < p.M) staging_store(&tmOut, stg, lane, col, row0, tile.b);
                    } else {
                        const bool bf = kEpi == GEMM16_DZ ? p.bf16 != 0 : p.out_type == DT_BF16;
                        if (!odd) staging_wait(lane);
#pragma unroll
                        for (uint32_t j = 0; j < 4; ++j)
                            st_shared_u4(stg_row + (((j + (odd ? 4u : 0u)) ^ sw) << 4), pack16(v[8 * j], v[8 * j + 1], bf),
                                         pack16(v[8 * j + 2], v[8 * j + 3], bf), pack16(v[8 * j + 4], v[8 * j + 5], bf),
                                         pack16(v[8 * j + 6], v[8 * j + 7], bf));
                        if ((odd || col + 32 >= p.N) && row0 < p.M)
                            staging_store(&tmOut, stg, lane, odd ? col - 32 : col, row0, tile.b);
                    }
                    if constexpr (kEpi == GEMM16_LINEAR) {
                        if (p.symmetric && tile.n > tile.m && row_ok) {          // the mirror image: lanes are 32 columns of a row
                            const size_t base = size_t(tile.b) * p.out_batch + row;
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (j < valid) store_elem(p.out, p.out_type, base + size_t(col + j) * p.out_ld, v[j]);
                        }
                        if (p.has_out2) {                                        // fp16 copy for the next product
                            staging_wait(lane);
#pragma unroll
                            for (uint32_t j = 0; j < 4; ++j) {
                                uint32_t w[4];
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    w[i] = pack16(v[8 * j + 2 * i] * p.scale2, v[8 * j + 2 * i + 1] * p.scale2, false);
                                st_shared_u4(stg + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4), w[0], w[1], w[2], w[3]);
                            }
                            if (row0 < p.M) staging_store(&tmOut2, stg, lane, col, row0, tile.b);
                        }
                    }
                }
            }
            // the accumulator set is read: hand it back
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (kPair) mbar_arrive_cluster(ae_dst0 + 8 * buf);
                else mbar_arrive(&acc_empty_bar[buf]);
            }
            if constexpr (kEpi == GEMM16_STATS) {
                if (row_ok) p.part[size_t(row) * p.part_ld + 2 * tile.n + half] = make_float2(mx, sum);
            }
        }
        if (lane == 0) bulk_wait_group0();
        __syncwarp();
    }

    tc_fence_before();
    __syncthreads();
    if constexpr (kPair) cluster_sync_all();     // neither CTA leaves while the pair's MMAs may read its tiles
    if (warp == 1) {
        tc_fence_after();
        if constexpr (kPair) tmem_dealloc_pair(tmem_base, 2 * kBN);
        else tmem_dealloc(tmem_base, 2 * kBN);
    }
}

// Tensor map over [batch][outer][inner] elements, swizzled over the box's inner extent (128 or 64 bytes).
int make_tmap16(CUtensorMap* out, const void* base, int type, uint64_t inner, uint64_t outer, uint64_t batch, long ld,
                long batch_stride, uint32_t box_inner, uint32_t box_outer) {
    encode_tiled_fn enc = get_encode_tiled();
    if (!enc) return PCL_ERR_CUDA;
    const size_t es = dtype_bytes(type);
    const cuuint64_t dims[3] = {inner, outer, batch};
    const cuuint64_t strides[2] = {cuuint64_t(ld) * es, cuuint64_t(batch > 1 ? batch_stride : ld) * es};
    const cuuint32_t box[3] = {box_inner, box_outer, 1}, ones[3] = {1, 1, 1};
    if (reinterpret_cast<uintptr_t>(base) & 15) return PCL_ERR_MISALIGNED;
    if (strides[0] % 16 || strides[1] % 16 || strides[0] >= (1ull << 40) || strides[1] >= (1ull << 40)) return PCL_ERR_UNSUPPORTED_SHAPE;
    const CUtensorMapDataType dt = type == DT_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                 : type == DT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const CUresult r = enc(out, dt, 3, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           box_inner * es == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? PCL_OK : PCL_ERR_CUDA;
}

int operand_tmap(CUtensorMap* tm, const Gemm16Operand& o, int rows, int K, int batch, bool bf16) {
    const int type = bf16 ? DT_BF16 : DT_F16;
    return o.mn_major ? make_tmap16(tm, o.ptr, type, rows, K, batch, o.ld, o.batch_stride, 64, 64)
                      : make_tmap16(tm, o.ptr, type, K, rows, batch, o.ld, o.batch_stride, 64, 128);
}

template <bool kPair, bool kAMn, bool kBMn, int kEpi>
int launch_variant(const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& to, const CUtensorMap& to2,
                   const Gemm16Params& p, cudaStream_t st) {
    static PerDeviceOnce once;
    auto kernel = tc_gemm16_kernel<kPair, kAMn, kBMn, kEpi>;
    const int rc = once.run([&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem16) == cudaSuccess ? PCL_OK
                                                                                                                 : PCL_ERR_CUDA;
    });
    if (rc != PCL_OK) return rc;
    const int slots = device_sm_count() / (kPair ? 2 : 1);
    const int grid = (p.total_tiles < slots ? p.total_tiles : slots) * (kPair ? 2 : 1);
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(grid);
    lc.blockDim = dim3(kThreads16);
    lc.dynamicSmemBytes = kSmem16;
    lc.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {kPair ? 2u : 1u, 1u, 1u};
    lc.attrs = attr;
    lc.numAttrs = 1;
    return cudaLaunchKernelEx(&lc, kernel, ta, tb, to, to2, p) == cudaSuccess ? PCL_OK : PCL_ERR_CUDA;
}

template <bool kPair>
int launch_form(const Gemm16Args& a, const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& to,
                const CUtensorMap& to2, const Gemm16Params& p, cudaStream_t st) {
    if (a.epi == GEMM16_STATS) return launch_variant<kPair, false, false, GEMM16_STATS>(ta, tb, to, to2, p, st);
    if (a.epi == GEMM16_DZ) return launch_variant<kPair, false, false, GEMM16_DZ>(ta, tb, to, to2, p, st);
    if (!a.a.mn_major && !a.b.mn_major) return launch_variant<kPair, false, false, GEMM16_LINEAR>(ta, tb, to, to2, p, st);
    if (!a.a.mn_major) return launch_variant<kPair, false, true, GEMM16_LINEAR>(ta, tb, to, to2, p, st);
    if (a.b.mn_major) return launch_variant<kPair, true, true, GEMM16_LINEAR>(ta, tb, to, to2, p, st);
    return PCL_ERR_UNSUPPORTED_SHAPE;        // (no product here has an MN-major A with a K-major B)
}

// Pairs or single CTAs: both need about as long for a tile's 64-deep block when the GPU is full (see the header), so the
// form with fewer waves is taken, and single CTAs, whose epilogue is half as long, where both fit one wave.
bool use_pairs(const Gemm16Args& a) {
    const long sms = device_sm_count();
    auto waves = [&](int tile, long slots) {
        const long mt = (a.M + tile - 1) / tile, nt = (a.N + tile - 1) / tile;
        const long tiles = (a.symmetric ? mt * (mt + 1) / 2 : mt * nt) * a.batch;
        return (tiles + slots - 1) / slots;
    };
    const long wp = waves(256, sms / 2), ws = waves(128, sms);
    return ws > 1 && wp <= ws;
}

}  // namespace

int gemm16_stats_parts(int M, int N) {
    Gemm16Args a{};
    a.M = M; a.N = N; a.batch = 1;
    const int tile = use_pairs(a) ? 256 : 128;
    return 2 * ((N + tile - 1) / tile);
}

int launch_gemm16(const Gemm16Args& a, cudaStream_t st) {
    if (a.M <= 0 || a.N <= 0 || a.K <= 0 || a.batch <= 0) return PCL_ERR_BAD_ARG;
    if (a.out2 && a.out && a.out_type != DT_F32) return PCL_ERR_BAD_ARG;      // (a 16-bit out holds its staging tile for two chunks)
    if (a.symmetric && (a.M != a.N || !a.out || a.out_type == DT_F32 || a.out2 || a.update)) return PCL_ERR_BAD_ARG;
    const bool pair = use_pairs(a);
    const int tile = pair ? 256 : 128;
    Gemm16Params p{};
    p.M = a.M; p.N = a.N; p.batch = a.batch;
    p.k_blocks = (a.K + 63) / 64;
    p.m_tiles = (a.M + tile - 1) / tile;
    p.n_tiles = (a.N + tile - 1) / tile;
    const double per = a.symmetric ? 0.5 * p.m_tiles * (p.m_tiles + 1.0) : double(p.m_tiles) * p.n_tiles;
    if (per * a.batch > 2e9) return PCL_ERR_UNSUPPORTED_SHAPE;
    p.tiles_per_matrix = int(per);
    p.total_tiles = p.tiles_per_matrix * a.batch;
    p.symmetric = a.symmetric; p.bf16 = a.bf16; p.epi = a.epi;
    p.alpha = a.alpha; p.beta = a.beta; p.scale2 = a.scale2; p.keep = a.keep; p.step = a.step; p.alpha_dev = a.alpha_dev;
    auto vec = [&](const void* ptr, int type, long ld, long bs) {
        const long per16 = 16 / long(dtype_bytes(type));
        return (reinterpret_cast<uintptr_t>(ptr) & 15) == 0 && ld % per16 == 0 && (a.batch == 1 || bs % per16 == 0);
    };
    p.src = a.src; p.src_type = a.src_type; p.src_ld = a.src_ld; p.src_batch = a.src_batch;
    p.src_vec = a.src && vec(a.src, a.src_type, a.src_ld, a.src_batch);
    p.out = a.out; p.out_type = a.out_type; p.out_ld = a.out_ld; p.out_batch = a.out_batch;
    p.has_out2 = a.out2 != nullptr; p.update = a.update;
    p.bias = a.bias; p.labels = a.labels; p.col0 = a.col0; p.part = a.part; p.part_ld = a.part_ld; p.label_z = a.label_z;
    p.lse = a.lse; p.row_scale = a.row_scale;
    p.status = device_status_ptr();
    if (!p.status) return PCL_ERR_CUDA;
    CUtensorMap ta, tb, to, to2;
    int rc = operand_tmap(&ta, a.a, a.M, a.K, a.batch, a.bf16);
    if (rc == PCL_OK) rc = operand_tmap(&tb, a.b, a.N, a.K, a.batch, a.bf16);
    if (rc != PCL_OK) return rc;
    to = ta; to2 = ta;
    if (a.out) {
        p.out_vec = vec(a.out, a.out_type, a.out_ld, a.out_batch);
        p.out_tma = p.out_vec;       // (a TMA store has the same conditions; other rows are stored element by element)
        if (p.out_tma)
            rc = make_tmap16(&to, a.out, a.out_type, a.N, a.M, a.batch, a.out_ld, a.out_batch, a.out_type == DT_F32 ? 32 : 64, 32);
        if (rc != PCL_OK) return rc;
    }
    if (a.out2) {
        rc = make_tmap16(&to2, a.out2, DT_F16, a.N, a.M, a.batch, a.out2_ld, a.out2_batch, 32, 32);
        if (rc != PCL_OK) return rc;
    }
    LaunchScope scope(KID_TC_GEMM16, 2.0 * a.M * double(a.N) * a.K * a.batch * (a.symmetric ? 0.5 : 1.0), st);
    return pair ? launch_form<true>(a, ta, tb, to, to2, p, st) : launch_form<false>(a, ta, tb, to, to2, p, st);
}

}  // namespace pcl

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
//
// Launches whose tiles do not fill whole waves cut the reduction of the last wave's tiles (all tiles, if there is less than one
// wave) into `splits` parts, each a work item of its own.  A part leaves its raw accumulators in the workspace and counts
// itself; whichever comes last adds the parts in their order and runs the epilogue.  Nobody waits for anybody, and the
// order of additions does not depend on who comes last.  (PARTS leaves the parts to its caller's next kernel instead.)
//
// The tensor core truncates when it adds to the accumulator, which biases a sum a little with every addition, more so with
// fp16 operands, whose products have 22 significant bits (bf16: 16).  The STATS epilogue, whose results are fp32, therefore takes
// long fp16 reductions in runs of kRunBlocks blocks and adds the runs in registers (kLong).
//
// Every kernel starts before the one in front of it has ended (programmatic dependent launch): barriers, TMEM and tensor maps
// are set up meanwhile, and griddepcontrol.wait stands before the first access to global memory.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <type_traits>

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
constexpr int kRunBlocks = 16;                               // kLong: 64-element blocks per accumulator run
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLoScale = 2048.f;                            // STEP: the second plane holds what rounding to 11 bits left, times this
// Up to here a logit times log2(e) stays in range, so that exp(z - ref) is one multiply-add and one ex2; beyond (classes masked
// with the type's lowest value) the difference is taken first.
constexpr float kScaledLimit = 1e38f;

// n / d for n < 2^31 by a multiplication (a division by a run-time value is some twenty instructions, which a short launch has to
// fetch before its first copy).
struct FastDiv { unsigned d, mul, shift; };
FastDiv fast_div(unsigned d) {
    unsigned s = 0;
    while ((1ull << s) < d) ++s;
    return {d, unsigned(((1ull << 32) * ((1ull << s) - d)) / d + 1), s};
}
__device__ __forceinline__ int divide(int n, const FastDiv& f) {
    return int((static_cast<unsigned long long>(__umulhi(unsigned(n), f.mul)) + unsigned(n)) >> f.shift);
}

struct Gemm16Params {
    int M, N, k_blocks, last_slices, batch;
    int m_tiles, n_tiles;
    FastDiv per_matrix, per_group, by_splits;        // tiles of a matrix; of kGroupM rows of tiles; parts of a tile
    int full_tiles, splits, part_blocks, items;      // tiles [0, full_tiles) are one item each, the others `splits`
    int* counters; float4* parts;                    // of the split tiles
    int symmetric, bf16;
    float alpha, beta, keep, step;
    const float* alpha_dev;
    const void* src; int src_type; long src_ld, src_batch;
    const __half* src_lo;
    void* out; int out_type; long out_ld, out_batch;
    int has_lo, update, quads;                       // quads: GENERAL rows start on multiples of four elements
    const void* bias;
    const int* labels;
    int col0;
    float2* part; int part_ld;
    float* label_z;
    const float* lse;
    const float* row_scale;
    unsigned int* status;
};

// 32 consecutive elements of a 16-bit vector as fp32; `valid` of them exist.  16-byte aligned.
__device__ __forceinline__ void load_chunk16(const void* base, bool bf16, size_t off, int valid, float (&o)[32]) {
    const uint16_t* s = static_cast<const uint16_t*>(base) + off;
    if (valid >= 32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint4 v = reinterpret_cast<const uint4*>(s)[j];
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                o[8 * j + 2 * i] = bf16 ? __uint_as_float(w[i] << 16) : f.x;
                o[8 * j + 2 * i + 1] = bf16 ? __uint_as_float(w[i] & 0xffff0000u) : f.y;
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const uint16_t u = j < valid ? s[j] : uint16_t(0);
            o[j] = bf16 ? __uint_as_float(uint32_t(u) << 16) : __half2float(__ushort_as_half(u));
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
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void st_shared_u4(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// Work item: a tile of one matrix and the reduction blocks [k0, k1) of it; part < 0: all of them.
struct Item16 { int b, m, n, k0, k1, part, split_tile; };
// Columns the MMAs of a tile compute: the last tile's are rounded up to 32.
__device__ __forceinline__ int tile_width(const Gemm16Params& p, int n, int bn) {
    const int left = p.N - n * bn;
    return left >= bn ? bn : (left + 31) / 32 * 32;
}
__device__ __forceinline__ Item16 decode_item(const Gemm16Params& p, int i) {
    Item16 o;
    int t = i;
    o.k0 = 0; o.k1 = p.k_blocks; o.part = -1; o.split_tile = 0;
    if (i >= p.full_tiles) {
        const int j = i - p.full_tiles;
        o.split_tile = divide(j, p.by_splits);
        t = p.full_tiles + o.split_tile;
        o.part = j - o.split_tile * p.splits;
        o.k0 = o.part * p.part_blocks;
        o.k1 = o.k0 + p.part_blocks < p.k_blocks ? o.k0 + p.part_blocks : p.k_blocks;
    }
    o.b = divide(t, p.per_matrix);
    int r = t - o.b * int(p.per_matrix.d);
    if (p.symmetric) {                       // tiles (m, n >= m), row by row
        int m = 0;
        while (r >= p.n_tiles - m) { r -= p.n_tiles - m; ++m; }
        o.m = m; o.n = m + r;
        return o;
    }
    const int g = divide(r, p.per_group);
    r -= g * int(p.per_group.d);
    const int left = p.m_tiles - g * kGroupM;
    if (left >= kGroupM) { o.n = r / kGroupM; o.m = g * kGroupM + (r - o.n * kGroupM); }
    else { o.n = r / left; o.m = g * kGroupM + (r - o.n * left); }
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

// GENERAL: a staged 32 x 32 chunk to and from memory.  kQuad: a lane takes four columns of every fourth row (rows start on
// multiples of four elements); else column `lane` of all rows.  Widths in bytes (0: no src).  The loads of eight (four
// columns) or sixteen rows are issued before any is used; rows past the last repeat it.
template <int kSrc, int kOut, bool kUpdate, bool kQuad>
__device__ __forceinline__ void general_rows(const Gemm16Params& p, uint32_t stg, int lane, int rows, size_t so, size_t oo, float alpha) {
    constexpr int kCols = kQuad ? 4 : 1, kBatch = kQuad ? 8 : 16;
    using S = std::conditional_t<kSrc == 4, uint32_t, uint16_t>;
    using O = std::conditional_t<kOut == 4, uint32_t, uint16_t>;
    struct alignas(sizeof(S) * kCols) SV { S e[kCols]; };
    struct alignas(sizeof(O) * kCols) OV { O e[kCols]; };
    auto value = [](auto raw, int type) {
        if constexpr (sizeof(raw) == 4) return __uint_as_float(raw);
        else return type == DT_BF16 ? __uint_as_float(uint32_t(raw) << 16) : __half2float(__ushort_as_half(raw));
    };
    const int first = kQuad ? lane >> 3 : 0, step = kQuad ? 4 : 1, col = kQuad ? (lane & 7) * 4 : lane;
    const S* src = static_cast<const S*>(p.src) + so + col;
    O* out = static_cast<O*>(p.out) + oo + col;
#pragma unroll 1
    for (int r0 = first; r0 < rows; r0 += kBatch * step) {
        SV s[kBatch];
        OV w[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int r = r0 + i * step < rows ? r0 + i * step : rows - 1;
            if constexpr (kSrc != 0) s[i] = *reinterpret_cast<const SV*>(src + size_t(r) * p.src_ld);
            if constexpr (kUpdate) w[i] = *reinterpret_cast<const OV*>(out + size_t(r) * p.out_ld);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const uint32_t r = (r0 + i * step) & 31;
            const uint32_t at = stg + r * 128 + (((uint32_t(col) >> 2) ^ (r & 7)) << 4);
            float x[kCols];
            if constexpr (kQuad) {
                const float4 q = ld_shared_v4(at);
                x[0] = q.x; x[1] = q.y; x[2] = q.z; x[3] = q.w;
            } else {
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x[0]) : "r"(at + (col & 3) * 4));
            }
            OV o;
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
                x[j] *= alpha;
                if constexpr (kSrc != 0) x[j] = fmaf(p.beta, value(s[i].e[j], p.src_type), x[j]);
                if constexpr (kUpdate) x[j] = fmaf(p.keep, value(w[i].e[j], p.out_type), -p.step * x[j]);
                if constexpr (kOut == 4) o.e[j] = __float_as_uint(x[j]);
                else o.e[j] = uint16_t(pack16(x[j], 0.f, p.out_type == DT_BF16) & 0xffffu);
            }
            if (r0 + i * step < rows) *reinterpret_cast<OV*>(out + size_t(r0 + i * step) * p.out_ld) = o;
        }
    }
}
template <int kSrc, int kOut, bool kUpdate>
__device__ __forceinline__ void general_chunk(const Gemm16Params& p, uint32_t stg, int lane, int rows, int valid, size_t so, size_t oo, float alpha) {
    if (p.quads) {
        if ((lane & 7) * 4 < valid) general_rows<kSrc, kOut, kUpdate, true>(p, stg, lane, rows, so, oo, alpha);
    } else if (lane < valid) {
        general_rows<kSrc, kOut, kUpdate, false>(p, stg, lane, rows, so, oo, alpha);
    }
}
// 32 rows of 64 bytes (32 fp16 values), swizzled over 64 bytes: sixteen-byte unit u of row r.
__device__ __forceinline__ uint32_t half_tile_addr(uint32_t tile, uint32_t r, uint32_t u) { return tile + r * 64 + ((u ^ ((r >> 1) & 3)) << 4); }
__device__ __forceinline__ void stage_half_row(uint32_t tile, int lane, const float (&v)[32]) {
#pragma unroll
    for (uint32_t u = 0; u < 4; ++u)
        st_shared_u4(half_tile_addr(tile, lane, u), pack16(v[8 * u], v[8 * u + 1], false), pack16(v[8 * u + 2], v[8 * u + 3], false),
                     pack16(v[8 * u + 4], v[8 * u + 5], false), pack16(v[8 * u + 6], v[8 * u + 7], false));
}

template <bool kPair, bool kAMn, bool kBMn, int kEpi, bool kLong>
__global__ void __launch_bounds__(kThreads16, 1)
tc_gemm16_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                 const __grid_constant__ CUtensorMap tmOut, const __grid_constant__ CUtensorMap tmLo, Gemm16Params p) {
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
    grid_dependency_wait();
    grid_dependents_launch();

    if (warp == 0) {
        // ---------------------------------------------------------------- producer (whole warp, an elected lane issues)
        const uint32_t full0 = smem_u32(&full_bar[0]), empty0 = smem_u32(&empty_bar[0]), ring0 = smem_u32(smem);
        const uint32_t full_dst0 = kPair ? map_to_cta(&full_bar[0], 0) : full0;
        int stage = 0;
        uint32_t phase = 0;
        long issued = 0;
        bool ok = true;
        for (int t = first; t < p.items && ok; t += stride) {
            const Item16 tile = decode_item(p, t);
            const int ra = tile.m * kTileM + int(pair_rank) * 128, rb = tile.n * kBN + (kPair ? int(pair_rank) * (tile_width(p, tile.n, kBN) / 2) : 0);
            for (int kb = tile.k0; kb < tile.k1; ++kb) {
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
            const uint32_t idesc0 = make_idesc_f16(0, p.bf16 != 0, kAMn, kBMn, kTileM);
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
            for (int t = first; t < p.items && ok; t += stride) {
                const Item16 tile = decode_item(p, t);
                const uint32_t idesc = idesc0 | (uint32_t(tile_width(p, tile.n, kBN)) >> 3 << 17);
                for (int kb = tile.k0; kb < tile.k1 && ok; ++it) {
                    const int run_end = kLong && kb + kRunBlocks < tile.k1 ? kb + kRunBlocks : tile.k1;
                    const uint32_t buf = it & 1;
                    if (!bounded_wait_addr_warp(ae0 + 8 * buf, ((it >> 1) & 1) ^ 1u, &abort_flag, p.status, WAIT_MMA_TMEM_EMPTY)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t d = tmem_base + buf * kBN;
                    uint32_t accum = 0;
                    for (; kb < run_end; ++kb) {
                        if (!bounded_wait_addr_warp(full0 + 8 * stage, phase, &abort_flag, p.status, WAIT_MMA_FULL)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t off = uint32_t(stage) * (kSlotBytes / 16);
                        if (kb + 1 < p.k_blocks || p.last_slices == 4)
                            umma_kstep_f16<kPair, kAMn ? 128 : 2, kBMn ? 128 : 2>(d, a_lo0 + off, b_lo0 + off, a_hi, b_hi, idesc, accum);
                        else                     // a short last block: only the K = 16 slices that hold anything
                            for (int s = 0; s < p.last_slices; ++s)
                                umma_f16<kPair>(d, (uint64_t(a_hi) << 32) | (a_lo0 + off + s * (kAMn ? 128 : 2)),
                                                (uint64_t(b_hi) << 32) | (b_lo0 + off + s * (kBMn ? 128 : 2)), idesc, accum | (s > 0));
                        accum = 1;
                        umma_commit_addr<kPair>(empty0 + 8 * stage);
                        if (++stage == kStages16) { stage = 0; phase ^= 1u; }
                    }
                    if (ok) umma_commit_addr<kPair>(af0 + 8 * buf);
                }
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
        constexpr bool kClasses = kEpi == GEMM16_STATS || kEpi == GEMM16_DZ;
        constexpr bool kJoins = kEpi != GEMM16_STATS && kEpi != GEMM16_PARTS;           // parts are joined by whichever comes last
        const float alpha = kClasses ? 1.f : p.alpha * (p.alpha_dev ? __ldg(p.alpha_dev) : 1.f);
        const uint32_t warp_slot = kPair ? pair_rank * 8 + (warp - 2) : warp - 2;      // of a tile's epilogue warps
        constexpr uint32_t kWarpSlots = kPair ? 16 : 8;
        constexpr int kChunks = kHalf / 32;
        constexpr size_t kWarpPart = size_t(kChunks) * 8 * 32;                          // float4 of one warp's part
        int it = 0;
        bool ok = true;
        auto release = [&](uint32_t buf) {       // the accumulator set is read: hand it back
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (kPair) mbar_arrive_cluster(ae_dst0 + 8 * buf);
                else mbar_arrive(&acc_empty_bar[buf]);
            }
        };
        for (int t = first; t < p.items && ok; t += stride) {
            const Item16 tile = decode_item(p, t);
            const int row0 = tile.m * kTileM + int(pair_rank) * 128 + quarter * 32, row = row0 + lane;
            const int cbase = tile.n * kBN + half * kHalf;
            const bool row_ok = row < p.M;
            int label = -1;
            float lse = 0.f, g = 0.f;
            if constexpr (kClasses) {
                if (row_ok) label = p.labels[row] - p.col0;
                if constexpr (kEpi == GEMM16_DZ) {
                    if (row_ok) { lse = p.lse[row]; g = p.row_scale[row]; }
                }
            }
            if constexpr (kEpi == GEMM16_GENERAL || kEpi == GEMM16_STEP || kEpi == GEMM16_SYM) {
                // what the epilogue reads is on its way to L2 while the main loop runs
                const long col_bytes = kEpi == GEMM16_GENERAL && p.src_type == DT_F32 ? 4 : 2;
                if (row_ok && cbase < p.N) {
                    if (p.src) {
                        const char* s = static_cast<const char*>(p.src) + (size_t(tile.b) * p.src_batch + size_t(row) * p.src_ld + cbase) * col_bytes;
                        for (int c = 0; c < kHalf * col_bytes && cbase + c / col_bytes < p.N; c += 128) prefetch_l2(s + c);
                    }
                    if (kEpi == GEMM16_STEP)
                        for (int c = 0; c < kHalf && cbase + c < p.N; c += 64)
                            prefetch_l2(p.src_lo + size_t(tile.b) * p.src_batch + size_t(row) * p.src_ld + cbase + c);
                    if (kEpi == GEMM16_GENERAL && p.update) {
                        const long es = p.out_type == DT_F32 ? 4 : 2;
                        const char* s = static_cast<const char*>(p.out) + (size_t(tile.b) * p.out_batch + size_t(row) * p.out_ld + cbase) * es;
                        for (int c = 0; c < kHalf * es && cbase + c / es < p.N; c += 128) prefetch_l2(s + c);
                    }
                }
            }
            float mx = -INFINITY, sum = 0.f;            // STATS: running maximum and sum of this thread's half row

            // ---- 32 columns of the finished accumulator (the code is kept short: a launch of a few microseconds fetches
            // every instruction from L2 once)
            auto process = [&](int c, float (&v)[32]) {
                const int col = cbase + c;
                const int valid = p.N - col < 32 ? p.N - col : 32;
                if constexpr (kClasses) {
                    if (p.bias) {
                        float s[32];
                        load_chunk16(p.bias, p.bf16 != 0, col, valid, s);
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] += s[j];
                    }
                }
                if constexpr (kEpi == GEMM16_STATS) {
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
                } else if constexpr (kEpi == GEMM16_SYM || kEpi == GEMM16_STEP) {
                    // fp16 tiles of 32 x 32; rows of src and out are padded to multiples of 8, so whole vectors exist
                    if (kEpi == GEMM16_STEP || p.src) {
                        float s[32];
                        const size_t off = size_t(tile.b) * p.src_batch + size_t(row_ok ? row : 0) * p.src_ld + col;
                        const int have = !row_ok ? 0 : valid;
                        if (kEpi == GEMM16_STEP) {                                // src + src_lo / 2^11: X to 22 bits
                            load_chunk16(p.src_lo, false, off, have, s);
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = fmaf(p.beta / kLoScale, s[j], v[j] * alpha);
                            load_chunk16(p.src, false, off, have, s);
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = fmaf(p.beta, s[j], v[j]);
                        } else {
                            load_chunk16(p.src, false, off, have, s);
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = fmaf(p.beta, s[j], v[j] * alpha);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] *= alpha;
                    }
                    staging_wait(lane);
                    stage_half_row(stg, lane, v);
                    const bool mirror = kEpi == GEMM16_SYM && tile.n > tile.m;
                    if (mirror) {                                                 // transposed: this lane's row is column `lane`
#pragma unroll
                        for (uint32_t j = 0; j < 32; ++j)
                            asm volatile("st.shared.b16 [%0], %1;" ::"r"(half_tile_addr(stg + 2048, j, lane >> 3) + (lane & 7) * 2),
                                         "h"(__half_as_ushort(__float2half_rn(v[j]))) : "memory");
                    }
                    if (kEpi == GEMM16_STEP && p.has_lo) {                        // what the rounding to fp16 left
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = (v[j] - __half2float(__float2half_rn(v[j]))) * kLoScale;
                        stage_half_row(stg + 2048, lane, v);
                    }
                    if (row0 < p.M) {
                        fence_proxy_async_shared();
                        __syncwarp();
                        if (lane == 0) {
                            tma_store_3d(&tmOut, stg, col, row0, tile.b);
                            if (mirror) tma_store_3d(&tmOut, stg + 2048, row0, col, tile.b);
                            if (kEpi == GEMM16_STEP && p.has_lo) tma_store_3d(&tmLo, stg + 2048, col, row0, tile.b);
                            bulk_commit_group();
                        }
                    }
                } else if constexpr (kEpi == GEMM16_GENERAL) {
                    // any type and alignment: the chunk is transposed through the staging tile, then all lanes take one row
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j)
                        st_shared_v4(stg_row + ((j ^ sw) << 4), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                    __syncwarp();
                    if (row0 < p.M) {
                        const int rows = p.M - row0 < 32 ? p.M - row0 : 32;
                        const size_t so = size_t(tile.b) * p.src_batch + size_t(row0) * p.src_ld + col;
                        const size_t oo = size_t(tile.b) * p.out_batch + size_t(row0) * p.out_ld + col;
                        const int sb = !p.src ? 0 : p.src_type == DT_F32 ? 4 : 2;
                        if (p.out_type == DT_F32) {
                            if (p.update) general_chunk<2, 4, true>(p, stg, lane, rows, valid, so, oo, alpha);
                            else if (sb == 2) general_chunk<2, 4, false>(p, stg, lane, rows, valid, so, oo, alpha);
                            else if (sb == 4) general_chunk<4, 4, false>(p, stg, lane, rows, valid, so, oo, alpha);
                            else general_chunk<0, 4, false>(p, stg, lane, rows, valid, so, oo, alpha);
                        } else {
                            if (p.update) general_chunk<2, 2, true>(p, stg, lane, rows, valid, so, oo, alpha);
                            else if (sb == 2) general_chunk<2, 2, false>(p, stg, lane, rows, valid, so, oo, alpha);
                            else if (sb == 4) general_chunk<4, 2, false>(p, stg, lane, rows, valid, so, oo, alpha);
                            else general_chunk<0, 2, false>(p, stg, lane, rows, valid, so, oo, alpha);
                        }
                    }
                    __syncwarp();
                } else if constexpr (kEpi == GEMM16_PARTS) {
                    staging_wait(lane);
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j)
                        st_shared_v4(stg_row + ((j ^ sw) << 4), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                    if (row0 < p.M) staging_store(&tmOut, stg, lane, col, row0, tile.part);
                } else {
                    if constexpr (kEpi == GEMM16_DZ) {
                        const int rel = label - col;
                        const float ref = lse == -INFINITY ? 0.f : lse;           // a row without any finite logit has p = 0
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
                    }
                    const bool odd = (c & 32) != 0;                               // 16-bit: two chunks fill the staging tile's rows
                    if (!odd) staging_wait(lane);
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j)
                        st_shared_u4(stg_row + (((j + (odd ? 4u : 0u)) ^ sw) << 4), pack16(v[8 * j], v[8 * j + 1], p.bf16 != 0),
                                     pack16(v[8 * j + 2], v[8 * j + 3], p.bf16 != 0), pack16(v[8 * j + 4], v[8 * j + 5], p.bf16 != 0),
                                     pack16(v[8 * j + 6], v[8 * j + 7], p.bf16 != 0));
                    if ((odd || col + 32 >= p.N) && row0 < p.M)
                        staging_store(&tmOut, stg, lane, odd ? col - 32 : col, row0, tile.b);
                }
            };
            // (a part of a split tile: the same place for all parts, and the counter they share)
            float4* part0 = nullptr;
            size_t part_step = 0;
            const bool joined = kJoins && tile.part >= 0;
            if (joined) {
                part0 = p.parts + (size_t(tile.split_tile) * p.splits * kWarpSlots + warp_slot) * kWarpPart + lane;
                part_step = kWarpSlots * kWarpPart;
            }
            auto part_done = [&]() -> bool {     // whether this part came last; warp-uniform
                __threadfence();
                __syncwarp();
                int last = 0;
                if (lane == 0) {
                    int* counter = p.counters + tile.split_tile * kWarpSlots + warp_slot;
                    last = atomicAdd(counter, 1) == p.splits - 1;
                    if (last) *counter = 0;
                    __threadfence();
                }
                return __shfl_sync(0xffffffffu, last, 0) != 0;
            };
            auto load_parts = [&](int c, float (&v)[32]) {       // in the parts' order, the next part on its way
                const float4* s = part0 + size_t(c / 32) * 8 * 32;
                float4 x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = __ldcg(s + j * 32);
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = 0.f;
#pragma unroll 1
                for (int q = 0; q < p.splits; ++q) {
                    float4 y[8];
                    s += part_step;
#pragma unroll
                    for (int j = 0; j < 8; ++j) y[j] = q + 1 < p.splits ? __ldcg(s + j * 32) : x[j];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        v[4 * j] += x[j].x; v[4 * j + 1] += x[j].y; v[4 * j + 2] += x[j].z; v[4 * j + 3] += x[j].w;
                        x[j] = y[j];
                    }
                }
            };
            bool finish = true;
            if constexpr (kLong) {
                float acc[kChunks][32];
                for (int kb = tile.k0; kb < tile.k1; kb += kRunBlocks, ++it) {
                    const uint32_t buf = it & 1;
                    if (!bounded_wait_warp_relaxed(&acc_full_bar[buf], (it >> 1) & 1, &abort_flag, p.status, WAIT_EPI_TMEM_FULL)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t taddr = tmem_base + buf * kBN + half * kHalf + (uint32_t(quarter * 32) << 16);
#pragma unroll
                    for (int c = 0; c < 2 * kChunks; ++c) {            // (16 columns at a time: the sums take most registers)
                        uint32_t u[16];
                        tmem_ld_32x16(taddr + c * 16, u);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            float& s = acc[c >> 1][(c & 1) * 16 + j];
                            s = kb == tile.k0 ? __uint_as_float(u[j]) : s + __uint_as_float(u[j]);
                        }
                    }
                    release(buf);
                }
                if (!ok) break;
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
                    if (cbase + c * 32 < p.N) process(c * 32, acc[c]);
            } else {
                const uint32_t buf = it & 1;
                if (!bounded_wait_warp_relaxed(&acc_full_bar[buf], (it >> 1) & 1, &abort_flag, p.status, WAIT_EPI_TMEM_FULL)) break;
                tc_fence_after();
                const uint32_t taddr = tmem_base + buf * kBN + half * kHalf + (uint32_t(quarter * 32) << 16);
                if (joined) {
                    float4* d = part0 + size_t(tile.part) * part_step;
                    for (int c = 0; c < kHalf; c += 32) {
                        uint32_t u[32];
                        tmem_ld_32x32(taddr + c, u);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            __stcg(d + (c / 4 + j) * 32, make_float4(__uint_as_float(u[4 * j]), __uint_as_float(u[4 * j + 1]),
                                                                     __uint_as_float(u[4 * j + 2]), __uint_as_float(u[4 * j + 3])));
                    }
                    release(buf);
                    finish = part_done();
                }
                if (finish) {
                    for (int c = 0; c < kHalf && cbase + c < p.N; c += 32) {
                        float v[32];
                        if (joined) {
                            load_parts(c, v);
                        } else {
                            uint32_t u[32];
                            tmem_ld_32x32(taddr + c, u);
                            tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(u[j]);
                        }
                        process(c, v);
                    }
                }
                if (!joined) release(buf);
                ++it;
            }
            if constexpr (kEpi == GEMM16_STATS) {
                if (row_ok) p.part[size_t(row) * p.part_ld + 2 * tile.n + half] = make_float2(mx, sum);
            }
        }
        if (lane == 0) bulk_wait_group_read0();      // (the staging tiles have been read; the grid's end completes the writes)
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

struct Maps16 { CUtensorMap a, b, out, lo; };

template <bool kPair, bool kAMn, bool kBMn, int kEpi, bool kLong = false>
int launch_variant(const Maps16& m, const Gemm16Params& p, cudaStream_t st) {
    static PerDeviceOnce once;
    auto kernel = tc_gemm16_kernel<kPair, kAMn, kBMn, kEpi, kLong>;
    const int rc = once.run([&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem16) == cudaSuccess ? PCL_OK
                                                                                                                 : PCL_ERR_CUDA;
    });
    if (rc != PCL_OK) return rc;
    const int slots = device_sm_count() / (kPair ? 2 : 1);
    const int grid = (p.items < slots ? p.items : slots) * (kPair ? 2 : 1);
    return launch_chained(kernel, dim3(grid), dim3(kThreads16), kSmem16, st, kPair ? 2 : 1, m.a, m.b, m.out, m.lo, p);
}

// The combinations of epilogue and operand layouts that the callers use.
template <bool kPair>
int launch_form(const Gemm16Args& a, int epi, const Maps16& m, const Gemm16Params& p, cudaStream_t st) {
    const int layout = (a.a.mn_major ? 2 : 0) | (a.b.mn_major ? 1 : 0);
    if constexpr (!kPair)
        if (epi == GEMM16_PARTS && layout == 0) return launch_variant<false, false, false, GEMM16_PARTS>(m, p, st);
    switch (epi * 4 + layout) {
        case GEMM16_STATS * 4:
            return p.k_blocks > 2 * kRunBlocks && !p.bf16 ? launch_variant<kPair, false, false, GEMM16_STATS, true>(m, p, st)
                                                          : launch_variant<kPair, false, false, GEMM16_STATS>(m, p, st);
        case GEMM16_DZ * 4: return launch_variant<kPair, false, false, GEMM16_DZ>(m, p, st);
        case GEMM16_STORE * 4 + 1: return launch_variant<kPair, false, true, GEMM16_STORE>(m, p, st);
        case GEMM16_STORE * 4 + 3: return launch_variant<kPair, true, true, GEMM16_STORE>(m, p, st);
        case GEMM16_SYM * 4: return launch_variant<kPair, false, false, GEMM16_SYM>(m, p, st);
        case GEMM16_SYM * 4 + 3: return launch_variant<kPair, true, true, GEMM16_SYM>(m, p, st);
        case GEMM16_STEP * 4: return launch_variant<kPair, false, false, GEMM16_STEP>(m, p, st);
        case GEMM16_STEP * 4 + 1: return launch_variant<kPair, false, true, GEMM16_STEP>(m, p, st);
        case GEMM16_GENERAL * 4: return launch_variant<kPair, false, false, GEMM16_GENERAL>(m, p, st);
        case GEMM16_GENERAL * 4 + 1: return launch_variant<kPair, false, true, GEMM16_GENERAL>(m, p, st);
        case GEMM16_GENERAL * 4 + 3: return launch_variant<kPair, true, true, GEMM16_GENERAL>(m, p, st);
    }
    return PCL_ERR_UNSUPPORTED_SHAPE;
}

// Pairs or single CTAs, and in how many parts the last wave's reductions are cut.  Times in microseconds, from launches of the
// four forms on a B200: a 64-deep block takes its MMAs' time (0.27 pair, 0.135 single) or that of its copies, 32 KB per CTA at
// the 11.8 TB/s that L2 delivers to all SMs together (0.40 when the GPU is full); start and a tile's epilogue that nothing
// overlaps 6 (pair) or 5; a part costs its trip through L2, 1.2 (128 KB per CTA) or 0.6, plus 4 for the count.
struct Plan16 { bool pair; int splits, part_blocks; long tiles, full_tiles; double time; };
constexpr long kMostParts = 256;                              // 64 MB of workspace
Plan16 plan16(const Gemm16Args& a) {
    const long sms = device_sm_count(), kb = (a.K + 63) / 64;
    Plan16 best{};
    best.time = 1e300;
    if (a.epi == GEMM16_PARTS) {
        const long tiles = long((a.M + 127) / 128) * ((a.N + 127) / 128), part = (kb + a.k_parts - 1) / a.k_parts;
        return Plan16{false, a.k_parts, int(part), tiles, 0, 0.0};
    }
    const bool joins = a.split_ws && a.epi != GEMM16_STATS;
    for (int form = 0; form < 2; ++form) {
        const bool pair = form == 0;
        const long tile = pair ? 256 : 128, slots = pair ? sms / 2 : sms;
        const long mt = (a.M + tile - 1) / tile, nt = (a.N + tile - 1) / tile;
        const long tiles = (a.epi == GEMM16_SYM ? mt * (mt + 1) / 2 : mt * nt) * a.batch;
        const double mma = pair ? 0.27 : 0.135, copy = (pair ? 2.0 : 1.0) * 32768.0 / 11.8e6, epi = pair ? 6.0 : 5.0;
        auto block = [&](long active) { return mma > copy * active ? mma : copy * active; };
        const long whole = tiles / slots, rest = tiles - whole * slots;
        for (long s = 1; s <= 16 && (s == 1 || (joins && rest > 0 && s * rest <= kMostParts)); ++s) {
            const long part = (kb + s - 1) / s, splits = (kb + part - 1) / part;
            if (splits != s) continue;
            const long waves = (rest * s + slots - 1) / slots;
            const double t = whole * kb * block(slots) + waves * part * block(waves > 1 ? slots : rest * s) + epi + (s > 1 ? 4.0 + s * (pair ? 1.2 : 0.6) : 0.0);
            if (t < best.time) best = Plan16{pair, int(s), int(part), tiles, s > 1 ? whole * slots : tiles, t};
        }
    }
    return best;
}

}  // namespace

int gemm16_stats_parts(const Gemm16Args& a) {
    const int tile = plan16(a).pair ? 256 : 128;
    return 2 * ((a.N + tile - 1) / tile);
}

size_t gemm16_split_ws_bytes(const Gemm16Args& args) {
    Gemm16Args a = args;
    a.split_ws = reinterpret_cast<void*>(256);          // (the plan with workspace)
    const Plan16 pl = plan16(a);
    if (pl.splits < 2 || a.epi == GEMM16_PARTS) return 0;
    return kGemm16CounterBytes + size_t(pl.tiles - pl.full_tiles) * pl.splits * (pl.pair ? 256 * 256 : 128 * 128) * 4;
}

int gemm16_parts(const Gemm16Args& a) {
    const long sms = device_sm_count(), kb = (a.K + 63) / 64, tiles = long((a.M + 127) / 128) * ((a.N + 127) / 128);
    long s = sms / tiles;
    if (s > kb / 4) s = kb / 4;                               // at least four blocks each
    if (s > 8) s = 8;
    if (s < 2) return 1;
    const long part = (kb + s - 1) / s;
    return int((kb + part - 1) / part);
}

int launch_gemm16(const Gemm16Args& a, cudaStream_t st) {
    if (a.M <= 0 || a.N <= 0 || a.K <= 0 || a.batch <= 0) return PCL_ERR_BAD_ARG;
    auto every = [&](const void* ptr, int type, long ld, long bs) {      // all rows start on multiples of 16 bytes
        const long n = 16 / long(dtype_bytes(type));
        return (reinterpret_cast<uintptr_t>(ptr) & 15) == 0 && ld % n == 0 && (a.batch == 1 || bs % n == 0);
    };
    int epi = a.epi;
    const int t16 = a.bf16 ? DT_BF16 : DT_F16;
    switch (epi) {
        case GEMM16_STATS:
            if (!a.part || !a.label_z || !a.labels) return PCL_ERR_BAD_ARG;
            break;
        case GEMM16_DZ:
            if (!a.out || !a.lse || !a.row_scale || !a.labels || !every(a.out, t16, a.out_ld, 0)) return PCL_ERR_BAD_ARG;
            break;
        case GEMM16_PARTS:
            if (a.k_parts < 1 || a.batch != 1 || a.out_type != DT_F32 || !every(a.out, DT_F32, a.out_ld, a.out_batch)) return PCL_ERR_BAD_ARG;
            break;
        case GEMM16_SYM:
            if (a.M != a.N || !every(a.out, DT_F16, a.out_ld, a.out_batch) || (a.src && !every(a.src, DT_F16, a.src_ld, a.src_batch))) return PCL_ERR_BAD_ARG;
            break;
        case GEMM16_STEP:
            if (!a.src || !a.src_lo || !every(a.out, DT_F16, a.out_ld, a.out_batch) || !every(a.src, DT_F16, a.src_ld, a.src_batch)) return PCL_ERR_BAD_ARG;
            break;
        case GEMM16_GENERAL:
            // a 16-bit result of the operands' type in aligned rows, and nothing added: through TMA stores
            if (a.update && (!a.src || a.src_type == DT_F32)) return PCL_ERR_BAD_ARG;
            if (!a.src && !a.update && a.out_type == t16 && every(a.out, t16, a.out_ld, a.out_batch)) epi = GEMM16_STORE;
            break;
        default: return PCL_ERR_BAD_ARG;
    }
    const Plan16 pl = plan16(a);
    const int tile = pl.pair ? 256 : 128;
    Gemm16Params p{};
    p.M = a.M; p.N = a.N; p.batch = a.batch;
    p.k_blocks = (a.K + 63) / 64;
    p.last_slices = (a.K - (p.k_blocks - 1) * 64 + 15) / 16;
    p.m_tiles = (a.M + tile - 1) / tile;
    p.n_tiles = (a.N + tile - 1) / tile;
    if (pl.tiles > 2000000000L) return PCL_ERR_UNSUPPORTED_SHAPE;
    p.per_matrix = fast_div(unsigned(pl.tiles / a.batch));
    p.per_group = fast_div(unsigned(kGroupM * p.n_tiles));
    p.by_splits = fast_div(unsigned(pl.splits));
    p.full_tiles = int(pl.full_tiles); p.splits = pl.splits; p.part_blocks = pl.part_blocks;
    p.items = int(pl.full_tiles + (pl.tiles - pl.full_tiles) * pl.splits);
    p.counters = static_cast<int*>(a.split_ws);
    p.parts = reinterpret_cast<float4*>(static_cast<char*>(a.split_ws) + kGemm16CounterBytes);
    p.symmetric = epi == GEMM16_SYM; p.bf16 = a.bf16;
    p.alpha = a.alpha; p.beta = a.beta; p.keep = a.keep; p.step = a.step; p.alpha_dev = a.alpha_dev;
    p.src = a.src; p.src_type = a.src_type; p.src_ld = a.src_ld; p.src_batch = a.src_batch;
    p.src_lo = static_cast<const __half*>(a.src_lo);
    p.out = a.out; p.out_type = a.out_type; p.out_ld = a.out_ld; p.out_batch = a.out_batch;
    p.has_lo = a.out_lo != nullptr; p.update = a.update;
    auto four = [&](const void* ptr, int type, long ld, long bs) {
        return !ptr || ((reinterpret_cast<uintptr_t>(ptr) & (4 * dtype_bytes(type) - 1)) == 0 && ld % 4 == 0 && (a.batch == 1 || bs % 4 == 0));
    };
    p.quads = a.N % 4 == 0 && four(a.src, a.src_type, a.src_ld, a.src_batch) && four(a.out, a.out_type, a.out_ld, a.out_batch);
    p.bias = a.bias; p.labels = a.labels; p.col0 = a.col0; p.part = a.part; p.part_ld = a.part_ld; p.label_z = a.label_z;
    p.lse = a.lse; p.row_scale = a.row_scale;
    p.status = device_status_ptr();
    if (!p.status) return PCL_ERR_CUDA;
    Maps16 m;
    int rc = operand_tmap(&m.a, a.a, a.M, a.K, a.batch, a.bf16);
    if (rc == PCL_OK) rc = operand_tmap(&m.b, a.b, a.N, a.K, a.batch, a.bf16);
    if (rc != PCL_OK) return rc;
    m.out = m.lo = m.a;
    const bool halves = epi == GEMM16_SYM || epi == GEMM16_STEP;
    if (halves || epi == GEMM16_STORE || epi == GEMM16_DZ)
        rc = make_tmap16(&m.out, a.out, halves ? int(DT_F16) : t16, a.N, a.M, a.batch, a.out_ld, a.out_batch, halves ? 32 : 64, 32);
    if (epi == GEMM16_PARTS) rc = make_tmap16(&m.out, a.out, DT_F32, a.N, a.M, pl.splits, a.out_ld, a.out_batch, 32, 32);
    if (rc == PCL_OK && p.has_lo)
        rc = make_tmap16(&m.lo, a.out_lo, DT_F16, a.N, a.M, a.batch, a.out_ld, a.out_batch, 32, 32);
    if (rc != PCL_OK) return rc;
    LaunchScope scope(KID_TC_GEMM16, 2.0 * a.M * double(a.N) * a.K * a.batch * (p.symmetric ? 0.5 : 1.0), st);
    return pl.pair ? launch_form<true>(a, epi, m, p, st) : launch_form<false>(a, epi, m, p, st);
}

}  // namespace pcl

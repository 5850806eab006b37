// Device side of the 16-bit tcgen05 GEMM: the roles of its kernels (see tc_gemm16.cu) as functions, shared with kernels that run
// several products in one launch (orthogonalize.cu).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <string.h>

#include <type_traits>

#include "pcl_internal.h"
#include "pcl_ptx.cuh"

namespace pcl {

namespace {

constexpr int kThreads16 = 320;
constexpr int kStages16 = 6;                                  // slots of the ring; kernels with SYM and STEP epilogues: 5
constexpr int kSlotBytes = 32768;
constexpr int kStaging = 4096;                                // per epilogue warp: one 32-row x 128-byte tile; SYM and STEP twice that
constexpr int kSmem16 = kStages16 * kSlotBytes + 8 * kStaging + 1024;
constexpr int kSmem16Fetch = (kStages16 - 1) * kSlotBytes + 16 * kStaging + 1024;
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
    // The order of the tiles: the whole ones of all matrices, then those of the ragged last row, then those of the ragged last
    // column (so the cheap ones come last).
    int m_whole, n_whole, core_tiles, bottom_tiles;  // whole rows and columns of tiles; tiles of the first two kinds
    FastDiv by_core, by_group, by_bottom, by_right;  // tiles of one matrix of each kind; of kGroupM rows of whole tiles
    FastDiv by_rest;                                 // split tiles
    int full_tiles, splits, part_blocks, items;      // tiles [0, full_tiles) are one item each, the others `splits`
    int* counters; float4* parts;                    // of the split tiles
    int symmetric, bf16;
    float alpha, beta, keep, step;
    const float* alpha_dev;
    const void* src; long src_ld, src_batch;
    void* out; int out_type; long out_ld, out_batch;
    int update, quads;                       // quads: GENERAL / FINAL rows start on multiples of four elements
    const void* bias;
    const int* labels;
    int col0;
    float2* part; int part_ld;
    float* label_z;
    unsigned* clear;
    const float* lse;
    const float* row_scale;
    unsigned int* status;
};

__device__ __forceinline__ float2 half2_value(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }
// Elements i .. i + 3 of a 16-bit vector of n (0 behind its end); i is a multiple of four, the vector 8-byte aligned.
__device__ __forceinline__ uint2 load_four16(const void* base, int i, int n) {
    const uint16_t* s = static_cast<const uint16_t*>(base) + i;
    if (i + 4 <= n) return __ldg(reinterpret_cast<const uint2*>(s));
    uint32_t e[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) e[j] = i + j < n ? __ldg(s + j) : 0u;
    return make_uint2(e[0] | e[1] << 16, e[2] | e[3] << 16);
}
__device__ __forceinline__ uint32_t pack16(float lo, float hi, bool bf16) {
    if (bf16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void pack16(const float (&v)[32], bool bf16, uint32_t (&h)[16]) {
    if (bf16) {
#pragma unroll
        for (int j = 0; j < 16; ++j) h[j] = pack16(v[2 * j], v[2 * j + 1], true);
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) h[j] = pack16(v[2 * j], v[2 * j + 1], false);
    }
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
// A CTA's (pair's) items: one of each wave, in turn from the wave's front and from its back, so that with items in the order of
// falling cost all CTAs get about the same (8200 x 4100 update, 4100 being 16 tiles and 4 columns: its square product 88 -> 75 us).  hop in the roles' loops: the steps to the next item, in turn.
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
        o.part = divide(j, p.by_rest);                       // (part by part: the same reduction blocks at the same time)
        o.split_tile = j - o.part * int(p.by_rest.d);
        t = p.full_tiles + o.split_tile;
        o.k0 = o.part * p.part_blocks;
        o.k1 = o.k0 + p.part_blocks < p.k_blocks ? o.k0 + p.part_blocks : p.k_blocks;
    }
    if (t < p.core_tiles) {
        o.b = divide(t, p.by_core);
        int r = t - o.b * int(p.by_core.d);
        if (p.symmetric) {                       // tiles (m, n >= m), row by row
            int m = 0;
            while (r >= p.n_whole - m) { r -= p.n_whole - m; ++m; }
            o.m = m; o.n = m + r;
            return o;
        }
        const int g = divide(r, p.by_group);
        r -= g * int(p.by_group.d);
        const int left = p.m_whole - g * kGroupM;
        if (left >= kGroupM) { o.n = r / kGroupM; o.m = g * kGroupM + (r - o.n * kGroupM); }
        else { o.n = r / left; o.m = g * kGroupM + (r - o.n * left); }
        return o;
    }
    t -= p.core_tiles;
    if (t < p.bottom_tiles) {
        o.b = divide(t, p.by_bottom);
        o.n = t - o.b * int(p.by_bottom.d);
        o.m = p.m_whole;
    } else {
        t -= p.bottom_tiles;
        o.b = divide(t, p.by_right);
        o.m = t - o.b * int(p.by_right.d);
        o.n = p.n_whole;
    }
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

template <class V>
__device__ __forceinline__ V load_l2(const V* p) {
    V v;
    if constexpr (sizeof(V) == 16) { const uint4 u = __ldcg(reinterpret_cast<const uint4*>(p)); memcpy(&v, &u, 16); }
    else if constexpr (sizeof(V) == 8) { const uint2 u = __ldcg(reinterpret_cast<const uint2*>(p)); memcpy(&v, &u, 8); }
    else if constexpr (sizeof(V) == 4) { const unsigned u = __ldcg(reinterpret_cast<const unsigned*>(p)); memcpy(&v, &u, 4); }
    else { const unsigned short u = __ldcg(reinterpret_cast<const unsigned short*>(p)); memcpy(&v, &u, 2); }
    return v;
}
// GENERAL, FINAL: a staged 32 x 32 chunk to and from memory.  kQuad: a lane takes four columns of every fourth row (rows start on
// multiples of four elements); else column `lane` of all rows.  Widths in bytes (src 0: none, 2: fp16, 4: fp32).  The loads of eight (four
// columns) or sixteen rows are issued before any is used; rows past the last repeat it.
template <int kSrc, int kOut, bool kUpdate, bool kQuad>
__device__ __forceinline__ void general_rows(const Gemm16Params& p, const void* src_base, void* out_base, uint32_t stg, int lane,
                                             int rows, size_t so, size_t oo, float alpha) {
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
    const S* src = static_cast<const S*>(src_base) + so + col;
    O* out = static_cast<O*>(out_base) + oo + col;
#pragma unroll 1
    for (int r0 = first; r0 < rows; r0 += kBatch * step) {
        SV s[kBatch];
        OV w[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int r = r0 + i * step < rows ? r0 + i * step : rows - 1;
            if constexpr (kSrc != 0) s[i] = load_l2(reinterpret_cast<const SV*>(src + size_t(r) * p.src_ld));
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
                if constexpr (kSrc != 0) x[j] = fmaf(p.beta, value(s[i].e[j], DT_F16), x[j]);
                if constexpr (kUpdate) x[j] = fmaf(p.keep, value(w[i].e[j], p.out_type), -p.step * x[j]);
                if constexpr (kOut == 4) o.e[j] = __float_as_uint(x[j]);
                else o.e[j] = uint16_t(pack16(x[j], 0.f, p.out_type == DT_BF16) & 0xffffu);
            }
            if (r0 + i * step < rows) *reinterpret_cast<OV*>(out + size_t(r0 + i * step) * p.out_ld) = o;
        }
    }
}
template <int kSrc, int kOut, bool kUpdate>
__device__ __forceinline__ void general_chunk(const Gemm16Params& p, const void* src, void* out, uint32_t stg, int lane, int rows,
                                              int valid, size_t so, size_t oo, float alpha) {
    if (p.quads) {
        if ((lane & 7) * 4 < valid) general_rows<kSrc, kOut, kUpdate, true>(p, src, out, stg, lane, rows, so, oo, alpha);
    } else if (lane < valid) {
        general_rows<kSrc, kOut, kUpdate, false>(p, src, out, stg, lane, rows, so, oo, alpha);
    }
}
// 32 rows of 64 bytes (32 fp16 values), swizzled over 64 bytes: sixteen-byte unit u of row r.
__device__ __forceinline__ uint32_t half_tile_addr(uint32_t tile, uint32_t r, uint32_t u) { return tile + r * 64 + ((u ^ ((r >> 1) & 3)) << 4); }
__device__ __forceinline__ void stage_half_row(uint32_t tile, int lane, const uint32_t (&h)[16]) {
#pragma unroll
    for (uint32_t u = 0; u < 4; ++u) st_shared_u4(half_tile_addr(tile, lane, u), h[4 * u], h[4 * u + 1], h[4 * u + 2], h[4 * u + 3]);
}
// Two fp32 multiply-adds in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 o;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
        "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(o.x), "=f"(o.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return o;
}

// What the warps of a CTA share.
struct Gemm16Shared {
    uint64_t full_bar[kStages16], empty_bar[kStages16], acc_full_bar[2], acc_empty_bar[2];
    uint64_t phase_end_bar, phase_go_bar;            // kernels of several products: see there
    uint64_t src_bar[8];                             // SYM, STEP: an epilogue warp's fetched chunk has arrived
    uint32_t tmem_base_slot, abort_flag;
};
// A thread's view of its CTA, and where the pipeline stands (a kernel may run several products one after another).
struct Gemm16Ctx {
    Gemm16Shared* sh;
    uint32_t ring, tmem, pair_rank;
    int warp, lane, first, stride;
    unsigned int* status;
    int stages;             // slots of the ring
    uint32_t src_phase = 0; // epilogue: of src_bar, and whether a fetched chunk is under way
    bool src_pending = false;
    int stage = 0;          // slot of the ring, and its barriers' phase (producer, issuer)
    uint32_t phase = 0;
    int it = 0;             // accumulator runs so far (issuer, epilogue)
    long issued = 0;        // producer
};

// Barriers, TMEM, and the context of the calling thread; ends with the CTA (pair) in step.
template <bool kPair>
__device__ __forceinline__ Gemm16Ctx gemm16_begin(Gemm16Shared* sh, uint8_t* smem_raw, unsigned int* status, int stages = kStages16) {
    constexpr int kBN = kPair ? 256 : 128;
    Gemm16Ctx c;
    c.sh = sh; c.status = status; c.stages = stages;
    c.warp = threadIdx.x >> 5; c.lane = threadIdx.x & 31;
    c.ring = (smem_u32(smem_raw) + 1023) & ~1023u;
    c.pair_rank = kPair ? cluster_ctarank() : 0u;
    c.first = kPair ? int(cluster_id_x()) : int(blockIdx.x);
    c.stride = kPair ? int(nclusters_x()) : int(gridDim.x);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages16; ++s) { mbar_init(&sh->full_bar[s], 1); mbar_init(&sh->empty_bar[s], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&sh->acc_full_bar[i], 1); mbar_init(&sh->acc_empty_bar[i], kPair ? 16 : 8); }
        mbar_init(&sh->phase_end_bar, 8);
        mbar_init(&sh->phase_go_bar, 1);
        for (int i = 0; i < 8; ++i) mbar_init(&sh->src_bar[i], 1);
        sh->abort_flag = 0;
        mbar_fence_init();
    }
    if (c.warp == 1) {
        if constexpr (kPair) { tmem_alloc_pair(&sh->tmem_base_slot, 2 * kBN); tmem_relinquish_pair(); }
        else { tmem_alloc(&sh->tmem_base_slot, 2 * kBN); tmem_relinquish(); }
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (kPair) cluster_sync_all();
    tc_fence_after();
    c.tmem = sh->tmem_base_slot;
    return c;
}
template <bool kPair>
__device__ __forceinline__ void gemm16_end(const Gemm16Ctx& c) {
    constexpr int kBN = kPair ? 256 : 128;
    tc_fence_before();
    __syncthreads();
    if constexpr (kPair) cluster_sync_all();     // neither CTA leaves while the pair's MMAs may read its tiles
    if (c.warp == 1) {
        tc_fence_after();
        if constexpr (kPair) tmem_dealloc_pair(c.tmem, 2 * kBN);
        else tmem_dealloc(c.tmem, 2 * kBN);
    }
}

// ---- producer: the whole warp, an elected lane issues.  tile: its first item, decoded by the caller before whatever it waits
// for (a lone warp's every instruction is some ten cycles).  false: a wait ran out.
template <bool kPair, bool kAMn, bool kBMn>
__device__ __forceinline__ bool produce_items(Gemm16Ctx& c, const Gemm16Params& p, Item16 tile, const CUtensorMap* tm_a, const CUtensorMap* tm_b) {
    constexpr int kTileM = kPair ? 256 : 128, kBN = kTileM;
    const uint32_t full0 = smem_u32(&c.sh->full_bar[0]), empty0 = smem_u32(&c.sh->empty_bar[0]);
    const uint32_t full_dst0 = kPair ? map_to_cta(&c.sh->full_bar[0], 0) : full0;
    for (int t = c.first, hop = 2 * (c.stride - c.first) - 1; t < p.items;) {
        const int ra = tile.m * kTileM + int(c.pair_rank) * 128;
        const int rb = tile.n * kBN + (kPair ? int(c.pair_rank) * (tile_width(p, tile.n, kBN) / 2) : 0);
        for (int kb = tile.k0; kb < tile.k1; ++kb) {
            if (!bounded_wait_addr_warp(empty0 + 8 * c.stage, c.phase ^ 1u, &c.sh->abort_flag, c.status, WAIT_PRODUCER_EMPTY)) return false;
            if (c.pair_rank == 0) mbar_expect_tx_addr(full0 + 8 * c.stage, kPair ? 2 * kSlotBytes : kSlotBytes);
            const uint32_t dst = c.ring + c.stage * kSlotBytes, bar = full_dst0 + 8 * c.stage;
            if constexpr (kAMn) {
                tma_load_3d_addr<kPair>(dst, tm_a, bar, ra, kb * 64, tile.b);
                tma_load_3d_addr<kPair>(dst + 8192, tm_a, bar, ra + 64, kb * 64, tile.b);
            } else {
                tma_load_3d_addr<kPair>(dst, tm_a, bar, kb * 64, ra, tile.b);
            }
            if constexpr (kBMn) {
                tma_load_3d_addr<kPair>(dst + 16384, tm_b, bar, rb, kb * 64, tile.b);
                tma_load_3d_addr<kPair>(dst + 24576, tm_b, bar, rb + 64, kb * 64, tile.b);
            } else {
                tma_load_3d_addr<kPair>(dst + 16384, tm_b, bar, kb * 64, rb, tile.b);
            }
            ++c.issued;
            if (++c.stage == c.stages) { c.stage = 0; c.phase ^= 1u; }
        }
        t += hop;
        hop = 2 * c.stride - hop;
        if (t < p.items) tile = decode_item(p, t);
    }
    return true;
}
// A producer that gave up: copies already issued still land in this CTA's shared memory; wait (bounded) for them.
__device__ __forceinline__ void drain_producer(Gemm16Ctx& c) {
    const int pending = c.issued < c.stages ? int(c.issued) : c.stages;
    for (int j = 0; j < pending; ++j) {
        if (--c.stage < 0) { c.stage = c.stages - 1; c.phase ^= 1u; }
        for (uint32_t spin = 0; spin < (1u << 20); ++spin)
            if (mbar_try_wait(&c.sh->full_bar[c.stage], c.phase)) break;
    }
}

// The same for an epilogue warp's fetched chunk.
__device__ __forceinline__ void drain_fetch(Gemm16Ctx& c) {
    if (!c.src_pending) return;
    for (uint32_t spin = 0; spin < (1u << 20); ++spin)
        if (mbar_try_wait(&c.sh->src_bar[c.warp - 2], c.src_phase)) break;
}

// ---- MMA issuer (of the leading CTA).  false: a wait ran out.
template <bool kPair, bool kAMn, bool kBMn, bool kLong>
__device__ __forceinline__ bool issue_items(Gemm16Ctx& c, const Gemm16Params& p) {
    constexpr int kTileM = kPair ? 256 : 128, kBN = kTileM;
    const uint32_t idesc0 = make_idesc_f16(0, p.bf16 != 0, kAMn, kBMn, kTileM);
    // K-major: 8-row groups 1 KB apart.  MN-major: 64-row groups 8 KB apart, 8-deep reduction groups 1 KB apart.
    const uint64_t da = make_smem_desc(c.ring, kAMn ? 8192 : 0, 1024, kSwizzle128B);
    const uint64_t db = make_smem_desc(c.ring + 16384, kBMn ? 8192 : 0, 1024, kSwizzle128B);
    const uint32_t a_hi = uint32_t(da >> 32), b_hi = uint32_t(db >> 32), a_lo0 = uint32_t(da), b_lo0 = uint32_t(db);
    const uint32_t full0 = smem_u32(&c.sh->full_bar[0]), empty0 = smem_u32(&c.sh->empty_bar[0]);
    const uint32_t af0 = smem_u32(&c.sh->acc_full_bar[0]), ae0 = smem_u32(&c.sh->acc_empty_bar[0]);
    for (int t = c.first, hop = 2 * (c.stride - c.first) - 1; t < p.items; t += hop, hop = 2 * c.stride - hop) {
        const Item16 tile = decode_item(p, t);
        const uint32_t idesc = idesc0 | (uint32_t(tile_width(p, tile.n, kBN)) >> 3 << 17);
        for (int kb = tile.k0; kb < tile.k1; ++c.it) {
            const int run_end = kLong && kb + kRunBlocks < tile.k1 ? kb + kRunBlocks : tile.k1;
            const uint32_t buf = c.it & 1;
            if (!bounded_wait_addr_warp(ae0 + 8 * buf, ((c.it >> 1) & 1) ^ 1u, &c.sh->abort_flag, c.status, WAIT_MMA_TMEM_EMPTY)) return false;
            tc_fence_after();
            const uint32_t d = c.tmem + buf * kBN;
            uint32_t accum = 0;
            for (; kb < run_end; ++kb) {
                if (!bounded_wait_addr_warp(full0 + 8 * c.stage, c.phase, &c.sh->abort_flag, c.status, WAIT_MMA_FULL)) return false;
                tc_fence_after();
                const uint32_t off = uint32_t(c.stage) * (kSlotBytes / 16);
                if (kb + 1 < p.k_blocks || p.last_slices == 4)
                    umma_kstep_f16<kPair, kAMn ? 128 : 2, kBMn ? 128 : 2>(d, a_lo0 + off, b_lo0 + off, a_hi, b_hi, idesc, accum);
                else                     // a short last block: only the K = 16 slices that hold anything
                    for (int s = 0; s < p.last_slices; ++s)
                        umma_f16<kPair>(d, (uint64_t(a_hi) << 32) | (a_lo0 + off + s * (kAMn ? 128 : 2)),
                                        (uint64_t(b_hi) << 32) | (b_lo0 + off + s * (kBMn ? 128 : 2)), idesc, accum | (s > 0));
                accum = 1;
                umma_commit_addr<kPair>(empty0 + 8 * c.stage);
                if (++c.stage == c.stages) { c.stage = 0; c.phase ^= 1u; }
            }
            umma_commit_addr<kPair>(af0 + 8 * buf);
        }
    }
    return true;
}

// ---- epilogue warps.  src, out: as in Gemm16Args (arguments, because a kernel of several products alternates its buffers).
// false: a wait ran out.
template <bool kPair, int kEpi, bool kLong>
__device__ __forceinline__ bool finish_items(Gemm16Ctx& c, const Gemm16Params& p, const CUtensorMap* tm_out, const CUtensorMap* tm_lo,
                                             const void* src, void* out, const CUtensorMap* tm_src = nullptr,
                                             const CUtensorMap* tm_src_lo = nullptr) {
    constexpr int kTileM = kPair ? 256 : 128, kBN = kTileM;
    constexpr int kHalf = kBN / 2;                   // columns per epilogue warp
    const int warp = c.warp, lane = c.lane;
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    constexpr bool kFetches = kEpi == GEMM16_SYM || kEpi == GEMM16_STEP;
    const uint32_t stg = c.ring + c.stages * kSlotBytes + (warp - 2) * (kFetches ? 2 * kStaging : kStaging);
    const uint32_t stg_row = stg + lane * 128;
    const uint32_t sw = lane & 7;
    const uint32_t ae0 = smem_u32(&c.sh->acc_empty_bar[0]);
    const uint32_t ae_dst0 = kPair ? map_to_cta(&c.sh->acc_empty_bar[0], 0) : ae0;
    constexpr bool kClasses = kEpi == GEMM16_STATS || kEpi == GEMM16_DZ;
    constexpr bool kJoins = kEpi != GEMM16_STATS && kEpi != GEMM16_PARTS;           // parts are joined by whichever comes last
    const float alpha = kClasses ? 1.f : p.alpha * (p.alpha_dev ? __ldg(p.alpha_dev) : 1.f);
    const uint32_t warp_slot = kPair ? c.pair_rank * 8 + (warp - 2) : warp - 2;      // of a tile's epilogue warps
    constexpr uint32_t kWarpSlots = kPair ? 16 : 8;
    constexpr int kChunks = kHalf / 32;
    constexpr size_t kWarpPart = size_t(kChunks) * 8 * 32;                          // float4 of one warp's part
    bool ok = true;
    auto release = [&](uint32_t buf) {       // the accumulator set is read: hand it back
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
            if constexpr (kPair) mbar_arrive_cluster_read(ae_dst0 + 8 * buf);
            else mbar_arrive(&c.sh->acc_empty_bar[buf]);
        }
    };
    for (int t = c.first, hop = 2 * (c.stride - c.first) - 1; t < p.items && ok; t += hop, hop = 2 * c.stride - hop) {
        const Item16 tile = decode_item(p, t);
        const int row0 = tile.m * kTileM + int(c.pair_rank) * 128 + quarter * 32, row = row0 + lane;
        const int cbase = tile.n * kBN + half * kHalf;
        const bool row_ok = row < p.M;
        int label = -1;
        float lse = 0.f, g = 0.f;
        uint2 bias = make_uint2(0u, 0u);
        if constexpr (kClasses) {
            // the bias of the warp's columns, four per lane: it arrives while the warp waits for the product (a chunk's 64 bytes loaded where
            // they are added took 500 cycles a chunk)
            if (p.bias) bias = load_four16(p.bias, cbase + 4 * (lane & (kHalf / 4 - 1)), p.N);
            if (row_ok) label = max(p.labels[row], -1) - p.col0;
            if constexpr (kEpi == GEMM16_DZ) {
                if (row_ok) { lse = p.lse[row]; g = lse == -INFINITY ? 0.f : p.row_scale[row]; }     // (no finite logit: no gradient)
            }
        }
        if constexpr (kEpi == GEMM16_GENERAL || kEpi == GEMM16_FINAL) {
            // what the epilogue reads is on its way to L2 while the main loop runs
            const long col_bytes = kEpi == GEMM16_GENERAL ? 4 : 2;
            if (row_ok && cbase < p.N) {
                if (src) {
                    const char* s = static_cast<const char*>(src) + (size_t(tile.b) * p.src_batch + size_t(row) * p.src_ld + cbase) * col_bytes;
                    for (int o = 0; o < kHalf * col_bytes && cbase + o / col_bytes < p.N; o += 128) prefetch_l2(s + o);
                }
                if (kEpi == GEMM16_FINAL && p.update) {
                    const long es = p.out_type == DT_F32 ? 4 : 2;
                    const char* s = static_cast<const char*>(out) + (size_t(tile.b) * p.out_batch + size_t(row) * p.out_ld + cbase) * es;
                    for (int o = 0; o < kHalf * es && cbase + o / es < p.N; o += 128) prefetch_l2(s + o);
                }
            }
        }
        float mx = -INFINITY, sum = 0.f;            // STATS: running maximum and sum of this thread's half row

        // SYM, STEP: what is added to a chunk comes through TMA, one chunk ahead, into the second half of the warp's staging
        // space (loads of one row per lane touch 32 lines each: the eight warps' loads took 2000 cycles a chunk)
        const uint32_t src_stg = stg + kStaging;
        uint64_t* src_bar = &c.sh->src_bar[warp - 2];
        const bool fetches = kFetches && tm_src != nullptr;
        auto fetch = [&](int col) {              // (the whole warp; every lane has read the chunk before)
            __syncwarp();
            c.src_pending = true;
            mbar_expect_tx(src_bar, kEpi == GEMM16_STEP ? 4096 : 2048);
            tma_load_3d_addr<false>(src_stg, tm_src, smem_u32(src_bar), col, row0, tile.b);
            if (kEpi == GEMM16_STEP) tma_load_3d_addr<false>(src_stg + 2048, tm_src_lo, smem_u32(src_bar), col, row0, tile.b);
        };

        // ---- 32 columns of the finished accumulator (the code is kept short: a launch of a few microseconds fetches
        // every instruction from L2 once)
        auto process = [&](int cc, float (&v)[32]) {
            const int col = cbase + cc;
            const int valid = p.N - col < 32 ? p.N - col : 32;
            if constexpr (kClasses) {
                if (p.bias) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const uint32_t two = __shfl_sync(0xffffffffu, j & 1 ? bias.y : bias.x, cc / 4 + j / 2);
                        const float2 h = half2_value(two);
                        v[2 * j] += p.bf16 ? __uint_as_float(two << 16) : h.x;
                        v[2 * j + 1] += p.bf16 ? __uint_as_float(two & 0xffff0000u) : h.y;
                    }
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
                    const float2 l2 = make_float2(kLog2e, kLog2e), ref2 = make_float2(-ref * kLog2e, -ref * kLog2e);
                    float2 two = make_float2(0.f, 0.f);
                    const float2 one = make_float2(1.f, 1.f);
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float2 e = fma2(make_float2(v[2 * j], v[2 * j + 1]), l2, ref2);
                        two = fma2(make_float2(ex2(e.x), ex2(e.y)), one, two);
                    }
                    add = two.x + two.y;
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) add += ex2((v[j] - ref) * kLog2e);
                }
                sum = sum * ex2((mx - ref) * kLog2e) + add;
                mx = nm;
            } else if constexpr (kEpi == GEMM16_SYM || kEpi == GEMM16_STEP) {
                // fp16 tiles of 32 x 32, two elements at a time
                float2 w[16];
                const float2 al = make_float2(alpha, alpha), zero = make_float2(0.f, 0.f);
#pragma unroll
                for (int j = 0; j < 16; ++j) w[j] = make_float2(v[2 * j], v[2 * j + 1]);
                if (fetches) {                                                    // STEP: src + src_lo / 2^11, X to 22 bits
                    if (!bounded_wait_warp(src_bar, c.src_phase, &c.sh->abort_flag, c.status, WAIT_EPI_TMEM_FULL)) { ok = false; return; }
                    c.src_pending = false;
                    c.src_phase ^= 1u;
                    const float2 be = make_float2(p.beta, p.beta), bl = make_float2(p.beta / kLoScale, p.beta / kLoScale);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float4 hi = ld_shared_v4(half_tile_addr(src_stg, lane, u));
                        float4 lo;
                        if constexpr (kEpi == GEMM16_STEP) lo = ld_shared_v4(half_tile_addr(src_stg + 2048, lane, u));
                        const float h4[4] = {hi.x, hi.y, hi.z, hi.w};
                        const float l4[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float2& x = w[4 * u + i];
                            float2 s = zero;
                            if constexpr (kEpi == GEMM16_STEP) s = fma2(half2_value(__float_as_uint(l4[i])), bl, zero);
                            x = fma2(x, al, fma2(half2_value(__float_as_uint(h4[i])), be, s));
                        }
                    }
                    if (cc + 32 < kHalf && col + 32 < p.N) fetch(col + 32);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[j] = fma2(w[j], al, zero);
                }
                uint32_t h[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) h[j] = pack16(w[j].x, w[j].y, false);
                staging_wait(lane);
                stage_half_row(stg, lane, h);
                const bool mirror = kEpi == GEMM16_SYM && p.symmetric && tile.n > tile.m;
                if (mirror) {                                                 // transposed: this lane's row is column `lane`
#pragma unroll
                    for (uint32_t j = 0; j < 32; ++j)
                        asm volatile("st.shared.b16 [%0], %1;" ::"r"(half_tile_addr(stg + 2048, j, lane >> 3) + (lane & 7) * 2),
                                     "h"(static_cast<unsigned short>(j & 1 ? h[j >> 1] >> 16 : h[j >> 1])) : "memory");
                }
                if (kEpi == GEMM16_STEP && tm_lo) {                           // what the rounding to fp16 left (exact in fp32)
                    const float2 minus = make_float2(-1.f, -1.f);
                    const __half2 up = __float2half2_rn(kLoScale);
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float2 r = fma2(half2_value(h[j]), minus, w[j]);
                        const uint32_t q = pack16(r.x, r.y, false);
                        const __half2 s = __hmul2(*reinterpret_cast<const __half2*>(&q), up);
                        h[j] = *reinterpret_cast<const uint32_t*>(&s);
                    }
                    stage_half_row(stg + 2048, lane, h);
                }
                if (row0 < p.M) {
                    fence_proxy_async_shared();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_3d(tm_out, stg, col, row0, tile.b);
                        if (mirror) tma_store_3d(tm_out, stg + 2048, row0, col, tile.b);
                        if (kEpi == GEMM16_STEP && tm_lo) tma_store_3d(tm_lo, stg + 2048, col, row0, tile.b);
                        bulk_commit_group();
                    }
                }
            } else if constexpr (kEpi == GEMM16_GENERAL || kEpi == GEMM16_FINAL) {
                // any type and alignment: the chunk is transposed through the staging tile, then all lanes take one row
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j)
                    st_shared_v4(stg_row + ((j ^ sw) << 4), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                __syncwarp();
                if (row0 < p.M) {
                    const int rows = p.M - row0 < 32 ? p.M - row0 : 32;
                    const size_t so = size_t(tile.b) * p.src_batch + size_t(row0) * p.src_ld + col;
                    const size_t oo = size_t(tile.b) * p.out_batch + size_t(row0) * p.out_ld + col;
                    const bool wide = p.out_type == DT_F32;
                    if constexpr (kEpi == GEMM16_FINAL) {
                        if (p.update) {
                            if (wide) general_chunk<2, 4, true>(p, src, out, stg, lane, rows, valid, so, oo, alpha);
                            else general_chunk<2, 2, true>(p, src, out, stg, lane, rows, valid, so, oo, alpha);
                        } else {
                            if (wide) general_chunk<2, 4, false>(p, src, out, stg, lane, rows, valid, so, oo, alpha);
                            else general_chunk<2, 2, false>(p, src, out, stg, lane, rows, valid, so, oo, alpha);
                        }
                    } else if (src) {
                        if (wide) general_chunk<4, 4, false>(p, src, out, stg, lane, rows, valid, so, oo, alpha);
                        else general_chunk<4, 2, false>(p, src, out, stg, lane, rows, valid, so, oo, alpha);
                    } else {
                        if (wide) general_chunk<0, 4, false>(p, src, out, stg, lane, rows, valid, so, oo, alpha);
                        else general_chunk<0, 2, false>(p, src, out, stg, lane, rows, valid, so, oo, alpha);
                    }
                }
                __syncwarp();
            } else if constexpr (kEpi == GEMM16_PARTS) {
                staging_wait(lane);
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j)
                    st_shared_v4(stg_row + ((j ^ sw) << 4), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                if (row0 < p.M) staging_store(tm_out, stg, lane, col, row0, tile.part);
            } else {
                if constexpr (kEpi == GEMM16_DZ) {
                    const int rel = label - col;
                    const float ref2 = lse * kLog2e;
                    if (fabsf(lse) < kScaledLimit) {
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const float2 e = fma2(make_float2(v[j], v[j + 1]), make_float2(kLog2e, kLog2e), make_float2(-ref2, -ref2));
                            v[j] = ex2(e.x); v[j + 1] = ex2(e.y);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = ex2((v[j] - lse) * kLog2e);
                    }
                    if (rel >= 0 && rel < 32)
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] -= j == rel ? 1.f : 0.f;
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] *= g;
                    if (g == 0.f)                                                 // rows left out or without a finite logit: exactly 0, whatever z is
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = 0.f;
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] *= alpha;
                }
                uint32_t h[16];
                pack16(v, p.bf16 != 0, h);
                const bool odd = (cc & 32) != 0;                               // 16-bit: two chunks fill the staging tile's rows
                if (!odd) staging_wait(lane);
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j)
                    st_shared_u4(stg_row + (((j + (odd ? 4u : 0u)) ^ sw) << 4), h[4 * j], h[4 * j + 1], h[4 * j + 2], h[4 * j + 3]);
                if ((odd || col + 32 >= p.N) && row0 < p.M)
                    staging_store(tm_out, stg, lane, odd ? col - 32 : col, row0, tile.b);
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
        auto load_parts = [&](int cc, float (&v)[32]) {       // in the parts' order, the next part on its way
            const float4* s = part0 + size_t(cc / 32) * 8 * 32;
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
            for (int kb = tile.k0; kb < tile.k1; kb += kRunBlocks, ++c.it) {
                const uint32_t buf = c.it & 1;
                if (!bounded_wait_warp(&c.sh->acc_full_bar[buf], (c.it >> 1) & 1, &c.sh->abort_flag, c.status, WAIT_EPI_TMEM_FULL)) { ok = false; break; }
                tc_fence_after();
                const uint32_t taddr = c.tmem + buf * kBN + half * kHalf + (uint32_t(quarter * 32) << 16);
#pragma unroll
                for (int h = 0; h < 2 * kChunks; ++h) {            // (16 columns at a time: the sums take most registers)
                    uint32_t u[16];
                    tmem_ld_32x16(taddr + h * 16, u);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float& s = acc[h >> 1][(h & 1) * 16 + j];
                        s = kb == tile.k0 ? __uint_as_float(u[j]) : s + __uint_as_float(u[j]);
                    }
                }
                release(buf);
            }
            if (!ok) break;
#pragma unroll
            for (int h = 0; h < kChunks; ++h)
                if (cbase + h * 32 < p.N) process(h * 32, acc[h]);
        } else {
            if (fetches && !joined && cbase < p.N) fetch(cbase);
            const uint32_t buf = c.it & 1;
            if (!bounded_wait_warp(&c.sh->acc_full_bar[buf], (c.it >> 1) & 1, &c.sh->abort_flag, c.status, WAIT_EPI_TMEM_FULL)) return false;
            tc_fence_after();
            const uint32_t taddr = c.tmem + buf * kBN + half * kHalf + (uint32_t(quarter * 32) << 16);
            if (joined) {
                float4* d = part0 + size_t(tile.part) * part_step;
                for (int cc = 0; cc < kHalf; cc += 32) {
                    uint32_t u[32];
                    tmem_ld_32x32(taddr + cc, u);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        __stcg(d + (cc / 4 + j) * 32, make_float4(__uint_as_float(u[4 * j]), __uint_as_float(u[4 * j + 1]),
                                                                 __uint_as_float(u[4 * j + 2]), __uint_as_float(u[4 * j + 3])));
                }
                release(buf);
                finish = part_done();
            }
            if (finish) {
                if (fetches && joined && cbase < p.N) fetch(cbase);
                bool held = !joined;
                for (int cc = 0; cc < kHalf && cbase + cc < p.N && ok; cc += 32) {
                    float v[32];
                    if (joined) {
                        load_parts(cc, v);
                    } else {
                        uint32_t u[32];
                        tmem_ld_32x32(taddr + cc, u);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(u[j]);
                        if (cc + 32 >= kHalf || cbase + cc + 32 >= p.N) { release(buf); held = false; }
                    }
                    process(cc, v);
                }
                if (held) release(buf);                        // (a tile without columns for this warp)
            }
            ++c.it;
        }
        if constexpr (kEpi == GEMM16_STATS) {
            if (row_ok) p.part[size_t(row) * p.part_ld + 2 * tile.n + half] = make_float2(mx, sum);
        }
    }
    return ok;
}

// ---- host
// Tensor map over [batch][outer][inner] elements, swizzled over the box's inner extent (128 or 64 bytes).
inline int make_tmap16(CUtensorMap* out, const void* base, int type, uint64_t inner, uint64_t outer, uint64_t batch, long ld,
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

inline int operand_tmap(CUtensorMap* tm, const Gemm16Operand& o, int rows, int K, int batch, bool bf16) {
    const int type = bf16 ? DT_BF16 : DT_F16;
    return o.mn_major ? make_tmap16(tm, o.ptr, type, rows, K, batch, o.ld, o.batch_stride, 64, 64)
                      : make_tmap16(tm, o.ptr, type, K, rows, batch, o.ld, o.batch_stride, 64, 128);
}

// Pairs or single CTAs, and in how many parts the last wave's reductions are cut.  Times in microseconds, from launches of the
// four forms on a B200: a 64-deep block takes its MMAs' time (0.27 pair, 0.135 single) or that of its copies, 32 KB per CTA at
// the 11.8 TB/s that L2 delivers to all SMs together (0.41 when the GPU is full); start and a tile's epilogue that nothing
// overlaps 6 (pair) or 5, and 1.5 more where it writes a mirror image (so the whole of a small symmetric result is computed
// where there are SMs to spare); a part costs its trip through L2, 1.2 (128 KB per CTA) or 0.6, plus 4 for the count.
struct Plan16 { bool pair, mirrored; int splits, part_blocks; long tiles, full_tiles; double time; };
constexpr long kMostParts = 256;                              // 64 MB of workspace
// Counters of a launch: one per split tile and epilogue warp of it.
inline long counter_words(const Plan16& pl) { return (pl.tiles - pl.full_tiles) * (pl.pair ? 16 : 8); }
static_assert(kMostParts / 2 * 16 * 4 <= long(kGemm16CounterBytes), "a tile in two parts has 16 counters");
inline Plan16 plan16(const Gemm16Args& a) {
    const long sms = device_sm_count(), kb = (a.K + 63) / 64;
    Plan16 best{};
    best.time = 1e300;
    if (a.epi == GEMM16_PARTS) {
        const long tiles = long((a.M + 127) / 128) * ((a.N + 127) / 128), part = (kb + a.k_parts - 1) / a.k_parts;
        return Plan16{false, false, a.k_parts, int(part), tiles, 0, 0.0};
    }
    const bool joins = a.split_ws && a.epi != GEMM16_STATS;
    const long least = a.most_blocks > 0 ? (kb + a.most_blocks - 1) / a.most_blocks : 1;          // parts of every tile
    for (int form = 0; form < 4; ++form) {
        const bool pair = form % 2 == 0, mirrored = form >= 2;
        if (a.form == GEMM16_FORM_PAIR ? !pair : a.form == GEMM16_FORM_SINGLE ? pair : false) continue;
        if (mirrored && a.epi != GEMM16_SYM) continue;
        const long tile = pair ? 256 : 128, slots = pair ? sms / 2 : sms;
        const long mt = (a.M + tile - 1) / tile, nt = (a.N + tile - 1) / tile;
        const long tiles = (mirrored ? mt * (mt + 1) / 2 : mt * nt) * a.batch;
        // whole tiles, and those of the ragged last row and column: the first copies less, the second also has narrower MMAs
        const long mw = a.M / tile, nw = a.N / tile;
        const long core = (mirrored ? nw * (nw + 1) / 2 : mw * nw) * a.batch, bottom = mirrored || mt == mw ? 0 : nw * a.batch;
        const long right = nt == nw ? 0 : mt * a.batch;
        const double fm = double(a.M - mw * tile) / tile, fn = double(a.N - nw * tile) / tile;
        const double mma = pair ? 0.27 : 0.135, copy = (pair ? 2.0 : 1.0) * 32768.0 / 11.8e6, epi = (pair ? 6.0 : 5.0) + (mirrored ? 1.5 : 0.0);
        struct Costs { double core, bottom, right; };
        auto block = [&](long active) {
            auto most = [](double x, double y) { return x > y ? x : y; };
            Costs c{most(mma, copy * active), most(mma, copy * active * (1.0 + fm) / 2), most(mma * most(fn, 0.5), copy * active * (1.0 + fn) / 2)};
            // STATS (without the spilling sums of kLong) of one row of tiles: B comes from memory, once, to pairs at 4.8 TB/s and to
            // single CTAs at 4.0 (2 rows, 2816 -> 105536: 125 and 147 us)
            if (mt == 1 && a.epi == GEMM16_STATS && (a.bf16 || kb <= 2 * kRunBlocks)) { const double feed = active * (pair ? 32768.0 / 4.8e6 : 16384.0 / 4.0e6); c.core = most(c.core, feed); c.bottom = most(c.bottom, feed); }
            return c;
        };
        const Costs full = block(slots);
        const long whole = least > 1 ? 0 : core / slots;
        for (long s = least; (s <= 16 || s == least) && (s == 1 || (joins && s * (tiles - whole * slots) <= kMostParts)); ++s) {
            const long part = (kb + s - 1) / s, splits = (kb + part - 1) / part;
            if (splits != s || (s > 1 && tiles == whole * slots)) continue;
            const long c1 = (core - whole * slots) * s, items = c1 + (bottom + right) * s;
            double last = 0.0;                               // of the items behind the whole waves
            if (items <= slots) {
                const Costs one = block(whole ? slots : items);
                last = c1 ? one.core : bottom ? one.bottom : right ? one.right : 0.0;
            } else {
                const double waves = double((c1 + slots - 1) / slots) * full.core, end = right ? full.right : bottom ? full.bottom : 0.0;
                const double even = (c1 * full.core + s * (bottom * full.bottom + right * full.right)) / slots + end / 2;
                last = waves > even ? waves : even;
            }
            const double t = whole * kb * full.core + part * last + epi + (s > 1 ? 4.0 + s * (pair ? 1.2 : 0.6) : 0.0);
            if (t < best.time) best = Plan16{pair, mirrored, int(s), int(part), tiles, s > 1 ? whole * slots : tiles, t};
        }
    }
    return best;
}

// Everything of the kernel's parameters but the tensor maps.
inline int fill_params16(Gemm16Params& p, const Gemm16Args& a, const Plan16& pl) {
    const int tile = pl.pair ? 256 : 128;
    p = Gemm16Params{};
    p.M = a.M; p.N = a.N; p.batch = a.batch;
    p.k_blocks = (a.K + 63) / 64;
    p.last_slices = (a.K - (p.k_blocks - 1) * 64 + 15) / 16;
    p.m_tiles = (a.M + tile - 1) / tile;
    p.n_tiles = (a.N + tile - 1) / tile;
    if (pl.tiles > 2000000000L || (pl.splits > 1 && a.epi != GEMM16_PARTS && counter_words(pl) * 4 > long(kGemm16CounterBytes))) return PCL_ERR_UNSUPPORTED_SHAPE;
    p.m_whole = a.M / tile;
    p.n_whole = a.N / tile;
    const long core = pl.mirrored ? long(p.n_whole) * (p.n_whole + 1) / 2 : long(p.m_whole) * p.n_whole;
    const int bottom = pl.mirrored || p.m_tiles == p.m_whole ? 0 : p.n_whole;
    p.core_tiles = int(core * a.batch);
    p.bottom_tiles = bottom * a.batch;
    auto divisor = [](long d) { return fast_div(unsigned(d > 0 ? d : 1)); };       // (0: no tile of the kind)
    p.by_core = divisor(core);
    p.by_group = divisor(long(kGroupM) * p.n_whole);
    p.by_bottom = divisor(bottom);
    p.by_right = divisor(p.m_tiles);
    p.by_rest = fast_div(unsigned(pl.tiles > pl.full_tiles ? pl.tiles - pl.full_tiles : 1));
    p.full_tiles = int(pl.full_tiles); p.splits = pl.splits; p.part_blocks = pl.part_blocks;
    p.items = int(pl.full_tiles + (pl.tiles - pl.full_tiles) * pl.splits);
    p.counters = static_cast<int*>(a.split_ws);
    p.parts = reinterpret_cast<float4*>(static_cast<char*>(a.split_ws) + kGemm16CounterBytes);
    p.symmetric = pl.mirrored; p.bf16 = a.bf16;
    p.alpha = a.alpha; p.beta = a.beta; p.keep = a.keep; p.step = a.step; p.alpha_dev = a.alpha_dev;
    p.src = a.src; p.src_ld = a.src_ld; p.src_batch = a.src_batch;
    p.out = a.out; p.out_type = a.out_type; p.out_ld = a.out_ld; p.out_batch = a.out_batch;
    p.update = a.update;
    auto four = [&](const void* ptr, int type, long ld, long bs) {
        return !ptr || ((reinterpret_cast<uintptr_t>(ptr) & (4 * dtype_bytes(type) - 1)) == 0 && ld % 4 == 0 && (a.batch == 1 || bs % 4 == 0));
    };
    p.quads = a.N % 4 == 0 && four(a.src, a.src_type, a.src_ld, a.src_batch) && four(a.out, a.out_type, a.out_ld, a.out_batch);
    p.bias = a.bias; p.labels = a.labels; p.col0 = a.col0; p.part = a.part; p.part_ld = a.part_ld; p.label_z = a.label_z; p.clear = a.clear;
    p.lse = a.lse; p.row_scale = a.row_scale;
    p.status = device_status_ptr();
    if (!p.status) return PCL_ERR_CUDA;
    return PCL_OK;
}

}  // namespace
}  // namespace pcl

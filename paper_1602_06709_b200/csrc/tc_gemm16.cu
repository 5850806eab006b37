// 16-bit GEMM on tcgen05 (kind::f16: bf16 or fp16 operands, fp32 accumulators in TMEM), the contraction behind the
// vocabulary loss and the orthogonalised update, and, with e4m3 operands (kind::f8f6f4), behind the 8-bit FC layer:  acc[r][c] = sum_k A(r, k) * B(c, k), either operand K-major or MN-major.
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
// long fp16 reductions in runs of kRunBlocks blocks and adds the runs in registers (kLong: 128 sums a thread, some of which the
// pair form spills; its main loops are long enough to hide that: 2 rows, 2856 -> 105536 forward 186 us).  bf16
// reductions stay in one run: their log-sum-exp is 2e-4 off at C = 4096 and 1.6e-3 at 16384 where all products have the same sign
// (z = 28), and 1e-5 and 4e-5 where they do not.  So do those of the DZ epilogue: fp16, C = 4096, dx is 1.7e-3 off where all
// products have the same sign, 2.4e-4 (the roundings') where they do not.
//
// e4m3 operands (Q8) go through the same ring two to a 16-bit element: a block is 128 of them, a slice of a block one K = 32 MMA of the same
// 32 bytes, and an MMA takes as long as one of 16-bit operands for twice the products.
//
// Every kernel starts before the one in front of it has ended (programmatic dependent launch): barriers, TMEM and tensor maps
// are set up meanwhile, and griddepcontrol.wait stands before the first access to global memory.
#include "gemm16_device.cuh"

namespace pcl {

namespace {

template <bool kPair, bool kAMn, bool kBMn, int kEpi, bool kLong>
__global__ void __launch_bounds__(kThreads16, 1)
tc_gemm16_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
                 const __grid_constant__ CUtensorMap tm_out, const __grid_constant__ Gemm16Params p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ Gemm16Shared sh;
    if (threadIdx.x == 0) { prefetch_tmap(&tm_a); prefetch_tmap(&tm_b); }
    constexpr bool kE4m3 = kEpi == GEMM16_Q8 || kEpi == GEMM16_Q8_STORE;
    Gemm16Ctx c = gemm16_begin<kPair>(&sh, smem_raw, p.status, kE4m3 ? kStagesQ8 : kStages16);
    const Item16 tile = decode_item(p, c.first);         // (the grid has at most p.items CTAs or pairs)
    grid_dependency_wait();
    grid_dependents_launch();
    if (kEpi == GEMM16_STATS || kEpi == GEMM16_PARTS)
        if (p.clear && blockIdx.x == 0 && threadIdx.x == 0) *p.clear = 0u;
    if (c.warp == 0) {
        if (!produce_items<kPair, kAMn, kBMn>(c, p, tile, &tm_a, &tm_b)) drain_producer(c);
    } else if (c.warp == 1) {
        if (c.pair_rank == 0) issue_items<kPair, kAMn, kBMn, kLong, kE4m3>(c, p);
        __syncwarp();
    } else {
        finish_items<kPair, kEpi, kLong>(c, p, &tm_out, nullptr, p.src, p.out);
        if (c.lane == 0) bulk_wait_group_read0();      // (the staging tiles have been read; the grid's end completes the writes)
        __syncwarp();
    }
    gemm16_end<kPair>(c);
}

struct Maps16 { CUtensorMap a, b, out; };

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
    return launch_chained(kernel, dim3(grid), dim3(kThreads16), kSmem16, st, kPair ? 2 : 1, m.a, m.b, m.out, p);
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
        case GEMM16_Q8 * 4: return launch_variant<kPair, false, false, GEMM16_Q8>(m, p, st);
        case GEMM16_Q8_STORE * 4: return launch_variant<kPair, false, false, GEMM16_Q8_STORE>(m, p, st);
        case GEMM16_STORE * 4 + 1: return launch_variant<kPair, false, true, GEMM16_STORE>(m, p, st);
        case GEMM16_STORE * 4 + 3: return launch_variant<kPair, true, true, GEMM16_STORE>(m, p, st);
        case GEMM16_GENERAL * 4 + 1: return launch_variant<kPair, false, true, GEMM16_GENERAL>(m, p, st);
        case GEMM16_GENERAL * 4 + 3: return launch_variant<kPair, true, true, GEMM16_GENERAL>(m, p, st);
    }
    return PCL_ERR_UNSUPPORTED_SHAPE;
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

bool gemm16_possible(const Gemm16Args& a) { return plan16(a).time < 1e299; }

int gemm16_parts(const Gemm16Args& a) {
    const long sms = device_sm_count(), kb = (a.K + 63) / 64, tiles = long((a.M + 127) / 128) * ((a.N + 127) / 128);
    long s = sms / tiles;
    if (s > kb / 4) s = kb / 4;                               // at least four blocks each
    if (s > 8) s = 8;
    if (s < 2) return 1;
    // ... and, of fp16, at most what the STATS epilogue takes in one run (256 x 16384 -> 3500, products of one sign: parts of 128 blocks
    // put the log-sum-exp 1.1e-3 off, at 28, in 54 us; now 76)
    const long least = a.bf16 ? 1 : (kb + 2 * kRunBlocks - 1) / (2 * kRunBlocks);
    if (s < least) s = least;
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
        case GEMM16_GENERAL:
            // a 16-bit result of the operands' type in aligned rows, and nothing added: through TMA stores
            if (a.update || (a.src && a.src_type != DT_F32)) return PCL_ERR_BAD_ARG;
            if (!a.src && a.out_type == t16 && every(a.out, t16, a.out_ld, a.out_batch)) epi = GEMM16_STORE;
            break;
        case GEMM16_Q8:
            if (!a.out || !a.row_scale || !a.col_scale || a.a.mn_major || a.b.mn_major || a.src) return PCL_ERR_BAD_ARG;
            if (a.out_type == t16 && every(a.out, t16, a.out_ld, a.out_batch)) epi = GEMM16_Q8_STORE;
            break;
        default: return PCL_ERR_BAD_ARG;
    }
    const Plan16 pl = plan16(a);
    if (pl.time >= 1e299) return PCL_ERR_UNSUPPORTED_SHAPE;
    Gemm16Params p;
    int rc = fill_params16(p, a, pl);
    if (rc != PCL_OK) return rc;
    Maps16 m;
    rc = operand_tmap(&m.a, a.a, a.M, a.K, a.batch, a.bf16);
    if (rc == PCL_OK) rc = operand_tmap(&m.b, a.b, a.N, a.K, a.batch, a.bf16);
    if (rc != PCL_OK) return rc;
    if (a.epi == GEMM16_Q8 && a.M <= 120) {
        // few rows: no more of them are copied (the others hold what was there before, in rows of the result that nobody reads); filling 128 rows, most
        // of them with zeros, took longer than the weights: 4096 -> 16384 in pairs, 1 row 23.4 -> 17.4 us, 16 rows 19.9 -> 17.6
        const int rows = int(align_up(a.M, 8));
        p.slot_bytes = (rows + 128) * 128;
        rc = make_tmap16(&m.a, a.a.ptr, t16, a.K, a.M, a.batch, a.a.ld, a.a.batch_stride, 64, uint32_t(rows));
        if (rc != PCL_OK) return rc;
    }
    m.out = m.a;
    if (epi == GEMM16_STORE || epi == GEMM16_DZ || epi == GEMM16_Q8_STORE) rc = make_tmap16(&m.out, a.out, t16, a.N, a.M, a.batch, a.out_ld, a.out_batch, 64, 32);
    if (epi == GEMM16_PARTS) rc = make_tmap16(&m.out, a.out, DT_F32, a.N, a.M, pl.splits, a.out_ld, a.out_batch, 32, 32);
    if (rc != PCL_OK) return rc;
    LaunchScope scope(KID_TC_GEMM16, (a.epi == GEMM16_Q8 ? 4.0 : 2.0) * a.M * double(a.N) * a.K * a.batch, st);
    return pl.pair ? launch_form<true>(a, epi, m, p, st) : launch_form<false>(a, epi, m, p, st);
}

}  // namespace pcl

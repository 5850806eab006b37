// Embedding lookup with scaling and its gradient by sorted tokens.  Everything here is bound by memory: a row of the table
// or of dy is read once, a row of the output written once.
//
// Gradient: dtable[v] = scale * sum over tokens n with ids[n] = v of dy[n].  The tokens are sorted by id (stable, so equal
// ids stay in index order): few of them by counting, more by one cluster of CTAs.  The other CTAs of that launch fetch dy into L2 where it
// fits and zero the gradient's last rows, as much as the sort's time allows (the sort is latency, the rest bandwidth).  Then
// every 8 or 16 consecutive sorted tokens are one work item.  An item sums the segments (runs of equal ids) that begin in it; only
// segments of more than twice that are cut at the items' borders into partial sums that a last pass adds in order.  The work is
// even whatever the ids' frequencies are, and the additions have a fixed order (no atomics).  Blocks that zero the remaining
// rows that do not occur run between the items' blocks.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <limits.h>

#include "pcl_internal.h"
#include "pcl_ptx.cuh"

namespace pcl {

namespace {

// Sorted tokens per work item, and the segment length from which a segment is cut at the items' borders: few tokens are spread
// over more warps (5000 tokens: 18.5 -> 13 us with items of 8), many leave fewer partial sums.
inline int item_tokens(int N) { return N <= 8192 ? 8 : 16; }
inline int long_segment(int N) { return 2 * item_tokens(N); }
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = 32;
constexpr int kMaxSortCtas = 8;          // portable cluster size
constexpr int kMaxBits = 9;              // bits of a digit
constexpr int kHistLd = (1 << kMaxBits) + 1;                  // (odd: a column over the warps meets every bank once)
constexpr size_t kBesideSort = size_t(100) << 20;             // bytes fetched and zeroed beside the sort (in about its 20 us)
constexpr int kMaxRun = 8192;            // tokens per CTA that the shared-memory sort takes
constexpr int kRankThreads = 512;
// Tokens that are sorted by counting: 1 token 7.1 -> 4.3 us, 100 10.1 -> 7.0, 2000 17.0 -> 12.3, 4096 19.7 -> 18.8 (whole gradient calls),
// but 6000 21.8 -> 27.0, because the work is quadratic.
constexpr int kMostRanked = 4096;
constexpr size_t kBesideRank = size_t(32) << 20;              // in its 5 us

template <class T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

template <class T, int kVec> struct alignas(sizeof(T) * kVec) Pack { T e[kVec]; };

// Output rows are not read again by these kernels: they should not push the table's rows out of L2.
template <class T, int kVec>
__device__ __forceinline__ void store_streaming(Pack<T, kVec>* p, const Pack<T, kVec>& v) {
    if constexpr (sizeof(T) * kVec == 16) __stcs(reinterpret_cast<uint4*>(p), *reinterpret_cast<const uint4*>(&v));
    else *p = v;
}

// Vectors per thread and row in the lookup; per lane and token in the gradient.  Rows are taken in the longest vectors that all of them
// start on a multiple of (32768 tokens, bf16 rows of 2048 / 2044 / 2046 / 2047: lookup 48 / 53 / 62 / 66 us, gradient
// 154 / 170 / 206 / 262 us; with single elements for the last three 75 and 420): short ones are bound by the number of instructions.
template <int kVec> constexpr int kLoads = kVec == 1 ? 8 : kVec == 2 ? 4 : 2;
template <int kVec, bool kSgd> constexpr int kReps = kVec == 1 && kSgd ? 2 : 1;

// ids that name no row (outside [0, V)) and the padding id
__device__ __forceinline__ bool row_exists(int id, int V, int pad_id, unsigned int* status) {
    if (is_special(id, pad_id)) return false;
    if (id < 0 || id >= V) {
        atomicCAS(status, 0u, static_cast<unsigned int>(kStatusBadLabel));
        return false;
    }
    return true;
}

// Two rows per pass of a thread group, and two vectors of each (more of shorter ones, where rows are not aligned for 16 bytes): that many
// independent loads per thread in flight.
template <class T, int kVec>
__global__ void __launch_bounds__(256) embedding_fwd_kernel(const int* __restrict__ ids, const T* __restrict__ table,
                                                            float scale, int pad_id, T* __restrict__ out, int N, int V, int C,
                                                            int tpr_log2, unsigned int* status) {
    constexpr int kHalves = kLoads<kVec>;
    const int tpr = 1 << tpr_log2;                   // threads per row
    grid_dependency_wait();
    grid_dependents_launch();
    const int vecs = C / kVec;
    const int lane = threadIdx.x & (tpr - 1);
    const long groups = long(gridDim.x) * (256 >> tpr_log2);
    for (long n = long(blockIdx.x) * (256 >> tpr_log2) + (threadIdx.x >> tpr_log2); n < N; n += 2 * groups) {
        bool there[2];
        const Pack<T, kVec>* src[2];
        Pack<T, kVec>* dst[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const long row = n + r * groups;
            const int id = row < N ? ids[row] : pad_id;
            there[r] = row < N && row_exists(id, V, pad_id, status);
            src[r] = reinterpret_cast<const Pack<T, kVec>*>(table + size_t(there[r] ? id : 0) * C);
            dst[r] = row < N ? reinterpret_cast<Pack<T, kVec>*>(out + size_t(row) * C) : nullptr;
        }
        for (int i = lane; i < vecs; i += kHalves * tpr) {
            Pack<T, kVec> v[2][kHalves];
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int h = 0; h < kHalves; ++h)
                    if (there[r] && i + h * tpr < vecs) v[r][h] = src[r][i + h * tpr];
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
                    if (!dst[r] || i + h * tpr >= vecs) continue;
                    Pack<T, kVec> o;
#pragma unroll
                    for (int j = 0; j < kVec; ++j) o.e[j] = from_f32<T>(there[r] ? scale * to_f32<T>(v[r][h].e[j]) : 0.f);
                    store_streaming(&dst[r][i + h * tpr], o);
                }
        }
    }
}

// A row of zeros by a warp, in 16-byte stores whatever its alignment (the bf16 gradient of 32768 tokens, 131072 x 2047:
// 420 -> 390 us).
template <class T>
__device__ __forceinline__ void zero_row(T* row, int C, int lane) {
    constexpr int kUnit = 16 / int(sizeof(T));
    int head = int((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / int(sizeof(T));
    if (head > C) head = C;
    const int units = (C - head) / kUnit, tail = C - head - units * kUnit;
    uint4* body = reinterpret_cast<uint4*>(row + head);
#pragma unroll 4
    for (int i = lane; i < units; i += 32) body[i] = make_uint4(0u, 0u, 0u, 0u);
    if (lane < head) row[lane] = from_f32<T>(0.f);
    if (lane < tail) row[head + units * kUnit + lane] = from_f32<T>(0.f);
}

// Stable radix sort of (id, token) by one cluster of CTAs.  Every warp owns a run of consecutive tokens; per pass it counts
// its digits, the counts are turned into positions (over digits, then CTAs, then warps, which keeps equal digits in
// token order), and the warp scatters its run in order.  Tokens without a row get the key V and end up last.  Each CTA
// owns a run of 2^run_log2 positions in its shared memory, and scattering writes the owner's (distributed shared memory);
// more tokens than that are kept in global memory instead (kShared = false).
// Leaves the sorted keys and tokens and, for each id that occurs, the bounds of its segment.
struct SortArgs {
    const int* ids;
    int N, V, pad_id;
    int passes, bits;             // digits of `bits` bits, least significant first
    int ctas;                     // of the sorting cluster (cluster 0)
    int run_log2;                 // positions per CTA (kShared)
    int per_warp;                 // tokens per warp, a multiple of 32
    int *keys0, *keys1;           // written by the even and the odd passes (kShared: the last pass's, once)
    int *idx0, *idx1;
    int2* bounds;                 // [V]: first position and end of the segment of an id; anything where it does not occur
    int* long_count;              // set to 0 here
    uint4* zero; size_t zero16;   // what the other CTAs clear: 16-byte units, and the bytes behind them
    unsigned char* zero_tail; int zero_tail_bytes;
    const char* dy; size_t dy_lines;                          // ... and fetch into L2: 128-byte lines of dy, and (sgd) the rows of
    const char* table; size_t row_bytes;                      // the table that the ids name
    unsigned int* status;
};
template <bool kShared>
__device__ __forceinline__ void sort_barrier(bool cluster) {
    if (!cluster) { __syncthreads(); return; }
    if (!kShared) __threadfence();
    cluster_sync_all();
    if (!kShared) __threadfence();                            // (drops stale L1 lines)
}
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
// The lanes of `act` (to which the calling lane belongs) that hold the same digit of `bits` bits.
__device__ __forceinline__ unsigned same_digit(unsigned act, int d, int bits) {
    unsigned same = act;
    for (int b = 0; b < bits; ++b) {
        const unsigned m = __ballot_sync(act, (d >> b) & 1);
        same &= (d >> b) & 1 ? m : ~m;
    }
    return same;
}
__device__ __forceinline__ int ld_cluster(uint32_t addr) {
    int v;
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster(uint32_t addr, int x, int y) {
    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ uint32_t map_addr(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

// What the blocks from `first` on do beside the sorting ones: fetch dy and the rows of the table that the ids name into L2, zeros.
__device__ __forceinline__ void beside_sort(const SortArgs& a, int first) {
    const int lane = threadIdx.x & 31;
    const uint4 z = make_uint4(0u, 0u, 0u, 0u);
    const size_t stride = size_t(gridDim.x - first) * blockDim.x;
    const size_t i0 = size_t(blockIdx.x - first) * blockDim.x + threadIdx.x;
    for (size_t i = i0; i < a.dy_lines; i += stride) prefetch_l2(a.dy + i * 128);
    if (a.table)
        for (size_t n = i0 >> 5; n < size_t(a.N); n += stride >> 5) {
            const int id = a.ids[n];
            if (id == a.pad_id || id < 0 || id >= a.V) continue;
            for (size_t o = size_t(lane) * 128; o < a.row_bytes; o += 32 * 128) prefetch_l2(a.table + size_t(id) * a.row_bytes + o);
        }
#pragma unroll 4
    for (size_t i = i0; i < a.zero16; i += stride) a.zero[i] = z;
    if (i0 < size_t(a.zero_tail_bytes)) a.zero_tail[i0] = 0;
}

// The same for few tokens, without passes: a token's position is the number of tokens with a smaller id, or the same id and a smaller
// index.  A block takes 32 tokens, one per lane, and its warps compare them with all tokens, 32 at a time (four integer instructions a
// comparison of 32 lanes, at half rate: N^2 / 2000 cycles with all SMs).  No block needs another's result.
__global__ void __launch_bounds__(kRankThreads) embedding_rank_kernel(SortArgs a) {
    constexpr int kWarps = kRankThreads / 32, kChunks = 4;
    __shared__ __align__(16) int others[kWarps][kChunks * 32];
    __shared__ int counts[kWarps][3][32];
    grid_dependency_wait();
    grid_dependents_launch();
    if (int(blockIdx.x) >= a.ctas) { beside_sort(a, a.ctas); return; }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, own = blockIdx.x;
    if (own == 0 && threadIdx.x == 0) *a.long_count = 0;
    const int chunks = (a.N + 31) / 32, n = own * 32 + lane;
    auto key_of = [&](int i) {               // (behind the last token: larger than all keys)
        const int id = i < a.N ? a.ids[i] : INT_MAX;
        return i >= a.N ? INT_MAX : id == a.pad_id || id < 0 || id >= a.V ? a.V : id;
    };
    const int key = key_of(n);
    int pos = 0, less = 0, upto = 0;         // tokens before this one; of smaller ids; of ids up to this one's
    for (int c0 = warp; c0 < chunks; c0 += kWarps * kChunks) {
        int k[kChunks];
#pragma unroll
        for (int i = 0; i < kChunks; ++i) k[i] = key_of((c0 + i * kWarps) * 32 + lane);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kChunks; ++i) others[warp][i * 32 + lane] = k[i];
        __syncwarp();
#pragma unroll 1
        for (int i = 0; i < kChunks; ++i) {
            const int c = c0 + i * kWarps;
            if (c >= chunks) break;
            int l = 0, u = 32, first = 0;     // first: of the ids up to this one's those of smaller indices (own chunk)
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const int4 o = *reinterpret_cast<const int4*>(&others[warp][i * 32 + j]);
                const int q[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    l += int(unsigned(q[e] - key) >> 31);        // (keys are not negative: the sign is the comparison)
                    u -= int(unsigned(key - q[e]) >> 31);
                }
            }
            if (c == own)
                for (int j = 0; j < 32; ++j) {
                    const int q = others[warp][i * 32 + j];
                    first += q < key || (q == key && j < lane);
                }
            less += l;
            upto += u;
            pos += c < own ? u : c > own ? l : first;
        }
    }
    counts[warp][0][lane] = pos; counts[warp][1][lane] = less; counts[warp][2][lane] = upto;
    __syncthreads();
    if (warp > 0 || n >= a.N) return;
    pos = less = upto = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) { pos += counts[w][0][lane]; less += counts[w][1][lane]; upto += counts[w][2][lane]; }
    if (key == a.V) row_exists(a.ids[n], a.V, a.pad_id, a.status);
    a.keys1[pos] = key;
    a.idx1[pos] = n;
    if (key < a.V && pos == less) a.bounds[key] = make_int2(less, upto);
}

template <bool kShared>
__global__ void __launch_bounds__(kSortThreads) embedding_sort_kernel(SortArgs a) {
    extern __shared__ int sort_smem[];       // hist [32][kHistLd], totals [512], (kShared) [2] runs of (key, token)
    __shared__ int warp_sum[16];
    grid_dependency_wait();
    grid_dependents_launch();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (int(blockIdx.x) >= a.ctas) { beside_sort(a, a.ctas); return; }
    int(*hist)[kHistLd] = reinterpret_cast<int(*)[kHistLd]>(sort_smem);
    int* totals = sort_smem + kSortWarps * kHistLd;
    int2* runs = reinterpret_cast<int2*>(totals + (1 << kMaxBits));           // [2][1 << run_log2]
    const int cta = blockIdx.x, ctas = a.ctas;
    const bool cluster = ctas > 1;
    if (cta == 0 && threadIdx.x == 0) *a.long_count = 0;
    const int bins = 1 << a.bits, run_size = 1 << a.run_log2;
    // this warp's tokens, as positions of the sequence; kShared: offsets in this CTA's run
    const long cta0 = kShared ? long(cta) << a.run_log2 : 0;
    const long r0 = (kShared ? cta0 : long(cta) * kSortWarps * a.per_warp) + long(warp) * a.per_warp;
    long r1 = r0 + a.per_warp;
    if (kShared && r1 > cta0 + run_size) r1 = cta0 + run_size;
    if (r1 > a.N) r1 = a.N;
    auto id_key = [&](long i) {
        const int id = a.ids[i];
        return row_exists(id, a.V, a.pad_id, a.status) ? id : a.V;
    };
    if (kShared) {
#pragma unroll 2
        for (long i = r0 + lane; i < r1; i += 32) runs[i - cta0] = make_int2(id_key(i), int(i));
        __syncwarp();
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.bits, from = pass & 1;     // kShared: buffer read in this pass
        const int2* run = runs + (size_t(from) << a.run_log2) - cta0;
        auto pair_of = [&](long i) {
            if (kShared) return run[i];
            return pass > 0 ? make_int2((from ? a.keys0 : a.keys1)[i], (from ? a.idx0 : a.idx1)[i]) : make_int2(id_key(i), int(i));
        };
        for (int d = lane; d < bins; d += 32) hist[warp][d] = 0;
        __syncwarp();
        for (long i0 = r0; i0 < r1; i0 += 32) {
            const long i = i0 + lane;
            const bool in = i < r1;
            const unsigned act = __ballot_sync(0xffffffffu, in);
            if (in) {
                const int d = (pair_of(i).x >> shift) & (bins - 1);
                const unsigned same = same_digit(act, d, a.bits);
                if (lane == __ffs(same) - 1) hist[warp][d] += __popc(same);
            }
            __syncwarp();
        }
        __syncthreads();
        const int d0 = threadIdx.x;                           // thread d: digit d's counts of the warps become offsets
        int total = 0;
        if (d0 < bins) {
#pragma unroll 8
            for (int w = 0; w < kSortWarps; ++w) { const int c = hist[w][d0]; hist[w][d0] = total; total += c; }
            totals[d0] = total;
        }
        sort_barrier<kShared>(cluster);
        int all = total, before = 0;                          // over the CTAs, and those before this one
        if (cluster && d0 < bins) {
            const uint32_t mine = smem_u32(totals + d0);
            all = 0;
#pragma unroll 4
            for (int c = 0; c < ctas; ++c) {
                const int v = ld_cluster(map_addr(mine, c));
                if (c < cta) before += v;
                all += v;
            }
        }
        if (d0 < (1 << kMaxBits)) {                           // exclusive scan over the digits
            if (d0 >= bins) all = 0;
            int inc = all;
            for (int o = 1; o < 32; o <<= 1) { const int u = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += u; }
            if (lane == 31) warp_sum[warp] = inc;
            before += inc - all;
        }
        __syncthreads();
        if (d0 < bins) {
            for (int w = 0; w < warp; ++w) before += warp_sum[w];
#pragma unroll 8
            for (int w = 0; w < kSortWarps; ++w) hist[w][d0] += before;
        }
        __syncthreads();
        const uint32_t dst_run = smem_u32(runs + ((from ^ 1) << a.run_log2));
        for (long i0 = r0; i0 < r1; i0 += 32) {
            const long i = i0 + lane;
            const bool in = i < r1;
            const unsigned act = __ballot_sync(0xffffffffu, in);
            if (in) {
                const int2 kt = pair_of(i);
                const int d = (kt.x >> shift) & (bins - 1);
                const unsigned same = same_digit(act, d, a.bits);
                const int pos = hist[warp][d] + __popc(same & ((1u << lane) - 1u));
                __syncwarp(act);
                if (lane == __ffs(same) - 1) hist[warp][d] += __popc(same);
                if (kShared) {
                    const uint32_t off = (uint32_t(pos) & uint32_t(run_size - 1)) * 8u;
                    if (cluster) st_cluster(map_addr(dst_run + off, uint32_t(pos) >> a.run_log2), kt.x, kt.y);
                    else runs[((from ^ 1) << a.run_log2) + pos] = kt;
                } else {
                    (from ? a.keys1 : a.keys0)[pos] = kt.x;
                    (from ? a.idx1 : a.idx0)[pos] = kt.y;
                }
            }
            __syncwarp();
        }
        sort_barrier<kShared>(cluster);
    }
    const int last = a.passes & 1;                            // kShared: the buffer of the last pass
    int* sorted = (a.passes & 1) ? a.keys0 : a.keys1;
    int* sorted_idx = (a.passes & 1) ? a.idx0 : a.idx1;
    const long e0 = kShared ? cta0 : 0;
    const long e1 = kShared ? (cta0 + run_size < a.N ? cta0 + run_size : a.N) : a.N;
    const long step = kShared ? kSortThreads : long(ctas) * kSortThreads;
    for (long i = e0 + (kShared ? 0 : long(cta) * kSortThreads) + threadIdx.x; i < e1; i += step) {
        int k, before = -1, after = -1;
        if (kShared) {
            const int o = int(i - cta0);
            const int2* mine = runs + (last << a.run_log2);
            k = mine[o].x;
            if (i > 0) before = o > 0 ? mine[o - 1].x : ld_cluster(map_addr(smem_u32(mine + run_size - 1), cta - 1));
            if (i + 1 < a.N) after = o + 1 < run_size ? mine[o + 1].x : ld_cluster(map_addr(smem_u32(mine), cta + 1));
            sorted[i] = k;
            sorted_idx[i] = mine[o].y;
        } else {
            k = sorted[i];
            if (i > 0) before = sorted[i - 1];
            if (i + 1 < a.N) after = sorted[i + 1];
        }
        if (k < a.V) {
            if (before != k) a.bounds[k].x = int(i);
            if (after != k) a.bounds[k].y = int(i) + 1;
        }
    }
    if (kShared && cluster) cluster_sync_all();               // (the neighbours may still read this CTA's run)
}

struct GradArgs {
    const int* keys;              // sorted ids (V: no row)
    const int* idx;               // their tokens
    const int2* bounds;           // [V] segment of an id that occurs
    int zero_rows;                // rows [0, zero_rows) that do not occur are zeroed here
    int item_blocks, zero_blocks;
    float* part;                  // [items][2][C]: sums of an item's share of a long segment begun before it, and begun in it
    float scale, lr;
    int N, V, C, items, item_tokens;
    int* long_count;              // long segments and the items they begin in
    int* long_items;
    int wpi_log2;                 // warps per item
    int sgd;
};

template <class T, int kVec>
__device__ __forceinline__ void write_row(const GradArgs& a, T* out, int key, int i, const float (&sum)[kVec], const Pack<T, kVec>& old) {
    Pack<T, kVec> o;
    if (a.sgd) {
#pragma unroll
        for (int j = 0; j < kVec; ++j) o.e[j] = from_f32<T>(fmaf(-a.lr, a.scale * sum[j], to_f32<T>(old.e[j])));
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) o.e[j] = from_f32<T>(a.scale * sum[j]);
    }
    reinterpret_cast<Pack<T, kVec>*>(out + size_t(key) * a.C)[i] = o;
}

// One warp per item and 32 vectors of a row (kSgd, single elements: 64).  The item's keys
// and tokens are held by the lanes (a window of 32 sorted positions), so that per batch of tokens only their rows are waited
// for; with kSgd the table's old rows come with them.
template <class T, int kVec, bool kSgd>
__global__ void __launch_bounds__(256, kSgd || kVec < 8 ? 4 : 3) embedding_grad_kernel(GradArgs a, const T* __restrict__ dy, T* __restrict__ out) {
    constexpr int kBatch = 4, kRep = kReps<kVec, kSgd>;             // tokens at a time; vectors per lane, 32 apart
    using P = Pack<T, kVec>;
    const int vecs = a.C / kVec, strips = (vecs + 32 * kRep - 1) / (32 * kRep);
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    grid_dependency_wait();
    grid_dependents_launch();
    // the zeroing blocks are spread evenly among the others
    const long all = long(a.item_blocks) + a.zero_blocks, b = blockIdx.x;
    const int zeros_before = int(b * a.zero_blocks / all);
    if (!kSgd && int((b + 1) * a.zero_blocks / all) != zeros_before) {
        for (int v = zeros_before * 8 + w; v < a.zero_rows; v += a.zero_blocks * 8) {
            const int at = a.bounds[v].x;                     // (of an id that does not occur: anything)
            if (unsigned(at) < unsigned(a.N) && a.keys[at] == v) continue;
            zero_row(out + size_t(v) * a.C, a.C, lane);
        }
        return;
    }
    const int wpi = 1 << a.wpi_log2;                          // warps per item
    const int item = int(b - zeros_before) * (8 >> a.wpi_log2) + (w >> a.wpi_log2);
    if (item >= a.items) return;
    const int p0 = item * a.item_tokens;
    const int p1 = p0 + a.item_tokens < a.N ? p0 + a.item_tokens : a.N;
    int wb = p0, key, tok;
    unsigned ends;
    auto load_window = [&]() {                                // (whether lane 31 ends a segment is not known in it)
        key = wb + lane < a.N ? a.keys[wb + lane] : -1;
        tok = wb + lane < a.N ? a.idx[wb + lane] : 0;
        const int next = __shfl_down_sync(0xffffffffu, key, 1);
        ends = __ballot_sync(0xffffffffu, lane < 31 && key != next);
    };
    load_window();
    const int k0 = __shfl_sync(0xffffffffu, key, 0);
    if (k0 >= a.V) return;
    // [.., rows_end): the item's tokens that have a row
    const int rows_end = p0 + __popc(__ballot_sync(0xffffffffu, p0 + lane < p1 && key < a.V));
    const int k1 = __shfl_sync(0xffffffffu, key, rows_end - 1 - p0);
    const int2 s0 = a.bounds[k0], s1 = a.bounds[k1];
    const int done = s0.x < p0 ? (s0.y < rows_end ? s0.y : rows_end) : p0;      // [p0, done): of a segment begun before
    const bool front = done > p0 && s0.y - s0.x > 2 * a.item_tokens;                 // ... whose share is summed here
    const bool goes_on = s1.x >= p0 && s1.y > p1;                               // the last segment begins here
    const bool back = goes_on && s1.y - s1.x > 2 * a.item_tokens;
    const int begin = front ? p0 : done, stop = back || !goes_on ? rows_end : s1.y;
    if (back && (w & (wpi - 1)) == 0 && lane == 0) a.long_items[atomicAdd(a.long_count, 1)] = item;
    for (int strip = w & (wpi - 1); strip < strips; strip += wpi) {
        const int i0 = strip * 32 * kRep + lane;
        float sum[kRep][kVec];
#pragma unroll
        for (int h = 0; h < kRep; ++h)
#pragma unroll
            for (int j = 0; j < kVec; ++j) sum[h][j] = 0.f;
        for (int p = begin; p < stop; p += kBatch) {
            if (p < wb || p + kBatch > wb + 31) { wb = p; load_window(); }
            P v[kBatch][kRep], old[kSgd ? kBatch : 1][kRep];
            bool row_ends[kBatch];
#pragma unroll
            for (int q = 0; q < kBatch; ++q) {
                const int o = p - wb + q;
                const size_t t = size_t(__shfl_sync(0xffffffffu, tok, o));
                const int k = kSgd ? __shfl_sync(0xffffffffu, key, o) : 0;
                row_ends[q] = (ends >> o) & 1u;
#pragma unroll
                for (int h = 0; h < kRep; ++h)
                    if (p + q < stop && i0 + 32 * h < vecs) {
                        v[q][h] = reinterpret_cast<const P*>(dy + t * a.C)[i0 + 32 * h];
                        if (kSgd && row_ends[q]) old[q][h] = reinterpret_cast<const P*>(out + size_t(k) * a.C)[i0 + 32 * h];
                    }
            }
#pragma unroll
            for (int q = 0; q < kBatch; ++q) {
                if (p + q >= stop) break;
                const int k = __shfl_sync(0xffffffffu, key, p - wb + q);
                const bool flush = row_ends[q] || p + q + 1 == stop;
                const bool share0 = front && p + q < done, share1 = back && p + q >= s1.x;
#pragma unroll
                for (int h = 0; h < kRep; ++h) {
                    const int i = i0 + 32 * h;
                    if (i >= vecs) continue;
#pragma unroll
                    for (int j = 0; j < kVec; ++j) sum[h][j] += to_f32<T>(v[q][h].e[j]);
                    if (!flush) continue;
                    if (share0 || share1) {
                        float* dst = a.part + (size_t(item) * 2 + (share0 ? 0 : 1)) * a.C + size_t(i) * kVec;
#pragma unroll
                        for (int j = 0; j < kVec; ++j) dst[j] = sum[h][j];
                    } else {
                        write_row<T, kVec>(a, out, k, i, sum[h], old[kSgd ? q : 0][h]);
                    }
#pragma unroll
                    for (int j = 0; j < kVec; ++j) sum[h][j] = 0.f;
                }
            }
        }
    }
}

// Long segments: the shares of a segment are added up in a fixed order, every eighth by one warp, then the warps' sums.
template <class T, int kVec>
__global__ void __launch_bounds__(256) embedding_grad_join_kernel(GradArgs a, T* __restrict__ out) {
    __shared__ float sums[8][32][kVec + 1];
    grid_dependency_wait();
    grid_dependents_launch();
    const int vecs = a.C / kVec, strips = (vecs + 31) / 32;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const long works = long(*a.long_count) * strips;
    for (long wk = blockIdx.x; wk < works; wk += gridDim.x) {
        const int item = a.long_items[wk / strips], i = int(wk % strips) * 32 + lane;
        const int key = a.keys[(item + 1) * a.item_tokens - 1];
        const int last = (a.bounds[key].y - 1) / a.item_tokens;
        float sum[kVec];
#pragma unroll
        for (int j = 0; j < kVec; ++j) sum[j] = 0.f;
        if (i < vecs) {
#pragma unroll 8
            for (int it = item + w; it <= last; it += 8) {
                const float* src = a.part + (size_t(it) * 2 + (it == item ? 1 : 0)) * a.C + size_t(i) * kVec;
#pragma unroll
                for (int j = 0; j < kVec; ++j) sum[j] += src[j];
            }
        }
#pragma unroll
        for (int j = 0; j < kVec; ++j) sums[w][lane][j] = sum[j];
        __syncthreads();
        if (w == 0 && i < vecs) {
            for (int o = 1; o < 8; ++o)
#pragma unroll
                for (int j = 0; j < kVec; ++j) sum[j] += sums[o][lane][j];
            Pack<T, kVec> old;
            if (a.sgd) old = reinterpret_cast<const Pack<T, kVec>*>(out + size_t(key) * a.C)[i];
            write_row<T, kVec>(a, out, key, i, sum, old);
        }
        __syncthreads();
    }
}

int log2_threads(int vecs) {
    int l = 5;
    while (l < 8 && (1 << l) < vecs) ++l;
    return l;
}

struct BwdLayout { size_t keys[2], idx[2], bounds, long_count, long_items, part, total; };
BwdLayout bwd_layout(int N, int V, int C) {
    BwdLayout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
    const size_t items = (size_t(N) + item_tokens(N) - 1) / item_tokens(N);
    for (int i = 0; i < 2; ++i) { l.keys[i] = take(size_t(N) * 4); l.idx[i] = take(size_t(N) * 4); }
    l.bounds = take(size_t(V) * 8);
    l.long_count = take(4);
    l.long_items = take((size_t(N) / long_segment(N) + 1) * 4);
    l.part = take(N > long_segment(N) ? items * 2 * C * 4 : 0);
    l.total = at;
    return l;
}

template <class T, int kVec>
int run_fwd(int N, int V, int C, const int* ids, const void* table, float scale, int pad_id, void* out, unsigned int* status,
            cudaStream_t st) {
    const int tl = log2_threads((C / kVec + kLoads<kVec> / 2 - 1) / (kLoads<kVec> / 2));
    const long rows_per_block = 256 >> tl;
    const long blocks = (N + 2 * rows_per_block - 1) / (2 * rows_per_block), cap = long(device_sm_count()) * 8;
    LaunchScope scope(KID_EMBEDDING, 2.0 * sizeof(T) * double(N) * C, st);
    return launch_chained(embedding_fwd_kernel<T, kVec>, dim3(unsigned(blocks < cap ? blocks : cap)), dim3(256), 0, st, 1, ids,
                          static_cast<const T*>(table), scale, pad_id, static_cast<T*>(out), N, V, C, tl, status);
}

template <class T, int kVec>
int run_grad(GradArgs a, const void* dy, void* out, cudaStream_t st) {
    const int vecs = a.C / kVec, per_strip = 32 * (a.sgd ? kReps<kVec, true> : kReps<kVec, false>), strips = (vecs + per_strip - 1) / per_strip;
    while (a.wpi_log2 < 3 && (1 << a.wpi_log2) < strips) ++a.wpi_log2;
    const int per_block = 8 >> a.wpi_log2, blocks = (a.items + per_block - 1) / per_block;
    {
        LaunchScope scope(KID_EMBEDDING, double(sizeof(T)) * a.C * double(a.N), st);
        a.item_blocks = blocks;
        const int zero_cap = device_sm_count() * 8;
        a.zero_blocks = (a.zero_rows + 7) / 8 < zero_cap ? (a.zero_rows + 7) / 8 : zero_cap;
        const int rc = launch_chained(a.sgd ? embedding_grad_kernel<T, kVec, true> : embedding_grad_kernel<T, kVec, false>,
                                      dim3(blocks + (a.sgd ? 0 : a.zero_blocks)), dim3(256), 0, st, 1, a, static_cast<const T*>(dy),
                                      static_cast<T*>(out));
        if (rc != PCL_OK) return rc;
    }
    if (a.N <= long_segment(a.N)) return PCL_OK;
    LaunchScope scope(KID_EMBEDDING, 0.0, st);
    const long most = (long(a.N) / long_segment(a.N)) * ((vecs + 31) / 32), cap = long(device_sm_count()) * 8;
    return launch_chained(embedding_grad_join_kernel<T, kVec>, dim3(unsigned(most < cap ? most : cap)), dim3(256), 0, st, 1, a, static_cast<T*>(out));
}

int log2_up(long v) {
    int l = 0;
    while ((1L << l) < v) ++l;
    return l;
}

template <bool kShared>
int run_sort(const SortArgs& s, size_t smem, int blocks, cudaStream_t st) {
    static PerDeviceOnce once;
    const int rc = once.run([&] {
        return cudaFuncSetAttribute(embedding_sort_kernel<kShared>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - 1024) ==
                       cudaSuccess ? PCL_OK : PCL_ERR_CUDA;
    });
    if (rc != PCL_OK) return rc;
    return launch_chained(embedding_sort_kernel<kShared>, dim3(blocks), dim3(kSortThreads), smem, st, unsigned(s.ctas), s);
}

}  // namespace

size_t embedding_workspace_bytes(int N, int V, int C) { return bwd_layout(N, V, C).total; }

int launch_embedding_fwd(int N, int V, int C, int type, const int* ids, const void* table, float scale, int pad_id, void* out,
                         cudaStream_t st) {
    unsigned int* status = device_status_ptr();
    if (!status) return PCL_ERR_CUDA;
    auto run = [&](auto zero) {              // with the longest vectors that every row starts on a multiple of
        using T = decltype(zero);
        if constexpr (sizeof(T) == 2)
            if (C % 8 == 0) return run_fwd<T, 8>(N, V, C, ids, table, scale, pad_id, out, status, st);
        return C % 4 == 0 ? run_fwd<T, 4>(N, V, C, ids, table, scale, pad_id, out, status, st)
             : C % 2 == 0 ? run_fwd<T, 2>(N, V, C, ids, table, scale, pad_id, out, status, st)
                          : run_fwd<T, 1>(N, V, C, ids, table, scale, pad_id, out, status, st);
    };
    return type == DT_F32 ? run(float{}) : type == DT_BF16 ? run(__nv_bfloat16{}) : run(__half{});
}

int launch_embedding_bwd(int N, int V, int C, int type, const int* ids, const void* dy, float scale, int pad_id, void* out,
                         bool sgd, float lr, void* ws, cudaStream_t st) {
    unsigned int* status = device_status_ptr();
    if (!status) return PCL_ERR_CUDA;
    const BwdLayout l = bwd_layout(N, V, C);
    char* base = static_cast<char*>(ws);
    SortArgs s{};
    s.ids = ids; s.N = N; s.V = V; s.pad_id = pad_id; s.status = status;
    const int key_bits = log2_up(long(V) + 1);                               // keys 0 .. V
    s.passes = (key_bits + kMaxBits - 1) / kMaxBits;
    s.bits = (key_bits + s.passes - 1) / s.passes;
    // Tokens per CTA: 1024 where one CTA takes them all, up to kMaxRun with eight; beyond, the sequence stays in global memory.
    const bool rank = N <= kMostRanked, shared = N <= kMaxSortCtas * kMaxRun;
    size_t smem = size_t(kSortWarps * kHistLd + (1 << kMaxBits)) * 4;
    if (rank) {
        s.ctas = (N + 31) / 32;
        s.passes = 0;
    } else if (shared) {
        s.run_log2 = log2_up((N + kMaxSortCtas - 1) / kMaxSortCtas);
        if (s.run_log2 < 10) s.run_log2 = 10;
        s.ctas = 1 << log2_up((long(N) + (1 << s.run_log2) - 1) >> s.run_log2);
        s.per_warp = (1 << s.run_log2) / kSortWarps;
        smem += size_t(16) << s.run_log2;
    } else {
        s.ctas = kMaxSortCtas;
        const long per_warp = (N + long(s.ctas) * kSortWarps - 1) / (long(s.ctas) * kSortWarps);
        s.per_warp = int((per_warp + 31) / 32 * 32);
    }
    s.keys0 = reinterpret_cast<int*>(base + l.keys[0]); s.keys1 = reinterpret_cast<int*>(base + l.keys[1]);
    s.idx0 = reinterpret_cast<int*>(base + l.idx[0]); s.idx1 = reinterpret_cast<int*>(base + l.idx[1]);
    s.bounds = reinterpret_cast<int2*>(base + l.bounds);
    s.long_count = reinterpret_cast<int*>(base + l.long_count);
    // What the other SMs do meanwhile: fetch dy (and the table's rows) into L2 if they fit, then zeros.
    const size_t row = size_t(C) * dtype_bytes(type);
    size_t fetched = size_t(N) * row * (sgd ? 2 : 1);
    const size_t beside = rank ? kBesideRank : kBesideSort;
    if (fetched > beside) fetched = size_t(N) * row <= beside ? size_t(N) * row : 0;
    if (fetched) {
        s.dy = static_cast<const char*>(dy);
        s.dy_lines = (size_t(N) * row + 127) / 128;
        if (sgd && fetched > size_t(N) * row) { s.table = static_cast<const char*>(out); s.row_bytes = row; }
    }
    int other_blocks = int((fetched + 127) / 128 / kSortThreads) + 1, zero_row0 = 0;
    const int most_blocks = device_sm_count() * 2;
    if (!sgd) {
        // whole rows from the end, of which the first starts on a 16-byte boundary (every eighth row does)
        const size_t rows = (beside - fetched) / row;
        if (rows < size_t(V)) zero_row0 = (V - int(rows)) / 8 * 8;
        const size_t bytes = size_t(V - zero_row0) * row;
        s.zero = reinterpret_cast<uint4*>(static_cast<char*>(out) + zero_row0 * row);
        s.zero16 = bytes / 16;
        s.zero_tail = reinterpret_cast<unsigned char*>(s.zero + s.zero16);
        s.zero_tail_bytes = int(bytes % 16);
        const size_t want = (s.zero16 + 4 * kSortThreads - 1) / (4 * kSortThreads) + 1;
        if (want > size_t(other_blocks)) other_blocks = int(want < size_t(most_blocks) ? want : size_t(most_blocks));
    }
    if (other_blocks > most_blocks) other_blocks = most_blocks;
    if (!rank) other_blocks = (other_blocks + s.ctas - 1) / s.ctas * s.ctas;     // (whole clusters)
    {
        LaunchScope scope(KID_EMBEDDING, 16.0 * double(N) * s.passes + (sgd ? 0.0 : double(V) * C * dtype_bytes(type)), st);
        const int rc = rank ? launch_chained(embedding_rank_kernel, dim3(s.ctas + other_blocks), dim3(kRankThreads), 0, st, 1, s)
                     : shared ? run_sort<true>(s, smem, s.ctas + other_blocks, st) : run_sort<false>(s, smem, s.ctas + other_blocks, st);
        if (rc != PCL_OK) return rc;
    }
    GradArgs g{};
    g.keys = (s.passes & 1) ? s.keys0 : s.keys1; g.idx = (s.passes & 1) ? s.idx0 : s.idx1; g.bounds = s.bounds;
    g.part = reinterpret_cast<float*>(base + l.part);
    g.long_count = s.long_count; g.long_items = reinterpret_cast<int*>(base + l.long_items);
    g.scale = scale; g.lr = lr; g.N = N; g.V = V; g.C = C; g.item_tokens = item_tokens(N); g.items = (N - 1) / g.item_tokens + 1; g.sgd = sgd;
    g.zero_rows = zero_row0;
    auto run = [&](auto zero) {
        using T = decltype(zero);
        if constexpr (sizeof(T) == 2)
            if (C % 8 == 0) return run_grad<T, 8>(g, dy, out, st);
        return C % 4 == 0 ? run_grad<T, 4>(g, dy, out, st) : C % 2 == 0 ? run_grad<T, 2>(g, dy, out, st) : run_grad<T, 1>(g, dy, out, st);
    };
    return type == DT_F32 ? run(float{}) : type == DT_BF16 ? run(__nv_bfloat16{}) : run(__half{});
}

}  // namespace pcl

// Embedding lookup with scaling and its gradient by sorted tokens.  Everything here is bound by memory: a row of the table
// or of dy is read once, a row of the output written once.
//
// Gradient: dtable[v] = scale * sum over tokens n with ids[n] = v of dy[n].  The tokens are sorted by id (stable, so equal
// ids stay in index order), then every 32 consecutive sorted tokens are one work item: segments that lie inside an item
// are summed and written directly, the two that may cross its borders leave partial sums that a second pass adds in
// order.  The work is even whatever the ids' frequencies are, and the additions have a fixed order (no atomics).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <limits.h>

#include "pcl_internal.h"
#include "pcl_ptx.cuh"

namespace pcl {

namespace {

constexpr int kItemTokens = 32;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = 32;
constexpr int kMaxSortCtas = 8;          // portable cluster size
constexpr int kMaxBins = 256;

template <class T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

template <class T, int kVec> struct alignas(sizeof(T) * kVec) Pack { T e[kVec]; };

// ids that name no row (outside [0, V)) and the padding id
__device__ __forceinline__ bool row_exists(int id, int V, int pad_id, unsigned int* status) {
    if (id == pad_id) return false;
    if (id < 0 || id >= V) {
        atomicCAS(status, 0u, static_cast<unsigned int>(kStatusBadLabel));
        return false;
    }
    return true;
}

template <class T, int kVec>
__global__ void __launch_bounds__(256) embedding_fwd_kernel(const int* __restrict__ ids, const T* __restrict__ table,
                                                            float scale, int pad_id, T* __restrict__ out, int N, int V, int C,
                                                            int tpr_log2, unsigned int* status) {
    const int tpr = 1 << tpr_log2;                   // threads per row
    const int vecs = C / kVec;
    const int lane = threadIdx.x & (tpr - 1);
    const long rows_per_pass = long(gridDim.x) * (256 >> tpr_log2);
    for (long n = long(blockIdx.x) * (256 >> tpr_log2) + (threadIdx.x >> tpr_log2); n < N; n += rows_per_pass) {
        const int id = ids[n];
        const bool there = row_exists(id, V, pad_id, status);
        const Pack<T, kVec>* src = reinterpret_cast<const Pack<T, kVec>*>(table + size_t(there ? id : 0) * C);
        Pack<T, kVec>* dst = reinterpret_cast<Pack<T, kVec>*>(out + size_t(n) * C);
        for (int i = lane; i < vecs; i += tpr) {
            Pack<T, kVec> v;
            if (there) {
                v = src[i];
#pragma unroll
                for (int j = 0; j < kVec; ++j) v.e[j] = from_f32<T>(scale * to_f32<T>(v.e[j]));
            } else {
#pragma unroll
                for (int j = 0; j < kVec; ++j) v.e[j] = from_f32<T>(0.f);
            }
            dst[i] = v;
        }
    }
}

// Stable radix sort of (id, token) by one cluster of CTAs.  Every warp owns a run of consecutive tokens; per pass it counts
// its digits, the counts are turned into positions (over digits, then CTAs, then warps, which keeps equal digits in
// token order), and the warp scatters its run in order.  Tokens without a row get the key V and end up last.
// Also leaves, per table row, the first sorted position of its tokens (-1: none).
struct SortArgs {
    const int* ids;
    int N, V, pad_id;
    int passes, bits;             // digits of `bits` bits, least significant first
    int per_warp;                 // tokens per warp, a multiple of 32
    int* keys[2];
    int* idx[2];
    int* totals;                  // [kMaxSortCtas][kMaxBins]
    int* head;                    // [V]
    unsigned int* status;
};
__device__ __forceinline__ void sort_barrier(bool cluster) {
    if (cluster) { __threadfence(); cluster_sync_all(); __threadfence(); }     // (also drops stale L1 lines)
    else __syncthreads();
}
__global__ void __launch_bounds__(kSortThreads) embedding_sort_kernel(SortArgs a, int ctas) {
    __shared__ int hist[kSortWarps][kMaxBins];
    __shared__ int base[kMaxBins];
    __shared__ int warp_sum[8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, cta = blockIdx.x;
    const bool cluster = ctas > 1;
    const long run0 = (long(cta) * kSortWarps + warp) * a.per_warp;
    const long run1 = run0 + a.per_warp < a.N ? run0 + a.per_warp : a.N;
    const int bins = 1 << a.bits;
    for (int v = cta * kSortThreads + threadIdx.x; v < a.V; v += ctas * kSortThreads) a.head[v] = -1;
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.bits;
        const int* src_key = a.keys[(pass & 1) ^ 1];
        const int* src_idx = a.idx[(pass & 1) ^ 1];
        int* dst_key = a.keys[pass & 1];
        int* dst_idx = a.idx[pass & 1];
        auto key_of = [&](long i) {
            if (pass > 0) return src_key[i];
            const int id = a.ids[i];
            return row_exists(id, a.V, a.pad_id, a.status) ? id : a.V;
        };
        for (int d = lane; d < bins; d += 32) hist[warp][d] = 0;
        __syncwarp();
        for (long i0 = run0; i0 < run1; i0 += 32) {
            const long i = i0 + lane;
            const bool in = i < run1;
            const unsigned act = __ballot_sync(0xffffffffu, in);
            if (in) {
                const int d = (key_of(i) >> shift) & (bins - 1);
                const unsigned same = __match_any_sync(act, d);
                if (lane == __ffs(same) - 1) hist[warp][d] += __popc(same);
            }
            __syncwarp();
        }
        __syncthreads();
        if (threadIdx.x < bins) {
            int run = 0;
            for (int w = 0; w < kSortWarps; ++w) { const int c = hist[w][threadIdx.x]; hist[w][threadIdx.x] = run; run += c; }
            a.totals[cta * kMaxBins + threadIdx.x] = run;
        }
        sort_barrier(cluster);
        if (threadIdx.x < kMaxBins) {
            const int d = threadIdx.x;
            int all = 0, before = 0;
            if (d < bins)
                for (int c = 0; c < ctas; ++c) {
                    const int v = *static_cast<volatile int*>(a.totals + c * kMaxBins + d);
                    if (c < cta) before += v;
                    all += v;
                }
            int inc = all;                               // inclusive scan over the digits
            for (int o = 1; o < 32; o <<= 1) { const int u = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += u; }
            if (lane == 31) warp_sum[warp] = inc;
            base[d] = inc - all + before;
        }
        __syncthreads();
        if (threadIdx.x < kMaxBins) {
            int off = 0;
            for (int w = 0; w < warp; ++w) off += warp_sum[w];
            base[threadIdx.x] += off;
        }
        __syncthreads();
        for (int d = lane; d < bins; d += 32) hist[warp][d] += base[d];
        __syncwarp();
        for (long i0 = run0; i0 < run1; i0 += 32) {
            const long i = i0 + lane;
            const bool in = i < run1;
            const unsigned act = __ballot_sync(0xffffffffu, in);
            if (in) {
                const int k = key_of(i), t = pass > 0 ? src_idx[i] : int(i);
                const int d = (k >> shift) & (bins - 1);
                const unsigned same = __match_any_sync(act, d);
                const int pos = hist[warp][d] + __popc(same & ((1u << lane) - 1u));
                __syncwarp(act);
                if (lane == __ffs(same) - 1) hist[warp][d] += __popc(same);
                dst_key[pos] = k;
                dst_idx[pos] = t;
            }
            __syncwarp();
        }
        sort_barrier(cluster);
    }
    const int* keys = a.keys[(a.passes - 1) & 1];
    for (long i = long(cta) * kSortThreads + threadIdx.x; i < a.N; i += long(ctas) * kSortThreads) {
        const int k = keys[i];
        if (k < a.V && (i == 0 || keys[i - 1] != k)) a.head[k] = int(i);
    }
}

struct GradArgs {
    const int* keys;              // sorted ids (V: no row)
    const int* idx;               // their tokens
    const int* head;              // [V]
    float* part;                  // [items][2][C]: sums of an item's first segment (begun before it) and of its last (goes on)
    float scale, lr;
    int N, V, C, items;
    int tpi_log2;                 // threads per item
    int item_blocks;              // blocks that take items; the others write the rows that do not occur
    int sgd;
};

template <class T, int kVec>
__device__ __forceinline__ void write_row(const GradArgs& a, T* out, int key, int i, const float (&sum)[kVec]) {
    Pack<T, kVec>* dst = reinterpret_cast<Pack<T, kVec>*>(out + size_t(key) * a.C) + i;
    Pack<T, kVec> o;
    if (a.sgd) {
        o = *dst;
#pragma unroll
        for (int j = 0; j < kVec; ++j) o.e[j] = from_f32<T>(fmaf(-a.lr, a.scale * sum[j], to_f32<T>(o.e[j])));
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) o.e[j] = from_f32<T>(a.scale * sum[j]);
    }
    *dst = o;
}

template <class T, int kVec>
__global__ void __launch_bounds__(256) embedding_grad_kernel(GradArgs a, const T* __restrict__ dy, T* __restrict__ out) {
    const int vecs = a.C / kVec;
    if (int(blockIdx.x) >= a.item_blocks) {          // rows that do not occur are zero: one warp per row
        const int warps = (gridDim.x - a.item_blocks) * 8, lane = threadIdx.x & 31;
        for (int v = (blockIdx.x - a.item_blocks) * 8 + (threadIdx.x >> 5); v < a.V; v += warps) {
            if (a.head[v] >= 0) continue;
            Pack<T, kVec> z;
#pragma unroll
            for (int j = 0; j < kVec; ++j) z.e[j] = from_f32<T>(0.f);
            Pack<T, kVec>* dst = reinterpret_cast<Pack<T, kVec>*>(out + size_t(v) * a.C);
            for (int i = lane; i < vecs; i += 32) dst[i] = z;
        }
        return;
    }
    const int tpi = 1 << a.tpi_log2, per_block = 256 >> a.tpi_log2;
    const int strips = (vecs + tpi - 1) >> a.tpi_log2;
    const long works = long(a.items) * strips;
    for (long wk = long(blockIdx.x) * per_block + (threadIdx.x >> a.tpi_log2); wk < works; wk += long(a.item_blocks) * per_block) {
        const int item = int(wk / strips);
        const int i = int(wk - long(item) * strips) * tpi + (threadIdx.x & (tpi - 1));
        if (i >= vecs) continue;
        const int p0 = item * kItemTokens;
        const int p1 = p0 + kItemTokens < a.N ? p0 + kItemTokens : a.N;
        int key = a.keys[p0];
        if (key >= a.V) continue;
        bool begun_before = p0 > 0 && a.keys[p0 - 1] == key;
        float sum[kVec];
#pragma unroll
        for (int j = 0; j < kVec; ++j) sum[j] = 0.f;
        for (int p = p0; p < p1; p += 4) {
            int k4[4];
            Pack<T, kVec> v4[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                k4[q] = p + q < p1 ? a.keys[p + q] : a.V;
                if (k4[q] < a.V) v4[q] = reinterpret_cast<const Pack<T, kVec>*>(dy + size_t(a.idx[p + q]) * a.C)[i];
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (k4[q] != key && key < a.V && p + q < p1) {          // the segment ends here
                    if (begun_before) {
#pragma unroll
                        for (int j = 0; j < kVec; ++j) a.part[(size_t(item) * 2) * a.C + size_t(i) * kVec + j] = sum[j];
                    } else {
                        write_row<T, kVec>(a, out, key, i, sum);
                    }
                    begun_before = false;
#pragma unroll
                    for (int j = 0; j < kVec; ++j) sum[j] = 0.f;
                    key = k4[q];
                }
                if (k4[q] < a.V)
#pragma unroll
                    for (int j = 0; j < kVec; ++j) sum[j] += to_f32<T>(v4[q].e[j]);
            }
        }
        if (key < a.V) {
            const bool goes_on = p1 < a.N && a.keys[p1] == key;
            if (begun_before || goes_on) {
                float* dst = a.part + (size_t(item) * 2 + (begun_before ? 0 : 1)) * a.C + size_t(i) * kVec;
#pragma unroll
                for (int j = 0; j < kVec; ++j) dst[j] = sum[j];
            } else {
                write_row<T, kVec>(a, out, key, i, sum);
            }
        }
    }
}

// Segments that cross items: the item in which one begins adds up the partial sums in order.
template <class T, int kVec>
__global__ void __launch_bounds__(256) embedding_grad_join_kernel(GradArgs a, T* __restrict__ out) {
    const int vecs = a.C / kVec;
    const int tpi = 1 << a.tpi_log2, per_block = 256 >> a.tpi_log2;
    const int strips = (vecs + tpi - 1) >> a.tpi_log2;
    const long works = long(a.items) * strips;
    for (long wk = long(blockIdx.x) * per_block + (threadIdx.x >> a.tpi_log2); wk < works; wk += long(gridDim.x) * per_block) {
        const int item = int(wk / strips);
        const int i = int(wk - long(item) * strips) * tpi + (threadIdx.x & (tpi - 1));
        const int p0 = item * kItemTokens, p1 = p0 + kItemTokens;
        if (i >= vecs || p1 >= a.N) continue;
        const int key = a.keys[p1 - 1];
        if (key >= a.V || a.keys[p1] != key) continue;                                   // does not go on
        if (a.keys[p0] == key && p0 > 0 && a.keys[p0 - 1] == key) continue;              // did not begin here
        float sum[kVec];
        const float* src = a.part + (size_t(item) * 2 + 1) * a.C + size_t(i) * kVec;
#pragma unroll
        for (int j = 0; j < kVec; ++j) sum[j] = src[j];
        for (int it = item + 1; it < a.items; ++it) {
            const float* f = a.part + size_t(it) * 2 * a.C + size_t(i) * kVec;
#pragma unroll
            for (int j = 0; j < kVec; ++j) sum[j] += f[j];
            const int e = (it + 1) * kItemTokens;
            if (e >= a.N || a.keys[e] != key) break;
        }
        write_row<T, kVec>(a, out, key, i, sum);
    }
}

int log2_threads(int vecs) {
    int l = 5;
    while (l < 8 && (1 << l) < vecs) ++l;
    return l;
}

struct BwdLayout { size_t keys[2], idx[2], totals, head, part, total; };
BwdLayout bwd_layout(int N, int V, int C) {
    BwdLayout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
    for (int i = 0; i < 2; ++i) { l.keys[i] = take(size_t(N) * 4); l.idx[i] = take(size_t(N) * 4); }
    l.totals = take(size_t(kMaxSortCtas) * kMaxBins * 4);
    l.head = take(size_t(V) * 4);
    l.part = take(size_t((N + kItemTokens - 1) / kItemTokens) * 2 * C * 4);
    l.total = at;
    return l;
}

template <class T, int kVec>
int run_fwd(int N, int V, int C, const int* ids, const void* table, float scale, int pad_id, void* out, unsigned int* status,
            cudaStream_t st) {
    const int tl = log2_threads(C / kVec);
    const long rows_per_block = 256 >> tl;
    const long blocks = (N + rows_per_block - 1) / rows_per_block, cap = long(device_sm_count()) * 8;
    LaunchScope scope(KID_EMBEDDING, 2.0 * sizeof(T) * double(N) * C, st);
    embedding_fwd_kernel<T, kVec><<<int(blocks < cap ? blocks : cap), 256, 0, st>>>(
        ids, static_cast<const T*>(table), scale, pad_id, static_cast<T*>(out), N, V, C, tl, status);
    return cudaGetLastError() == cudaSuccess ? PCL_OK : PCL_ERR_CUDA;
}

template <class T, int kVec>
int run_grad(GradArgs a, const void* dy, void* out, cudaStream_t st) {
    a.tpi_log2 = log2_threads(a.C / kVec);
    const int tpi = 1 << a.tpi_log2;
    const long strips = (a.C / kVec + tpi - 1) / tpi, works = long(a.items) * strips, per_block = 256 / tpi;
    const long cap = long(device_sm_count()) * 16;
    const long want = (works + per_block - 1) / per_block;
    a.item_blocks = int(want < cap ? want : cap);
    const int zero_blocks = a.sgd ? 0 : int((a.V + 7) / 8 < device_sm_count() * 8 ? (a.V + 7) / 8 : device_sm_count() * 8);
    {
        LaunchScope scope(KID_EMBEDDING, double(sizeof(T)) * a.C * (double(a.N) + a.V), st);
        embedding_grad_kernel<T, kVec><<<a.item_blocks + zero_blocks, 256, 0, st>>>(a, static_cast<const T*>(dy), static_cast<T*>(out));
    }
    if (cudaGetLastError() != cudaSuccess) return PCL_ERR_CUDA;
    if (a.items > 1) {
        LaunchScope scope(KID_EMBEDDING, 0.0, st);
        embedding_grad_join_kernel<T, kVec><<<a.item_blocks, 256, 0, st>>>(a, static_cast<T*>(out));
    }
    return cudaGetLastError() == cudaSuccess ? PCL_OK : PCL_ERR_CUDA;
}

}  // namespace

size_t embedding_workspace_bytes(int N, int V, int C) { return bwd_layout(N, V, C).total; }

int launch_embedding_fwd(int N, int V, int C, int type, const int* ids, const void* table, float scale, int pad_id, void* out,
                         cudaStream_t st) {
    unsigned int* status = device_status_ptr();
    if (!status) return PCL_ERR_CUDA;
    if (type == DT_F32)
        return C % 4 == 0 ? run_fwd<float, 4>(N, V, C, ids, table, scale, pad_id, out, status, st)
                          : run_fwd<float, 1>(N, V, C, ids, table, scale, pad_id, out, status, st);
    if (type == DT_BF16)
        return C % 8 == 0 ? run_fwd<__nv_bfloat16, 8>(N, V, C, ids, table, scale, pad_id, out, status, st)
                          : run_fwd<__nv_bfloat16, 1>(N, V, C, ids, table, scale, pad_id, out, status, st);
    return C % 8 == 0 ? run_fwd<__half, 8>(N, V, C, ids, table, scale, pad_id, out, status, st)
                      : run_fwd<__half, 1>(N, V, C, ids, table, scale, pad_id, out, status, st);
}

int launch_embedding_bwd(int N, int V, int C, int type, const int* ids, const void* dy, float scale, int pad_id, void* out,
                         bool sgd, float lr, void* ws, cudaStream_t st) {
    unsigned int* status = device_status_ptr();
    if (!status) return PCL_ERR_CUDA;
    const BwdLayout l = bwd_layout(N, V, C);
    char* base = static_cast<char*>(ws);
    SortArgs s{};
    s.ids = ids; s.N = N; s.V = V; s.pad_id = pad_id; s.status = status;
    int key_bits = 1;
    while (key_bits < 31 && (long(V) >> key_bits) != 0) ++key_bits;          // keys 0 .. V
    s.passes = (key_bits + 7) / 8;
    s.bits = (key_bits + s.passes - 1) / s.passes;
    int ctas = 1;
    while (ctas < kMaxSortCtas && long(ctas) * kSortThreads * 4 < N) ctas *= 2;
    const long per_warp = (N + long(ctas) * kSortWarps - 1) / (long(ctas) * kSortWarps);
    s.per_warp = int((per_warp + 31) / 32 * 32);
    for (int i = 0; i < 2; ++i) {
        s.keys[i] = reinterpret_cast<int*>(base + l.keys[i]);
        s.idx[i] = reinterpret_cast<int*>(base + l.idx[i]);
    }
    s.totals = reinterpret_cast<int*>(base + l.totals);
    s.head = reinterpret_cast<int*>(base + l.head);
    {
        LaunchScope scope(KID_EMBEDDING, 16.0 * double(N) * s.passes, st);
        cudaLaunchConfig_t lc = {};
        lc.gridDim = dim3(ctas);
        lc.blockDim = dim3(kSortThreads);
        lc.stream = st;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim = {unsigned(ctas), 1u, 1u};
        lc.attrs = attr;
        lc.numAttrs = 1;
        if (cudaLaunchKernelEx(&lc, embedding_sort_kernel, s, ctas) != cudaSuccess) return PCL_ERR_CUDA;
    }
    GradArgs g{};
    g.keys = s.keys[(s.passes - 1) & 1]; g.idx = s.idx[(s.passes - 1) & 1]; g.head = s.head;
    g.part = reinterpret_cast<float*>(base + l.part);
    g.scale = scale; g.lr = lr; g.N = N; g.V = V; g.C = C; g.items = (N + kItemTokens - 1) / kItemTokens; g.sgd = sgd;
    if (type == DT_F32)
        return C % 4 == 0 ? run_grad<float, 4>(g, dy, out, st) : run_grad<float, 1>(g, dy, out, st);
    if (type == DT_BF16)
        return C % 8 == 0 ? run_grad<__nv_bfloat16, 8>(g, dy, out, st) : run_grad<__nv_bfloat16, 1>(g, dy, out, st);
    return C % 8 == 0 ? run_grad<__half, 8>(g, dy, out, st) : run_grad<__half, 1>(g, dy, out, st);
}

}  // namespace pcl

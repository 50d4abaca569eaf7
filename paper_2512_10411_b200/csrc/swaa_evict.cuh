// Eviction from a key/value cache by accumulated attention weight.
//
// App. A: FA decode has to retain the cache of the whole context; where that outgrows memory, the entries that gathered
// little attention can go (sinks and recent entries stay, as in the trimmed cache of a pure-SWA layer).  For every (sequence, kv
// head) of len > budget entries: the first n_sink and the last `recent` entries stay, and of those between the
// budget - n_sink - recent with the largest weights, the lower index first among equals.  The survivors keep their order, so that the
// first entries are still the sinks and the last ones still the recent ones.
//
// Two kernels.  select: one cluster per (sequence, kv head) finds the weight of the last survivor by three counting passes over 11, 11
// and 10 bits of the weights' order-preserving integer form, held in shared memory (one read of the weights), and lists the survivors
// in order.  gather: copies their rows of K and V, 16 bytes a lane, eight rows of each in flight per warp.  The order of
// every step is fixed: the result does not depend on scheduling.
//
// What bounds it: the copy.  Rows of one head are 2 D bytes, Hkv of them from places of their own make one row of the new cache.
#pragma once

#include <cooperative_groups.h>

#include "swaa_internal.cuh"
#include "swaa_ptx.cuh"

namespace swaa {

struct EvictParams {
    const __nv_bfloat16 *k, *v;
    const float* weights;          // [B, Hkv, weights_rows]
    const int32_t *seqlens, *block_table, *block_table_out;  // tables null: dense
    int B, rows /* Lmax, or max_blocks * page_size */, weights_rows, Hkv;
    int max_blocks, num_pages, page_size;
    int budget, n_sink, recent;
    __nv_bfloat16 *k_out, *v_out;
    int rows_out, weights_out_rows, max_blocks_out, num_pages_out, page_size_out;
    float* weights_out;            // [B, Hkv, weights_out_rows]
    int32_t *kept, *seqlens_out;   // [B, Hkv, budget], [B]
    int cap;                       // keys of a block that shared memory holds
};

constexpr int kEvictThreads = 1024;
constexpr int kEvictWarps = kEvictThreads / 32;
constexpr int kEvictBins = 2048;
constexpr int kEvictMaxCluster = 8;
constexpr int kEvictPerThread = 4;  // neighbouring keys of a thread in the listing pass
constexpr int kEvictTile = kEvictThreads * kEvictPerThread;

// Integers in the order of the weights: -0 and 0 are equal, NaN is above everything.
__device__ __forceinline__ uint32_t evict_key(float w) {
    if (w != w) return 0xffffffffu;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u ^ ((u >> 31) != 0u ? 0xffffffffu : 0x80000000u);
}

// Inclusive sum over the block's threads; sm: kEvictWarps words.  Every thread calls it.
__device__ __forceinline__ uint32_t evict_scan(uint32_t x, uint32_t* sm, uint32_t* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) sm[warp] = x;
    __syncthreads();
    uint32_t w = sm[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += y;
    }
    *total = __shfl_sync(0xffffffffu, w, 31);
    if (warp > 0) x += __shfl_sync(0xffffffffu, w, warp - 1);
    __syncthreads();
    return x;
}

__global__ void __launch_bounds__(kEvictThreads, 1) evict_select_kernel(const EvictParams p) {
    namespace cg = cooperative_groups;
    extern __shared__ uint32_t sm_keys[];
    __shared__ uint32_t hist[3][kEvictBins];
    __shared__ uint32_t sm_scan[32], sm_gt, sm_eq, sm_bin, sm_above;
    static_assert(kEvictWarps == 32, "one word per lane in evict_scan");
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, row = (int)(blockIdx.x / (unsigned)ranks);
    const int b = row / p.Hkv;
    grid_wait();
    const int n = p.seqlens[b];
    const bool bad = n < 0 || n > p.rows || n > p.weights_rows;
    if (bad && tid == 0) record_device_error(SWAA_ERR_BAD_SEQLENS);
    const int left = bad ? 0 : n < p.budget ? n : p.budget;
    if (row == b * p.Hkv && rank == 0 && tid == 0) p.seqlens_out[b] = left;
    if (left == 0) return;  // the whole cluster
    const float* w = p.weights + (size_t)row * p.weights_rows;
    int32_t* kept = p.kept + (size_t)row * p.budget;
    float* w_out = p.weights_out + (size_t)row * p.weights_out_rows;
    if (n <= p.budget) {  // all stay
        for (int j = rank * kEvictThreads + tid; j < n; j += ranks * kEvictThreads) {
            kept[j] = j;
            w_out[j] = w[j];
        }
        return;
    }
    const int m = p.budget - p.n_sink - p.recent;       // to keep of the entries [n_sink, n - recent), fewer than those
    const int candidates = n - p.recent - p.n_sink;
    for (int j = rank * kEvictThreads + tid; j < p.n_sink + p.recent; j += ranks * kEvictThreads) {
        const int from = j < p.n_sink ? j : n - p.recent + (j - p.n_sink), to = j < p.n_sink ? j : m + j;
        kept[to] = from;
        w_out[to] = w[from];
    }
    if (m == 0) return;
    // this block's share of the candidates, a multiple of kEvictPerThread each
    const int share = ((candidates + ranks - 1) / ranks + kEvictPerThread - 1) / kEvictPerThread * kEvictPerThread;
    const int c0 = min(rank * share, candidates), cn = min(share, candidates - c0);
    const float* wc = w + p.n_sink + c0;
    auto key = [&](int i) -> uint32_t { return i < p.cap ? sm_keys[i] : evict_key(wc[i]); };
    for (int i = tid; i < 3 * kEvictBins; i += kEvictThreads) (&hist[0][0])[i] = 0u;
    __syncthreads();
    for (int i = tid; i < cn; i += kEvictThreads) {  // the first pass reads the weights
        const uint32_t k = evict_key(wc[i]);
        if (i < p.cap) sm_keys[i] = k;
        atomicAdd(&hist[0][k >> 21], 1u);
    }
    // digits of the last survivor's key, from the top; `need` survivors share the digits found so far
    uint32_t prefix = 0, need = (uint32_t)m;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        if (pass > 0) {
            for (int i = tid; i < cn; i += kEvictThreads) {
                const uint32_t k = key(i);
                if ((k >> (shift + bits)) == prefix) atomicAdd(&hist[pass][(k >> shift) & ((1u << bits) - 1u)], 1u);
            }
        }
        if (ranks > 1) cluster.sync();
        else __syncthreads();
        // thread t: bins kEvictBins - 1 - 2 t and the one below it, so that the running sum counts from the top
        uint32_t c[2] = {0u, 0u};
        const int top = kEvictBins - 1 - 2 * tid;
        for (int r = 0; r < ranks; ++r) {
            const uint32_t* h = ranks > 1 ? cluster.map_shared_rank(&hist[pass][0], r) : &hist[pass][0];
            c[0] += h[top];
            c[1] += h[top - 1];
        }
        uint32_t total;
        const uint32_t upto = evict_scan(c[0] + c[1], sm_scan, &total), before = upto - c[0] - c[1];
        if (before < need && need <= upto) {  // one thread
            const bool first = need <= before + c[0];
            sm_bin = (uint32_t)(first ? top : top - 1);
            sm_above = first ? before : before + c[0];
        }
        __syncthreads();
        prefix = (prefix << bits) | sm_bin;
        need -= sm_above;
        __syncthreads();
    }
    // `prefix` is the key; survivors are all above it and the first `need` equal to it.  Where does this block's list start?
    uint32_t gt0 = 0, eq0 = 0;
    if (ranks > 1) {
        uint32_t gt = 0, eq = 0;
        for (int i = tid; i < cn; i += kEvictThreads) {
            const uint32_t k = key(i);
            gt += k > prefix;
            eq += k == prefix;
        }
        uint32_t total_gt, total_eq;
        evict_scan(gt, sm_scan, &total_gt);
        evict_scan(eq, sm_scan, &total_eq);
        if (tid == 0) {
            sm_gt = total_gt;
            sm_eq = total_eq;
        }
        cluster.sync();
        for (int r = 0; r < rank; ++r) {
            gt0 += *cluster.map_shared_rank(&sm_gt, r);
            eq0 += *cluster.map_shared_rank(&sm_eq, r);
        }
    }
    for (int base = 0; base < cn; base += kEvictTile) {
        const int i0 = base + kEvictPerThread * tid;
        uint32_t k[kEvictPerThread], gt = 0, eq = 0;
#pragma unroll
        for (int e = 0; e < kEvictPerThread; ++e) {
            k[e] = i0 + e < cn ? key(i0 + e) : 0u;
            gt += i0 + e < cn && k[e] > prefix;
            eq += i0 + e < cn && k[e] == prefix;
        }
        uint32_t total;
        const uint32_t before = evict_scan(gt << 16 | eq, sm_scan, &total) - (gt << 16 | eq);  // a tile has at most 4096 of each
        uint32_t g = gt0 + (before >> 16), q = eq0 + (before & 0xffffu);
#pragma unroll
        for (int e = 0; e < kEvictPerThread; ++e) {
            if (i0 + e >= cn) continue;
            const bool above = k[e] > prefix, equal = k[e] == prefix;
            if (above || (equal && q < need)) {
                const int to = p.n_sink + (int)(g + min(q, need));
                kept[to] = p.n_sink + c0 + i0 + e;
                w_out[to] = wc[i0 + e];
            }
            g += above;
            q += equal;
        }
        gt0 += total >> 16;
        eq0 += total & 0xffffu;
    }
    if (ranks > 1) cluster.sync();  // no block leaves while another reads its counts
}

constexpr int kGatherThreads = 256;
constexpr int kGatherRows = 4;  // rows of K and of V per lane

template <int D>
__global__ void __launch_bounds__(kGatherThreads) evict_gather_kernel(const EvictParams p) {
    constexpr int kLanes = D / 8, kPerWarp = 32 / kLanes;
    grid_wait();
    const int b = (int)blockIdx.y, n = p.seqlens[b];
    if (n < 0 || n > p.rows || n > p.weights_rows) return;  // reported by the selection
    const long long items = (long long)min(n, p.budget) * p.Hkv;
    const int lane = threadIdx.x & 31, l = lane % kLanes;
    // items (entry, kv head), heads first: the lanes of a warp write one stretch of the new cache
    const long long i0 = ((long long)blockIdx.x * (kGatherThreads / 32) + (threadIdx.x >> 5)) * (kPerWarp * kGatherRows) + lane / kLanes;
    uint4 kx[kGatherRows], vx[kGatherRows];
    long long to[kGatherRows];
#pragma unroll
    for (int u = 0; u < kGatherRows; ++u) {
        const long long i = i0 + u * kPerWarp;
        to[u] = -1;
        if (i >= items) continue;
        const int e = (int)(i / p.Hkv), h = (int)(i - (long long)e * p.Hkv);
        const int j = p.kept[((size_t)b * p.Hkv + h) * p.budget + e];
        long long from, dst;
        if (p.block_table == nullptr) {
            from = (long long)b * p.rows + j;
            dst = (long long)b * p.rows_out + e;
        } else {
            const int page = p.block_table[(size_t)b * p.max_blocks + j / p.page_size];
            const int page_out = p.block_table_out[(size_t)b * p.max_blocks_out + e / p.page_size_out];
            if (page < 0 || page >= p.num_pages || page_out < 0 || page_out >= p.num_pages_out) {
                record_device_error(SWAA_ERR_BAD_SEQLENS);
                continue;
            }
            from = (long long)page * p.page_size + j % p.page_size;
            dst = (long long)page_out * p.page_size_out + e % p.page_size_out;
        }
        const long long at = (from * p.Hkv + h) * D + 8 * l;
        to[u] = (dst * p.Hkv + h) * D + 8 * l;
        kx[u] = *reinterpret_cast<const uint4*>(p.k + at);
        vx[u] = *reinterpret_cast<const uint4*>(p.v + at);
    }
#pragma unroll
    for (int u = 0; u < kGatherRows; ++u) {
        if (to[u] < 0) continue;
        *reinterpret_cast<uint4*>(p.k_out + to[u]) = kx[u];
        *reinterpret_cast<uint4*>(p.v_out + to[u]) = vx[u];
    }
}

}  // namespace swaa

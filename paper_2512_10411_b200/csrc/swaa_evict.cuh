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
// 16 caches of 32768 entries, 8 heads of 128, to 4096: 26 us of selection and 95 of copying (537 MB); one of 20011 entries, 4 heads of 64, to
// 2048: 18 us in all, most of it the chain of passes.
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
// A row is cut over up to four blocks while each keeps 8192 weights.  One row of 8 heads, us with one, two, four and eight blocks: 32768
// weights 27.4, 23.7, 22.8, -; 65536 -, 31.2, 27.0, 31.9; 131072 -, -, 33.4, 35.2 (an exchange between blocks takes about 1.5 us of a pass).
constexpr int kEvictMaxCluster = 4;
constexpr int kEvictShare = 8192;
constexpr int kEvictBatch = 16;     // weights of a thread on their way at a time

// Integers in the order of the weights: -0 and 0 are equal, NaN is above everything.
__device__ __forceinline__ uint32_t evict_key(float w) {
    if (w != w) return 0xffffffffu;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u ^ ((u >> 31) != 0u ? 0xffffffffu : 0x80000000u);
}

// The weight of a key, but for zeros and NaN, of which there are several.
__device__ __forceinline__ bool evict_key_is_one(uint32_t k) { return k != 0x80000000u && k != 0xffffffffu; }
__device__ __forceinline__ float evict_weight(uint32_t k) { return __uint_as_float((k >> 31) != 0u ? k ^ 0x80000000u : ~k); }

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
    extern __shared__ __align__(16) uint32_t sm_keys[];
    __shared__ uint32_t hist[3][kEvictBins];
    __shared__ uint32_t sm_scan[32], sm_gt, sm_eq, sm_bin, sm_above;
    __shared__ uint2 sm_count[kEvictWarps];
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
    const int share = (candidates + ranks - 1) / ranks;  // of the candidates, this block's
    const int c0 = min(rank * share, candidates), cn = min(share, candidates - c0);
    const float* wc = w + p.n_sink + c0;
    auto key = [&](int i) -> uint32_t { return i < p.cap ? sm_keys[i] : evict_key(wc[i]); };
    for (int i = tid; i < 3 * kEvictBins; i += kEvictThreads) (&hist[0][0])[i] = 0u;
    __syncthreads();
    for (int i0 = tid; i0 < cn; i0 += kEvictBatch * kEvictThreads) {  // the first pass reads the weights, several on their way at a time
        float x[kEvictBatch];
#pragma unroll
        for (int u = 0; u < kEvictBatch; ++u) x[u] = i0 + u * kEvictThreads < cn ? wc[i0 + u * kEvictThreads] : 0.f;
#pragma unroll
        for (int u = 0; u < kEvictBatch; ++u) {
            const int i = i0 + u * kEvictThreads;
            if (i >= cn) break;
            const uint32_t k = evict_key(x[u]);
            if (i < p.cap) sm_keys[i] = k;
            atomicAdd(&hist[0][k >> 21], 1u);
        }
    }
    // digits of the last survivor's key, from the top; `need` survivors share the digits found so far
    uint32_t prefix = 0, need = (uint32_t)m;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        if (pass > 0) {
            auto count = [&](uint32_t k) {
                if ((k >> (shift + bits)) == prefix) atomicAdd(&hist[pass][(k >> shift) & ((1u << bits) - 1u)], 1u);
            };
            const int held = min(cn, p.cap) / 4;  // four keys at a time from shared memory, then the rest
            for (int i = tid; i < held; i += kEvictThreads) {
                const uint4 k = reinterpret_cast<const uint4*>(sm_keys)[i];
                count(k.x);
                count(k.y);
                count(k.z);
                count(k.w);
            }
            for (int i = 4 * held + tid; i < cn; i += kEvictThreads) count(key(i));
        }
        if (ranks > 1) cluster.sync();
        else __syncthreads();
        // thread t: bins kEvictBins - 1 - 2 t and the one below it, so that the running sum counts from the top
        uint32_t c[2] = {0u, 0u};
        const int top = kEvictBins - 1 - 2 * tid;
        if (ranks == 1) {
            c[0] = hist[pass][top];
            c[1] = hist[pass][top - 1];
        } else {
            uint32_t x[2 * kEvictMaxCluster];
#pragma unroll
            for (int r = 0; r < kEvictMaxCluster; ++r) {
                const uint32_t* h = cluster.map_shared_rank(&hist[pass][0], r < ranks ? r : 0);
                x[2 * r] = r < ranks ? h[top] : 0u;
                x[2 * r + 1] = r < ranks ? h[top - 1] : 0u;
            }
#pragma unroll
            for (int r = 0; r < kEvictMaxCluster; ++r) {
                c[0] += x[2 * r];
                c[1] += x[2 * r + 1];
            }
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
    // `prefix` is the key; survivors are all above it and the first `need` equal to it.  A warp lists a stretch of the share, 32 keys
    // at a time; how many there are before it is counted first.
    const int lane = tid & 31, warp = tid >> 5;
    const int stretch = ((cn + kEvictWarps - 1) / kEvictWarps + 127) / 128 * 128, i0 = min(warp * stretch, cn), i1 = min(i0 + stretch, cn);
    uint32_t gt = 0, eq = 0;
    auto tell = [&](uint32_t k) {
        gt += k > prefix;
        eq += k == prefix;
    };
    const int held = max(min(i1, p.cap) - i0, 0) / 4;
    for (int i = lane; i < held; i += 32) {
        const uint4 k = reinterpret_cast<const uint4*>(sm_keys + i0)[i];
        tell(k.x);
        tell(k.y);
        tell(k.z);
        tell(k.w);
    }
    for (int i = i0 + 4 * held + lane; i < i1; i += 32) tell(key(i));
    gt = __reduce_add_sync(0xffffffffu, gt);
    eq = __reduce_add_sync(0xffffffffu, eq);
    if (lane == 0) sm_count[warp] = make_uint2(gt, eq);
    __syncthreads();
    const uint2 theirs = sm_count[lane];
    uint32_t before_gt = lane < warp ? theirs.x : 0u, before_eq = lane < warp ? theirs.y : 0u, all_gt = theirs.x, all_eq = theirs.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        before_gt += __shfl_xor_sync(0xffffffffu, before_gt, o);
        before_eq += __shfl_xor_sync(0xffffffffu, before_eq, o);
        all_gt += __shfl_xor_sync(0xffffffffu, all_gt, o);
        all_eq += __shfl_xor_sync(0xffffffffu, all_eq, o);
    }
    if (ranks > 1) {
        if (tid == 0) {
            sm_gt = all_gt;
            sm_eq = all_eq;
        }
        cluster.sync();
        for (int r = 0; r < rank; ++r) {
            before_gt += *cluster.map_shared_rank(&sm_gt, r);
            before_eq += *cluster.map_shared_rank(&sm_eq, r);
        }
    }
    const unsigned below = (1u << lane) - 1u;
#pragma unroll 4
    for (int i = i0; i < i1; i += 32) {
        const uint32_t k = i + lane < i1 ? key(i + lane) : 0u;
        const bool above = i + lane < i1 && k > prefix, equal = i + lane < i1 && k == prefix;
        const unsigned gts = __ballot_sync(0xffffffffu, above), eqs = __ballot_sync(0xffffffffu, equal);
        const uint32_t q = before_eq + __popc(eqs & below);
        if (above || (equal && q < need)) {
            const int to = p.n_sink + (int)(before_gt + __popc(gts & below) + min(q, need));
            kept[to] = p.n_sink + c0 + i + lane;
            w_out[to] = evict_key_is_one(k) ? evict_weight(k) : wc[i + lane];
        }
        before_gt += __popc(gts);
        before_eq += __popc(eqs);
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

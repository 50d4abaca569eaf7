// Attention weight that the entries of a key/value cache gather, per kv head (summed over the query heads of its group), as
// the eviction of swaa_evict.cuh wants it.
//
// Decode step.  decode_kernel computes every score once, on its way to the output; its kScores instance also stores them (4 bytes per
// query head and entry next to the 4 D bytes of an entry's K and V) and the logarithm of each row's sum.  The kernel here then forms
//     weights_out[b, g, j] = weights_in[b, g, j] + sum over heads h of g of 2^(score_hj * sl2 - lse2_h)
// one thread per entry.  A second pass over K instead would move 2 D bytes an entry.  The entry of the new token itself starts from 0.
// Bound by memory: 16 sequences of 65536 entries, 32 heads, 8 key heads of 128: 659 us with the scores stored, then 40 (201 MB).
//
// Prompt.  With the log-sum-exp rows of the attention (lse of the prefill calls),
//     weights_out[b, g, j] = weights_in[b, g, j] + sum over the queries i and heads h of g that see j of exp(scale q_ih . k_j - lse_ih)
// One block owns 128 keys of one (sequence, kv head) and walks the 128-query tiles that see them, for every head of the group:
//     S^T = K Q^T [128 keys x 128 queries], tcgen05.mma, accumulators in tensor memory
// so that a key is a tensor-memory lane and the sum over queries stays in its thread.  Two groups of four warps take the steps in
// turn; the log-sum-exps of a step's columns come by cp.async.  A tile seen by more than 16 query tiles (fewer in small calls, more in
// long ones, so that the sums of all chunks take 32 KB per SM at most) is cut into chunks for blocks of their own (every tile under full
// attention, the sinks under a window); the chunks' sums are added in order by a second kernel, so results do not depend on scheduling.  Where few queries count (the last ones of a prompt) a step takes 64 queries
// of two heads, in groups of an even number of them, and a block several tiles of keys one after another.
//
// What bounds it: shared memory and the exponentials, one per visible pair.  A step of 128 x 128 moves through shared memory the operands of its
// products (512 cycles at D = 128), its queries (256) and four readings of the log-sum-exps (128), and takes 1024 cycles of
// the SM's special-function units; it lasts about 1300.  32k tokens, 32 heads of 128, 8 key heads, window 2048: 715 us, 820 called back to back (1000 W,
// 1.78 GHz); full causal 16k 1385; the last 64 queries of eight prompts of 145610 tokens in all 130.  64-column steps: 883 and 220 us; a
// polynomial for an eighth to a half of the exponentials 883 to 995; 256 keys a block, which halves the queries' arrivals, 780 and 132.
#pragma once

#include "swaa_backward_tc.cuh"
#include "swaa_decode.cuh"
#include "swaa_internal.cuh"
#include "swaa_ptx.cuh"

namespace swaa {

struct DecodeWeightsParams {
    const float *scores, *lse2;
    const float* weights_in;  // null: zeros; may be weights_out
    float* weights_out;       // [B, Hkv, weights_rows]
    const int32_t* seqlens;
    int Lmax, weights_rows, Hq, Hkv, G, score_rows, score_heads;
    int window, n_sink, is_full, paged;
    float sl2;
};

constexpr int kDecodeWeightsThreads = 256;
constexpr int kDecodeWeightsKeys = 4;  // per thread

__global__ void __launch_bounds__(kDecodeWeightsThreads) decode_weights_kernel(const DecodeWeightsParams p) {
    extern __shared__ float sm_lse[];  // [G]
    grid_wait();
    const int b = (int)blockIdx.z, hk = (int)blockIdx.y;
    const SeqGeom s = decode_seq_geom(p.seqlens[b], p.Lmax, p.window, p.n_sink, p.is_full, p.paged != 0);  // len 0: out of range, reported by the decode kernel
    const int j0 = (int)blockIdx.x * (kDecodeWeightsThreads * kDecodeWeightsKeys);
    if (s.len > p.weights_rows) {
        if (threadIdx.x == 0) record_device_error(SWAA_ERR_BAD_SEQLENS);
        return;
    }
    if (j0 >= s.len) return;
    for (int h = threadIdx.x; h < p.G; h += kDecodeWeightsThreads) sm_lse[h] = p.lse2[(size_t)b * p.Hq + hk * p.G + h];
    __syncthreads();
    const size_t row = (size_t)b * p.Hkv + hk;
    const float* in = p.weights_in != nullptr ? p.weights_in + row * p.weights_rows : nullptr;
    float* out = p.weights_out + row * p.weights_rows;
#pragma unroll
    for (int u = 0; u < kDecodeWeightsKeys; ++u) {
        const int j = j0 + u * kDecodeWeightsThreads + (int)threadIdx.x;
        if (j >= s.len) continue;
        const bool seen = j >= s.wb || j < s.se;
        if (!seen && in == out) continue;  // stays as it is
        float sum = in != nullptr && j < s.len - 1 ? in[j] : 0.f;
        if (seen) {
            const int at = j >= s.wb ? s.nst * kDecodeTileKeys + (j - s.w0) : j;
            const float* x = p.scores + (row * p.score_rows + at) * p.score_heads;
            float got = 0.f;
            for (int h = 0; h < p.G; ++h) got += ex2f(fmaf(x[h], p.sl2, -sm_lse[h]));
            sum += got;
        }
        out[j] = sum;
    }
}

// ------------------------------------------------------------------------------------------- prompt
struct KeyWeightsParams {
    const float* lse;             // [Hq, Tq]
    const float* weights_in;      // null: zeros; may be weights_out
    float* weights_out;           // [B, Hkv, weights_rows]
    const int32_t *cu_q, *cu_k;   // cu_k null: paged
    const int32_t *seqlens_k, *block_table;
    int max_blocks, page_size, num_pages;
    int B, Tq, Tk, max_q, max_k, weights_rows, Hq, Hkv, G;
    int window, n_sink, is_full, last;
    float sl2;
    // chunks: [chunks][B][Hkv][128 key_tiles] sums of all tiles, [sink_chunks][B][Hkv][128 sink_tiles] of the tiles that hold sinks
    int key_tiles, chunks, sink_tiles, sink_chunks;
    int run;                      // key tiles of a block, one after another; above 1 nothing is cut into chunks
    int chunk_log;                // a tile seen by more than 2^chunk_log query tiles is cut
    int heads_per_step;           // 2: a step takes 64 queries of two heads (at most 64 queries of a sequence count)
    float *part, *sink_part;
};

constexpr int kKeyWeightsKeys = 128;
constexpr int kKeyWeightsRows = 128;   // columns of a step: queries, or queries of two heads in turn
constexpr int kKeyWeightsChunkLog = 4;  // log2 of the query tiles of a block, less in small calls
constexpr int kKeyWeightsThreads = 320;  // two groups of four warps, producer, issuer
constexpr int kKeyWeightsSumSteps = 512;  // steps of a key tile, a power of two, after which the two groups start new sums
constexpr int kKeyWeightsPartTiles = 64;  // key tiles per SM, each chunk counted, whose sums the chunks of a call may take
constexpr int kKeyWeightsRunSteps = 16;  // steps below which a block takes more key tiles
constexpr int kKeyWeightsLse = 4;      // steps whose log-sum-exps are in shared memory

// One sequence of a call, checked against what the call says of it.
struct KeyWeightsSeq {
    bool ok;
    int q0, len_q, k0, len_k;  // first packed query and key, lengths
    int nq, pos0;              // queries that count (the last ones) and the position of the first
};
__device__ __forceinline__ KeyWeightsSeq key_weights_seq(const KeyWeightsParams& p, int b) {
    KeyWeightsSeq s;
    s.q0 = p.cu_q[b];
    const int q1 = p.cu_q[b + 1];
    s.k0 = p.cu_k != nullptr ? p.cu_k[b] : 0;
    const long long len_q = (long long)q1 - s.q0, len_k = p.cu_k != nullptr ? (long long)p.cu_k[b + 1] - s.k0 : p.seqlens_k[b];
    s.ok = s.q0 >= 0 && q1 <= p.Tq && len_q >= 0 && len_q <= len_k && len_q <= p.max_q && len_k <= p.max_k && len_k <= p.weights_rows &&
           (p.cu_k != nullptr ? s.k0 >= 0 && (long long)s.k0 + len_k <= p.Tk : len_k <= (long long)p.max_blocks * p.page_size);
    s.len_q = (int)len_q;
    s.len_k = (int)len_k;
    s.nq = p.last > 0 && p.last < s.len_q ? p.last : s.len_q;
    s.pos0 = s.len_k - s.nq;
    return s;
}
// Query tiles [lo, hi] (128 rows from pos0 on) that see a key of the tile at j0, and their chunks; none: hi < lo, 0 chunks.
struct KeyWeightsSpan {
    int lo, hi, chunks;
};
__device__ __forceinline__ KeyWeightsSpan key_weights_span(const KeyWeightsParams& p, const KeyWeightsSeq& s, int j0) {
    KeyWeightsSpan t;
    const int tiles = (s.nq + kKeyWeightsRows - 1) / kKeyWeightsRows;
    t.lo = j0 > s.pos0 ? (j0 - s.pos0) / kKeyWeightsRows : 0;
    t.hi = tiles - 1;
    if (!p.is_full && j0 >= p.n_sink) {
        const long long end = (long long)j0 + kKeyWeightsKeys - 1 + p.window - 1 - s.pos0;  // last query, from pos0, that sees the tile's last key
        t.hi = end < 0 ? -1 : (int)(end / kKeyWeightsRows < t.hi ? end / kKeyWeightsRows : t.hi);
    }
    t.chunks = t.hi < t.lo ? 0 : ((t.hi - t.lo) >> p.chunk_log) + 1;
    return t;
}
// The page of a key tile; the pages are multiples of the tile.  -1: not a page of the pool.
__device__ __forceinline__ int key_weights_page(const KeyWeightsParams& p, int b, int j0) {
    const int page = p.block_table[(size_t)b * p.max_blocks + j0 / p.page_size];
    return page >= 0 && page < p.num_pages ? page : -1;
}
__device__ __forceinline__ float key_weights_old(const KeyWeightsParams& p, const KeyWeightsSeq& s, size_t row, int j) {
    return p.weights_in != nullptr && j < s.len_k - s.len_q ? p.weights_in[row * p.weights_rows + j] : 0.f;  // the call's own tokens start from 0
}

template <int D>
struct KeyWeightsSmem {
    static constexpr int kPanels = D / 64;
    static constexpr int kStages = D == 128 ? 2 : 4;  // two blocks per SM at either size
    static constexpr int kPanelBytes = 128 * 128;     // 128 rows of 64 channels
    static constexpr int kTileBytes = kPanels * kPanelBytes;
    static constexpr int kOffRing = kTileBytes;       // K first
    static constexpr int kOffLse = kOffRing + kStages * kTileBytes;
    static constexpr int kOffSum = kOffLse + kKeyWeightsLse * kKeyWeightsRows * 4;
    static constexpr int kOffFar = kOffSum + 2 * kKeyWeightsKeys * 4;
    static constexpr int kOffBar = kOffFar + 2 * kKeyWeightsKeys * 4;
    static constexpr int kNumBars = 2 + 2 * kStages + 2 * kKeyWeightsLse + 4 + 1;
    static constexpr int kOffMisc = kOffBar + kNumBars * 8;
    static constexpr int kBytes = kOffMisc + 16;
    static_assert(2 * (kBytes + 1024) <= 228 * 1024, "two blocks per SM");
};

// 4 bytes from global to shared memory, zero where the source does not count.
__device__ __forceinline__ void cp_async_4(uint32_t dst, const float* src, bool on) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(on ? 4 : 0) : "memory");
}
// An arrival on `bar` when the thread's copies so far have landed.
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

// Keeps the uses of 16 registers that an asynchronous tensor-memory load fills behind the wait for it.
__device__ __forceinline__ void pin16(uint32_t* r) {
#pragma unroll
    for (int i = 0; i < 16; ++i) asm volatile("" : "+r"(r[i]));
}

template <int D>
__global__ void __launch_bounds__(kKeyWeightsThreads, 2)
key_weights_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const KeyWeightsParams p) {
    using L = KeyWeightsSmem<D>;
    constexpr int BK = kKeyWeightsKeys, BR = kKeyWeightsRows, NQ = L::kStages, NL = kKeyWeightsLse;
    constexpr uint32_t kIdS = make_idesc(BK, BR, 0);
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t smem_base = smem_u32(smem_raw);
    if ((smem_base & 1023u) != 0u) {  // the swizzled tiles need it; uniform, before any barrier or allocation
        if (threadIdx.x == 0) record_device_error(SWAA_ERR_CUDA);
        return;
    }
    float* s_lse = reinterpret_cast<float*>(smem_raw + L::kOffLse);
    float* s_sum = reinterpret_cast<float*>(smem_raw + L::kOffSum);
    float* far = reinterpret_cast<float*>(smem_raw + L::kOffFar);  // a word of each thread that sums (a register would spill)
    const uint32_t sK = smem_base, sRing = smem_base + L::kOffRing, bars = smem_base + L::kOffBar;
    auto bar = [&](int i) -> uint32_t { return bars + 8u * (uint32_t)i; };
    constexpr int BAR_KF = 0, BAR_KE = 1, BAR_QF = 2, BAR_QE = BAR_QF + NQ, BAR_LF = BAR_QE + NQ, BAR_LE = BAR_LF + NL, BAR_SF = BAR_LE + NL;
    constexpr int BAR_SE = BAR_SF + 2, BAR_FIN = BAR_SE + 2;
    static_assert(BAR_FIN + 1 == L::kNumBars, "barrier count");
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_raw + L::kOffMisc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    grid_wait();
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int b = (int)blockIdx.x / p.Hkv, hk = (int)blockIdx.x - b * p.Hkv;
    // blocks start in the order of their index, x first: the tiles that hold sinks, then all tiles from the first key on
    int slot = (int)(blockIdx.z * gridDim.y + blockIdx.y), tile0, chunk;
    const bool sinks = slot < p.sink_tiles * p.sink_chunks;
    if (sinks) {
        tile0 = slot / p.sink_chunks;
        chunk = slot - tile0 * p.sink_chunks;
    } else {
        slot -= p.sink_tiles * p.sink_chunks;
        tile0 = slot / p.chunks;
        chunk = slot - tile0 * p.chunks;
        tile0 *= p.run;
        if (tile0 < p.sink_tiles || tile0 >= p.key_tiles) return;
    }
    const KeyWeightsSeq s = key_weights_seq(p, b);
    if (!s.ok) {
        if (threadIdx.x == 0 && chunk == 0) record_device_error(SWAA_ERR_BAD_SEQLENS);
        return;
    }
    if (tile0 * BK >= s.len_k) return;
    const int tile1 = min(tile0 + (sinks ? 1 : p.run), (s.len_k + BK - 1) / BK);
    const size_t row = (size_t)b * p.Hkv + hk;

    // One tile of the run: the query tiles m_lo .. m_lo + nm - 1 that this block takes, for every group of heads_per_step heads.
    const int hs = p.heads_per_step, shift = hs - 1, head_steps = p.G / hs;
    struct Tile {
        int m_lo, nm, page;
        KeyWeightsSpan span;
    };
    auto tile_of = [&](int t) {
        Tile x;
        x.span = key_weights_span(p, s, t * BK);
        x.m_lo = x.nm = x.page = 0;
        if (x.span.chunks == 1 && chunk == 0) {
            x.m_lo = x.span.lo;
            x.nm = x.span.hi - x.span.lo + 1;
        } else if (chunk < x.span.chunks) {  // an even share of the span
            const int n = x.span.hi - x.span.lo + 1, share = (n + x.span.chunks - 1) / x.span.chunks;
            x.m_lo = x.span.lo + chunk * share;
            x.nm = max(min(x.span.hi, x.m_lo + share - 1) - x.m_lo + 1, 0);
        }
        // (keys that no query sees need no page: what lies before the windows of a long sequence may have been given up)
        if (p.cu_k == nullptr && x.nm > 0 && (x.page = key_weights_page(p, b, t * BK)) < 0) x.nm = 0;
        return x;
    };
    // What the block found out for key j of tile t: the whole sum, or that of its chunk.
    auto store = [&](const Tile& x, int j, float total) {
        if (j >= s.len_k) return;
        if (x.page < 0) {
            record_device_error(SWAA_ERR_BAD_SEQLENS);
        } else if (x.span.chunks <= 1) {
            if (chunk == 0) p.weights_out[row * p.weights_rows + j] = key_weights_old(p, s, row, j) + total;
        } else if (chunk < x.span.chunks) {
            if (sinks) p.sink_part[((size_t)chunk * p.B * p.Hkv + row) * (p.sink_tiles * BK) + j] = total;
            else p.part[((size_t)chunk * p.B * p.Hkv + row) * ((size_t)p.key_tiles * BK) + j] = total;
        }
    };
    bool any = false;  // uniform
    for (int t = tile0; t < tile1; ++t) any = any || tile_of(t).nm > 0;
    if (!any) {  // no query of the block sees a key of it
        for (int t = tile0; t < tile1; ++t)
            if ((int)threadIdx.x < BK) store(tile_of(t), t * BK + (int)threadIdx.x, 0.f);
        return;
    }

    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int i = 0; i < L::kNumBars; ++i) {
            uint32_t count = 1u;
            if (i >= BAR_LF && i < BAR_LF + NL) count = 32u;  // the lanes that copy
            if ((i >= BAR_LE && i < BAR_LE + NL) || (i >= BAR_SE && i < BAR_SE + 2)) count = 4u;  // the warps of a group
            mbar_init(bar(i), count);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(256u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    static_assert(2 * BR == 256, "tensor memory columns");
    bool ok = true;

    if (warp == 8) {
        // ================================================================================= producer
        const int first = s.q0 + s.len_q - s.nq;  // packed row of the query at pos0
        int tiles = 0, loads = 0, steps = 0;      // so far
        for (int t = tile0; t < tile1 && ok; ++t) {
            const Tile x = tile_of(t);
            if (x.nm == 0) continue;
            if (tiles > 0) ok = warp_wait(bar(BAR_KE), (uint32_t)(tiles - 1) & 1u, abort_flag);
            if (!ok) break;
            ++tiles;
            if (lane == 0) {
                mbar_arrive_expect_tx(bar(BAR_KF), (uint32_t)L::kTileBytes);
#pragma unroll
                for (int pn = 0; pn < L::kPanels; ++pn) {
                    if (p.cu_k != nullptr) tma_load_3d(sK + pn * L::kPanelBytes, &tm_k, pn * 64, hk, s.k0 + t * BK, bar(BAR_KF));
                    else tma_load_4d(sK + pn * L::kPanelBytes, &tm_k, pn * 64, hk, t * BK % p.page_size, x.page, bar(BAR_KF));
                }
            }
            for (int h = 0; h < head_steps && ok; ++h)
                for (int m = 0; m < x.nm; ++m) {
                    const int head = hk * p.G + h * hs, i0 = (x.m_lo + m) * BR;  // from pos0
                    const int st = steps % NQ;
                    if (steps >= NQ) ok = warp_wait(bar(BAR_QE + st), (uint32_t)(steps / NQ - 1) & 1u, abort_flag);
                    if (!ok) break;
                    if (lane == 0) {
                        mbar_arrive_expect_tx(bar(BAR_QF + st), (uint32_t)L::kTileBytes);
#pragma unroll
                        for (int pn = 0; pn < L::kPanels; ++pn)
                            tma_load_3d(sRing + (uint32_t)(st * L::kTileBytes + pn * L::kPanelBytes), &tm_q, pn * 64, head, first + i0, bar(BAR_QF + st));
                    }
                    ++loads;
                    const int sl = steps % NL;
                    if (steps >= NL) ok = warp_wait(bar(BAR_LE + sl), (uint32_t)(steps / NL - 1) & 1u, abort_flag);
                    if (!ok) break;
#pragma unroll
                    for (int e = 0; e < BR / 32; ++e) {
                        const int c = lane + 32 * e, r = i0 + (c >> shift);
                        const bool on = r < s.nq;
                        cp_async_4(smem_u32(s_lse + sl * BR + c), p.lse + (size_t)(head + (c & shift)) * p.Tq + first + (on ? r : 0), on);
                    }
                    cp_async_arrive(bar(BAR_LF + sl));
                    ++steps;
                }
        }
        if (!ok) {  // give outstanding copies a bounded chance to land before the block's memory is released
            asm volatile("cp.async.wait_all;" ::: "memory");
            const uint64_t t0 = global_timer_ns();
            bool landed = false;
            while (!landed && global_timer_ns() - t0 < kWaitLimitNs) {
                landed = tiles == 0 || mbar_try_wait(bar(BAR_KF), (uint32_t)(tiles - 1) & 1u);
                for (int n = max(0, loads - NQ); n < loads; ++n) landed = landed && mbar_try_wait(bar(BAR_QF + n % NQ), (uint32_t)(n / NQ) & 1u);
            }
        }
        __syncwarp();
    } else if (warp == 9) {
        // =================================================================================== issuer
        const bool el = elect_one();
        const uint32_t hi = (uint32_t)(smem_desc_sw128(0, 0, 1024) >> 32);
        const uint32_t k_a = (uint32_t)smem_desc_sw128(sK, 16, 1024), q_b = (uint32_t)smem_desc_sw128(sRing, 16, 1024);
        int tiles = 0, n = 0;  // n: steps so far
        for (int t = tile0; t < tile1 && ok; ++t) {
            const Tile x = tile_of(t);
            const int n_steps = x.nm * head_steps;
            if (n_steps == 0) continue;
            ok = warp_wait(bar(BAR_KF), (uint32_t)tiles & 1u, abort_flag);
            ++tiles;
            for (int i = 0; i < n_steps && ok; ++i, ++n) {
                const int st = n % NQ, buf = n & 1;
                ok = warp_wait(bar(BAR_QF + st), (uint32_t)(n / NQ) & 1u, abort_flag) &&
                     warp_wait(bar(BAR_SE + buf), ((uint32_t)(n >> 1) & 1u) ^ 1u, abort_flag);  // the buffers start out free
                if (!ok) break;
                tc_fence_after();
                if (el) {
                    const uint32_t d = tmem_base + (uint32_t)(BR * buf), q = q_b + (((uint32_t)st * L::kTileBytes) >> 4);
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint32_t o = ((uint32_t)(kk >> 2) * L::kPanelBytes + (uint32_t)(kk & 3) * 32u) >> 4;
                        mma_ss_lh(d, k_a + o, q + o, hi, kIdS, kk > 0 ? 1u : 0u);
                    }
                    tc_commit(bar(BAR_SF + buf));
                    tc_commit(bar(BAR_QE + st));
                    if (i == n_steps - 1) tc_commit(bar(BAR_KE));
                }
            }
        }
        // all products issued by this warp must have retired before the tensor memory is freed
        if (el) tc_commit(bar(BAR_FIN));
        warp_wait(bar(BAR_FIN), 0u, abort_flag);
        __syncwarp();
    } else {
        // =============================================================================== exponentials
        // Group n & 1 takes step n of the block; the groups' sums of a tile meet in the warps of the first.
        const int grp = warp >> 2, quad = warp & 3, kl = 32 * quad + lane;
        const bool full = p.is_full != 0;
        const uint32_t tS = tmem_base + ((uint32_t)(32 * quad) << 16) + (uint32_t)(BR * grp);
        const uint64_t sl2x2 = pack_f32x2(p.sl2, p.sl2), nlog2e = pack_f32x2(-1.4426950408889634f, -1.4426950408889634f);
        int base = 0;  // steps of the tiles before
        for (int t = tile0; t < tile1; ++t) {
            const Tile x = tile_of(t);
            const int j0 = t * BK, jw = j0 + 32 * quad, j = j0 + kl, n_steps = x.nm * head_steps;
            const int vis_hi = (full || j < p.n_sink) ? s.len_k : (int)min((long long)s.len_k, (long long)j + p.window);
            float total = 0.f;
            const int first = (base ^ grp) & 1;  // step of this group, then every other one
            int m = first;
            for (int i = first; i < n_steps && ok; i += 2) {
                const int n = base + i, sl = n % NL;
                while (m >= x.nm) m -= x.nm;
                const int i0 = s.pos0 + (x.m_lo + m) * BR;  // position of the first query
                m += 2;
                ok = warp_wait(bar(BAR_LF + sl), (uint32_t)(n / NL) & 1u, abort_flag) && warp_wait(bar(BAR_SF + grp), (uint32_t)(n >> 1) & 1u, abort_flag);
                if (!ok) break;
                tc_fence_after();
                const int i1 = i0 + ((BR - 1) >> shift);
                const bool edge = i1 >= s.len_k || tile_needs_mask(i0, i1, j0, j0 + BK - 1, p.window, p.n_sink, full);
                uint64_t sum[2] = {0ull, 0ull};
                const float* lse = s_lse + sl * BR;
                // 32 columns from c0 on, whose scores are in sv
                auto columns = [&](auto mask_tag, auto count_tag, int c0, const uint32_t* sv) {
                    constexpr bool kMask = decltype(mask_tag)::value;
                    constexpr int kCount = decltype(count_tag)::value;
                    const int r_lo = min(max(j - i0, 0), BR) * hs - c0, r_hi = min(max(vis_hi - i0, 0), BR) * hs - c0;  // visible ones
#pragma unroll
                    for (int e = 0; e < kCount; e += 4) {
                        const float4 l4 = *reinterpret_cast<const float4*>(lse + c0 + e);
#pragma unroll
                        for (int u = 0; u < 4; u += 2) {
                            uint64_t c;
                            asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(c) : "l"(u ? pack_f32x2(l4.z, l4.w) : pack_f32x2(l4.x, l4.y)), "l"(nlog2e));
                            const uint64_t v = fma_f32x2(pack_f32x2(__uint_as_float(sv[e + u]), __uint_as_float(sv[e + u + 1])), sl2x2, c);
                            float x0, x1;
                            unpack_f32x2(v, x0, x1);
                            x0 = ex2f(x0);
                            x1 = ex2f(x1);
                            if (kMask) {
                                x0 = e + u >= r_lo && e + u < r_hi ? x0 : 0.f;
                                x1 = e + u + 1 >= r_lo && e + u + 1 < r_hi ? x1 : 0.f;
                            }
                            sum[u >> 1] = add_f32x2(sum[u >> 1], pack_f32x2(x0, x1));
                        }
                    }
                };
                auto release = [&] {  // the products of the group's next step may overwrite the scores
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(BAR_SE + grp));
                    __syncwarp();
                };
                if (!edge) {  // the next columns on their way while the exponentials of these are taken
                    using N = std::integral_constant<int, 16>;
                    uint32_t sa[16], sb[16];
                    tmem_ld16(tS, sa);
                    tc_wait_ld();
                    pin16(sa);
#pragma unroll
                    for (int c0 = 0; c0 < BR; c0 += 32) {
                        tmem_ld16(tS + (uint32_t)(c0 + 16), sb);
                        columns(std::false_type{}, N{}, c0, sa);
                        tc_wait_ld();
                        pin16(sb);
                        if (c0 + 32 < BR) tmem_ld16(tS + (uint32_t)(c0 + 32), sa);
                        else release();
                        columns(std::false_type{}, N{}, c0 + 16, sb);
                        if (c0 + 32 < BR) {
                            tc_wait_ld();
                            pin16(sa);
                        }
                    }
                } else {
                    using N = std::integral_constant<int, 32>;
#pragma unroll 1
                    for (int c0 = 0; c0 < BR; c0 += 32) {
                        const int ia = i0 + (c0 >> shift), ib = i0 + ((c0 + 31) >> shift);
                        // the warp's 32 keys and these queries: nothing visible, nothing hidden, or both
                        if (ib < jw || ia >= s.len_k || !(full || jw < p.n_sink || (long long)ia < (long long)jw + 31 + p.window)) continue;
                        uint32_t sv[32];
                        tmem_ld32(tS + (uint32_t)c0, sv);
                        tc_wait_ld();
                        if (ib < s.len_k && !tile_needs_mask(ia, ib, jw, jw + 31, p.window, p.n_sink, full)) columns(std::false_type{}, N{}, c0, sv);
                        else columns(std::true_type{}, N{}, c0, sv);
                    }
                    release();
                }
                float a, c, d, e;
                unpack_f32x2(sum[0], a, c);
                unpack_f32x2(sum[1], d, e);
                total += (a + c) + (d + e);  // a step's terms at a time, so that long sums keep their bits
                if ((i & (kKeyWeightsSumSteps - 1)) >= kKeyWeightsSumSteps - 2) {  // half of that is the group's: a sum of sums in long chunks
                    far[threadIdx.x] = (i < kKeyWeightsSumSteps ? 0.f : far[threadIdx.x]) + total;
                    total = 0.f;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(BAR_LE + sl));
                __syncwarp();
            }
            base += n_steps;
            if (((kKeyWeightsSumSteps - 2) | first) < n_steps) total += far[threadIdx.x];
            // The two warps that hold the same keys meet here, whatever their waits gave.  (The first group reads its buffer before it
            // gets to the next meeting, the second writes it again after that one.)
            float* meet = s_sum + (t & 1) * BK;
            if (grp == 1) meet[kl] = total;
            __syncwarp();
            asm volatile("bar.sync %0, 64;" ::"r"(1 + quad) : "memory");
            if (grp == 0 && *abort_flag == 0) store(x, j, total + meet[kl]);
            __syncwarp();
        }
    }

    // ---- every thread arrives here (also after a failed wait)
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(256u) : "memory");
    }
}

// Sums of the chunks, in their order, of the keys whose tile was cut.
__global__ void __launch_bounds__(kKeyWeightsKeys) key_weights_join_kernel(const KeyWeightsParams p) {
    grid_wait();
    const int b = (int)blockIdx.x / p.Hkv, hk = (int)blockIdx.x - b * p.Hkv;
    const int tile = (int)(blockIdx.z * gridDim.y + blockIdx.y), j0 = tile * kKeyWeightsKeys, j = j0 + (int)threadIdx.x;
    if (tile >= p.key_tiles) return;
    const KeyWeightsSeq s = key_weights_seq(p, b);
    if (!s.ok || j >= s.len_k) return;
    const KeyWeightsSpan span = key_weights_span(p, s, j0);
    if (span.chunks < 2 || (p.cu_k == nullptr && key_weights_page(p, b, j0) < 0)) return;
    const size_t row = (size_t)b * p.Hkv + hk, rows = (size_t)p.B * p.Hkv;
    const bool sinks = tile < p.sink_tiles;
    const size_t keys = (size_t)(sinks ? p.sink_tiles : p.key_tiles) * kKeyWeightsKeys;
    const float* part = (sinks ? p.sink_part : p.part) + row * keys + j;
    float sum = 0.f;
    for (int c = 0; c < span.chunks; ++c) sum += part[(size_t)c * rows * keys];
    p.weights_out[row * p.weights_rows + j] = key_weights_old(p, s, row, j) + sum;
}

}  // namespace swaa

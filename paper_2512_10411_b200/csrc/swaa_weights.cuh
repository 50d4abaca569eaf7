// Attention weight that the entries of a key/value cache gather, per kv head (summed over the query heads of its group), as
// the eviction of swaa_evict.cuh wants it.
//
// Decode step.  decode_kernel computes every score once, on its way to the output; its kScores instance also stores them (4 bytes per
// query head and entry next to the 4 D bytes of an entry's K and V) and the logarithm of each row's sum.  The kernel here then forms
//     weights_out[b, g, j] = weights_in[b, g, j] + sum over heads h of g of 2^(score_hj * sl2 - lse2_h)
// one thread per entry.  A second pass over K instead would move 2 D bytes an entry.  The entry of the new token itself starts from 0.
//
// Prompt.  With the log-sum-exp rows of the attention (lse of the prefill calls),
//     weights_out[b, g, j] = weights_in[b, g, j] + sum over the queries i and heads h of g that see j of exp(scale q_ih . k_j - lse_ih)
// One block owns 128 keys of one (sequence, kv head) and walks the 64-query tiles that see them, for every head of the group:
//     S^T = K Q^T [128 keys x 64 queries], tcgen05.mma, accumulators in tensor memory
// so that a key is a tensor-memory lane and the sum over queries stays in its thread.  Two groups of four warps take the steps in
// turn, four of them in flight; the log-sum-exps of a step's rows come with its queries (cp.async).  A tile seen by more than kKeyWeightsChunk
// query tiles is cut into chunks for blocks of their own (every tile under full attention, the sinks under a window); the chunks'
// sums are added in order by a second kernel, so results do not depend on scheduling.
//
// What bounds it: the exponentials, one per visible pair: 64 x 128 of them take 512 cycles of an SM's special-function units, the
// products of a step at D = 128 256 cycles of its tensor cores.
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
    float *part, *sink_part;
};

constexpr int kKeyWeightsKeys = 128;
constexpr int kKeyWeightsRows = 64;    // queries of a step
constexpr int kKeyWeightsChunk = 32;   // query tiles of a block
constexpr int kKeyWeightsThreads = 320;  // two groups of four warps, producer, issuer
constexpr int kKeyWeightsBuffers = 4;  // S^T in tensor memory; half of it per block, two blocks per SM

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
// Query tiles [lo, hi] (64 rows from pos0 on) that see a key of the tile at j0, and their chunks; none: hi < lo, 0 chunks.
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
    t.chunks = t.hi < t.lo ? 0 : (t.hi - t.lo + kKeyWeightsChunk) / kKeyWeightsChunk;
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
    static constexpr int kStages = D == 128 ? 4 : 8;  // two blocks per SM at either size
    static constexpr int kKPanelBytes = kKeyWeightsKeys * 128, kKBytes = kPanels * kKPanelBytes;
    static constexpr int kQPanelBytes = kKeyWeightsRows * 128, kQBytes = kPanels * kQPanelBytes;
    static constexpr int kOffRing = kKBytes;
    static constexpr int kOffLse = kOffRing + kStages * kQBytes;
    static constexpr int kOffSum = kOffLse + kStages * kKeyWeightsRows * 4;
    static constexpr int kOffBar = kOffSum + kKeyWeightsKeys * 4;
    static constexpr int kNumBars = 1 + 2 * kStages + 2 * kKeyWeightsBuffers + 1;
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

template <int D>
__global__ void __launch_bounds__(kKeyWeightsThreads, 2)
key_weights_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const KeyWeightsParams p) {
    using L = KeyWeightsSmem<D>;
    constexpr int BK = kKeyWeightsKeys, BR = kKeyWeightsRows, NQ = L::kStages, NB = kKeyWeightsBuffers;
    constexpr uint32_t kIdS = make_idesc(BK, BR, 0);
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t smem_base = smem_u32(smem_raw);
    if ((smem_base & 1023u) != 0u) {  // the swizzled tiles need it; uniform, before any barrier or allocation
        if (threadIdx.x == 0) record_device_error(SWAA_ERR_CUDA);
        return;
    }
    float* s_lse = reinterpret_cast<float*>(smem_raw + L::kOffLse);
    float* s_sum = reinterpret_cast<float*>(smem_raw + L::kOffSum);
    const uint32_t sK = smem_base, sRing = smem_base + L::kOffRing, bars = smem_base + L::kOffBar;
    auto bar = [&](int i) -> uint32_t { return bars + 8u * (uint32_t)i; };
    constexpr int BAR_K = 0, BAR_QF = 1, BAR_QE = BAR_QF + NQ, BAR_SF = BAR_QE + NQ, BAR_SE = BAR_SF + NB, BAR_FIN = BAR_SE + NB;
    static_assert(BAR_FIN + 1 == L::kNumBars, "barrier count");
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_raw + L::kOffMisc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    grid_wait();
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int b = (int)blockIdx.x / p.Hkv, hk = (int)blockIdx.x - b * p.Hkv;
    // blocks start in the order of their index, x first: the tiles that hold sinks, then all tiles from the first key on
    int slot = (int)(blockIdx.z * gridDim.y + blockIdx.y), tile, chunk;
    const bool sinks = slot < p.sink_tiles * p.sink_chunks;
    if (sinks) {
        tile = slot / p.sink_chunks;
        chunk = slot - tile * p.sink_chunks;
    } else {
        slot -= p.sink_tiles * p.sink_chunks;
        tile = slot / p.chunks;
        chunk = slot - tile * p.chunks;
        if (tile < p.sink_tiles || tile >= p.key_tiles) return;
    }
    const KeyWeightsSeq s = key_weights_seq(p, b);
    const int j0 = tile * BK;
    if (!s.ok) {
        if (threadIdx.x == 0 && chunk == 0) record_device_error(SWAA_ERR_BAD_SEQLENS);
        return;
    }
    if (j0 >= s.len_k) return;
    const KeyWeightsSpan span = key_weights_span(p, s, j0);
    const size_t row = (size_t)b * p.Hkv + hk;
    if (span.chunks == 0) {  // no query of the call sees the tile
        const int j = j0 + (int)threadIdx.x;
        if (chunk == 0 && (int)threadIdx.x < BK && j < s.len_k) p.weights_out[row * p.weights_rows + j] = key_weights_old(p, s, row, j);
        return;
    }
    if (chunk >= span.chunks) return;
    int page = 0;
    if (p.cu_k == nullptr && (page = key_weights_page(p, b, j0)) < 0) {
        if (threadIdx.x == 0) record_device_error(SWAA_ERR_BAD_SEQLENS);
        return;
    }
    // an even share of the span's tiles
    const int span_tiles = span.hi - span.lo + 1, share = (span_tiles + span.chunks - 1) / span.chunks;
    const int m_lo = span.lo + chunk * share, m_hi = min(span.hi, m_lo + share - 1);
    const int nm = max(m_hi - m_lo + 1, 0), n_steps = nm * p.G;

    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int i = 0; i < L::kNumBars; ++i) {
            uint32_t count = 1u;
            if (i >= BAR_QF && i < BAR_QF + NQ) count = 33u;  // the copy of the queries, and 32 lanes with the log-sum-exps
            if (i >= BAR_QE && i < BAR_QE + NQ) count = 5u;   // the products, and four warps that have read the log-sum-exps
            if (i >= BAR_SE && i < BAR_SE + NB) count = 4u;   // four warps that have read S^T
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
    static_assert(NB * BR == 256, "tensor memory columns");
    bool ok = true;
    float total = 0.f;

    if (warp == 8) {
        // ================================================================================= producer
        if (lane == 0) {
            mbar_arrive_expect_tx(bar(BAR_K), (uint32_t)L::kKBytes);
#pragma unroll
            for (int pn = 0; pn < L::kPanels; ++pn) {
                if (p.cu_k != nullptr) tma_load_3d(sK + pn * L::kKPanelBytes, &tm_k, pn * 64, hk, s.k0 + j0, bar(BAR_K));
                else tma_load_4d(sK + pn * L::kKPanelBytes, &tm_k, pn * 64, hk, j0 % p.page_size, page, bar(BAR_K));
            }
        }
        const int first = s.q0 + s.len_q - s.nq;  // packed row of the query at pos0
        int issued = 0;
        for (int st = 0, n = 0, h = 0, m = 0; n < n_steps; ++n) {
            if (n >= NQ) ok = mbar_wait(bar(BAR_QE + st), (uint32_t)(n / NQ - 1) & 1u, abort_flag);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const int head = hk * p.G + h, i0 = (m_lo + m) * BR;  // from pos0
            if (lane == 0) {
                mbar_arrive_expect_tx(bar(BAR_QF + st), (uint32_t)L::kQBytes);
#pragma unroll
                for (int pn = 0; pn < L::kPanels; ++pn)
                    tma_load_3d(sRing + (uint32_t)(st * L::kQBytes + pn * L::kQPanelBytes), &tm_q, pn * 64, head, first + i0, bar(BAR_QF + st));
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = lane + 32 * e;
                const bool on = i0 + r < s.nq;
                cp_async_4(smem_u32(s_lse + st * BR + r), p.lse + (size_t)head * p.Tq + first + (on ? i0 + r : 0), on);
            }
            cp_async_arrive(bar(BAR_QF + st));
            issued = n + 1;
            if (++m == nm) {
                m = 0;
                ++h;
            }
            if (++st == NQ) st = 0;
        }
        if (!ok) {  // give outstanding copies a bounded chance to land before the block's memory is released
            asm volatile("cp.async.wait_all;" ::: "memory");
            const uint64_t t0 = global_timer_ns();
            bool landed = false;
            while (!landed && global_timer_ns() - t0 < kWaitLimitNs) {
                landed = mbar_try_wait(bar(BAR_K), 0u);
                for (int n = max(0, issued - NQ); n < issued; ++n) landed = landed && mbar_try_wait(bar(BAR_QF + n % NQ), (uint32_t)(n / NQ) & 1u);
            }
        }
        __syncwarp();
    } else if (warp == 9) {
        // =================================================================================== issuer
        const bool el = elect_one();
        const uint32_t hi = (uint32_t)(smem_desc_sw128(0, 0, 1024) >> 32);
        const uint32_t k_a = (uint32_t)smem_desc_sw128(sK, 16, 1024), q_b = (uint32_t)smem_desc_sw128(sRing, 16, 1024);
        ok = warp_wait(bar(BAR_K), 0u, abort_flag);
        int st = 0, buf = 0;
        uint32_t st_ph = 0, buf_ph = 1;  // the buffers start out free
        for (int n = 0; n < n_steps && ok; ++n) {
            ok = warp_wait(bar(BAR_QF + st), st_ph, abort_flag) && warp_wait(bar(BAR_SE + buf), buf_ph, abort_flag);
            if (!ok) break;
            tc_fence_after();
            if (el) {
                const uint32_t d = tmem_base + (uint32_t)(BR * buf), q = q_b + (((uint32_t)st * L::kQBytes) >> 4);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    const uint32_t oa = ((uint32_t)(kk >> 2) * L::kKPanelBytes + (uint32_t)(kk & 3) * 32u) >> 4;
                    const uint32_t ob = ((uint32_t)(kk >> 2) * L::kQPanelBytes + (uint32_t)(kk & 3) * 32u) >> 4;
                    mma_ss_lh(d, k_a + oa, q + ob, hi, kIdS, kk > 0 ? 1u : 0u);
                }
                tc_commit(bar(BAR_SF + buf));
                tc_commit(bar(BAR_QE + st));
            }
            if (++st == NQ) {
                st = 0;
                st_ph ^= 1u;
            }
            if (++buf == NB) {
                buf = 0;
                buf_ph ^= 1u;
            }
        }
        // all products issued by this warp must have retired before the tensor memory is freed
        if (el) tc_commit(bar(BAR_FIN));
        warp_wait(bar(BAR_FIN), 0u, abort_flag);
        __syncwarp();
    } else {
        // =============================================================================== exponentials
        const int grp = warp >> 2, quad = warp & 3, kl = 32 * quad + lane;
        const int j = j0 + kl;
        const bool full = p.is_full != 0;
        const int vis_hi = (full || j < p.n_sink) ? s.len_k : (int)min((long long)s.len_k, (long long)j + p.window);
        const uint64_t sl2x2 = pack_f32x2(p.sl2, p.sl2), nlog2e = pack_f32x2(-1.4426950408889634f, -1.4426950408889634f);
        for (int n = grp; n < n_steps; n += 2) {
            const int st = n % NQ, buf = n % NB, i0 = s.pos0 + (m_lo + n % nm) * BR;  // position of the tile's first query
            ok = warp_wait(bar(BAR_QF + st), (uint32_t)(n / NQ) & 1u, abort_flag) && warp_wait(bar(BAR_SF + buf), (uint32_t)(n / NB) & 1u, abort_flag);
            if (!ok) break;
            tc_fence_after();
            const bool need_mask = i0 + BR > s.len_k || tile_needs_mask(i0, i0 + BR - 1, j0, j0 + BK - 1, p.window, p.n_sink, full);
            uint64_t sum[2] = {0ull, 0ull};
            auto half = [&](auto mask_tag, int c0) {
                constexpr bool kMask = decltype(mask_tag)::value;
                uint32_t sv[32];
                tmem_ld32(tmem_base + ((uint32_t)(32 * quad) << 16) + (uint32_t)(BR * buf + c0), sv);
                tc_wait_ld();
                const float* lse = s_lse + st * BR + c0;
                const int r_lo = j - i0 - c0, r_hi = vis_hi - i0 - c0;  // visible queries of this half
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                    const float4 l4 = *reinterpret_cast<const float4*>(lse + e);
#pragma unroll
                    for (int u = 0; u < 4; u += 2) {
                        uint64_t c;
                        asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(c) : "l"(u ? pack_f32x2(l4.z, l4.w) : pack_f32x2(l4.x, l4.y)), "l"(nlog2e));
                        const uint64_t x = fma_f32x2(pack_f32x2(__uint_as_float(sv[e + u]), __uint_as_float(sv[e + u + 1])), sl2x2, c);
                        float x0, x1;
                        unpack_f32x2(x, x0, x1);
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
            if (need_mask) {
                half(std::true_type{}, 0);
                half(std::true_type{}, 32);
            } else {
                half(std::false_type{}, 0);
                half(std::false_type{}, 32);
            }
            float a, c, d, e;
            unpack_f32x2(sum[0], a, c);
            unpack_f32x2(sum[1], d, e);
            total += (a + c) + (d + e);  // 64 terms at a time, so that long sums keep their bits
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(bar(BAR_SE + buf));
                mbar_arrive(bar(BAR_QE + st));
            }
            __syncwarp();
        }
        if (grp == 1) s_sum[kl] = total;
    }

    // ---- every thread arrives here (also after a failed wait)
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(256u) : "memory");
    } else if (warp < 4 && *abort_flag == 0) {
        const int kl = (int)threadIdx.x, j = j0 + kl;
        if (j < s.len_k) {
            total += s_sum[kl];
            if (span.chunks == 1) p.weights_out[row * p.weights_rows + j] = key_weights_old(p, s, row, j) + total;
            else if (sinks) p.sink_part[((size_t)chunk * p.B * p.Hkv + row) * (p.sink_tiles * BK) + j] = total;
            else p.part[((size_t)chunk * p.B * p.Hkv + row) * ((size_t)p.key_tiles * BK) + j] = total;
        }
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

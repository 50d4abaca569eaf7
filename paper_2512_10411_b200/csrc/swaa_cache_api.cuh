// C-ABI entry points of the operators around the key/value cache: validation, planning and launches (see include/swaa.h).
// Part of the translation unit of swaa_lib.cu, which includes it last.
#pragma once

#include "swaa_evict.cuh"
#include "swaa_rope.cuh"

namespace swaa {

static bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
static bool stride_ok(long long stride, int heads, int D) { return stride % 8 == 0 && stride >= (long long)heads * D; }

// What the packed form, the cache form and the gradient have in common.
static int check_rope(int T, int Hq, int Hkv, int D, int rotary_dim, const float* inv_freq, const float* qw, const float* kw, float eps) {
    if (T < 0 || Hq < 1 || Hkv < 1 || rotary_dim < 0 || !(eps >= 0.f)) return SWAA_ERR_INVALID_ARG;
    if (Hq % Hkv != 0 || (D != 64 && D != 128)) return SWAA_ERR_UNSUPPORTED;
    if (rotary_dim > D || rotary_dim % 16 != 0) return SWAA_ERR_UNSUPPORTED;
    if ((rotary_dim > 0 && !inv_freq) || !aligned4(inv_freq) || !aligned4(qw) || !aligned4(kw)) return SWAA_ERR_INVALID_ARG;
    if (Hq > (1 << 20)) return SWAA_ERR_UNSUPPORTED;
    return SWAA_OK;
}

template <bool kCache>
static int launch_rope(const RopeParams& p, int D, bool pairs, int sms, cudaStream_t st) {
    const dim3 grid(rope_blocks(p.T, RopeSplit(p.Hq, p.Hkv, D, kRopeRows, p.v != nullptr), sms));
    auto* kernel = D == 128 ? (pairs ? rope_kernel<128, true, kCache> : rope_kernel<128, false, kCache>)
                            : (pairs ? rope_kernel<64, true, kCache> : rope_kernel<64, false, kCache>);
    static std::atomic<bool> attr_done[4][64];
    if (ensure_dynamic_smem(kernel, kRopeSmem, attr_done[(D == 128 ? 2 : 0) + (pairs ? 1 : 0)]) != SWAA_OK) return SWAA_ERR_CUDA;
    return launch_overlapped(kernel, grid, kRopeThreads, kRopeSmem, st, p);
}

static int current_sm100(DeviceInfo* info) {
    const int rc = current_device_info(info);
    if (rc != SWAA_OK) return rc;
    return info->cc_major == 10 ? SWAA_OK : SWAA_ERR_UNSUPPORTED;
}

static RopeParams rope_params(const void* q, const void* k, const void* v, long long q_stride, long long k_stride, long long v_stride,
                              const float* qw, const float* kw, float eps, const float* inv_freq, const int32_t* positions, int T, int Hq,
                              int Hkv, int D, int rotary_dim, void* q_out, void* k_out, void* v_out) {
    RopeParams p = {};
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k = static_cast<const __nv_bfloat16*>(k);
    p.v = static_cast<const __nv_bfloat16*>(v);
    p.q_stride = q_stride;
    p.k_stride = k_stride;
    p.v_stride = v_stride;
    p.qw = qw;
    p.kw = kw;
    p.eps = eps;
    p.inv_freq = inv_freq;
    p.positions = positions;
    p.T = T;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.rot = rotary_dim;
    p.q_out = static_cast<__nv_bfloat16*>(q_out);
    p.k_out = static_cast<__nv_bfloat16*>(k_out);
    p.v_out = static_cast<__nv_bfloat16*>(v_out);
    return p;
}

// Shared body of swaa_cache_append (block_table == nullptr) and swaa_cache_append_paged.
static int append_impl(const void* q, const void* k, const void* v, long long q_stride, long long k_stride, long long v_stride,
                       const float* qw, const float* kw, float eps, const float* inv_freq, int rotary_dim, int interleaved,
                       const int32_t* positions, const int32_t* cu_seqlens_q, const int32_t* seqlens_k, const int32_t* block_table, int B,
                       int Tq, int rows, int max_blocks, int num_pages, int page_size, int Hq, int Hkv, int D, int window, int n_sink,
                       void* q_out, void* kcache, void* vcache, void* stream) {
    if (B < 0 || rows < 1 || window < 0 || n_sink < 0) return SWAA_ERR_INVALID_ARG;
    int rc = check_rope(Tq, Hq, Hkv, D, rotary_dim, inv_freq, qw, kw, eps);
    if (rc != SWAA_OK) return rc;
    if (!stride_ok(q_stride, Hq, D) || !stride_ok(k_stride, Hkv, D) || !stride_ok(v_stride, Hkv, D)) return SWAA_ERR_INVALID_ARG;
    if (window > 0 && (long long)n_sink + window > rows) return SWAA_ERR_INVALID_ARG;  // the ring does not fit the cache
    if (B == 0 || Tq == 0) return SWAA_OK;
    if (!q || !k || !v || !cu_seqlens_q || !seqlens_k || !q_out || !kcache || !vcache) return SWAA_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(kcache) || !aligned16(vcache)) return SWAA_ERR_INVALID_ARG;
    if (!aligned4(positions) || !aligned4(cu_seqlens_q) || !aligned4(seqlens_k) || !aligned4(block_table)) return SWAA_ERR_INVALID_ARG;
    DeviceInfo info;
    if ((rc = current_sm100(&info)) != SWAA_OK) return rc;
    RopeParams p = rope_params(q, k, v, q_stride, k_stride, v_stride, qw, kw, eps, inv_freq, positions, Tq, Hq, Hkv, D, rotary_dim, q_out,
                               kcache, vcache);
    p.cu = cu_seqlens_q;
    p.seqlens = seqlens_k;
    p.block_table = block_table;
    p.B = B;
    p.rows = rows;
    p.max_blocks = max_blocks;
    p.page_size = page_size;
    p.num_pages = num_pages;
    p.ring = window;
    p.n_sink = n_sink;
    return launch_rope<true>(p, D, interleaved != 0, info.sm_count, reinterpret_cast<cudaStream_t>(stream));
}

}  // namespace swaa

// ----------------------------------------------------------------------------------- norm and rotation
extern "C" int swaa_qk_norm_rope(const void* q, const void* k, const void* v, long long q_stride, long long k_stride, long long v_stride,
                                 const float* q_weight, const float* k_weight, float eps, const float* inv_freq, int rotary_dim,
                                 int interleaved, const int32_t* positions, int T, int Hq, int Hkv, int D, void* q_out, void* k_out,
                                 void* v_out, void* stream) {
    int rc = check_rope(T, Hq, Hkv, D, rotary_dim, inv_freq, q_weight, k_weight, eps);
    if (rc != SWAA_OK) return rc;
    if (!stride_ok(q_stride, Hq, D) || !stride_ok(k_stride, Hkv, D) || (v && !stride_ok(v_stride, Hkv, D))) return SWAA_ERR_INVALID_ARG;
    if (T == 0) return SWAA_OK;
    if (!q || !k || !q_out || !k_out || !positions || (v == nullptr) != (v_out == nullptr)) return SWAA_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(k_out) || !aligned16(v_out) || !aligned4(positions))
        return SWAA_ERR_INVALID_ARG;
    DeviceInfo info;
    if ((rc = current_sm100(&info)) != SWAA_OK) return rc;
    const RopeParams p = rope_params(q, k, v, q_stride, k_stride, v_stride, q_weight, k_weight, eps, inv_freq, positions, T, Hq, Hkv, D,
                                     rotary_dim, q_out, k_out, v_out);
    return launch_rope<false>(p, D, interleaved != 0, info.sm_count, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" size_t swaa_qk_norm_rope_backward_workspace_size(int T, int Hq, int Hkv, int D) {
    if (T < 1 || check_rope(T, Hq, Hkv, D, 0, nullptr, nullptr, nullptr, 0.f) != SWAA_OK) return 256;
    DeviceInfo info;
    if (current_device_info(&info) != SWAA_OK) info.sm_count = 148;
    // with values or without: the more blocks
    return (size_t)rope_blocks(T, RopeSplit(Hq, Hkv, D, kRopeBwdRows, true), info.sm_count) * 2 * D * sizeof(float);
}

extern "C" int swaa_qk_norm_rope_backward(const void* q, const void* k, long long q_stride, long long k_stride, const void* dq_out,
                                          const void* dk_out, const void* dv_out, const float* q_weight, const float* k_weight, float eps,
                                          const float* inv_freq, int rotary_dim, int interleaved, const int32_t* positions, int T, int Hq,
                                          int Hkv, int D, void* dq, void* dk, void* dv, long long dq_stride, long long dk_stride,
                                          long long dv_stride, float* dq_weight, float* dk_weight, void* workspace, size_t workspace_bytes,
                                          void* stream) {
    int rc = check_rope(T, Hq, Hkv, D, rotary_dim, inv_freq, q_weight, k_weight, eps);
    if (rc != SWAA_OK) return rc;
    if ((q_weight && !stride_ok(q_stride, Hq, D)) || (k_weight && !stride_ok(k_stride, Hkv, D)) || !stride_ok(dq_stride, Hq, D) ||
        !stride_ok(dk_stride, Hkv, D) || (dv && !stride_ok(dv_stride, Hkv, D)))
        return SWAA_ERR_INVALID_ARG;
    // a weight and its gradient come together
    if ((q_weight == nullptr) != (dq_weight == nullptr) || (k_weight == nullptr) != (dk_weight == nullptr)) return SWAA_ERR_INVALID_ARG;
    if (!aligned4(dq_weight) || !aligned4(dk_weight)) return SWAA_ERR_INVALID_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (T == 0) {  // sums over no tokens
        if (dq_weight && cudaMemsetAsync(dq_weight, 0, D * sizeof(float), st) != cudaSuccess) return SWAA_ERR_CUDA;
        if (dk_weight && cudaMemsetAsync(dk_weight, 0, D * sizeof(float), st) != cudaSuccess) return SWAA_ERR_CUDA;
        return SWAA_OK;
    }
    if ((q_weight && !q) || (k_weight && !k) || !dq_out || !dk_out || !dq || !dk || !positions || (dv_out == nullptr) != (dv == nullptr))
        return SWAA_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k) || !aligned16(dq_out) || !aligned16(dk_out) || !aligned16(dv_out) || !aligned16(dq) || !aligned16(dk) ||
        !aligned16(dv) || !aligned4(positions))
        return SWAA_ERR_INVALID_ARG;
    const bool weights = q_weight != nullptr || k_weight != nullptr;
    if (weights && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)) return SWAA_ERR_WORKSPACE;
    DeviceInfo info;
    if ((rc = current_sm100(&info)) != SWAA_OK) return rc;
    RopeGradParams p = {};
    const unsigned blocks = rope_blocks(T, RopeSplit(Hq, Hkv, D, kRopeBwdRows, dv != nullptr), info.sm_count);
    if (weights && workspace_bytes < (size_t)blocks * 2 * D * sizeof(float)) return SWAA_ERR_WORKSPACE;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k = static_cast<const __nv_bfloat16*>(k);
    p.q_stride = q_stride;
    p.k_stride = k_stride;
    p.dq_out = static_cast<const __nv_bfloat16*>(dq_out);
    p.dk_out = static_cast<const __nv_bfloat16*>(dk_out);
    p.dv_out = static_cast<const __nv_bfloat16*>(dv_out);
    p.qw = q_weight;
    p.kw = k_weight;
    p.eps = eps;
    p.inv_freq = inv_freq;
    p.positions = positions;
    p.T = T;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.rot = rotary_dim;
    p.dq = static_cast<__nv_bfloat16*>(dq);
    p.dk = static_cast<__nv_bfloat16*>(dk);
    p.dv = static_cast<__nv_bfloat16*>(dv);
    p.dq_stride = dq_stride;
    p.dk_stride = dk_stride;
    p.dv_stride = dv_stride;
    p.partial = weights ? static_cast<float*>(workspace) : nullptr;
    auto* kernel = D == 128 ? (interleaved ? rope_backward_kernel<128, true> : rope_backward_kernel<128, false>)
                            : (interleaved ? rope_backward_kernel<64, true> : rope_backward_kernel<64, false>);
    static std::atomic<bool> attr_done[4][64];
    if (ensure_dynamic_smem(kernel, kRopeSmem, attr_done[(D == 128 ? 2 : 0) + (interleaved ? 1 : 0)]) != SWAA_OK) return SWAA_ERR_CUDA;
    rc = launch_overlapped(kernel, dim3(blocks), kRopeThreads, kRopeSmem, st, p);
    if (rc != SWAA_OK || !weights) return rc;
    return launch_overlapped(rope_weight_grad_kernel, dim3((unsigned)(2 * D / 32)), 1024, 0, st, p.partial, (int)blocks, D, dq_weight, dk_weight);
}

// -------------------------------------------------------------------------------------- cache append
extern "C" int swaa_cache_append(const void* q, const void* k, const void* v, long long q_stride, long long k_stride, long long v_stride,
                                 const float* q_weight, const float* k_weight, float eps, const float* inv_freq, int rotary_dim,
                                 int interleaved, const int32_t* positions, const int32_t* cu_seqlens_q, const int32_t* seqlens_k, int B,
                                 int Tq, int Lmax, int Hq, int Hkv, int D, int window, int n_sink, void* q_out, void* kcache, void* vcache,
                                 void* stream) {
    return append_impl(q, k, v, q_stride, k_stride, v_stride, q_weight, k_weight, eps, inv_freq, rotary_dim, interleaved, positions,
                       cu_seqlens_q, seqlens_k, nullptr, B, Tq, Lmax, 0, 0, 0, Hq, Hkv, D, window, n_sink, q_out, kcache, vcache, stream);
}

extern "C" int swaa_cache_append_paged(const void* q, const void* k, const void* v, long long q_stride, long long k_stride,
                                       long long v_stride, const float* q_weight, const float* k_weight, float eps, const float* inv_freq,
                                       int rotary_dim, int interleaved, const int32_t* positions, const int32_t* cu_seqlens_q,
                                       const int32_t* seqlens_k, const int32_t* block_table, int B, int Tq, int max_blocks, int num_pages,
                                       int page_size, int Hq, int Hkv, int D, void* q_out, void* kpages, void* vpages, void* stream) {
    const int rc = check_paged_shape(max_blocks, num_pages, page_size);
    if (rc != SWAA_OK) return rc;
    if (!block_table) return SWAA_ERR_INVALID_ARG;
    return append_impl(q, k, v, q_stride, k_stride, v_stride, q_weight, k_weight, eps, inv_freq, rotary_dim, interleaved, positions,
                       cu_seqlens_q, seqlens_k, block_table, B, Tq, max_blocks * page_size, max_blocks, num_pages, page_size, Hq, Hkv, D, 0,
                       0, q_out, kpages, vpages, stream);
}

// ------------------------------------------------------------------------------------------- eviction
namespace swaa {

static bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

// Blocks of a cluster that works on one (sequence, kv head): more while the launch does not fill the SMs and a block still has
// several thousand weights.
static int evict_cluster(long long rows, int length, int sms) {
    int c = 1;
    while (c < kEvictMaxCluster && 2 * c * rows <= sms && (length + 2 * c - 1) / (2 * c) >= kEvictShare) c *= 2;
    return c;
}

static int evict_impl(EvictParams p, int D, bool paged, cudaStream_t st) {
    if (p.B < 0 || p.rows < 1 || p.weights_rows < 1 || p.Hkv < 1 || p.budget < 1 || p.n_sink < 0 || p.recent < 0 || p.rows_out < 1)
        return SWAA_ERR_INVALID_ARG;
    if ((long long)p.n_sink + p.recent > p.budget || p.rows_out < p.budget || p.weights_out_rows < p.budget) return SWAA_ERR_INVALID_ARG;
    if (D != 64 && D != 128) return SWAA_ERR_UNSUPPORTED;
    if (p.B > 65535 || (long long)p.B * p.Hkv > 0x7fffffffLL / kEvictMaxCluster) return SWAA_ERR_UNSUPPORTED;  // grid dimensions
    const int length = std::min(p.rows, p.weights_rows);
    if (length > 0x7fff0000) return SWAA_ERR_UNSUPPORTED;  // the selection goes through a row in int steps of up to 16384 entries
    if (p.B == 0) return SWAA_OK;
    if (!p.k || !p.v || !p.weights || !p.seqlens || !p.k_out || !p.v_out || !p.weights_out || !p.kept || !p.seqlens_out) return SWAA_ERR_INVALID_ARG;
    if (paged && (!p.block_table || !p.block_table_out)) return SWAA_ERR_INVALID_ARG;
    if (!aligned16(p.k) || !aligned16(p.v) || !aligned16(p.k_out) || !aligned16(p.v_out)) return SWAA_ERR_INVALID_ARG;
    if (!aligned4(p.weights) || !aligned4(p.seqlens) || !aligned4(p.block_table) || !aligned4(p.block_table_out) || !aligned4(p.weights_out) ||
        !aligned4(p.kept) || !aligned4(p.seqlens_out))
        return SWAA_ERR_INVALID_ARG;
    const size_t heads = (size_t)p.B * p.Hkv, in = heads * p.rows * D * 2, out = heads * p.rows_out * D * 2;
    if (!paged && (overlap(p.k, in, p.k_out, out) || overlap(p.v, in, p.v_out, out) || overlap(p.k, in, p.v_out, out) || overlap(p.v, in, p.k_out, out) ||
                   overlap(p.k_out, out, p.v_out, out)))
        return SWAA_ERR_INVALID_ARG;
    if (overlap(p.weights, heads * p.weights_rows * 4, p.weights_out, heads * p.weights_out_rows * 4) ||
        overlap(p.seqlens, (size_t)p.B * 4, p.seqlens_out, (size_t)p.B * 4))
        return SWAA_ERR_INVALID_ARG;
    DeviceInfo info;
    int rc = current_sm100(&info);
    if (rc != SWAA_OK) return rc;
    const int ranks = evict_cluster((long long)heads, length, info.sm_count);
    constexpr int kMostKeys = 48 * 1024;
    p.cap = std::min(((length + ranks - 1) / ranks + 3) / 4 * 4, kMostKeys);
    static std::atomic<bool> attr_done[64];
    if (ensure_dynamic_smem(evict_select_kernel, kMostKeys * 4, attr_done) != SWAA_OK) return SWAA_ERR_CUDA;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)ranks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(heads * ranks));
    cfg.blockDim = dim3(kEvictThreads);
    cfg.dynamicSmemBytes = (size_t)p.cap * 4;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, evict_select_kernel, p) != cudaSuccess) {
        (void)cudaGetLastError();
        return SWAA_ERR_CUDA;
    }
    launch_counter().fetch_add(1, std::memory_order_relaxed);
    const int per_block = (kGatherThreads / 32) * (32 / (D / 8)) * kGatherRows;
    const long long blocks = ((long long)std::min(p.budget, length) * p.Hkv + per_block - 1) / per_block;
    if (blocks > 0x7fffffffLL) return SWAA_ERR_UNSUPPORTED;
    return launch_overlapped(D == 128 ? evict_gather_kernel<128> : evict_gather_kernel<64>, dim3((unsigned)blocks, (unsigned)p.B), kGatherThreads, 0, st, p);
}

static EvictParams evict_params(const void* k, const void* v, const float* weights, const int32_t* seqlens, int B, int weights_rows, int Hkv,
                                int budget, int n_sink, int recent, void* k_out, void* v_out, float* weights_out, int weights_out_rows,
                                int32_t* kept, int32_t* seqlens_out) {
    EvictParams p = {};
    p.k = static_cast<const __nv_bfloat16*>(k);
    p.v = static_cast<const __nv_bfloat16*>(v);
    p.weights = weights;
    p.seqlens = seqlens;
    p.B = B;
    p.weights_rows = weights_rows;
    p.Hkv = Hkv;
    p.budget = budget;
    p.n_sink = n_sink;
    p.recent = recent;
    p.k_out = static_cast<__nv_bfloat16*>(k_out);
    p.v_out = static_cast<__nv_bfloat16*>(v_out);
    p.weights_out = weights_out;
    p.weights_out_rows = weights_out_rows;
    p.kept = kept;
    p.seqlens_out = seqlens_out;
    return p;
}

}  // namespace swaa

extern "C" int swaa_cache_evict(const void* kcache, const void* vcache, const float* weights, const int32_t* seqlens, int B, int Lmax,
                                int weights_rows, int Hkv, int D, int budget, int n_sink, int recent, void* kcache_out, void* vcache_out,
                                int Lmax_out, float* weights_out, int weights_out_rows, int32_t* kept, int32_t* seqlens_out, void* stream) {
    EvictParams p = evict_params(kcache, vcache, weights, seqlens, B, weights_rows, Hkv, budget, n_sink, recent, kcache_out, vcache_out,
                                 weights_out, weights_out_rows, kept, seqlens_out);
    p.rows = Lmax;
    p.rows_out = Lmax_out;
    return evict_impl(p, D, false, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" int swaa_cache_evict_paged(const void* kpages, const void* vpages, const float* weights, const int32_t* seqlens,
                                      const int32_t* block_table, int B, int max_blocks, int num_pages, int page_size, int weights_rows,
                                      int Hkv, int D, int budget, int n_sink, int recent, void* kpages_out, void* vpages_out,
                                      const int32_t* block_table_out, int max_blocks_out, int num_pages_out, int page_size_out,
                                      float* weights_out, int weights_out_rows, int32_t* kept, int32_t* seqlens_out, void* stream) {
    int rc = check_paged_shape(max_blocks, num_pages, page_size);
    if (rc == SWAA_OK) rc = check_paged_shape(max_blocks_out, num_pages_out, page_size_out);
    if (rc != SWAA_OK) return rc;
    EvictParams p = evict_params(kpages, vpages, weights, seqlens, B, weights_rows, Hkv, budget, n_sink, recent, kpages_out, vpages_out,
                                 weights_out, weights_out_rows, kept, seqlens_out);
    p.block_table = block_table;
    p.max_blocks = max_blocks;
    p.num_pages = num_pages;
    p.page_size = page_size;
    p.rows = max_blocks * page_size;
    p.block_table_out = block_table_out;
    p.max_blocks_out = max_blocks_out;
    p.num_pages_out = num_pages_out;
    p.page_size_out = page_size_out;
    p.rows_out = max_blocks_out * page_size_out;
    return evict_impl(p, D, true, reinterpret_cast<cudaStream_t>(stream));
}

// -------------------------------------------------------------------------------- decode with weights
namespace swaa {

static int check_decode_weights(int B, int Lmax, int Hq, int Hkv, const float* in, const float* out, int rows) {
    if (rows < 1) return SWAA_ERR_INVALID_ARG;
    if (Lmax > 0x7fffff00) return SWAA_ERR_UNSUPPORTED;  // its tiles, in entries, are counted in an int
    if (B > 65535 || Hkv > 65535 || Hq / Hkv > 4096) return SWAA_ERR_UNSUPPORTED;  // grid dimensions, shared memory
    if (B <= 0) return SWAA_OK;
    const size_t bytes = (size_t)B * Hkv * rows * sizeof(float);
    if (!out || !aligned4(in) || !aligned4(out) || (in && in != out && overlap(in, bytes, out, bytes))) return SWAA_ERR_INVALID_ARG;
    return SWAA_OK;
}

}  // namespace swaa

extern "C" size_t swaa_decode_weighted_workspace_size(int B, int Hq, int Hkv, int D, int Lmax, int window, int n_sink, int is_full) {
    if (check_decode_shape(B, Hq, Hkv, D, Lmax, window, n_sink, is_full) != SWAA_OK || B == 0 || Lmax > 0x7fffff00) return 256;
    DeviceInfo info;
    if (current_device_info(&info) != SWAA_OK) info.sm_count = 148;
    size_t bytes = 0;
    for (int paged = 0; paged < 2; ++paged) {
        const DecodePlan pl = plan_decode(B, Hq, Hkv, D, Lmax, window, n_sink, is_full, info.sm_count, paged != 0);
        bytes = std::max(bytes, score_plan(pl, B, Hq, Hkv, D, Lmax, window, n_sink, is_full, paged != 0).bytes);
    }
    return bytes;
}

extern "C" int swaa_decode_weighted(const void* q, const void* kcache, const void* vcache, void* out, const float* weights_in,
                                    float* weights_out, const int32_t* seqlens, int B, int Lmax, int weights_rows, int Hq, int Hkv, int D,
                                    int window, int n_sink, int is_full, float scale, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_decode_shape(B, Hq, Hkv, D, Lmax, window, n_sink, is_full);
    if (rc == SWAA_OK) rc = check_decode_weights(B, Lmax, Hq, Hkv, weights_in, weights_out, weights_rows);
    if (rc != SWAA_OK) return rc;
    const DecodeWeights w = {weights_in, weights_out, weights_rows};
    return decode_impl(q, kcache, vcache, out, seqlens, nullptr, 0, 0, 0, B, Lmax, Hq, Hkv, D, window, n_sink, is_full, scale, workspace,
                       workspace_bytes, stream, nullptr, 0, &w);
}

extern "C" int swaa_decode_weighted_paged(const void* q, const void* kpages, const void* vpages, void* out, const float* weights_in,
                                          float* weights_out, const int32_t* block_table, const int32_t* seqlens, int B, int max_blocks,
                                          int num_pages, int page_size, int weights_rows, int Hq, int Hkv, int D, int window, int n_sink,
                                          int is_full, float scale, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_paged_shape(max_blocks, num_pages, page_size);
    if (rc != SWAA_OK) return rc;
    if (!block_table) return SWAA_ERR_INVALID_ARG;
    rc = check_decode_shape(B, Hq, Hkv, D, max_blocks * page_size, window, n_sink, is_full);
    if (rc == SWAA_OK) rc = check_decode_weights(B, max_blocks * page_size, Hq, Hkv, weights_in, weights_out, weights_rows);
    if (rc != SWAA_OK) return rc;
    const DecodeWeights w = {weights_in, weights_out, weights_rows};
    return decode_impl(q, kpages, vpages, out, seqlens, block_table, max_blocks, num_pages, page_size, B, max_blocks * page_size, Hq, Hkv, D,
                       window, n_sink, is_full, scale, workspace, workspace_bytes, stream, nullptr, 0, &w);
}

// ----------------------------------------------------------------------------------- weights of a prompt
namespace swaa {

// Launch shape and workspace: chunks of the key tiles, [chunks of all tiles | chunks of the tiles that hold sinks].
struct KeyWeightsPlan {
    int heads_per_step, chunk_log, key_tiles, chunks, sink_tiles, sink_chunks;
    long long steps;  // query tiles of a sequence times groups of heads
    size_t off_sink, bytes;
};
static KeyWeightsPlan key_weights_plan(int B, int max_q, int max_k, int G, int Hkv, int window, int n_sink, bool full, int last, int sms) {
    KeyWeightsPlan pl;
    const long long rows = last > 0 && last < max_q ? last : max_q;
    // Up to 64 queries fill half of a step's columns: two heads share it where the group has an even number of them.  The last 64 queries of
    // eight prompts of 145610 tokens in all, 32 heads of 128, 8 key heads: 191 us with a head a step, 130 with two.  An odd group keeps a head a step
    // with half of its columns empty: 28 + 4 heads 158 us where 24 + 4 take 102.
    pl.heads_per_step = G % 2 == 0 && 2 * rows <= kKeyWeightsRows ? 2 : 1;
    const long long most = (rows + kKeyWeightsRows - 1) / kKeyWeightsRows;  // query tiles of a sequence
    pl.steps = std::max(1ll, most) * (G / pl.heads_per_step);
    // a key tile meets the queries of `window + 127` positions, which start anywhere in a tile
    const long long band = full ? most : std::min(most, ((long long)window + kKeyWeightsKeys - 1) / kKeyWeightsRows + 2);
    pl.key_tiles = (int)(((long long)max_k + kKeyWeightsKeys - 1) / kKeyWeightsKeys);
    const size_t tile = (size_t)B * Hkv * kKeyWeightsKeys * sizeof(float);
    auto cut = [&](int chunk_log) {
        auto chunks = [&](long long tiles) { return (int)std::max(1ll, (tiles + (1ll << chunk_log) - 1) >> chunk_log); };
        pl.chunk_log = chunk_log;
        pl.chunks = chunks(band);
        pl.sink_chunks = full ? 1 : chunks(most);
        pl.sink_tiles = pl.sink_chunks > pl.chunks ? (int)std::min<long long>(((long long)n_sink + kKeyWeightsKeys - 1) / kKeyWeightsKeys, pl.key_tiles) : 0;
        pl.off_sink = pl.chunks > 1 ? tile * pl.chunks * pl.key_tiles : 0;
        pl.bytes = pl.off_sink + tile * pl.sink_chunks * pl.sink_tiles;
    };
    cut(kKeyWeightsChunkLog);
    // Under full attention (and for many sinks) chunks of one length would take a workspace quadratic in the prompt's: they get longer instead, so
    // that their sums stay within kKeyWeightsPartTiles key tiles per SM, which are blocks enough.  One prompt, 32 + 8 heads of 128, ms and
    // workspace of 16 query tiles a chunk and of this: 32k tokens 6.0 (17 MB) and 5.2 (4.8 MB), 128k 121 (268 MB) and 87 (4.8 MB); with 256 key
    // tiles per SM 6.0 and 112.  16 prompts of 32k, window 2048: 14 to 16 either way.
    const size_t bound = kKeyWeightsPartTiles * (size_t)sms * kKeyWeightsKeys * sizeof(float);
    const size_t wanted = std::min(pl.bytes, bound);
    while (pl.bytes > bound) cut(pl.chunk_log + 1);
    // Calls of few key tiles are cut finer, down to 8 steps a block, until there are two blocks per SM.  Window 2048, us uncut and cut: 1024 tokens,
    // 32 + 8 heads of 128 32.2 and 20.8; 2048 tokens, 28 + 4 heads 94.4 and 44.5; 4096 tokens, window 512 92.8 and 49.5; 500 and 300 tokens 19.9
    // and 15.6; 8192 tokens, 4 + 2 heads 51.6 and 38.  Until there are four or eight: the same within 4 %.  What that takes of the
    // workspace stays within a bound of its own, which every call is asked for: a workspace for longer sequences does for shorter ones.
    const size_t fine = 4 * (size_t)sms * kKeyWeightsKeys * sizeof(float);
    while (pl.chunk_log > 0 && (G / pl.heads_per_step) << pl.chunk_log >= 16 && (long long)B * Hkv * pl.key_tiles * pl.chunks < 2ll * sms) {
        const KeyWeightsPlan before = pl;
        cut(pl.chunk_log - 1);
        if (pl.bytes > fine) {
            pl = before;
            break;
        }
    }
    pl.bytes = std::max(wanted, fine);  // at least what the chunks take, and no less than a smaller call asks for
    return pl;
}

static int check_key_weights(int B, int max_q, int max_k, int Hq, int Hkv, int window, int n_sink, int is_full, int last) {
    if (B < 0 || max_q < 0 || max_k < 0 || Hq < 1 || Hkv < 1 || n_sink < 0 || last < 0) return SWAA_ERR_INVALID_ARG;
    if (!is_full && window < 1) return SWAA_ERR_INVALID_ARG;
    if (Hq % Hkv != 0) return SWAA_ERR_UNSUPPORTED;
    if ((long long)B * Hkv > 0x7fffffffLL || max_k > 0x7fffff00) return SWAA_ERR_UNSUPPORTED;  // grid, positions of a tile
    return SWAA_OK;
}

template <int D>
static int launch_key_weights(const CUtensorMap& tq, const CUtensorMap& tk, const KeyWeightsParams& p, cudaStream_t st) {
    using L = KeyWeightsSmem<D>;
    static std::atomic<bool> attr_done[64];
    if (ensure_dynamic_smem(key_weights_kernel<D>, L::kBytes, attr_done) != SWAA_OK) return SWAA_ERR_CUDA;
    long long slots = (long long)p.sink_tiles * p.sink_chunks + (long long)p.key_tiles * p.chunks;
    auto grid = [&](long long n) {
        const unsigned y = n < 32768 ? (unsigned)n : 32768u;
        return dim3((unsigned)(p.B * p.Hkv), y, (unsigned)((n + y - 1) / y));
    };
    if (p.run > 1) slots = (p.key_tiles + p.run - 1) / p.run;
    if (slots > 32768ll * 65535) return SWAA_ERR_UNSUPPORTED;
    const int rc = launch_overlapped(key_weights_kernel<D>, grid(slots), kKeyWeightsThreads, L::kBytes, st, tq, tk, p);
    if (rc != SWAA_OK || (p.chunks == 1 && p.sink_tiles == 0)) return rc;
    return launch_overlapped(key_weights_join_kernel, grid(p.chunks > 1 ? p.key_tiles : p.sink_tiles), kKeyWeightsKeys, 0, st, p);
}

static int key_weights_impl(const void* q, const void* k, const float* lse, const float* weights_in, float* weights_out, const int32_t* cu_q,
                            const int32_t* cu_k, const int32_t* seqlens_k, const PagedKV& paged, int B, int Tq, int Tk, int max_q, int max_k,
                            int weights_rows, int Hq, int Hkv, int D, int window, int n_sink, int is_full, float scale, int last,
                            void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_key_weights(B, max_q, max_k, Hq, Hkv, window, n_sink, is_full, last);
    if (rc != SWAA_OK) return rc;
    if (Tq < 0 || Tk < 0 || weights_rows < 1) return SWAA_ERR_INVALID_ARG;
    if (D != 64 && D != 128) return SWAA_ERR_UNSUPPORTED;
    if (B == 0 || max_k == 0) return SWAA_OK;
    if (!cu_q || !weights_out || (Tq > 0 && (!q || !lse)) || (Tk > 0 && !k)) return SWAA_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k) || !aligned4(lse) || !aligned4(weights_in) || !aligned4(weights_out) || !aligned4(cu_q) || !aligned4(cu_k) ||
        !aligned4(seqlens_k) || !aligned4(paged.block_table))
        return SWAA_ERR_INVALID_ARG;
    const size_t bytes = (size_t)B * Hkv * weights_rows * sizeof(float);
    if (weights_in && weights_in != weights_out && overlap(weights_in, bytes, weights_out, bytes)) return SWAA_ERR_INVALID_ARG;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return SWAA_ERR_WORKSPACE;
    DeviceInfo info;
    if ((rc = current_sm100(&info)) != SWAA_OK) return rc;
    const int G = Hq / Hkv;
    const KeyWeightsPlan pl = key_weights_plan(B, max_q, max_k, G, Hkv, window, n_sink, is_full != 0, last, info.sm_count);
    if (workspace_bytes < pl.bytes) return SWAA_ERR_WORKSPACE;
    const int hs = pl.heads_per_step;
    CUtensorMap tq = {}, tk = {};
    if (Tq > 0 && (rc = make_token_major_map(&tq, q, Tq, Hq, D, kKeyWeightsRows / hs, hs)) != SWAA_OK) return rc;
    if (Tk > 0) {
        rc = cu_k != nullptr ? make_token_major_map(&tk, k, Tk, Hkv, D, kKeyWeightsKeys)
                             : make_cache_map(&tk, k, paged.num_pages, paged.page_size, Hkv, D, kKeyWeightsKeys);
        if (rc != SWAA_OK) return rc;
    }
    KeyWeightsParams p = {};
    p.lse = lse;
    p.weights_in = weights_in;
    p.weights_out = weights_out;
    p.cu_q = cu_q;
    p.cu_k = cu_k;
    p.seqlens_k = seqlens_k;
    p.block_table = paged.block_table;
    p.max_blocks = paged.max_blocks;
    p.page_size = paged.page_size;
    p.num_pages = paged.num_pages;
    p.B = B;
    p.Tq = Tq;
    p.Tk = Tk;
    p.max_q = max_q;
    p.max_k = max_k;
    p.weights_rows = weights_rows;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.G = G;
    p.window = window;
    p.n_sink = n_sink;
    p.is_full = is_full ? 1 : 0;
    p.last = last;
    p.sl2 = (scale > 0.f ? scale : 1.0f / sqrtf((float)D)) * 1.4426950408889634f;
    p.key_tiles = pl.key_tiles;
    p.chunks = pl.chunks;
    p.sink_tiles = pl.sink_tiles;
    p.sink_chunks = pl.sink_chunks;
    p.heads_per_step = hs;
    p.chunk_log = pl.chunk_log;
    // A block of few steps is mostly set-up: it takes more key tiles, up to 16 steps, while there are several blocks per SM all the same.  The same
    // call with 4, 8, 16 and 32 steps: 192, 158, 149 and 150 us (an earlier form of the kernel); one prompt of 32768 tokens 48 throughout.
    p.run = 1;
    while (pl.chunks == 1 && pl.sink_tiles == 0 && p.run * pl.steps < kKeyWeightsRunSteps && (long long)B * Hkv * (pl.key_tiles / (2 * p.run)) >= 8ll * info.sm_count) p.run *= 2;
    p.part = static_cast<float*>(workspace);
    p.sink_part = reinterpret_cast<float*>(static_cast<char*>(workspace) + pl.off_sink);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    return D == 128 ? launch_key_weights<128>(tq, tk, p, st) : launch_key_weights<64>(tq, tk, p, st);
}

}  // namespace swaa

extern "C" size_t swaa_key_weights_workspace_size(int B, int max_seqlen_q, int max_seqlen_k, int Hq, int Hkv, int window, int n_sink,
                                                  int is_full, int last) {
    if (check_key_weights(B, max_seqlen_q, max_seqlen_k, Hq, Hkv, window, n_sink, is_full, last) != SWAA_OK || B == 0) return 256;
    DeviceInfo info;
    if (current_device_info(&info) != SWAA_OK) info.sm_count = 148;
    return key_weights_plan(B, max_seqlen_q, max_seqlen_k, Hq / Hkv, Hkv, window, n_sink, is_full != 0, last, info.sm_count).bytes;
}

extern "C" int swaa_key_weights(const void* q, const void* k, const float* lse, const float* weights_in, float* weights_out,
                                const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int B, int Tq, int Tk, int max_seqlen_q,
                                int max_seqlen_k, int weights_rows, int Hq, int Hkv, int D, int window, int n_sink, int is_full, float scale,
                                int last, void* workspace, size_t workspace_bytes, void* stream) {
    if (!cu_seqlens_k && B > 0) return SWAA_ERR_INVALID_ARG;
    return key_weights_impl(q, k, lse, weights_in, weights_out, cu_seqlens_q, cu_seqlens_k, nullptr, PagedKV(), B, Tq, Tk, max_seqlen_q,
                            max_seqlen_k, weights_rows, Hq, Hkv, D, window, n_sink, is_full, scale, last, workspace, workspace_bytes, stream);
}

extern "C" int swaa_key_weights_paged(const void* q, const void* kpages, const float* lse, const float* weights_in, float* weights_out,
                                      const int32_t* cu_seqlens_q, const int32_t* seqlens_k, const int32_t* block_table, int B, int Tq,
                                      int max_seqlen_q, int max_blocks, int num_pages, int page_size, int weights_rows, int Hq, int Hkv, int D,
                                      int window, int n_sink, int is_full, float scale, int last, void* workspace, size_t workspace_bytes,
                                      void* stream) {
    const int rc = check_paged_shape(max_blocks, num_pages, page_size);
    if (rc != SWAA_OK) return rc;
    if (page_size % kKeyWeightsKeys != 0) return SWAA_ERR_UNSUPPORTED;
    if (!block_table || (!seqlens_k && B > 0)) return SWAA_ERR_INVALID_ARG;
    PagedKV paged;
    paged.block_table = block_table;
    paged.max_blocks = max_blocks;
    paged.num_pages = num_pages;
    paged.page_size = page_size;
    const int max_k = std::min(max_blocks * page_size, weights_rows);  // longer sequences have no room for their weights
    return key_weights_impl(q, kpages, lse, weights_in, weights_out, cu_seqlens_q, nullptr, seqlens_k, paged, B, Tq, 1, max_seqlen_q, max_k,
                            weights_rows, Hq, Hkv, D, window, n_sink, is_full, scale, last, workspace, workspace_bytes, stream);
}

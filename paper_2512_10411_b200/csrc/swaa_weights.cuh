// Attention weight that the entries of a key/value cache gather, per kv head (summed over the query heads of its group), as
// the eviction of swaa_evict.cuh wants it.
//
// Decode step.  decode_kernel computes every score once, on its way to the output; its kScores instance also stores them (4 bytes per
// query head and entry next to the 4 D bytes of an entry's K and V) and the logarithm of each row's sum.  The kernel here then forms
//     weights_out[b, g, j] = weights_in[b, g, j] + sum over heads h of g of 2^(score_hj * sl2 - lse2_h)
// one thread per entry.  A second pass over K instead would move 2 D bytes an entry.  The entry of the new token itself starts from 0.
#pragma once

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

}  // namespace swaa

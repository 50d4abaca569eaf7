// Queries, keys and values on their way from the projection to the attention: a norm of every query and key head, the
// rotation by the token's position, and the store into what the attention reads (packed rows, or the rows of a
// dense, ring or paged key/value cache), in one pass; and the gradient of the packed form.
//
//     u = x / sqrt(mean(x^2) + eps)          over the D channels of one head of one token
//     y = w u                                 (w: one weight per channel; without weights y = x)
//     (z_a, z_b) = (y_a cos - y_b sin, y_b cos + y_a sin)      for every pair (a, b) of the first R channels
// with the angle position * frequency of the pair; pairs are (i, i + R/2), or (2i, 2i + 1) when interleaved.  The channels from R on
// keep y.  Gradient, with g = the rotation by the negative angle of dz:
//     dw = sum over tokens and heads of g u,     dx = (w g - u mean(w g u)) / sqrt(mean(x^2) + eps)
//
// Angles are formed in double: position * frequency / 2 pi keeps its fraction to 2^-24 for positions up to 2^30 and to 2^-23 for every other
// 32-bit one (frequencies up to 1), and sincospif takes the fraction; there is no table whose length bounds the positions.  For |position| up
// to 2^k the rounded product adds 2^(k - 54) / 2 pi, 1 / 2 pi as a double 2^(k - 56), its product 2^(k - 56) and the fraction in fp32 2^-26.  All sums and products are
// fp32, rounded to bf16 once, at the store.
//
// What bounds it: memory, every channel read and written once (2 * 2 bytes a channel; the gradient 3 * 2).  A head is D / 16 lanes,
// each with two 16-byte pieces that hold both channels of its pairs, so the rotation needs no exchange and the norm log2(D / 16)
// shuffles.  A warp takes kRopeRows groups of 32 / (D / 16) heads (1 KiB) of one token after another; these shares come by bulk
// copies through a ring in shared memory.  The angles of a token are spread over the lanes that hold the same channels of
// different heads: a lane forms 8 / (heads per group) of its 8 and takes the others by shuffle.
//
// 32k tokens, 32 + 8 heads of 128: 131 us on one GPU, 147 on another (805 MB; a plain copy of as much takes 123).  16k tokens, forward
// and gradient: 66 + 114 + 4.  Loads into registers instead of the ring 150; three blocks per SM at 80 registers 147 where two take 131.
#pragma once

#include <algorithm>

#include "swaa_internal.cuh"
#include "swaa_ptx.cuh"

namespace swaa {

constexpr int kRopeThreads = 256;
constexpr int kRopeWarps = kRopeThreads / 32;
constexpr int kRopeBlocksPerSm = 2;
constexpr int kRopeRows = 4;     // groups of heads of a warp's share of a token: forward
constexpr int kRopeBwdRows = 2;  // and gradient, which takes two rows of each head
constexpr int kRopeShare = kRopeRows * 1024;  // bytes of a share: a group is 4 heads of 128 channels or 8 of 64
constexpr int kRopeStages = 2;   // shares of a warp in shared memory
constexpr int kRopeSmem = kRopeWarps * kRopeStages * kRopeShare;
static_assert(kRopeBwdRows * 2 == kRopeRows, "the gradient's two inputs fill a share");

// Work of a token: its heads in groups of 32 / (D / 16), a share of `rows` groups for every warp.  Shares hold query groups, or key and
// value groups in turn, so that those with values, which are only copied, are about as long as the others.
struct RopeSplit {
    int groups_q, groups_kv;  // groups of query heads; of key heads and, where there are any, value heads
    int seg_q, segs;          // shares of query groups, of all
    bool values;
    __host__ __device__ RopeSplit(int Hq, int Hkv, int D, int rows, bool with_values) {
        const int per = 32 / (D / 16);
        values = with_values;
        groups_q = (Hq + per - 1) / per;
        groups_kv = (Hkv + per - 1) / per * (values ? 2 : 1);
        seg_q = (groups_q + rows - 1) / rows;
        segs = seg_q + (groups_kv + rows - 1) / rows;
    }
};
// Blocks of a launch: a warp per share of a token, as many as the SMs hold at a time; the warps go on through the tokens.
inline unsigned rope_blocks(int T, const RopeSplit& s, int sms) {
    const long long most = std::max((long long)sms * kRopeBlocksPerSm, ((long long)s.segs + kRopeWarps - 1) / kRopeWarps);
    return (unsigned)std::min(((long long)T * s.segs + kRopeWarps - 1) / kRopeWarps, most);
}
// A warp's place among them: share `seg` of the tokens stream, stream + streams, ...  Neighbouring warps have the shares of one token, which
// are neighbours in memory: 16k tokens of 16 + 4 heads of 64, forward and gradient, 63 us; with streams of their own for every kind of head,
// as many as its work asks for, the kinds drift apart and it takes 97.
template <int D, int kRows>
struct RopeWarp {
    static constexpr int kHeads = 32 / (D / 16);
    int seg, stream, streams, groups;
    bool keys;  // keys and values
    __host__ __device__ __forceinline__ RopeWarp(const RopeSplit& p, unsigned warp, unsigned warps) {
        seg = (int)(warp % (unsigned)p.segs);
        stream = (int)(warp / (unsigned)p.segs);
        streams = (int)(warps / (unsigned)p.segs);
        keys = seg >= p.seg_q;
        const int left = keys ? p.groups_kv - (seg - p.seg_q) * kRows : p.groups_q - seg * kRows;
        groups = left < kRows ? left : kRows;
    }
    // Whether the warp has any of the T tokens.  A grid is whole blocks: the last warps may make up no stream of their own, and in a call of
    // few tokens a stream may start behind the last one.
    __host__ __device__ __forceinline__ bool works(int T) const { return stream < streams && stream < T; }
    // group u of the share: whether it holds values, and its first head
    __host__ __device__ __forceinline__ bool value(const RopeSplit& p, int u) const { return keys && p.values && ((seg - p.seg_q) * kRows + u) % 2 != 0; }
    __host__ __device__ __forceinline__ int head(const RopeSplit& p, int u) const {
        const int g = (keys ? seg - p.seg_q : seg) * kRows + u;
        return (keys && p.values ? g / 2 : g) * kHeads;
    }
};

struct RopeParams {
    const __nv_bfloat16 *q, *k, *v;              // [T, heads, D] with a stride between tokens
    long long q_stride, k_stride, v_stride;      // elements
    const float *qw, *kw;                        // [D] or null
    float eps;
    const float* inv_freq;                       // [rot / 2]
    const int32_t* positions;                    // [T]; cache form: may be null
    int T, Hq, Hkv, rot;
    __nv_bfloat16 *q_out, *k_out, *v_out;        // packed [T, heads, D]; cache form: k_out, v_out are the cache
    // cache form
    const int32_t *cu, *seqlens, *block_table;   // block_table null: dense [B, rows, Hkv, D]
    int B, rows /* of a sequence: Lmax, or max_blocks * page_size */, max_blocks, page_size, num_pages;
    int ring, n_sink;                            // ring > 0: slots n_sink .. n_sink + ring - 1 are a ring
};

struct RopeGradParams {
    const __nv_bfloat16 *q, *k;                  // inputs of the forward pass (null where not normalised)
    long long q_stride, k_stride;
    const __nv_bfloat16 *dq_out, *dk_out, *dv_out;  // packed
    const float *qw, *kw;
    float eps;
    const float* inv_freq;
    const int32_t* positions;
    int T, Hq, Hkv, rot;
    __nv_bfloat16 *dq, *dk, *dv;
    long long dq_stride, dk_stride, dv_stride;
    float* partial;                              // [blocks][2][D]: weight gradients of a block
};

// What a lane holds of a head: 8 channels from a0 and 8 from b0; pair i is (a_i, b_i), or, interleaved, pairs 0..3 are the
// neighbours in a and 4..7 those in b.  rot_a, rot_b: whether the pieces are rotated.
template <int D, bool kPairs>
struct RopeLane {
    static constexpr int kLanes = D / 16, kHeads = 32 / kLanes, kAngles = 8 / kHeads;
    int l, sub, a0, b0;
    bool rot_a, rot_b;
    float f[kAngles];
    __device__ __forceinline__ RopeLane(int lane, const float* inv_freq, int rot) {
        l = lane % kLanes;
        sub = lane / kLanes;
        const int np = rot / 16;  // half-split: lanes whose pieces are the two halves of pairs
        if (kPairs) {
            a0 = 8 * l;
            b0 = 8 * (l + kLanes);
            rot_a = a0 < rot;
            rot_b = b0 < rot;
        } else {
            a0 = l < np ? 8 * l : 16 * np + 16 * (l - np);
            b0 = l < np ? 8 * (l + np) : a0 + 8;
            rot_a = rot_b = l < np;
        }
#pragma unroll
        for (int i = 0; i < kAngles; ++i) {
            const int pair = sub * kAngles + i;  // of the lane's 8
            const bool turned = kPairs ? (pair < 4 ? rot_a : rot_b) : rot_a;
            const int at = kPairs ? (pair < 4 ? a0 / 2 + pair : b0 / 2 + pair - 4) : 8 * l + pair;
            f[i] = turned ? inv_freq[at] : 0.f;
        }
    }
    // cos and sin of the lane's 8 pairs at a position
    __device__ __forceinline__ void turn(int position, float (&c)[8], float (&s)[8]) const {
        float cm[kAngles], sm[kAngles];
#pragma unroll
        for (int i = 0; i < kAngles; ++i) {
            const double t = (double)position * (double)f[i] * 0.15915494309189533577;  // 1 / (2 pi)
            sincospif(2.f * (float)(t - rint(t)), &sm[i], &cm[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            c[i] = __shfl_sync(0xffffffffu, cm[i % kAngles], (i / kAngles) * kLanes + l);
            s[i] = __shfl_sync(0xffffffffu, sm[i % kAngles], (i / kAngles) * kLanes + l);
        }
    }
    // Rotation by the angle, or by its negative.  Pieces that are not rotated pass as they are (no 0 * inf).
    template <bool kBack>
    __device__ __forceinline__ void rotate(float (&a)[8], float (&b)[8], const float (&c)[8], const float (&s)[8]) const {
        auto pair = [](float& x, float& y, float co, float si, bool on) {
            const float sn = kBack ? -si : si;
            const float x1 = x * co - y * sn, y1 = y * co + x * sn;
            x = on ? x1 : x;
            y = on ? y1 : y;
        };
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!kPairs) pair(a[i], b[i], c[i], s[i], rot_a);
            else if (i < 4) pair(a[2 * i], a[2 * i + 1], c[i], s[i], rot_a);
            else pair(b[2 * i - 8], b[2 * i - 7], c[i], s[i], rot_b);
        }
    }
    static __device__ __forceinline__ float sum(float x) {  // over the lanes of a head
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        return x;
    }
};

__device__ __forceinline__ void unpack_bf16x8(const uint4& v, float (&x)[8]) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack_bf16x8(const float (&x)[8]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
// 8 weights of a piece; ones where there are none
__device__ __forceinline__ void load_weights(const float* w, int at, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = w != nullptr ? w[at + i] : 1.f;
}

// Sequence that owns packed token t: the smallest b with cu[b + 1] > t, or B behind the last one.  All lanes of the warp
// look at 32 places at a time.  Whatever cu holds, every index stays in [0, B].
__device__ __forceinline__ int sequence_of(const int32_t* cu, int B, int t, int lane) {
    int lo = 0, n = B;
    while (n > 0) {
        const int step = (n + 31) / 32;
        const long long ahead = (long long)(lane + 1) * step;
        const int at = lo + (int)(ahead < n ? ahead : n);  // cu[at] ends a stretch of `step` sequences
        const unsigned hit = __ballot_sync(0xffffffffu, cu[at] > t);
        if (hit == 0u) return B;
        const int first = (__ffs((int)hit) - 1) * step;
        lo += first < n ? first : n - 1;
        if (step == 1) return lo;
        n = n - first < step ? n - first : step;
    }
    return B;
}

// The sequence of a token of the cache form, kept while a warp's tokens stay in it.
struct RopeSeq {
    int b, end, len;  // tokens up to `end` are its, the last of `len` entries
    bool ok;
};
__device__ __forceinline__ RopeSeq rope_seq(const RopeParams& p, int t, int lane) {
    RopeSeq q = {sequence_of(p.cu, p.B, t, lane), p.T, 0, false};
    if (q.b >= p.B) return q;  // behind the last sequence: padding, left alone
    const int start = p.cu[q.b];
    q.end = p.cu[q.b + 1];
    q.len = p.seqlens[q.b];
    // (start > t or a length beyond the tokens shows a cu that decreases)
    q.ok = start >= 0 && start <= t && q.end <= p.T && (long long)q.end - start <= q.len && (p.ring > 0 || q.len <= p.rows);
    if (!q.ok) {
        record_device_error(SWAA_ERR_BAD_SEQLENS);
        q.end = t + 1;  // looked at token by token
    }
    return q;
}
// Row of the cache, seen as [rows, Hkv, D], for entry e of a sequence; -1: not stored.
__device__ __forceinline__ long long rope_row(const RopeParams& p, const RopeSeq& q, int e) {
    int slot = e;
    if (p.ring > 0 && e >= p.n_sink) {
        if ((long long)e + p.ring < q.len) return -1;  // a later token of the call has the slot
        slot = p.n_sink + (e - p.n_sink) % p.ring;
    }
    if (p.block_table == nullptr) return (long long)q.b * p.rows + slot;
    const int page = p.block_table[(size_t)q.b * p.max_blocks + slot / p.page_size];
    if (page >= 0 && page < p.num_pages) return (long long)page * p.page_size + slot % p.page_size;
    record_device_error(SWAA_ERR_BAD_SEQLENS);
    return -1;
}

// A warp's ring of shares: bulk copies land in shared memory while earlier shares are worked on, so the bytes in flight do not
// depend on registers.  Waits are bounded; a warp that gives up waits (again with a limit) for its copies in flight.
struct RopeRing {
    uint32_t data, bars;
    volatile int* abort_flag;
    int stage;
    uint32_t phase;
    __device__ __forceinline__ RopeRing(uint32_t smem, uint64_t* bar_words, volatile int* flag, int warp, int lane) {
        data = smem + (uint32_t)(warp * kRopeStages * kRopeShare);
        bars = smem_u32(bar_words + warp * kRopeStages);
        abort_flag = flag;
        stage = 0;
        phase = 0;
        if (lane == 0) {
            for (int i = 0; i < kRopeStages; ++i) mbar_init(bars + 8u * (uint32_t)i, 1u);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
    }
    // One lane: announces `bytes` to come into stage i; copies (16-byte aligned, a multiple of 16 bytes) into its `at`-th byte.
    __device__ __forceinline__ void expect(int i, uint32_t bytes) const { mbar_arrive_expect_tx(bars + 8u * (uint32_t)i, bytes); }
    __device__ __forceinline__ void copy(int i, int at, const void* src, uint32_t bytes) const {
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(data + (uint32_t)(i * kRopeShare + at)),
                     "l"(src), "r"(bytes), "r"(bars + 8u * (uint32_t)i)
                     : "memory");
    }
    __device__ __forceinline__ bool wait() const { return __all_sync(0xffffffffu, mbar_wait(bars + 8u * (uint32_t)stage, phase, abort_flag)) != 0; }
    __device__ __forceinline__ uint32_t share() const { return data + (uint32_t)(stage * kRopeShare); }
    __device__ __forceinline__ void next() {
        if (++stage == kRopeStages) {
            stage = 0;
            phase ^= 1u;
        }
    }
    // After a wait that ran out at the present share, with `ahead` shares filled from there on.
    __device__ __forceinline__ void drain(int ahead) {
        const uint64_t t0 = global_timer_ns();
        for (; ahead > 0; --ahead, next())
            while (!mbar_try_wait(bars + 8u * (uint32_t)stage, phase) && global_timer_ns() - t0 < kWaitLimitNs) {
            }
    }
};
__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

template <int D, bool kPairs, bool kCache>
__global__ void __launch_bounds__(kRopeThreads, 2) rope_kernel(const RopeParams p) {
    using L = RopeLane<D, kPairs>;
    extern __shared__ __align__(128) uint8_t rope_smem[];
    __shared__ uint64_t bar_words[kRopeWarps * kRopeStages];
    __shared__ int abort_word;
    if (threadIdx.x == 0) abort_word = 0;
    __syncthreads();
    grid_wait();
    const int lane = threadIdx.x & 31;
    const RopeSplit split(p.Hq, p.Hkv, D, kRopeRows, p.v != nullptr);
    const RopeWarp<D, kRopeRows> me(split, blockIdx.x * kRopeWarps + (threadIdx.x >> 5), gridDim.x * kRopeWarps);
    const int stream = me.stream, streams = me.streams;
    if (!me.works(p.T)) return;
    const int heads = me.keys ? p.Hkv : p.Hq;
    const float* w = me.keys ? p.kw : p.qw;
    const L ln(lane, p.inv_freq, p.rot);
    const bool norm = w != nullptr;
    float wa[8], wb[8];
    load_weights(w, ln.a0, wa);
    load_weights(w, ln.b0, wb);
    RopeRing ring(smem_u32(rope_smem), bar_words, &abort_word, (int)threadIdx.x >> 5, lane);
    uint32_t bytes = 0;  // of a share
#pragma unroll
    for (int u = 0; u < kRopeRows; ++u)
        if (u < me.groups) bytes += (uint32_t)(min(heads - me.head(split, u), L::kHeads) * D * 2);
    auto fill = [&](int i, long long t) {
        ring.expect(i, bytes);
#pragma unroll
        for (int u = 0; u < kRopeRows; ++u) {
            if (u >= me.groups) break;
            const int h0 = me.head(split, u);
            const __nv_bfloat16* src = !me.keys ? p.q + t * p.q_stride : me.value(split, u) ? p.v + t * p.v_stride : p.k + t * p.k_stride;
            ring.copy(i, u * 1024, src + (long long)h0 * D, (uint32_t)(min(heads - h0, L::kHeads) * D * 2));
        }
    };
    int filled = 0;  // shares from the present one on
    for (int t = stream; filled < kRopeStages && t < p.T; t += streams, ++filled)
        if (lane == 0) fill(filled, t);
    bool ok = true;
    RopeSeq seq = {0, -1, 0, false};
    // The next token's position on its way during this one: 16k tokens of 16 + 4 heads of 64, forward and gradient, 63.0 -> 58.3 us; not
    // for heads of 128 (32k tokens, 32 + 8 heads: packed 145 us without, 153 with; appended to a cache 146 and 154; 16 generated tokens and a
    // step of chunks next to tokens the same either way).
    constexpr bool kAhead = D == 64;
    int given = kAhead && p.positions != nullptr ? p.positions[stream] : 0;
    for (int t = stream; t < p.T; t += streams) {
        int position = given;
        if (p.positions != nullptr) {
            if (!kAhead) position = p.positions[t];
            else if (t < p.T - streams) given = p.positions[t + streams];
        }
        long long row = t;
        bool store = true;
        if (kCache) {  // the same for the whole warp
            if (t >= seq.end) seq = rope_seq(p, t, lane);
            const int e = seq.len - (seq.end - t);  // index of the token in its sequence
            if (p.positions == nullptr) position = e;
            if (seq.ok && me.keys) row = rope_row(p, seq, e);
            store = seq.ok && row >= 0;
        }
        float c[8], s[8];
        ln.turn(position, c, s);
        ok = ring.wait();
        if (!ok) break;
        if (store) {
#pragma unroll
            for (int u = 0; u < kRopeRows; ++u) {
                if (u >= me.groups) break;  // uniform
                const bool value = me.value(split, u);
                const int h = me.head(split, u) + ln.sub;
                const bool on = h < heads;
                const uint32_t x = ring.share() + (uint32_t)(u * 1024 + (on ? ln.sub : 0) * D * 2);
                uint4 va = ld_shared_v4(x + 2u * (uint32_t)ln.a0), vb = ld_shared_v4(x + 2u * (uint32_t)ln.b0);
                if (!value) {
                    float a[8], b[8];
                    unpack_bf16x8(va, a);
                    unpack_bf16x8(vb, b);
                    if (norm) {
                        float ss = 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) ss += a[i] * a[i] + b[i] * b[i];
                        const float r = rsqrtf(L::sum(ss) * (1.f / D) + p.eps);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            a[i] *= r * wa[i];
                            b[i] *= r * wb[i];
                        }
                    }
                    ln.template rotate<false>(a, b, c, s);
                    va = pack_bf16x8(a);
                    vb = pack_bf16x8(b);
                }
                if (on) {
                    __nv_bfloat16* y = (!me.keys ? p.q_out : value ? p.v_out : p.k_out) + (row * heads + h) * D;
                    *reinterpret_cast<uint4*>(y + ln.a0) = va;
                    *reinterpret_cast<uint4*>(y + ln.b0) = vb;
                }
            }
        }
        __syncwarp();  // the share has been read
        const long long ahead = (long long)t + (long long)kRopeStages * streams;
        if (ahead < p.T) {
            if (lane == 0) fill(ring.stage, ahead);
        } else {
            --filled;
        }
        ring.next();
    }
    if (!ok) ring.drain(filled);
}

template <int D, bool kPairs>
__global__ void __launch_bounds__(kRopeThreads, 2) rope_backward_kernel(const RopeGradParams p) {
    using L = RopeLane<D, kPairs>;
    extern __shared__ __align__(128) uint8_t rope_smem[];
    __shared__ float sm_w[kRopeWarps][D];
    __shared__ uint64_t bar_words[kRopeWarps * kRopeStages];
    __shared__ int abort_word;
    if (threadIdx.x == 0) abort_word = 0;
    __syncthreads();
    grid_wait();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const RopeSplit split(p.Hq, p.Hkv, D, kRopeBwdRows, p.dv != nullptr);
    const RopeWarp<D, kRopeBwdRows> me(split, blockIdx.x * kRopeWarps + wid, gridDim.x * kRopeWarps);
    const int heads = me.keys ? p.Hkv : p.Hq, streams = me.streams;
    const float* w = me.keys ? p.kw : p.qw;
    const L ln(lane, p.inv_freq, p.rot);
    const bool norm = w != nullptr;
    float wa[8], wb[8], da[8], db[8];
    load_weights(w, ln.a0, wa);
    load_weights(w, ln.b0, wb);
#pragma unroll
    for (int i = 0; i < 8; ++i) da[i] = db[i] = 0.f;
    RopeRing ring(smem_u32(rope_smem), bar_words, &abort_word, wid, lane);
    uint32_t bytes = 0;  // of a share
#pragma unroll
    for (int u = 0; u < kRopeBwdRows; ++u)
        if (u < me.groups) bytes += (uint32_t)(min(heads - me.head(split, u), L::kHeads) * D * 2) * (norm && !me.value(split, u) ? 2u : 1u);
    auto fill = [&](int i, long long t) {
        ring.expect(i, bytes);
#pragma unroll
        for (int u = 0; u < kRopeBwdRows; ++u) {
            if (u >= me.groups) break;
            const int h0 = me.head(split, u);
            const bool value = me.value(split, u);
            const uint32_t n = (uint32_t)(min(heads - h0, L::kHeads) * D * 2);
            ring.copy(i, u * 1024, (!me.keys ? p.dq_out : value ? p.dv_out : p.dk_out) + (t * heads + h0) * D, n);
            if (norm && !value) ring.copy(i, kRopeShare / 2 + u * 1024, (me.keys ? p.k + t * p.k_stride : p.q + t * p.q_stride) + (long long)h0 * D, n);
        }
    };
    const int T = me.works(p.T) ? p.T : 0;  // a warp without tokens still joins the sums of its block
    int filled = 0;
    for (int t = me.stream; filled < kRopeStages && t < T; t += streams, ++filled)
        if (lane == 0) fill(filled, t);
    bool ok = true;
    int given = T > 0 ? p.positions[me.stream] : 0;
    for (int t = me.stream; t < T; t += streams) {
        const int position = given;
        if (t < T - streams) given = p.positions[t + streams];  // of the next token, on its way meanwhile
        float c[8], s[8];
        ln.turn(position, c, s);
        ok = ring.wait();
        if (!ok) break;
#pragma unroll
        for (int u = 0; u < kRopeBwdRows; ++u) {
            if (u >= me.groups) break;  // uniform
            const bool value = me.value(split, u);
            const int h = me.head(split, u) + ln.sub;
            const bool on = h < heads;
            const uint32_t from = ring.share() + (uint32_t)(u * 1024 + (on ? ln.sub : 0) * D * 2), oa = 2u * (uint32_t)ln.a0, ob = 2u * (uint32_t)ln.b0;
            uint4 va = ld_shared_v4(from + oa), vb = ld_shared_v4(from + ob);
            if (!value) {
                float ga[8], gb[8];
                unpack_bf16x8(va, ga);
                unpack_bf16x8(vb, gb);
                ln.template rotate<true>(ga, gb, c, s);
                if (norm) {
                    float a[8], b[8], ss = 0.f;
                    unpack_bf16x8(ld_shared_v4(from + kRopeShare / 2 + oa), a);
                    unpack_bf16x8(ld_shared_v4(from + kRopeShare / 2 + ob), b);
#pragma unroll
                    for (int i = 0; i < 8; ++i) ss += a[i] * a[i] + b[i] * b[i];
                    const float r = rsqrtf(L::sum(ss) * (1.f / D) + p.eps);
                    float dot = 0.f;  // sum of (w g) u
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        a[i] *= r;
                        b[i] *= r;
                        da[i] += on ? ga[i] * a[i] : 0.f;
                        db[i] += on ? gb[i] * b[i] : 0.f;
                        ga[i] *= wa[i];
                        gb[i] *= wb[i];
                        dot += ga[i] * a[i] + gb[i] * b[i];
                    }
                    dot = L::sum(dot) * (1.f / D);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        ga[i] = r * (ga[i] - a[i] * dot);
                        gb[i] = r * (gb[i] - b[i] * dot);
                    }
                }
                va = pack_bf16x8(ga);
                vb = pack_bf16x8(gb);
            }
            if (on) {
                __nv_bfloat16* x = (!me.keys ? p.dq + t * p.dq_stride : value ? p.dv + t * p.dv_stride : p.dk + t * p.dk_stride) + (long long)h * D;
                *reinterpret_cast<uint4*>(x + ln.a0) = va;
                *reinterpret_cast<uint4*>(x + ln.b0) = vb;
            }
        }
        __syncwarp();  // the share has been read
        const long long ahead = (long long)t + (long long)kRopeStages * streams;
        if (ahead < T) {
            if (lane == 0) fill(ring.stage, ahead);
        } else {
            --filled;
        }
        ring.next();
    }
    if (!ok) ring.drain(filled);
    if (p.partial == nullptr) return;
    // weight gradients: the lanes with the same channels, then the block's warps in order, then (the next kernel) the blocks in order
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int o = L::kLanes; o < 32; o <<= 1) {
            da[i] += __shfl_xor_sync(0xffffffffu, da[i], o);
            db[i] += __shfl_xor_sync(0xffffffffu, db[i], o);
        }
        if (ln.sub == 0) {
            sm_w[wid][ln.a0 + i] = da[i];
            sm_w[wid][ln.b0 + i] = db[i];
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kRopeThreads) {
        float sum = 0.f;
        for (int o = 0; o < kRopeWarps; ++o) {
            if ((RopeWarp<D, kRopeBwdRows>(split, blockIdx.x * kRopeWarps + o, gridDim.x * kRopeWarps).keys ? 1 : 0) == i / D) sum += sm_w[o][i % D];
        }
        p.partial[(size_t)blockIdx.x * 2 * D + i] = sum;
    }
}

// dqw, dkw [D] = sums of the blocks' parts, in the same order every time.  One block per 32 of the 2 D channels, 32 rows of threads.
__global__ void __launch_bounds__(1024) rope_weight_grad_kernel(const float* partial, int blocks, int D, float* dqw, float* dkw) {
    __shared__ float sm[32][33];
    grid_wait();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, i = blockIdx.x * 32 + x;
    float sum = 0.f;
    for (int b = y; b < blocks; b += 32) sum += partial[(size_t)b * 2 * D + i];
    sm[y][x] = sum;
    __syncthreads();
    if (y == 0) {
        sum = 0.f;
        for (int r = 0; r < 32; ++r) sum += sm[r][x];
        float* out = i < D ? dqw : dkw;
        if (out != nullptr) out[i % D] = sum;
    }
}

}  // namespace swaa

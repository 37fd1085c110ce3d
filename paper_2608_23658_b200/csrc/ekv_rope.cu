// ekv_rope_write_kv: what stands between a layer's projection and its attention, in one pass over the rows.
//
//   y = x * rsqrt(mean(x^2) + eps) * (offset + w)                     (queries and keys, if the layer norms them; a row is a head)
//   (a, b) -> factor * (a cos t - b sin t, b cos t + a sin t)          (pairs of channels), t = position[axis of the pair] * inv_freq[pair]
//   queries -> q_out, keys and values -> their slots of the cache      (rounded to bf16 once, at the end)
//
// Bound by memory: every element is read once and written once, and 768 bytes of a row's arithmetic hide behind it.  A row of head_dim
// channels belongs to D / 8 neighbouring lanes, 16 bytes each, so that the sum of squares and the exchange of a pair's halves are shuffles.
// A CTA takes one or a few whole tokens: their sines and cosines are worked out once, into shared memory, for all heads, while the
// first rows are on their way.  The angle is taken in turns in 64 bits (position * inv_freq needs up to 55 bits; in fp32 a position of 10^6
// would be off by 0.06 rad) and only its fraction goes to sincospi.
#include <cuda_bf16.h>

#include "ekv_internal.h"
#include "ptx.cuh"

namespace ekv {

static constexpr int kRopeThreads = 256;
static constexpr int kRopeUnroll = 4;      // rows a thread has under way
static constexpr int kRopeMaxTokens = 4;   // of a CTA

enum RopeStyle { kHalves = 0, kAdjacent = 1, kHalvesAnywhere = 2 };  // the last: halves that do not begin at a multiple of 8 channels

struct RopeParams {
    const __nv_bfloat16 *q, *k, *v;
    __nv_bfloat16 *q_out;
    __nv_bfloat16 *k_out;   // 8-bit pools: the finished keys go here, and values nowhere
    uint8_t *cache;
    const long long *slots;
    const int *positions;
    const float *inv_freq;
    const __nv_bfloat16 *q_weight, *k_weight;  // null: no norm
    const long long *live;
    unsigned *status;
    long long q_stride, k_stride, v_stride, q_out_stride;  // elements between tokens
    long long block_stride;
    int T, num_q_heads, num_kv_heads, pairs, tokens;  // tokens: of a CTA
    float eps, offset, factor;
    uint8_t axis[64];
};

__device__ __forceinline__ float2 bf16x2_to_float2(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }

template <int D, int kStyle>
__global__ void __launch_bounds__(kRopeThreads) rope_write_kernel(const __grid_constant__ RopeParams p) {
    constexpr int kLanes = D / 8;  // of a row
    constexpr int kRows = kRopeThreads / kLanes;
    __shared__ float2 turn[kRopeMaxTokens][D / 2];
    __shared__ float2 row_of[kStyle == kHalvesAnywhere ? kRopeThreads * 4 : 1];  // each thread's 8 channels
    const int lane = threadIdx.x % kLanes, first = threadIdx.x / kLanes;
    const int per_token = p.num_q_heads + (p.k_out ? 1 : 2) * p.num_kv_heads;
    const int t0 = blockIdx.x * p.tokens;
    const int n_tokens = min(p.tokens, p.T - t0), n_rows = n_tokens * per_token;
    const long long live = *p.live;

    uint4 x[kRopeUnroll];
    int tok[kRopeUnroll], head[kRopeUnroll];
    auto load = [&](int r0) {
#pragma unroll
        for (int u = 0; u < kRopeUnroll; ++u) {
            const int r = r0 + u * kRows;
            tok[u] = -1;
            if (r >= n_rows) continue;
            const int i = r / per_token, h = r - i * per_token;
            tok[u] = i;
            head[u] = h;
            const long long t = t0 + i;
            const __nv_bfloat16 *from = h < p.num_q_heads ? p.q + t * p.q_stride + h * D
                                        : h < p.num_q_heads + p.num_kv_heads ? p.k + t * p.k_stride + (h - p.num_q_heads) * D
                                                                              : p.v + t * p.v_stride + (h - p.num_q_heads - p.num_kv_heads) * D;
            x[u] = reinterpret_cast<const uint4 *>(from)[lane];
        }
    };
    load(first);
    for (int i = threadIdx.x; i < n_tokens * p.pairs; i += kRopeThreads) {
        const int t = i / p.pairs, pair = i - t * p.pairs;
        const double turns = (double)p.positions[(long long)p.axis[pair] * p.T + t0 + t] * (double)p.inv_freq[pair] * 0.15915494309189535;
        float s, c;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        turn[t][pair] = make_float2(c * p.factor, s * p.factor);
    }
    __syncthreads();
    // (the bound is the same for all threads: the shuffles below need whole warps)
    for (int r0 = 0; r0 < n_rows; r0 += kRows * kRopeUnroll) {
        if (r0 > 0) load(r0 + first);
#pragma unroll
        for (int u = 0; u < kRopeUnroll; ++u) {
            const int h = tok[u] < 0 ? 0 : head[u], i = max(tok[u], 0);
            const bool is_q = h < p.num_q_heads, is_v = h >= p.num_q_heads + p.num_kv_heads;
            const long long t = t0 + i;
            if (tok[u] < 0) x[u] = make_uint4(0u, 0u, 0u, 0u);
            const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
            float y[8];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float2 a = bf16x2_to_float2(w[c]);
                y[2 * c] = a.x, y[2 * c + 1] = a.y;
            }
            if (p.q_weight || p.k_weight) {
                float sum = 0.f;
#pragma unroll
                for (int c = 0; c < 8; ++c) sum += y[c] * y[c];
#pragma unroll
                for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                const __nv_bfloat16 *weight = is_q ? p.q_weight : p.k_weight;
                if (weight && !is_v) {
                    const float f = rsqrtf(sum * (1.f / D) + p.eps);
                    const uint4 g = reinterpret_cast<const uint4 *>(weight)[lane];
                    const uint32_t gw[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const float2 a = bf16x2_to_float2(gw[c]);
                        y[2 * c] *= f * (p.offset + a.x), y[2 * c + 1] *= f * (p.offset + a.y);
                    }
                }
            }
            if (kStyle == kAdjacent) {
                if (!is_v) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int pair = 4 * lane + c;
                        if (pair < p.pairs) {
                            const float2 cs = turn[i][pair];
                            const float a = y[2 * c], b = y[2 * c + 1];
                            y[2 * c] = a * cs.x - b * cs.y, y[2 * c + 1] = b * cs.x + a * cs.y;
                        }
                    }
                }
            } else if (kStyle == kHalves) {
                const int half = p.pairs / 8;  // lanes that hold first channels of pairs; as many behind them hold the second ones
                const bool low = lane < half, there = lane < 2 * half;
                float other[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) other[c] = __shfl_sync(0xffffffffu, y[c], low ? lane + half : lane - half, kLanes);
                if (there && !is_v) {
                    const float2 *cs = &turn[i][8 * (low ? lane : lane - half)];
#pragma unroll
                    for (int c = 0; c < 8; ++c) y[c] = y[c] * cs[c].x + (low ? -other[c] : other[c]) * cs[c].y;
                }
            } else {
                float *mine = reinterpret_cast<float *>(row_of) + (threadIdx.x - lane) * 8;  // the row of this thread's lanes
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 8; ++c) mine[8 * lane + c] = y[c];
                __syncwarp();
                if (!is_v) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const int ch = 8 * lane + c;
                        if (ch < 2 * p.pairs) {
                            const bool low = ch < p.pairs;
                            const float2 cs = turn[i][low ? ch : ch - p.pairs];
                            const float other = mine[low ? ch + p.pairs : ch - p.pairs];
                            y[c] = y[c] * cs.x + (low ? -other : other) * cs.y;
                        }
                    }
                }
            }
            if (tok[u] < 0) continue;
            const uint4 out = is_v ? x[u] : make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
            if (is_q) {
                reinterpret_cast<uint4 *>(p.q_out + t * p.q_out_stride + h * D)[lane] = out;
                continue;
            }
            const int kv_row = h - p.num_q_heads;  // K heads, then V heads: as they lie in a block
            if (p.k_out) {
                if (!is_v) reinterpret_cast<uint4 *>(p.k_out + (t * p.num_kv_heads + kv_row) * D)[lane] = out;
                continue;
            }
            const long long s = p.slots[t];
            if (s < 0) continue;
            const long long n = s >> 4;
            if (n >= live) {
                if (kv_row == 0 && lane == 0) atomicOr(p.status, EKV_DEV_FLAG_OOB);
                continue;
            }
            reinterpret_cast<uint4 *>(p.cache + n * p.block_stride + (kv_row * 16 + (int)(s & 15)) * (2 * D))[lane] = out;
        }
    }
}

template <int D>
static cudaError_t launch_rope(const RopeParams &p, bool adjacent, cudaStream_t stream) {
    const unsigned grid = (unsigned)(((long long)p.T + p.tokens - 1) / p.tokens);
    if (adjacent) rope_write_kernel<D, kAdjacent><<<grid, kRopeThreads, 0, stream>>>(p);
    else if (p.pairs % 8 == 0) rope_write_kernel<D, kHalves><<<grid, kRopeThreads, 0, stream>>>(p);
    else rope_write_kernel<D, kHalvesAnywhere><<<grid, kRopeThreads, 0, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace ekv

using namespace ekv;

extern "C" ekv_status_t ekv_rope_write_kv(ekv_pool_t *pool, int32_t layer, const ekv_rope_t *rope, const void *q, int64_t q_stride,
                                          const void *k, int64_t k_stride, const void *v, int64_t v_stride, void *q_out, int64_t q_out_stride,
                                          void *k_out, const int64_t *slot_mapping, int32_t T, void *stream) {
    ekv_status_t st = check_compute(pool, layer, "ekv_rope_write_kv");
    if (st != EKV_OK) return st;
    const int D = pool->desc.head_dim, Hq = pool->desc.num_q_heads, Hk = pool->desc.num_kv_heads;
    if (!rope || T < 0 || rope->rotary_dim < 0 || rope->rotary_dim > D || (rope->rotary_dim & 1) || rope->num_axes < 1 || rope->num_axes > 4 ||
        (rope->flags & ~(uint32_t)EKV_ROPE_ADJACENT) || (rope->num_axes > 1 && rope->rotary_dim > 0 && !rope->pair_axis) || !(rope->eps >= 0.f)) {
        set_error("ekv_rope_write_kv: bad rotation (rotary_dim=%d, num_axes=%d, flags=%u) or T=%d", rope ? rope->rotary_dim : -1,
                  rope ? rope->num_axes : -1, rope ? rope->flags : 0u, T);
        return EKV_ERR_INVALID;
    }
    for (int i = 0; rope->num_axes > 1 && i < rope->rotary_dim / 2; ++i)
        if (rope->pair_axis[i] >= rope->num_axes) {
            set_error("ekv_rope_write_kv: pair %d turns by axis %d of %d", i, rope->pair_axis[i], rope->num_axes);
            return EKV_ERR_INVALID;
        }
    if (T == 0) return EKV_OK;
    const uintptr_t at = (uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out | (uintptr_t)k_out | (uintptr_t)rope->q_weight | (uintptr_t)rope->k_weight;
    if (!q || !k || !v || !q_out || !slot_mapping || (rope->rotary_dim > 0 && (!rope->inv_freq || !rope->positions)) || (at & 15) ||
        ((q_stride | k_stride | v_stride | q_out_stride) & 7)) {
        set_error("ekv_rope_write_kv: bad argument (q=%p, k=%p, v=%p, q_out=%p, slot_mapping=%p, inv_freq=%p, positions=%p; rows and weights on 16-byte boundaries)",
                  q, k, v, q_out, (const void *)slot_mapping, (const void *)rope->inv_freq, (const void *)rope->positions);
        return EKV_ERR_INVALID;
    }
    if (T > 1 && (q_stride < (int64_t)Hq * D || q_out_stride < (int64_t)Hq * D || k_stride < (int64_t)Hk * D || v_stride < (int64_t)Hk * D)) {
        set_error("ekv_rope_write_kv: rows of different tokens overlap (strides %lld, %lld, %lld, %lld)", (long long)q_stride, (long long)k_stride,
                  (long long)v_stride, (long long)q_out_stride);
        return EKV_ERR_INVALID;
    }
    if (pool->e4m3() != (k_out != nullptr)) {
        set_error("ekv_rope_write_kv: k_out is for EKV_E4M3 pools, and needed there");
        return EKV_ERR_INVALID;
    }
    RopeParams p;
    p.q = (const __nv_bfloat16 *)q, p.k = (const __nv_bfloat16 *)k, p.v = (const __nv_bfloat16 *)v;
    p.q_out = (__nv_bfloat16 *)q_out, p.k_out = (__nv_bfloat16 *)k_out;
    p.cache = (uint8_t *)pool->layer_base(layer);
    p.slots = (const long long *)slot_mapping;
    p.positions = rope->positions, p.inv_freq = rope->inv_freq;
    p.q_weight = (const __nv_bfloat16 *)rope->q_weight, p.k_weight = (const __nv_bfloat16 *)rope->k_weight;
    p.live = pool->d_live, p.status = pool->d_status;
    p.q_stride = q_stride, p.k_stride = k_stride, p.v_stride = v_stride, p.q_out_stride = q_out_stride;
    p.block_stride = (long long)pool->block_stride;
    p.T = T, p.num_q_heads = Hq, p.num_kv_heads = Hk, p.pairs = rope->rotary_dim / 2;
    p.eps = rope->eps, p.offset = rope->weight_offset, p.factor = rope->factor;
    for (int i = 0; i < 64; ++i) p.axis[i] = rope->num_axes > 1 && i < p.pairs ? rope->pair_axis[i] : 0;
    // A CTA's tokens share its start (positions, angles); with few tokens every one gets a CTA of its own.
    p.tokens = 1;
    while (p.tokens < kRopeMaxTokens && (long long)T >= (long long)pool->sm_count * 8 * 2 * p.tokens) p.tokens *= 2;
    const cudaError_t e = D == 128 ? launch_rope<128>(p, rope->flags & EKV_ROPE_ADJACENT, (cudaStream_t)stream)
                                   : launch_rope<64>(p, rope->flags & EKV_ROPE_ADJACENT, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail(e, "ekv_rope_write_kv launch");
    if (pool->e4m3()) return write_kv8(pool, layer, k_out, (int64_t)Hk * D, v, v_stride, slot_mapping, T, (cudaStream_t)stream);
    return EKV_OK;
}

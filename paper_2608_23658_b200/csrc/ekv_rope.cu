// ekv_rope_write_kv: what stands between a layer's projection and its attention, in one pass over the rows.
//
//   y = x * rsqrt(mean(x^2) + eps) * (offset + w)                     (queries and keys, if the layer norms them; a row is a head)
//   (a, b) -> factor * (a cos t - b sin t, b cos t + a sin t)          (pairs of channels), t = position[axis of the pair] * inv_freq[pair]
//   queries -> q_out, keys and values -> their slots of the cache      (rounded to bf16 once, at the end)
//
// Every element is read once and written once: 403 MB for 16384 tokens of 32q/8kv, 76 to 80 us = 5.0 to 5.3 TB/s of the 6.5 that a copy gets; the
// arithmetic between takes two thirds of the issue slots and is what keeps it from the rest.  2049 tokens of 28q/4kv 11 us, 256 of 32q/8kv 4, 31 of
// 4q/2kv 3, on the device.
// A row of head_dim channels belongs to D / 16 neighbouring lanes, two pieces of 16 bytes each; where pairs are halves of a row the pieces are
// chosen so that both channels of a pair are in one thread, so a rotation is register arithmetic and only the sum of squares is shuffled.
// (With one piece a thread, and the partners' values by shuffles: 16384 tokens of 32q/8kv 119 us.)  A CTA takes some whole tokens: their sines
// and cosines are worked out once, into shared memory, for all heads, while the first rows are on their way, and the next rows are always on
// theirs.  The angle is taken in turns in 64 bits (position * inv_freq needs up to 55 bits; in fp32 a position of 10^6 would be off by 0.06 rad) and
// only its fraction is turned into a sine and a cosine.
#include <cuda_bf16.h>

#include <algorithm>

#include "ekv_internal.h"
#include "ptx.cuh"

namespace ekv {

static constexpr int kRopeThreads = 128;
static constexpr int kRopeCtas = 4;        // an SM
static constexpr int kRopeUnroll = 3;      // rows a thread works on, with as many of the next token under way
static constexpr int kRopeTokens = 16;     // tokens whose angles a CTA works out at a time

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
    int T, num_q_heads, num_kv_heads, pairs;
    float eps, offset, factor;
    uint8_t axis[64];
};


// Two fp32 side by side in 64 bits.  (Through the intrinsics on float2 the halves were moved about between the operations.)
typedef unsigned long long Pair;
__device__ __forceinline__ Pair pair_of(float lo, float hi) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 halves(Pair a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a));
    return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint32_t to_bf16x2(Pair a) {
    const float2 v = halves(a);
    return pack_bf16x2(v.x, v.y);
}

template <int D, int kStyle>
__global__ void __launch_bounds__(kRopeThreads, kRopeCtas) rope_write_kernel(const __grid_constant__ RopeParams p) {
    constexpr int kLanes = D / 16;  // of a row
    constexpr int kRows = kRopeThreads / kLanes, kStep = kRows * kRopeUnroll;
    __shared__ __align__(16) float2 turn[kRopeTokens][D / 2];
    __shared__ __align__(16) float weights[2][D];
    __shared__ __align__(16) float row_of[kStyle == kHalvesAnywhere ? kRopeThreads * 16 : 4];  // each thread's 16 channels
    const int lane = threadIdx.x % kLanes, first = threadIdx.x / kLanes;
    const int q_heads = p.num_q_heads, qk_heads = q_heads + p.num_kv_heads, per_token = p.k_out ? qk_heads : qk_heads + p.num_kv_heads;
    const int t0 = (int)((long long)p.T * blockIdx.x / gridDim.x), n_tokens = (int)((long long)p.T * (blockIdx.x + 1) / gridDim.x) - t0;
    const int base = blockIdx.y * kStep;  // this CTA's rows of every token: base .. base + kStep - 1
    const long long live = *p.live;
    // This thread's two pieces of a row.  Halves: the first channels of eight pairs and the second ones, or what lies behind the pairs.
    const int half = kStyle == kHalves ? p.pairs / 8 : kLanes;
    const bool turns = lane < half;
    const int piece0 = turns ? lane : 2 * half + 2 * (lane - half), piece1 = turns ? lane + half : piece0 + 1;

    // The thread's rows stand at the same heads of every token, so their addresses only step.  The next token's are on their way while one's
    // are worked on.
    const uint4 *src[kRopeUnroll];
    uint4 x[kRopeUnroll][2], next[kRopeUnroll][2];
    auto stride_of = [&](int h) { return h < q_heads ? p.q_stride : h < qk_heads ? p.k_stride : p.v_stride; };
#pragma unroll
    for (int u = 0; u < kRopeUnroll; ++u) {
        const int h = min(base + first + u * kRows, per_token - 1);
        const __nv_bfloat16 *row = h < q_heads ? p.q + h * D : h < qk_heads ? p.k + (h - q_heads) * D : p.v + (h - qk_heads) * D;
        src[u] = reinterpret_cast<const uint4 *>(row + t0 * stride_of(h)) + piece0;
    }
    auto load = [&]() {
#pragma unroll
        for (int u = 0; u < kRopeUnroll; ++u) {
            next[u][0] = src[u][0];
            next[u][1] = src[u][piece1 - piece0];
            src[u] += stride_of(min(base + first + u * kRows, per_token - 1)) / 8;  // (a thread without a row takes the last one)
        }
    };
    load();
    const bool norms = p.q_weight || p.k_weight;
    for (int i = threadIdx.x; norms && i < 2 * D; i += kRopeThreads) {
        const __nv_bfloat16 *w = i < D ? p.q_weight : p.k_weight;
        weights[i / D][i % D] = w ? p.offset + __bfloat162float(w[i % D]) : 1.f;
    }
    // A thread works out the angles of one pair, of every kAngleRows-th token.  (|error| of the fast sine and cosine within half a turn: some 2^-21, so
    // some 2^-20 of the larger channel of the pair in the result, however small that comes out; the rounding to bf16 is up to 2^-8 of the result.)
    constexpr int kAngleRows = kRopeThreads / (D / 2);
    const int pair = threadIdx.x % (D / 2);
    const bool has_pair = pair < p.pairs;
    const double turns_per = has_pair ? (double)p.inv_freq[pair] * 0.15915494309189535 : 0.;
    const int *position = p.positions + (has_pair ? (long long)p.axis[pair] * p.T + t0 : 0);
    // (halves: eight pairs of a thread, laid out so that neighbouring lanes read neighbouring words)
    const int angle_at = kStyle == kHalves ? pair % 8 / 2 * (2 * half) + pair / 8 * 2 + pair % 2 : pair;
    auto angles = [&](int from) {  // of the tokens from there on
        const int n = has_pair ? min(kRopeTokens, n_tokens - from) : 0;
#pragma unroll 4
        for (int t = threadIdx.x / (D / 2); t < n; t += kAngleRows) {
            const double a = (double)position[from + t] * turns_per;
            const float b = (float)(a - rint(a)) * 6.283185307179586f;
            turn[t][angle_at] = make_float2(__cosf(b) * p.factor, __sinf(b) * p.factor);
        }
    };
    Pair cos2[4], sin2[4], minus[4];  // halves: of this thread's eight pairs, two at a time
    long long slot = p.k_out ? -1 : p.slots[t0];
    __nv_bfloat16 *q_to = p.q_out + t0 * p.q_out_stride;
    for (int i = 0; i < n_tokens; ++i, q_to += p.q_out_stride) {
        const int in_batch = i % kRopeTokens;
        if (in_batch == 0) {
            if (i > 0) __syncthreads();
            angles(i);
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < kRopeUnroll; ++u) x[u][0] = next[u][0], x[u][1] = next[u][1];
        if (i + 1 < n_tokens) load();
        const long long s = slot;
        if (i + 1 < n_tokens && !p.k_out) slot = p.slots[t0 + i + 1];
        __nv_bfloat16 *kv_to = nullptr;  // the token's first K row; a row of another head lies kv_step further on
        const int kv_step = p.k_out ? D : 16 * D;
        if (p.k_out) kv_to = p.k_out + (long long)(t0 + i) * p.num_kv_heads * D;
        else if (s >= 0 && (s >> 4) < live) kv_to = reinterpret_cast<__nv_bfloat16 *>(p.cache + (s >> 4) * p.block_stride) + (int)(s & 15) * D;
        else if (s >= 0 && threadIdx.x == 0) atomicOr(p.status, EKV_DEV_FLAG_OOB);
        if (kStyle == kHalves && turns) {  // a token's angles stay in registers for all its rows
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float4 a = *reinterpret_cast<const float4 *>(&turn[in_batch][c * (2 * half) + lane * 2]);
                cos2[c] = pair_of(a.x, a.z), sin2[c] = pair_of(a.y, a.w), minus[c] = pair_of(-a.y, -a.w);
            }
        }
        // All rows' sums side by side: one alone is a chain of shuffles and a root that nothing hides (16384 tokens of 32q/8kv one by one: 89 us).
        float f[kRopeUnroll];
        if (norms) {
#pragma unroll
            for (int u = 0; u < kRopeUnroll; ++u) {
                const uint32_t w[8] = {x[u][0].x, x[u][0].y, x[u][0].z, x[u][0].w, x[u][1].x, x[u][1].y, x[u][1].z, x[u][1].w};
                Pair sum = 0;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const Pair y = pair_of(__uint_as_float(w[c] << 16), __uint_as_float(w[c] & 0xffff0000u));
                    sum = fma2(y, y, sum);
                }
                f[u] = halves(sum).x + halves(sum).y;
            }
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1)
#pragma unroll
                for (int u = 0; u < kRopeUnroll; ++u) f[u] += __shfl_xor_sync(0xffffffffu, f[u], o);
#pragma unroll
            for (int u = 0; u < kRopeUnroll; ++u) {
                const float g = rsqrtf(f[u] * (1.f / D) + p.eps);
                f[u] = (base + first + u * kRows < q_heads ? p.q_weight : p.k_weight) ? g : 1.f;
            }
        }
#pragma unroll
        for (int u = 0; u < kRopeUnroll; ++u) {
            const int h = base + first + u * kRows;
            const uint32_t w[8] = {x[u][0].x, x[u][0].y, x[u][0].z, x[u][0].w, x[u][1].x, x[u][1].y, x[u][1].z, x[u][1].w};
            Pair y[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) y[c] = pair_of(__uint_as_float(w[c] << 16), __uint_as_float(w[c] & 0xffff0000u));
            if (norms) {
                const Pair f2 = pair_of(f[u], f[u]);
                const ulonglong2 *g = reinterpret_cast<const ulonglong2 *>(weights[h < q_heads ? 0 : 1]);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const ulonglong2 a = g[(c < 2 ? piece0 : piece1) * 2 + c % 2];
                    y[2 * c] = mul2(mul2(y[2 * c], f2), a.x), y[2 * c + 1] = mul2(mul2(y[2 * c + 1], f2), a.y);
                }
            }
            if (kStyle == kHalves) {
                if (turns) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const Pair a = y[c], b = y[4 + c];
                        y[c] = fma2(b, minus[c], mul2(a, cos2[c]));
                        y[4 + c] = fma2(a, sin2[c], mul2(b, cos2[c]));
                    }
                }
            } else if (kStyle == kAdjacent) {
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const int pair = 4 * (c < 4 ? piece0 : piece1) + c % 4;
                    if (pair < p.pairs) {
                        const float2 cs = turn[in_batch][pair], a = halves(y[c]);
                        y[c] = pair_of(a.x * cs.x - a.y * cs.y, a.y * cs.x + a.x * cs.y);
                    }
                }
            } else {
                float *mine = row_of + (threadIdx.x - lane) * 16;  // the row of this thread's lanes
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 8; ++c) *reinterpret_cast<float2 *>(mine + 8 * (c < 4 ? piece0 : piece1) + 2 * (c % 4)) = halves(y[c]);
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const int ch0 = 8 * (c < 4 ? piece0 : piece1) + 2 * (c % 4);
                    auto turned = [&](int ch, float own) {
                        if (ch >= 2 * p.pairs) return own;
                        const bool lower = ch < p.pairs;
                        const float2 a = turn[in_batch][lower ? ch : ch - p.pairs];
                        const float other = mine[lower ? ch + p.pairs : ch - p.pairs];
                        return own * a.x + (lower ? -other : other) * a.y;
                    };
                    const float2 own = halves(y[c]);
                    y[c] = pair_of(turned(ch0, own.x), turned(ch0 + 1, own.y));
                }
            }
            __nv_bfloat16 *row = h < q_heads ? q_to + h * D : kv_to ? kv_to + (h - q_heads) * kv_step : nullptr;  // K heads, then V heads: as they lie in a block
            if (!row || h >= per_token) continue;
            uint4 *to = reinterpret_cast<uint4 *>(row);
            if (h >= qk_heads) {
                to[piece0] = x[u][0];
                to[piece1] = x[u][1];
            } else {
                to[piece0] = make_uint4(to_bf16x2(y[0]), to_bf16x2(y[1]), to_bf16x2(y[2]), to_bf16x2(y[3]));
                to[piece1] = make_uint4(to_bf16x2(y[4]), to_bf16x2(y[5]), to_bf16x2(y[6]), to_bf16x2(y[7]));
            }
        }
    }
}

template <int D>
static cudaError_t launch_rope(const RopeParams &p, int sm_count, bool adjacent, cudaStream_t stream) {
    constexpr int kStep = kRopeThreads / (D / 16) * kRopeUnroll;
    const int per_token = p.num_q_heads + (p.k_out ? 1 : 2) * p.num_kv_heads;
    const int steps = (per_token + kStep - 1) / kStep, fit = std::max(1, sm_count * kRopeCtas / steps);
    const dim3 grid(std::min(p.T, fit), steps);  // CTAs that are all there at once share the tokens evenly
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
        (T > 1 && ((q_stride | k_stride | v_stride | q_out_stride) & 7))) {
        set_error("ekv_rope_write_kv: bad argument (q=%p, k=%p, v=%p, q_out=%p, slot_mapping=%p, inv_freq=%p, positions=%p; rows and weights on 16-byte boundaries)",
                  q, k, v, q_out, (const void *)slot_mapping, (const void *)rope->inv_freq, (const void *)rope->positions);
        return EKV_ERR_INVALID;
    }
    if (T > 1 && (q_stride < (int64_t)Hq * D || q_out_stride < (int64_t)Hq * D || k_stride < (int64_t)Hk * D || v_stride < (int64_t)Hk * D ||
                  (q == q_out && q_stride != q_out_stride))) {
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
    const cudaError_t e = D == 128 ? launch_rope<128>(p, pool->sm_count, rope->flags & EKV_ROPE_ADJACENT, (cudaStream_t)stream)
                                   : launch_rope<64>(p, pool->sm_count, rope->flags & EKV_ROPE_ADJACENT, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail(e, "ekv_rope_write_kv launch");
    if (pool->e4m3()) return write_kv8(pool, layer, k_out, (int64_t)Hk * D, v, v_stride, slot_mapping, T, (cudaStream_t)stream);
    return EKV_OK;
}

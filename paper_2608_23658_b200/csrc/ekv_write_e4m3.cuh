// ekv_write_kv on an 8-bit pool: rows of bf16 -> e4m3 codes with one power-of-two scale per (block, K|V, kv-head).
//
//   e = min{ e : max|x| <= 448 * 2^e },  s = max(old, 2^e),  code(x) = rne(x / s),  kept codes *= old / s  (rne again)
//
// The scale ties all tokens of a block together, so the unit of work is a BLOCK the call names, not a token: one
// CTA finds the block's tokens in the slot mapping, and each of its warps takes (K|V, head) pairs whole -- 16 rows of
// head_dim channels, at most 4 KiB, held in registers between the maximum and the conversion, so a row is read once
// and nothing is shared between warps.  A slot mapping may be in any order; the CTA that does a block's work
// is the one of its first token in the mapping:
//   T <= kScanTokens   one launch, a CTA per token; each looks through the whole mapping (8 KiB at most, from L2) for its block
//   more               a first launch leaves the range [first, last] of every block's tokens in two words per block
//                      (atomic maxima: no order matters), the second takes 16 tokens a CTA, does the blocks that begin
//                      there and puts their words back to zero
// Measured, 8 kv-heads of 128, write and read_kv together, us: 1024 tokens in a row 11.6 by the first form and 13.0 by the second, one
// token a block 23 and 43; 2048 in a row 16.6 and 14.1, one token a block 46 and 58.  So the second form is for long prompts.  Its tasks each
// look through the mapping from their block's first token to its last: nothing for runs, T squared for blocks whose tokens are spread
// over the call (16384 shuffled tokens, 8 kv-heads of 128: 0.97 ms for 31 us with the call's launches).
// 16384 tokens (101 MB: 4 bytes in and 2 out a channel pair of K and V, scales and mapping beside it) take 28.3 us = 3.6 TB/s, 4.7 of it the
// claims.  Not bound by memory (device memory is 29 % busy): a warp's chain of mapping, claim, row, maximum and store, gone through
// once, with half the issue slots taken.  256 tokens 5.8 us, a launch and four loads that wait for one another (slot, mapping, row and
// scale, then the rounding).
#pragma once
#include "e4m3.cuh"
#include "ekv_internal.h"

namespace ekv {

static constexpr int kW8Threads = 256;
static constexpr int kW8Warps = kW8Threads / 32;
static constexpr int kW8ClaimedThreads = 512;  // a warp for each (K|V, head) of a block with 8 kv-heads: all its rows are on their way at once
static constexpr int kW8TokensPerCta = 16;
static constexpr int kScanTokens = 1024;

struct Write8Params {
    uint8_t *cache;         // layer base
    float *scales;          // of the layer: [block][2][Hk]
    int2 *claims;           // of the layer: [block]
    const uint4 *k, *v;
    const long long *slots;
    const long long *live;
    unsigned *status;
    long long block_stride;
    int T, num_kv_heads;
};

// One (block, K|V, head): tok[t] = 1 + index of the row for slot t of the block, or 0.
template <int D>
__device__ __forceinline__ void write8_task(const Write8Params &p, long long n, int kv, int h, const int *tok, int lane) {
    constexpr int kLanesPerRow = D / 8;  // 8 channels a lane: 16 bytes of bf16, 8 of codes
    constexpr int kRows = 32 / kLanesPerRow;
    constexpr int kIts = 16 / kRows;
    const int sub = lane / kLanesPerRow, piece = lane % kLanesPerRow;
    const uint4 *src = (kv ? p.v : p.k) + (long long)h * kLanesPerRow + piece;
    const long long row_pieces = (long long)p.num_kv_heads * kLanesPerRow;
    float *scale_at = p.scales + (n * 2 + kv) * p.num_kv_heads + h;
    const float old = tok[0] ? 0.f : *scale_at;
    uint4 x[kIts];
    uint32_t m2 = 0;  // maxima of the magnitudes, two channels side by side (magnitudes of bf16 are ordered as integers)
#pragma unroll
    for (int it = 0; it < kIts; ++it) {
        const int t = tok[it * kRows + sub];
        x[it] = t ? __ldg(src + (t - 1) * row_pieces) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int it = 0; it < kIts; ++it) {
        m2 = __vmaxu2(m2, __vmaxu2(__vmaxu2(x[it].x & 0x7fff7fffu, x[it].y & 0x7fff7fffu), __vmaxu2(x[it].z & 0x7fff7fffu, x[it].w & 0x7fff7fffu)));
    }
    uint32_t m = max(m2 & 0xffffu, m2 >> 16);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    const bool nonfinite = m >= 0x7f80u;  // same in every lane
    if (nonfinite) {  // the maximum again, over the finite ones
        m = 0;
#pragma unroll
        for (int it = 0; it < kIts; ++it) {
            const uint32_t w[4] = {x[it].x, x[it].y, x[it].z, x[it].w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t a = (w[i >> 1] >> (16 * (i & 1))) & 0x7fffu;
                if (a < 0x7f80u) m = max(m, a);
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    }
    const float s = fmaxf(old, scale_of_bf16_bits(m));
    const float inv = pow2_inverse(s);
    const bool special = nonfinite || s >= kMaxScale;
    uint8_t *tile = p.cache + n * p.block_stride + (long long)(kv * p.num_kv_heads + h) * (16 * D);
#pragma unroll
    for (int it = 0; it < kIts; ++it) {
        const int row = it * kRows + sub;
        if (!tok[row]) continue;
        const uint32_t w[4] = {x[it].x, x[it].y, x[it].z, x[it].w};
        uint32_t c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a = __uint_as_float(w[i] << 16) * inv, b = __uint_as_float(w[i] & 0xffff0000u) * inv;
            if (special) {  // 256 * 2^120 is not a finite bf16, and a conversion would make 448 of an infinity
                const uint32_t la = w[i] & 0x7fffu, lb = (w[i] >> 16) & 0x7fffu;
                if (s >= kMaxScale) a = fminf(fmaxf(a, -240.f), 240.f), b = fminf(fmaxf(b, -240.f), 240.f);
                if (la >= 0x7f80u) a = __uint_as_float(0x7fffffffu);
                if (lb >= 0x7f80u) b = __uint_as_float(0x7fffffffu);
            }
            c[i] = floats_to_e4m3x2(a, b);
        }
        *reinterpret_cast<uint2 *>(tile + row * D + piece * 8) = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
    }
    if (s > old) {
        if (old > 0.f) {  // the scale rises: the codes that stay are brought to it
            const float f = __uint_as_float(__float_as_uint(old) & 0x7f800000u) * inv;  // 2^(old - new); an underflow to 0 is what rounding gives too
#pragma unroll
            for (int it = 0; it < kIts; ++it) {
                const int row = it * kRows + sub;
                if (tok[row]) continue;
                uint2 *at = reinterpret_cast<uint2 *>(tile + row * D + piece * 8);
                const uint2 v = *at;
                const uint32_t w[2] = {v.x, v.y};
                uint32_t c[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float2 a = f16x2_to_float2(e4m3_lo(w[i])), b = f16x2_to_float2(e4m3_hi(w[i]));
                    c[i] = floats_to_e4m3x2(a.x * f, a.y * f) | floats_to_e4m3x2(b.x * f, b.y * f) << 16;
                }
                *at = make_uint2(c[0], c[1]);
            }
        }
        if (lane == 0) *scale_at = s;
    }
}

template <int D>
__device__ __forceinline__ void write8_block(const Write8Params &p, long long n, const int *tok) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = warp; i < 2 * p.num_kv_heads; i += kW8Warps) {
        const int kv = i >= p.num_kv_heads;
        write8_task<D>(p, n, kv, i - kv * p.num_kv_heads, tok, lane);
    }
}

// A CTA per token: goes on only for the first token of its block.
template <int D>
__global__ void __launch_bounds__(kW8Threads) write8_scan_kernel(const Write8Params p) {
    __shared__ int tok[16];
    __shared__ int earlier;
    const int t = blockIdx.x;
    const long long s = p.slots[t];
    if (s < 0) return;
    const long long n = s >> 4;
    if (n >= *p.live) {
        if (threadIdx.x == 0) atomicOr(p.status, EKV_DEV_FLAG_OOB);
        return;
    }
    if (threadIdx.x < 16) tok[threadIdx.x] = 0;
    if (threadIdx.x == 16) earlier = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < p.T; i += kW8Threads) {
        const long long o = p.slots[i];
        if (o >= 0 && (o >> 4) == n) {
            if (i < t) earlier = 1;
            atomicMax(&tok[(int)(o & 15)], i + 1);  // of duplicate slots the last one
        }
    }
    __syncthreads();
    if (earlier) return;
    write8_block<D>(p, n, tok);
}

// claims[n] = {T - first token, last token + 1} of block n, both by atomic maximum over zeros
__global__ void __launch_bounds__(256) write8_claim_kernel(const Write8Params p) {
    const int t = blockIdx.x * 256 + threadIdx.x;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (t >= p.T) return;
    const long long s = p.slots[t];
    if (s < 0) return;
    const long long n = s >> 4;
    if (n >= *p.live) {
        atomicOr(p.status, EKV_DEV_FLAG_OOB);
        return;
    }
    atomicMax(&p.claims[n].x, p.T - t);
    atomicMax(&p.claims[n].y, t + 1);
}

// A CTA takes the blocks that begin in its 16 tokens; its warps share out their (block, K|V, head) tasks.  Everything a warp needs
// to know it works out itself, from the caches: the only meeting is the one after which the claims may go.
template <int D>
__global__ void __launch_bounds__(kW8ClaimedThreads, 2) write8_claimed_kernel(const Write8Params p) {
    __shared__ int tok_of[kW8ClaimedThreads / 32][16];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int t0 = blockIdx.x * kW8TokensPerCta, t = t0 + lane;
    asm volatile("griddepcontrol.wait;" ::: "memory");  // the claims are complete (this launch's CTAs come up beside the last of them)
    bool mine = false;
    int last = 0;
    long long n = -1;
    if (lane < kW8TokensPerCta && t < p.T) {
        const long long s = p.slots[t];
        if (s >= 0 && (s >> 4) < *p.live) {
            n = s >> 4;
            const volatile int2 *c = p.claims + n;
            mine = c->x == p.T - t;  // first token of its block; a block done already reads 0, which no token is
            last = c->y - 1;
        }
    }
    const unsigned mask = __ballot_sync(0xffffffffu, mine);
    __syncthreads();
    if (warp == 0 && mine) p.claims[n] = make_int2(0, 0);
    const int per_block = 2 * p.num_kv_heads, tasks = __popc(mask) * per_block;
    int *tok = tok_of[warp];
    for (int i = warp; i < tasks; i += kW8ClaimedThreads / 32) {
        const int b = i / per_block, pair = i - b * per_block;
        const int lead = (int)__fns(mask, 0, b + 1);  // lane of the b-th block's first token
        const long long block = __shfl_sync(0xffffffffu, n, lead);
        const int to = __shfl_sync(0xffffffffu, last, lead);
        __syncwarp();
        if (lane < 16) tok[lane] = 0;
        __syncwarp();
        for (int k = t0 + lead + lane; k <= to; k += 32) {
            const long long o = p.slots[k];
            if (o >= 0 && (o >> 4) == block) atomicMax(&tok[(int)(o & 15)], k + 1);  // of duplicate slots the last one
        }
        __syncwarp();
        const int kv = pair >= p.num_kv_heads;
        write8_task<D>(p, block, kv, pair - kv * p.num_kv_heads, tok, lane);
    }
}

template <int D>
static ekv_status_t launch_write8(ekv_pool *pool, const Write8Params &p, cudaStream_t stream) {
    if (p.T <= kScanTokens) {
        write8_scan_kernel<D><<<p.T, kW8Threads, 0, stream>>>(p);
    } else {
        write8_claim_kernel<<<(unsigned)(((long long)p.T + 255) / 256), 256, 0, stream>>>(p);
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return cuda_fail(e, "ekv_write_kv: claim launch");
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cfg.gridDim = dim3((unsigned)(((long long)p.T + kW8TokensPerCta - 1) / kW8TokensPerCta));
        cfg.blockDim = dim3(kW8ClaimedThreads);
        cfg.stream = stream;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        e = cudaLaunchKernelEx(&cfg, write8_claimed_kernel<D>, p);
        if (e != cudaSuccess) return cuda_fail(e, "ekv_write_kv launch");
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_fail(e, "ekv_write_kv launch");
    return EKV_OK;
}

}  // namespace ekv

// ekv_write_kv: slot-mapped KV write = exact scatter of bf16 bit patterns into the paged pool.
// HBM-bound copy: every thread moves one 16-byte piece; a token's K (and V) row of one kv-head is
// head_dim*2 contiguous bytes on both sides, so loads and stores are fully coalesced.
// 8-bit pools: ekv_write_e4m3.cuh.  ekv_read_kv, the inverse, is here for both.
#include "e4m3.cuh"
#include "ekv_internal.h"
#include "ekv_write_e4m3.cuh"
#include "ptx.cuh"

namespace ekv {

// One token's K and V rows are 2 * Hkv * (head_dim*2/16) pieces of 16 bytes.  A CTA walks over tokens; its
// threads cover a contiguous chunk of pieces at a time, issuing all loads of the chunk before its stores so
// that several 16-byte requests per thread are in flight.
static constexpr int kWriteThreads = 256;
static constexpr int kWriteUnroll = 4;

__global__ void __launch_bounds__(kWriteThreads) write_kv_kernel(uint4 *__restrict__ cache, const uint4 *__restrict__ k,
                                                                 const uint4 *__restrict__ v,
                                                                 const long long *__restrict__ slot_mapping, int T,
                                                                 int num_kv_heads, int block_size, int block_shift, int pieces_per_row, int row_shift, int token_shift,
                                                                 long long block_stride_pieces,
                                                                 const long long *__restrict__ live_ptr, unsigned *status) {
    const long long live = *live_ptr;
    const int row_pieces = num_kv_heads * pieces_per_row;  // one token's K (or V) over all heads
    const int token_pieces = 2 * row_pieces;
    const long long total = (long long)T * token_pieces;
    // a CTA takes contiguous chunks of kWriteThreads * kWriteUnroll pieces (16 KiB of source rows)
    const long long chunk = (long long)kWriteThreads * kWriteUnroll;
    for (long long base = (long long)blockIdx.x * chunk + threadIdx.x; base < total + threadIdx.x; base += (long long)gridDim.x * chunk) {
        uint4 val[kWriteUnroll];
        long long dst[kWriteUnroll];
        // one 64-bit division per trip; the pieces of the trip are then located with 32-bit arithmetic
        const long long i0 = base / token_pieces;
        const int rem0 = (int)(base - i0 * token_pieces);
#pragma unroll
        for (int u = 0; u < kWriteUnroll; ++u) {
            dst[u] = -1;
            if (base + (long long)u * kWriteThreads >= total) continue;
            const int r = rem0 + u * kWriteThreads;
            int di, rem;
            if (token_shift >= 0) {  // pieces per token a power of two (kv-head count is): no division
                di = r >> token_shift;
                rem = r & (token_pieces - 1);
            } else {
                di = r / token_pieces;
                rem = r - di * token_pieces;
            }
            const long long i = i0 + di;
            const int kv = rem >= row_pieces;
            const int hp = rem - kv * row_pieces;  // head * pieces_per_row + piece
            const int h = hp >> row_shift, c = hp & (pieces_per_row - 1);  // pieces_per_row is 8 or 16
            const long long s = slot_mapping[i];
            if (s < 0) continue;
            const long long n = s >> block_shift;  // block_size is a power of two (checked at pool creation)
            const int t = (int)(s & (block_size - 1));
            if (n >= live) {
                if (rem == 0) atomicOr(status, EKV_DEV_FLAG_OOB);
                continue;
            }
            val[u] = (kv ? v : k)[i * row_pieces + hp];
            dst[u] = n * block_stride_pieces + (((long long)(kv * num_kv_heads + h) * block_size + t) * pieces_per_row) + c;
        }
#pragma unroll
        for (int u = 0; u < kWriteUnroll; ++u)
            if (dst[u] >= 0) cache[dst[u]] = val[u];
    }
}

// ekv_read_kv: a thread takes kReadUnroll pieces of 16 channels of one row each -- 32 bytes of bf16, or 16 codes and their scale --
// and has the loads of all of them on their way before it stores.  A code times a power of two needs 4 significant bits, so the bf16 is
// exact.  Bound by the chain of mapping, codes and scale, gone through once a thread (device memory is 25 % busy on an 8-bit pool).  Outputs on 32-byte boundaries are stored 32 bytes at a time (kWhole).  Measured, 8 kv-heads of 128:
// 16384 tokens from an 8-bit pool (101 MB) 22.3 us = 4.5 TB/s, with two stores of 16 bytes 24.2; 2048 tokens 3.9 and 5.3; from a
// bf16 pool (134 MB) 24.0 = 5.6 TB/s and 26.1.
static constexpr int kReadUnroll = 4;

template <bool kE4m3, bool kWhole>
__global__ void __launch_bounds__(256) read_kv_kernel(const uint8_t *__restrict__ cache, const float *__restrict__ scales,
                                                      uint4 *__restrict__ k, uint4 *__restrict__ v, const long long *__restrict__ slot_mapping,
                                                      long long pieces, int num_kv_heads, int pieces_per_row, int token_shift,
                                                      long long block_stride, const long long *__restrict__ live_ptr, unsigned *status) {
    const long long live = *live_ptr;
    const int row_pieces = num_kv_heads * pieces_per_row, token_pieces = 2 * row_pieces;
    long long to[kReadUnroll];  // piece of k_out or v_out (16 channels); -1: none
    int rem[kReadUnroll];
    const uint8_t *src[kReadUnroll];
    const float *sc[kReadUnroll];
#pragma unroll
    for (int u = 0; u < kReadUnroll; ++u) {
        const long long i = ((long long)blockIdx.x * kReadUnroll + u) * 256 + threadIdx.x;
        to[u] = -1;
        if (i >= pieces) continue;
        const long long t = token_shift >= 0 ? i >> token_shift : i / token_pieces;
        rem[u] = (int)(i - t * token_pieces);
        const int kv = rem[u] >= row_pieces, hp = rem[u] - kv * row_pieces;
        const int h = hp / pieces_per_row, c = hp - h * pieces_per_row;
        const long long s = slot_mapping[t];
        if (s < 0) continue;
        const long long n = s >> 4;
        if (n >= live) {
            if (rem[u] == 0) atomicOr(status, EKV_DEV_FLAG_OOB);
            continue;
        }
        const int row = (kv * num_kv_heads + h) * 16 + (int)(s & 15);
        src[u] = cache + n * block_stride + ((long long)row * pieces_per_row + c) * (kE4m3 ? 16 : 32);
        if (kE4m3) sc[u] = scales + (n * 2 + kv) * num_kv_heads + h;
        to[u] = t * row_pieces + hp;
    }
    uint4 a[kReadUnroll], b[kReadUnroll];
    float scale[kReadUnroll];
#pragma unroll
    for (int u = 0; u < kReadUnroll; ++u) {
        if (to[u] < 0) continue;
        a[u] = *reinterpret_cast<const uint4 *>(src[u]);
        if (kE4m3) scale[u] = *sc[u];
        else b[u] = *reinterpret_cast<const uint4 *>(src[u] + 16);
    }
#pragma unroll
    for (int u = 0; u < kReadUnroll; ++u) {
        if (to[u] < 0) continue;
        if (kE4m3) {
            if (!(scale[u] > 0.f)) a[u] = make_uint4(0u, 0u, 0u, 0u);  // never written: 0, as attention reads it, whatever the codes
            const uint32_t w[4] = {a[u].x, a[u].y, a[u].z, a[u].w};
            uint32_t o[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 lo = f16x2_to_float2(e4m3_lo(w[j])), hi = f16x2_to_float2(e4m3_hi(w[j]));
                o[2 * j] = pack_bf16x2(lo.x * scale[u], lo.y * scale[u]);
                o[2 * j + 1] = pack_bf16x2(hi.x * scale[u], hi.y * scale[u]);
            }
            a[u] = make_uint4(o[0], o[1], o[2], o[3]);
            b[u] = make_uint4(o[4], o[5], o[6], o[7]);
        }
        uint4 *dst = (rem[u] >= row_pieces ? v : k) + 2 * to[u];
        if (kWhole) {
            st_global_32(dst, a[u], b[u]);
        } else {
            dst[0] = a[u];
            dst[1] = b[u];
        }
    }
}

}  // namespace ekv

using namespace ekv;

extern "C" ekv_status_t ekv_read_kv(ekv_pool_t *pool, int32_t layer, void *k_out, void *v_out, const int64_t *slot_mapping, int32_t T,
                                    void *stream) {
    ekv_status_t st = check_compute(pool, layer, "ekv_read_kv");
    if (st != EKV_OK) return st;
    if (T < 0 || (T > 0 && (!k_out || !v_out || !slot_mapping)) || ((uintptr_t)k_out & 15) || ((uintptr_t)v_out & 15)) {
        set_error("ekv_read_kv: bad argument (T=%d, k_out=%p, v_out=%p, slot_mapping=%p)", T, k_out, v_out, (const void *)slot_mapping);
        return EKV_ERR_INVALID;
    }
    if (T == 0) return EKV_OK;
    const int pieces_per_row = pool->desc.head_dim / 16, token_pieces = 2 * pool->desc.num_kv_heads * pieces_per_row;
    int token_shift = -1;
    if ((token_pieces & (token_pieces - 1)) == 0)
        for (token_shift = 0; (1 << token_shift) < token_pieces;) ++token_shift;
    const long long pieces = (long long)T * token_pieces, per_cta = 256 * kReadUnroll;
    if ((pieces + per_cta - 1) / per_cta > 0x7fffffffLL) {
        set_error("ekv_read_kv: too many rows (T=%d)", T);
        return EKV_ERR_INVALID;
    }
    const bool whole = (((uintptr_t)k_out | (uintptr_t)v_out) & 31) == 0;
    const auto kernel = pool->e4m3() ? (whole ? read_kv_kernel<true, true> : read_kv_kernel<true, false>)
                                     : (whole ? read_kv_kernel<false, true> : read_kv_kernel<false, false>);
    kernel<<<(unsigned)((pieces + per_cta - 1) / per_cta), 256, 0, (cudaStream_t)stream>>>(
        (const uint8_t *)pool->layer_base(layer), pool->e4m3() ? pool->layer_scales(layer) : nullptr, (uint4 *)k_out, (uint4 *)v_out,
        (const long long *)slot_mapping, pieces, pool->desc.num_kv_heads, pieces_per_row, token_shift, (long long)pool->block_stride, pool->d_live,
        pool->d_status);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_fail(e, "ekv_read_kv launch");
    return EKV_OK;
}

extern "C" ekv_status_t ekv_write_kv(ekv_pool_t *pool, int32_t layer, const void *k, const void *v,
                                     const int64_t *slot_mapping, int32_t T, void *stream) {
    ekv_status_t st = check_compute(pool, layer, "ekv_write_kv");
    if (st != EKV_OK) return st;
    if (T < 0 || (T > 0 && (!k || !v || !slot_mapping)) || ((uintptr_t)k & 15) || ((uintptr_t)v & 15)) {
        set_error("ekv_write_kv: bad argument (T=%d, k=%p, v=%p, slot_mapping=%p)", T, k, v, (const void *)slot_mapping);
        return EKV_ERR_INVALID;
    }
    if (T == 0) return EKV_OK;
    if (pool->e4m3()) {
        Write8Params p;
        p.cache = (uint8_t *)pool->layer_base(layer);
        p.scales = pool->layer_scales(layer);
        p.claims = pool->d_claims + (size_t)layer * pool->total_blocks();
        p.k = (const uint4 *)k;
        p.v = (const uint4 *)v;
        p.slots = (const long long *)slot_mapping;
        p.live = pool->d_live;
        p.status = pool->d_status;
        p.block_stride = (long long)pool->block_stride;
        p.T = T;
        p.num_kv_heads = pool->desc.num_kv_heads;
        return pool->desc.head_dim == 128 ? launch_write8<128>(pool, p, (cudaStream_t)stream) : launch_write8<64>(pool, p, (cudaStream_t)stream);
    }
    const int pieces_per_row = pool->desc.head_dim * 2 / 16;
    int block_shift = 0, row_shift = 0, token_shift = -1;
    while ((1 << block_shift) < pool->desc.block_size) ++block_shift;
    while ((1 << row_shift) < pieces_per_row) ++row_shift;
    const int token_pieces = 2 * pool->desc.num_kv_heads * pieces_per_row;
    if ((token_pieces & (token_pieces - 1)) == 0)
        for (token_shift = 0; (1 << token_shift) < token_pieces;) ++token_shift;
    const long long total = (long long)T * 2 * pool->desc.num_kv_heads * pieces_per_row;
    long long blocks = (total + kWriteThreads * kWriteUnroll - 1) / (kWriteThreads * kWriteUnroll);
    const long long cap = (long long)pool->sm_count * 64;
    if (blocks > cap) blocks = cap;
    write_kv_kernel<<<(unsigned)blocks, kWriteThreads, 0, (cudaStream_t)stream>>>(
        (uint4 *)pool->layer_base(layer), (const uint4 *)k, (const uint4 *)v, (const long long *)slot_mapping, T,
        pool->desc.num_kv_heads, pool->desc.block_size, block_shift, pieces_per_row, row_shift, token_shift, (long long)(pool->block_stride / 16), pool->d_live,
        pool->d_status);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_fail(e, "ekv_write_kv launch");
    return EKV_OK;
}

// ekv_attn_prefill_chunk: host entry point.  Validates, sizes the launch from the host copy of
// cu_q_lens (no device synchronisation) and dispatches the kernel for the pool's head_dim.
#include "ekv_internal.h"
#include "ekv_prefill_mma.cuh"
#include "ekv_prefill_tc.cuh"
#include "ekv_prefill_tc1.cuh"
#include "ekv_prefill_e4m3.cuh"
#include "ekv_prefill_e4m3_few.cuh"
#include "ekv_prefill_tcs.cuh"

using namespace ekv;

extern "C" ekv_status_t ekv_attn_prefill_chunk(ekv_pool_t *pool, int32_t layer, const void *q, void *out,
                                               const int32_t *block_tables, int32_t max_blocks_per_seq,
                                               const int32_t *cu_q_lens, const int32_t *cu_q_lens_host,
                                               const int32_t *seq_lens, int32_t R, float scale, void *stream) {
    ekv_status_t st = check_compute(pool, layer, "ekv_attn_prefill_chunk");
    if (st != EKV_OK) return st;
    if (R < 0 || max_blocks_per_seq < 1 || max_blocks_per_seq > (1 << 26) ||
        (R > 0 && (!q || !out || !block_tables || !cu_q_lens || !cu_q_lens_host || !seq_lens)) || ((uintptr_t)q & 15) ||
        ((uintptr_t)out & 15)) {
        set_error("ekv_attn_prefill_chunk: bad argument (R=%d, max_blocks_per_seq=%d)", R, max_blocks_per_seq);
        return EKV_ERR_INVALID;
    }
    if (R == 0) return EKV_OK;
    if (cu_q_lens_host[0] != 0) {
        set_error("ekv_attn_prefill_chunk: cu_q_lens[0] must be 0");
        return EKV_ERR_INVALID;
    }
    // Kernels (scale > 0 unless stated):
    //   two-head tcgen05 kernel   head_dim 128, query groups of 2 or more: a persistent CTA per SM, every K/V tile feeds two
    //                             heads (an odd group is cut into pairs and one single-head item per kv-head).
    //                             Measured, 32768 query tokens in one call, 32q/8kv: 256 x 128 fresh prompts 130 us against
    //                             161 us for the two-slot kernel; 64 x 512: 198 against 335-364; 16 x 2048: 508 against
    //                             769.  28q/4kv (groups of 7): a 16384-token prompt 1.63 against 2.11 ms, 64 x 512 215
    //                             against 299 us
    //   two-slot tcgen05 kernel   head_dim 128, one head per work item, the CTA's two TMEM slots on their own clocks: query
    //                             groups of one (no two heads share a K/V tile)
    //   one-head tcgen05 kernel   head_dim 64 (one CTA per tile and head, two CTAs per SM)
    //   warp-level MMA kernel     non-positive scales, and every call on a pool created with EKV_PREFILL_WARP_MMA (which
    //                             the tests use to check the kernel families against each other)
    // EKV_PREFILL_ONE_HEAD forces the one-head family on any group; EKV_PREFILL_TWO_HEAD is what a group of two or more at
    // head_dim 128 gets anyway (kept so that a caller can say so).
    const int group = pool->desc.num_q_heads / pool->desc.num_kv_heads;
    const uint32_t pf = pool->desc.flags;
    enum { K_TWO_HEAD, K_ONE_HEAD, K_WARP_MMA } kernel;
    if ((pf & EKV_PREFILL_WARP_MMA) || !(scale > 0.f)) {
        kernel = K_WARP_MMA;
    } else if ((pf & EKV_PREFILL_ONE_HEAD) || pool->desc.head_dim != 128 || group == 1) {
        kernel = K_ONE_HEAD;
    } else {
        kernel = K_TWO_HEAD;
    }
    // An 8-bit pool has one kernel, whose items are rows of all heads of a group (ekv_prefill_e4m3.cuh).
    const bool e4m3 = pool->e4m3();
    const int bm = e4m3 ? tc8::kItemRows : kernel == K_WARP_MMA ? kPmBM : tc::kBM;
    // Of an 8-bit pool's requests those with few rows go to a kernel of their own (ekv_prefill_e4m3_few.cuh): one launch each if a
    // call has both kinds, the second in the tail of the first (a chunk of 2048 over 8000 keys and 128 single rows 425 -> 400 us, 100
    // tokens over 500 keys and 8 requests of 4 31 -> 22).
    long long few = 0;
    PrefillParams p;
    p.n_prefix = R <= kPrefixMax ? 1 : 0;
    long long q_tiles = 0;
    for (int r = 0; r < R; ++r) {
        const long long c = ((long long)cu_q_lens_host[r + 1] - cu_q_lens_host[r]) * (e4m3 ? group : 1);
        if (c < 0) {
            set_error("ekv_attn_prefill_chunk: cu_q_lens decreases at request %d", r);
            return EKV_ERR_INVALID;
        }
        if (p.n_prefix) p.tile_prefix[r] = (int)q_tiles;
        if (e4m3 && c <= few8::kMaxRows) {
            if (c > 0) ++few;
            continue;
        }
        q_tiles += (c + bm - 1) / bm;
        if (q_tiles > 0x7fffffffLL) break;
    }
    if (p.n_prefix && q_tiles <= 0x7fffffffLL) p.tile_prefix[R] = (int)q_tiles;
    if (q_tiles == 0 && few == 0) return EKV_OK;
    if (q_tiles > 0x7fffffffLL || (e4m3 && ((q_tiles + R) * pool->desc.num_kv_heads * tc8::kMaxCluster > 0x7fffffffLL || (long long)cu_q_lens_host[R] * group >= (1LL << 29)))) {
        set_error("ekv_attn_prefill_chunk: too many query tiles");
        return EKV_ERR_INVALID;
    }
    p.q = (const __nv_bfloat16 *)q;
    p.out = (__nv_bfloat16 *)out;
    p.block_tables = block_tables;
    p.cu_q_lens = cu_q_lens;
    p.seq_lens = seq_lens;
    p.live = pool->d_live;
    p.status = pool->d_status;
    // every launch over a bf16 pool gets a device word of its own (abort flag + item counter), so that launches of one pool on
    // different streams do not share them; the launcher clears the word on the stream before the kernel
    p.abort_word = e4m3 ? nullptr : reinterpret_cast<int *>(pool->d_live + 1 + __atomic_fetch_add(&pool->launch_seq, 1u, __ATOMIC_RELAXED) % EKV_LAUNCH_SLOTS);
    p.max_blocks = max_blocks_per_seq;
    p.num_q_heads = pool->desc.num_q_heads;
    p.num_kv_heads = pool->desc.num_kv_heads;
    p.group = pool->desc.num_q_heads / pool->desc.num_kv_heads;
    p.R = R;
    p.q_tiles = (int)q_tiles;
    p.scale_log2 = scale * 1.4426950408889634f;
    const bool d128 = pool->desc.head_dim == 128;
    if (e4m3) {
        tc8::Params pp;
        pp.p = p;
        pp.p.scale_log2 = fabsf(p.scale_log2);
        pp.q_sign = scale < 0.f ? -1.f : scale == 0.f ? 0.f : 1.f;
        pp.cache = (const uint8_t *)pool->layer_base(layer);
        pp.scales = pool->layer_scales(layer);
        pp.block_stride = (long long)pool->block_stride;
        pp.few_rows = few8::kMaxRows;
        pp.cluster = 1;  // the launchers choose
        pp.group_magic = group > 1 ? (unsigned)(((1ull << 32) + group - 1) / group) : 0u;
        if (q_tiles > 0) {
            st = d128 ? tc8::launch_prefill8<128>(pool, pp, (cudaStream_t)stream) : tc8::launch_prefill8<64>(pool, pp, (cudaStream_t)stream);
            if (st != EKV_OK) return st;
        }
        if (few > 0)
            st = d128 ? few8::launch<128>(pool, layer, pp, few, q_tiles > 0, (cudaStream_t)stream) : few8::launch<64>(pool, layer, pp, few, q_tiles > 0, (cudaStream_t)stream);
        return st;
    }
    if (kernel == K_TWO_HEAD) return tc::launch_prefill_tc(pool, layer, p, q, out, cu_q_lens_host[R], (cudaStream_t)stream);
    if (kernel == K_ONE_HEAD)
        return d128 ? tcs::launch_prefill_tcs(pool, layer, p, q, out, cu_q_lens_host[R], (cudaStream_t)stream)
                    : tc1::launch_prefill_tc1<64>(pool, layer, p, (int)q_tiles, (cudaStream_t)stream);
    return d128 ? launch_prefill_mma<128>(pool, layer, p, (int)q_tiles, (cudaStream_t)stream)
                : launch_prefill_mma<64>(pool, layer, p, (int)q_tiles, (cudaStream_t)stream);
}

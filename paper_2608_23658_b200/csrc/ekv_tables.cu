// ekv_extend_tables: block tables, slot mapping, offsets and lengths of a step, made on the GPU.
//
//   need_r = ceil((len_r + new_r) / 16) - ceil(len_r / 16),  cu = exclusive sum of new,  first = cursor + exclusive sum of need
//   slot(cu_r + i) = 16 * id(r, p / 16) + p % 16, p = len_r + i; id = the table's entry if the block was there, else
//   free_ids[first_r + p / 16 - ceil(len_r / 16)]
//
// A step is a few thousand integers, so the cost is latency: one launch, no pass over device memory waits for another.  Every
// CTA reads all lengths (8 bytes a request) and scans them itself into shared memory; after that every window of 32 tokens and
// every new block finds its request there by bisection.  The mapping of a long step is split over a cluster of CTAs, whose barrier
// is also what lets lengths and cursor be updated in place: nobody writes before all have read.  All checks are made
// by every CTA on the same data before that barrier, so that a refused call changes nothing anywhere.
//
// Measured on the device: 64 requests of one token 5.5 us; 500 of 1..65 tokens 9.0 us; 1024 prompts of up to 127 tokens (65 000
// tokens) 12.2 us.  What a CTA does alone -- a launch, a read, a scan -- is 5 us of each; the rest goes with the tokens a CTA
// has to place: the last of the three took 81 us on one CTA, 46 on two, 16.0 on eight, 12.2 on the sixteen that a cluster can have.
// A bisection over all requests for each token, in place of a window's, took 19.5 us on eight; 512 threads a CTA 20.4.
#include <cooperative_groups.h>

#include "ekv_internal.h"

namespace ekv {

namespace cg = cooperative_groups;

static constexpr int kTabThreads = 1024;
static constexpr int kTabCluster = 16;
static constexpr int kTabMaxRequests = 16384;

struct TablesParams {
    const int *new_tokens, *seq_lens;
    int *tables;
    const int *free_ids, *cursor;
    long long *slots;
    int *cu, *lens_out, *cursor_out;
    const long long *live;
    unsigned *status;
    int R, max_blocks, n_free, T_cap;
};

// the last r in [lo, hi] with first[r] <= x; first is ascending, first[lo] <= x
__device__ __forceinline__ int last_at_most(const int *first, int lo, int hi, int x) {
    for (int w = hi > lo ? 1 << (31 - __clz(hi - lo)) : 0; w > 0; w >>= 1)
        if (lo + w <= hi && first[lo + w] <= x) lo += w;
    return lo;
}

__global__ void __launch_bounds__(kTabThreads) extend_tables_kernel(const TablesParams p) {
    extern __shared__ int smem[];
    int *len = smem, *cu = smem + p.R, *need = cu + p.R;  // lengths before; exclusive sums of new tokens and of new blocks
    __shared__ longlong2 warp_sum[kTabThreads / 32 + 1];  // tokens, blocks
    __shared__ unsigned bad;
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
    if (tid == 0) bad = 0;
    __syncthreads();

    // each thread sums a run of requests, the threads' sums are scanned, then each writes its run's exclusive sums
    const long long live = *p.live;
    const int cursor = *p.cursor;
    const int per = (p.R + kTabThreads - 1) / kTabThreads;
    const int r0 = min(p.R, tid * per), r1 = min(p.R, r0 + per);
    long long tokens = 0, blocks = 0;
    unsigned wrong = 0;
    for (int r = r0; r < r1; ++r) {
        const int n = p.new_tokens[r], l = p.seq_lens[r];
        len[r] = l;
        if (n < 0 || l < 0 || (long long)l + n > (long long)p.max_blocks * 16) {
            wrong |= EKV_DEV_FLAG_BAD_LEN;
        } else {
            tokens += n;
            blocks += (l + n + 15) / 16 - (l + 15) / 16;
            if (n > 0 && (l & 15)) {
                const int id = p.tables[(size_t)r * p.max_blocks + l / 16];
                if (id < 0 || id >= live) wrong |= EKV_DEV_FLAG_OOB;
            }
        }
    }
    long long ts = tokens, bs = blocks;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long a = __shfl_up_sync(0xffffffffu, ts, o), b = __shfl_up_sync(0xffffffffu, bs, o);
        if (lane >= o) ts += a, bs += b;
    }
    if (lane == 31) warp_sum[warp] = make_longlong2(ts, bs);
    if (wrong) atomicOr(&bad, wrong);
    __syncthreads();
    if (warp == 0) {  // the warps' sums -> exclusive, and the totals behind them
        longlong2 v = make_longlong2(0, 0);
        if (lane < kTabThreads / 32) v = warp_sum[lane];
        long long tw = v.x, bw = v.y;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long a = __shfl_up_sync(0xffffffffu, tw, o), b = __shfl_up_sync(0xffffffffu, bw, o);
            if (lane >= o) tw += a, bw += b;
        }
        if (lane < kTabThreads / 32) warp_sum[lane] = make_longlong2(tw - v.x, bw - v.y);
        if (lane == 31) warp_sum[kTabThreads / 32] = make_longlong2(tw, bw);
    }
    __syncthreads();
    const long long t_before = warp_sum[warp].x, b_before = warp_sum[warp].y;
    const long long t_total = warp_sum[kTabThreads / 32].x, b_total = warp_sum[kTabThreads / 32].y;
    if (tid == 0) {
        unsigned f = 0;
        if (t_total > p.T_cap) f |= EKV_DEV_FLAG_BAD_LEN;
        if (cursor < 0 || cursor + b_total > p.n_free) f |= EKV_DEV_FLAG_NO_BLOCKS;
        if (f) atomicOr(&bad, f);
    }
    __syncthreads();
    if (bad == 0) {
        int t_at = (int)(t_before + ts - tokens), b_at = (int)(b_before + bs - blocks);
        for (int r = r0; r < r1; ++r) {
            const int n = p.new_tokens[r], l = len[r];
            cu[r] = t_at;
            need[r] = b_at;
            t_at += n;
            b_at += (l + n + 15) / 16 - (l + 15) / 16;
        }
        bool out = false;
        for (int i = tid; i < (int)b_total; i += kTabThreads) {
            const int id = p.free_ids[cursor + i];
            out |= id < 0 || id >= live;
        }
        if (out) atomicOr(&bad, EKV_DEV_FLAG_OOB);
    }
    __syncthreads();
    const unsigned refused = bad;
    const int step = ctas * kTabThreads, me = rank * kTabThreads + tid;
    if (ctas > 1) cluster.sync();  // all CTAs have read lengths, cursor and partly filled blocks' ids

    if (refused) {
        if (me == 0) {
            atomicOr(p.status, refused);
            *p.cursor_out = cursor;
        }
        for (int i = me; i < p.T_cap; i += step) p.slots[i] = -1;
        for (int r = me; r <= p.R; r += step) {
            p.cu[r] = 0;
            if (r < p.R) p.lens_out[r] = len[r];
        }
        return;
    }
    // A warp takes a run of tokens, 32 at a time: once it knows the request of a window's first and last token -- one look, while
    // a request goes on -- the lanes have at most the requests in between to search.
    const int warps = step / 32, my_warp = rank * (kTabThreads / 32) + warp;
    const int run = ((p.T_cap + warps - 1) / warps + 31) / 32 * 32;
    const int run_end = (int)min((long long)p.T_cap, (long long)(my_warp + 1) * run);
    int rf = 0;
    for (int w = (int)min((long long)p.T_cap, (long long)my_warp * run); w < run_end; w += 32) {
        const int t = w + lane, t_last = (int)min(t_total, (long long)min(w + 32, run_end)) - 1;
        long long slot = -1;
        if (t_last >= w) {  // (else the window lies behind the last token)
            if (w == my_warp * run) rf = last_at_most(cu, 0, p.R - 1, w);
            const int rl = rf + 1 < p.R && cu[rf + 1] <= t_last ? last_at_most(cu, rf, p.R - 1, t_last) : rf;
            if (t <= t_last) {
                const int r = rl > rf ? last_at_most(cu, rf, rl, t) : rf;
                const int pos = len[r] + t - cu[r], have = (len[r] + 15) / 16, j = pos / 16;
                const int id = j < have ? p.tables[(size_t)r * p.max_blocks + j] : p.free_ids[cursor + need[r] + j - have];
                slot = (long long)id * 16 + (pos & 15);
            }
            // the next window's first token: of rl, or of a request behind it that starts there (empty ones between them or not)
            rf = rl + 1 < p.R && cu[rl + 1] <= w + 32 ? last_at_most(cu, rl, p.R - 1, w + 32) : rl;
        }
        if (t < run_end) p.slots[t] = slot;
    }
    for (int i = me; i < (int)b_total; i += step) {
        const int r = last_at_most(need, 0, p.R - 1, i);
        p.tables[(size_t)r * p.max_blocks + (len[r] + 15) / 16 + i - need[r]] = p.free_ids[cursor + i];
    }
    for (int r = me; r < p.R; r += step) {
        const int next = r + 1 < p.R ? cu[r + 1] : (int)t_total;
        p.cu[r] = cu[r];
        p.lens_out[r] = len[r] + next - cu[r];
    }
    if (me == 0) {
        p.cu[p.R] = (int)t_total;
        *p.cursor_out = cursor + (int)b_total;
    }
}

}  // namespace ekv

using namespace ekv;

extern "C" ekv_status_t ekv_extend_tables(ekv_pool_t *pool, const int32_t *new_tokens, const int32_t *seq_lens, int32_t R,
                                          int32_t *block_tables, int32_t max_blocks_per_seq, const int32_t *free_ids, int32_t n_free,
                                          const int32_t *free_cursor, int64_t *slot_mapping, int32_t T_cap, int32_t *cu_q_lens,
                                          int32_t *seq_lens_out, int32_t *free_cursor_out, void *stream) {
    ekv_status_t st = check_compute(pool, 0, "ekv_extend_tables");
    if (st != EKV_OK) return st;
    if (R < 0 || R > kTabMaxRequests || max_blocks_per_seq < 1 || max_blocks_per_seq > (1 << 26) || n_free < 0 || T_cap < 0 ||
        T_cap > (1 << 30) || !free_cursor || !free_cursor_out || !cu_q_lens || (n_free > 0 && !free_ids) || (T_cap > 0 && !slot_mapping) ||
        (R > 0 && (!new_tokens || !seq_lens || !block_tables || !seq_lens_out))) {
        set_error("ekv_extend_tables: bad argument (R=%d of at most %d, max_blocks_per_seq=%d, n_free=%d, T_cap=%d)", R, kTabMaxRequests,
                  max_blocks_per_seq, n_free, T_cap);
        return EKV_ERR_INVALID;
    }
    TablesParams p;
    p.new_tokens = new_tokens;
    p.seq_lens = seq_lens;
    p.tables = block_tables;
    p.free_ids = free_ids;
    p.cursor = free_cursor;
    p.slots = (long long *)slot_mapping;
    p.cu = cu_q_lens;
    p.lens_out = seq_lens_out;
    p.cursor_out = free_cursor_out;
    p.live = pool->d_live;
    p.status = pool->d_status;
    p.R = R;
    p.max_blocks = max_blocks_per_seq;
    p.n_free = n_free;
    p.T_cap = T_cap;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 1;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    static int max_cluster[64] = {0};  // per device: the cluster that fits at the largest R
    const int dev = pool->desc.device;
    int widest = dev < 64 ? max_cluster[dev] : 0;
    if (widest == 0) {
        cudaError_t e = cudaFuncSetAttribute(extend_tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * kTabMaxRequests * (int)sizeof(int));
        if (e == cudaSuccess) e = cudaFuncSetAttribute(extend_tables_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return cuda_fail(e, "ekv_extend_tables: kernel attributes");
        cfg.gridDim = dim3(kTabCluster);
        cfg.blockDim = dim3(kTabThreads);
        cfg.dynamicSmemBytes = 3 * kTabMaxRequests * sizeof(int);
        attr.val.clusterDim.x = kTabCluster;
        int n = 0;
        widest = cudaOccupancyMaxActiveClusters(&n, extend_tables_kernel, &cfg) == cudaSuccess && n > 0 ? kTabCluster : 8;
        (void)cudaGetLastError();
        if (dev < 64) max_cluster[dev] = widest;
    }
    // a token a thread of one CTA, then a cluster
    const int ctas = T_cap > kTabThreads ? widest : 1;
    attr.val.clusterDim.x = (unsigned)ctas;
    cfg.numAttrs = ctas > 1 ? 1 : 0;
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kTabThreads);
    cfg.dynamicSmemBytes = 3 * (size_t)R * sizeof(int);
    cfg.stream = (cudaStream_t)stream;
    cudaError_t e = cudaLaunchKernelEx(&cfg, extend_tables_kernel, p);
    if (e != cudaSuccess) return cuda_fail(e, "ekv_extend_tables launch");
    return EKV_OK;
}

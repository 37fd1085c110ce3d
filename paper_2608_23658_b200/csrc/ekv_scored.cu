// Host side of ekv_attn_decode_scored, ekv_attn_prefill_chunk_scored and ekv_attn_decode_shared: checks, plans, launches.
#include <cuda_bf16.h>
#include <math.h>
#include <string.h>

#include "ekv_decode_ext.cuh"
#include "ekv_internal.h"
#include "ekv_rows.cuh"

namespace ekv {

static constexpr float kLog2e = 1.4426950408889634f;
static constexpr float kSmallest = 1.17549435e-38f;  // stands for a scale of 0: -inf times it is still -inf
static constexpr float kLargest = 1e30f;             // bounds scale / cap: a score of 0 times it is still 0

// scale / cap and cap * log2 e as the kernels take them: fp32 numbers that are neither flushed to 0 (an infinite score still reaches the cap) nor infinite.
static float cap_scale_of(float scale, float cap) { return copysignf(fmaxf(kSmallest, fminf(fabsf(scale) / cap, kLargest)), scale); }
static float cap_log2_of(float cap) { return fminf(cap * kLog2e, 3.402823466e38f); }

// Shared-memory attributes of a kernel, once per device.
template <typename Kernel>
static cudaError_t ready(Kernel kernel, int bytes, int device, bool (&done)[64]) {
    if (device < 64 && done[device]) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && device < 64) done[device] = true;
    return e;
}

template <typename... P, typename... A>
static cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, int bytes, bool early, int cluster, cudaStream_t stream, A... args) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 0;
    if (early) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[cfg.numAttrs].val.clusterDim.x = (unsigned)cluster;
        attr[cfg.numAttrs].val.clusterDim.y = 1;
        attr[cfg.numAttrs++].val.clusterDim.z = 1;
    }
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int D, int kMode, bool kCap, bool kBias>
static cudaError_t launch_rows(ekv_pool *pool, int layer, const rows::Params &p, long long q_rows, cudaStream_t stream) {
    static bool done[64] = {false};
    cudaError_t e = ready(rows::rows_kernel<D, kMode, kCap, kBias>, rows::Geo<D>::kSmemBytes, pool->desc.device, done);
    if (e != cudaSuccess) return e;
    // Q by TMA: a box of all heads of a group x as many tokens as make a tile
    CUtensorMap qmap = pool->kv_map[layer];
    if (p.q_tma && encode_q_map(p.q, (uint64_t)q_rows, p.num_q_heads, D, rows::kBM / p.group, &qmap, p.group) != EKV_OK) return cudaErrorInvalidValue;
    return launch(rows::rows_kernel<D, kMode, kCap, kBias>, dim3(p.num_kv_heads * (kMode == rows::kShared ? 1 : p.parts), p.tiles), rows::kThreads, rows::Geo<D>::kSmemBytes, false, 1, stream, pool->kv_map[layer], qmap, p,
                  (const uint8_t *)pool->layer_base(layer), (long long)pool->block_stride);
}

template <int D>
static constexpr int ext_bytes() { return ext::kWarps * ext::kStages * (2 * (D / 64) * ext::kBoxBytes + 8) + 1024; }

template <int D, bool kShared, bool kCap, bool kBias>
static cudaError_t ready_ext(int device) {
    static bool done[64] = {false}, wide[64] = {false};
    cudaError_t e = ready(ext::decode_ext_kernel<D, kShared, kCap, kBias>, ext_bytes<D>(), device, done);
    if (e != cudaSuccess || (device < 64 && wide[device])) return e;
    e = cudaFuncSetAttribute(ext::decode_ext_kernel<D, kShared, kCap, kBias>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);  // more than eight CTAs
    if (e == cudaSuccess && device < 64) wide[device] = true;
    return e;
}

static int clusters_of(const ekv_pool *pool, long long clusters);

template <int D, bool kShared, bool kCap, bool kBias>
static cudaError_t launch_ext(ekv_pool *pool, int layer, ext::Params p, int B, bool early, cudaStream_t stream) {
    constexpr int kBytes = ext_bytes<D>();
    cudaError_t e = ready_ext<D, kShared, kCap, kBias>(pool->desc.device);
    if (e != cudaSuccess) return e;
    // Ranges that are few, and all there at once, add themselves up as a cluster.  (In larger calls CTAs that wait for their cluster would keep others out.)
    p.cluster = !p.beside && p.nsplit > 1 && p.nsplit <= clusters_of(pool, (long long)B * p.num_kv_heads);
    e = launch(ext::decode_ext_kernel<D, kShared, kCap, kBias>, dim3(p.nsplit, p.num_kv_heads, B), ext::kWarps * 32, kBytes, early, p.cluster ? p.nsplit : 1, stream, pool->kv_map[layer], p);
    if (e != cudaSuccess || ((p.nsplit == 1 || p.cluster) && !p.beside)) return e;
    const int n = B * p.num_q_heads;
    return launch(ext::combine_ext_kernel<D, kShared>, dim3((n + ext::kCombineWarps - 1) / ext::kCombineWarps), ext::kCombineWarps * 32, 0, true, 1, stream, p, n);
}

static size_t align256(size_t n) { return (n + 255) / 256 * 256; }
// (m, l) pairs and rows of fp32 partial results
static size_t parts_bytes(const ekv_pool *pool, size_t n) { return align256(n * sizeof(float2)) + align256(n * pool->desc.head_dim * sizeof(float)); }

static ekv_status_t check_workspace(const char *who, const void *workspace, size_t bytes, size_t need) {
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 255) || bytes < need)) {
        set_error("%s: workspace %p of %zu bytes; need %zu bytes, 256-byte aligned", who, workspace, bytes, need);
        return EKV_ERR_WORKSPACE;
    }
    return EKV_OK;
}

static ekv_status_t check_scores(const char *who, const ekv_pool *pool, const ekv_scores_t *s, float scale) {
    if (pool->e4m3()) {
        set_error("%s: EKV_BF16 pools only", who);
        return EKV_ERR_INVALID;
    }
    if (!s || !(s->cap >= 0.f) || isinf(s->cap) || s->window < 0 || isnan(scale) || isinf(scale)) {
        set_error("%s: bad scores (cap=%g, window=%d, scale=%g)", who, s ? (double)s->cap : 0., s ? s->window : 0, (double)scale);
        return EKV_ERR_INVALID;
    }
    return EKV_OK;
}

static ekv_status_t check_decode(const char *who, const void *q, const void *out, const int32_t *block_tables, int32_t max_blocks, const int32_t *seq_lens, int32_t B) {
    if (B < 0 || max_blocks < 1 || max_blocks > (1 << 26) || B > 65535 || (B > 0 && (!q || !out || !block_tables || !seq_lens)) ||
        (((uintptr_t)q | (uintptr_t)out) & 15)) {
        set_error("%s: bad argument (B=%d, max_blocks_per_seq=%d)", who, B, max_blocks);
        return EKV_ERR_INVALID;
    }
    return EKV_OK;
}

static void fill_ext(ext::Params &p, const ekv_pool *pool, const void *q, void *out, const int32_t *block_tables, int32_t max_blocks, const int32_t *seq_lens,
                     const DecodePlan &plan) {
    p.q = (const __nv_bfloat16 *)q, p.out = (__nv_bfloat16 *)out;
    p.block_tables = block_tables, p.seq_lens = seq_lens;
    p.live = pool->d_live, p.status = pool->d_status;
    p.slopes = nullptr, p.prefix_lens = nullptr;
    p.shared_o = nullptr, p.shared_ml = nullptr;
    p.max_blocks = max_blocks, p.num_q_heads = pool->desc.num_q_heads, p.num_kv_heads = pool->desc.num_kv_heads;
    p.group = p.num_q_heads / p.num_kv_heads;
    p.chunk_tokens = plan.chunk_tokens, p.nsplit = plan.nsplit;
    p.window = 0, p.parts = 0, p.G = 0, p.beside = 0;
    p.cap_scale = p.cap_log2 = 0.f;
}

static void fill_rows(rows::Params &p, const ekv_pool *pool, const void *q, void *out, const int32_t *block_tables, int32_t max_blocks) {
    p.q = (const __nv_bfloat16 *)q, p.out = (__nv_bfloat16 *)out;
    p.block_tables = block_tables, p.cu_q_lens = nullptr, p.seq_lens = nullptr;
    p.live = pool->d_live, p.status = pool->d_status;
    p.slopes = nullptr, p.prefix_lens = nullptr;
    p.max_blocks = max_blocks, p.num_q_heads = pool->desc.num_q_heads, p.num_kv_heads = pool->desc.num_kv_heads;
    p.group = p.num_q_heads / p.num_kv_heads;
    p.group_magic = p.group > 1 ? (unsigned)(((1ull << 32) + p.group - 1) / p.group) : 0u;
    p.window = 0, p.parts = 1, p.chunk_tiles = 0, p.q_flip = 0;
    p.q_tma = rows::kBM % p.group == 0;
    p.cap_scale = p.cap_log2 = p.near_limit = 0.f;
    for (float &c : p.near) c = 0.f;
}

template <int D>
static cudaError_t scored_decode(ekv_pool *pool, int layer, const ext::Params &p, bool cap, int B, cudaStream_t stream) {
    if (cap) return p.slopes ? launch_ext<D, false, true, true>(pool, layer, p, B, false, stream) : launch_ext<D, false, true, false>(pool, layer, p, B, false, stream);
    return p.slopes ? launch_ext<D, false, false, true>(pool, layer, p, B, false, stream) : launch_ext<D, false, false, false>(pool, layer, p, B, false, stream);
}

template <int D>
static cudaError_t scored_prefill(ekv_pool *pool, int layer, const rows::Params &p, bool cap, long long q_rows, cudaStream_t stream) {
    using namespace rows;
    if (cap) return p.slopes ? launch_rows<D, kScored, true, true>(pool, layer, p, q_rows, stream) : launch_rows<D, kScored, true, false>(pool, layer, p, q_rows, stream);
    return p.slopes ? launch_rows<D, kScored, false, true>(pool, layer, p, q_rows, stream) : launch_rows<D, kScored, false, false>(pool, layer, p, q_rows, stream);
}

// Parts that an item's keys are cut into: as many as let all items run at the same time, while a part keeps two key tiles of the most that an item can see.
static int plan_parts(const ekv_pool *pool, long long items, int max_blocks, int window, bool prefix, int max_rows) {
    long long tiles = ((long long)max_blocks * 16 + rows::kBN - 1) / rows::kBN;
    if (window > 0 && !prefix) {  // positions of an item, their windows, and a tile cut at each end
        const long long span = ((long long)window + max_rows + rows::kBN - 1) / rows::kBN + 1;
        if (span < tiles) tiles = span;
    }
    long long parts = pool->sm_count / (items > 0 ? items : 1);
    if (parts > tiles / 2) parts = tiles / 2;
    return parts < 1 ? 1 : (int)parts;
}

// CTAs of the largest cluster of which so many are there at once; 1: of none.
static int clusters_of(const ekv_pool *pool, long long clusters) {
    static int fit[64][ext::kCluster + 1] = {};  // by device and size, + 1; the same for all of the kernels, whose registers let three CTAs into an SM
    const int device = pool->desc.device;
    int size = ext::kCluster;
    for (; size > 1; --size) {
        int known = device < 64 ? fit[device][size] : 0;
        if (known == 0) {
            cudaLaunchConfig_t cfg = {};
            cudaLaunchAttribute attr;
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = (unsigned)size, attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
            cfg.gridDim = dim3((unsigned)size), cfg.blockDim = dim3(ext::kWarps * 32), cfg.dynamicSmemBytes = ext_bytes<128>();
            cfg.attrs = &attr, cfg.numAttrs = 1;
            int n = 0, current = device;
            if (cudaGetDevice(&current) != cudaSuccess || cudaSetDevice(device) != cudaSuccess || ready_ext<128, false, false, false>(device) != cudaSuccess ||
                cudaOccupancyMaxActiveClusters(&n, ext::decode_ext_kernel<128, false, false, false>, &cfg) != cudaSuccess)
                n = 0, (void)cudaGetLastError();
            if (current != device) (void)cudaSetDevice(current);
            known = n + 1;
            if (device < 64) fit[device][size] = known;
        }
        if (clusters <= known - 1) break;
    }
    return size;
}

// Ranges of decode's sequences: those of ekv_attn_decode, or, where they can be a cluster, or one, with up to 1024 keys each, as few as that takes.
// Device, us: a sequence of 16000, 32q/8kv 28.8 -> 17.6, 4 of 4000 19.7 -> 13.5, 8 of up to 4000 17.7 -> 13.7; 20 of 2000, 28q/4kv 20.1 -> 14.3;
// 64 of up to 700, 32q/8kv, as one range each 19.5 -> 15.5.  With 2048 keys, 4 of 16000 53.9 -> 55.9.
static constexpr int kRangeKeys = 1024;
static DecodePlan plan_ranges(const ekv_pool *pool, int B, int blocks) {
    DecodePlan plan = plan_decode(pool, B, blocks);
    const long long units = (long long)B * pool->desc.num_kv_heads, len = (long long)blocks * 16;
    const int n = plan.nsplit > 1 ? clusters_of(pool, units) : 1;
    if (plan.nsplit <= n) return plan;
    const long long chunk = ((len + n - 1) / n + 63) / 64 * 64;
    if (chunk > kRangeKeys) return plan;
    plan.chunk_tokens = (int)chunk;
    plan.nsplit = (int)((len + chunk - 1) / chunk);
    return plan;
}

// How a shared call's groups are cut: items of the rows kernel are 256 (request, head) rows x chunk_tiles key tiles.
struct SharedPlan {
    int chunk_tiles, parts, tiles;  // tiles: items per kv-head
    int own_blocks;                 // the longest table behind shared blocks
    double own_work;                // estimate of the pass over the requests' own keys, in key tiles
    bool worth, any;                // shared keys are read for all requests of a group at once; some group has any
};

static bool takes_shared(int requests, int shared) { return requests > 1 && shared > 0; }

static SharedPlan plan_shared(const ekv_pool *pool, const int32_t *starts, const int32_t *shared, int G, int max_blocks) {
    const int group = pool->desc.num_q_heads / pool->desc.num_kv_heads, Hk = pool->desc.num_kv_heads;
    SharedPlan s;
    s.any = s.worth = false;
    s.chunk_tiles = 1, s.parts = 0, s.tiles = 0, s.own_blocks = 1, s.own_work = 0.;
    int longest = 0, longest_shared = 0;
    long long row_tiles = 0, saved = 0;
    long long requests = 0, alone = 0, room = max_blocks;
    for (int g = 0; g < G; ++g)
        if (takes_shared(starts[g + 1] - starts[g], shared[g])) {
            saved += (long long)(starts[g + 1] - starts[g] - 1) * shared[g];
            if (shared[g] > longest_shared) longest_shared = shared[g];
        }
    // Worth it?  The pass over the shared keys costs a launch more and its items' starts and ends; it saves their bytes, read from L2 for the most part.
    // Measured with own parts of up to 200 keys, us with / without: 32q/8kv, 2 requests over 8192 keys 16.5 / 14.5, 4 over 4096 14.7 / 12.9, over 8192 16.5 /
    // 18.5; 16 over 1024 14.7 / 12.7, over 2048 17.2 / 16.7, over 4096 17.3 / 33.6; 64 over 512 16.6 / 23.0; 28q/4kv, 16 over 2048 16.1 / 13.3, over 4096
    // 17.2 / 18.2, 64 over 1024 20.3 / 28.7; 4q/2kv d64, 16 over 4096 10.3 / 9.8.  (16 over 2048 of 32q/8kv are shared all the same: half a microsecond lost, for
    // a rule of two terms.)
    s.worth = saved * Hk * pool->desc.head_dim * 4 / 9e6 + longest_shared * (0.4 / 1024) > 13.;
    for (int g = 0; g < G; ++g) {
        const int n = starts[g + 1] - starts[g];
        if (n == 0) continue;
        const bool takes = s.worth && takes_shared(n, shared[g]);
        const int own = max_blocks - (takes ? shared[g] / 16 : 0);
        requests += n;
        if (!takes) alone += (long long)n * (shared[g] / 16);
        if (max_blocks - shared[g] / 16 < room) room = max_blocks - shared[g] / 16;
        if (own > s.own_blocks) s.own_blocks = own;
        if (!takes) continue;
        s.any = true;
        const int kt = (shared[g] + rows::kBN - 1) / rows::kBN;
        if (kt > longest) longest = kt;
        row_tiles += ((long long)n * group + rows::kItemRows - 1) / rows::kItemRows;
    }
    if (!s.any) return s;
    // Keys of their own that requests have are known as an upper bound, the room in the tables; taken as half of what the longest prefix leaves.  In units
    // of a tile's time on an SM (2.1 us), of which an SM reads 84 KB.
    s.own_work = (alone + 0.5 * requests * room) * (64 * Hk * pool->desc.head_dim) / 84e3;
    // The cut with the shortest estimated time: rounds of the machine times an item's tiles and what it costs besides them; or, as the own keys
    // are read on SMs that this pass leaves free, all of both (an item's SM comes free late: 8 tiles; own work counts up to as much as the shared, since
    // tables may be far wider than the sequences are long); and the adding up of parts.  Measured, us, by items: nine groups of 28q/4kv 32 items 97, 64 41,
    // 68 37, 96 42, 136 50; 256 requests over 16384 keys 64 items 137, 96 114, 128 124, 256 134; 16 over 8192 64 items 21.3, 128 20.5, 256 25.3.
    const double fixed = 4.0;  // tiles' worth of an item's start and write-out
    double best = 1e30;
    long long most = 4LL * pool->sm_count / (row_tiles * Hk) + 1;
    if (most > ext::kMaxParts) most = ext::kMaxParts;
    if (most < 8) most = 8;
    for (int ns = 1; ns <= most && ns <= longest; ++ns) {
        const int chunk = (longest + ns - 1) / ns;
        long long items = 0;
        double work = 0., worst = 0.;
        int parts = 0;
        for (int g = 0; g < G; ++g) {
            const int n = starts[g + 1] - starts[g];
            if (!takes_shared(n, shared[g])) continue;
            const long long rt = ((long long)n * group + rows::kItemRows - 1) / rows::kItemRows * Hk, kt = (shared[g] + rows::kBN - 1) / rows::kBN;
            const int mine = rows::part_tiles(chunk, (long long)n * group), cut = (int)((kt + mine - 1) / mine);
            const double tile = (double)chunk / mine;  // time of a tile
            items += rt * cut;
            work += rt * kt * tile;
            worst = fmax(worst, fmin((double)kt, (double)mine) * tile);
            if (cut > parts) parts = cut;
        }
        const double rounds = (double)((items + pool->sm_count - 1) / pool->sm_count), mean = work / items + fixed;
        const double beside = fmin(s.own_work / work, 1.);
        const double t = fmax(fmax(rounds * mean, worst + fixed), (items * (mean + 8. * beside) + work * beside) / pool->sm_count) + 0.08 * parts;
        if (t < best) best = t, s.chunk_tiles = chunk, s.parts = parts;
    }
    return s;
}

static size_t shared_need(const ekv_pool *pool, const SharedPlan &s, const DecodePlan &own, int B) {
    const size_t rows = (size_t)B * pool->desc.num_q_heads;
    return (own.nsplit > 1 || s.any ? parts_bytes(pool, rows * own.nsplit) : 0) + (s.any ? parts_bytes(pool, rows * s.parts) : 0);
}

static ekv_status_t check_groups(const char *who, const ekv_pool *pool, const int32_t *starts, const int32_t *shared, int G, int max_blocks, int B) {
    if (G < 0 || G > rows::kMaxGroups || (G > 0 && (!starts || !shared)) || (G == 0 && B > 0) || max_blocks < 1 || max_blocks > (1 << 26)) {
        set_error("%s: bad groups (G=%d, B=%d, max_blocks_per_seq=%d; at most %d groups)", who, G, B, max_blocks, rows::kMaxGroups);
        return EKV_ERR_INVALID;
    }
    for (int g = 0; g < G; ++g)
        if (starts[g + 1] < starts[g] || (g == 0 && starts[0] != 0) || shared[g] < 0 || shared[g] % pool->desc.block_size != 0 ||
            shared[g] / pool->desc.block_size > max_blocks) {
            set_error("%s: bad group %d (requests %d .. %d, %d shared tokens)", who, g, starts[g], starts[g + 1], shared[g]);
            return EKV_ERR_INVALID;
        }
    if (B >= 0 && G > 0 && starts[G] != B) {
        set_error("%s: the groups hold %d requests, the call %d", who, starts[G], B);
        return EKV_ERR_INVALID;
    }
    return EKV_OK;
}

template <int D>
static cudaError_t shared_decode(ekv_pool *pool, int layer, const rows::Params &rp, const ext::Params &p, bool any, int B, cudaStream_t stream) {
    if (any) {
        const cudaError_t e = launch_rows<D, rows::kShared, false, false>(pool, layer, rp, B, stream);
        if (e != cudaSuccess) return e;
    }
    return launch_ext<D, true, false, false>(pool, layer, p, B, any, stream);
}

}  // namespace ekv

using namespace ekv;

extern "C" ekv_status_t ekv_attn_decode_scored(ekv_pool_t *pool, int32_t layer, const void *q, void *out, const int32_t *block_tables,
                                               int32_t max_blocks_per_seq, const int32_t *seq_lens, int32_t B, float scale,
                                               const ekv_scores_t *scores, void *workspace, size_t workspace_bytes, void *stream) {
    static const char who[] = "ekv_attn_decode_scored";
    ekv_status_t st = check_compute(pool, layer, who);
    if (st == EKV_OK) st = check_decode(who, q, out, block_tables, max_blocks_per_seq, seq_lens, B);
    if (st == EKV_OK) st = check_scores(who, pool, scores, scale);
    if (st != EKV_OK || B == 0) return st;
    int seen = max_blocks_per_seq;  // blocks that a sequence reads at most
    if (scores->window > 0 && !scores->prefix_lens && scores->window / 16 + 2 < seen) seen = scores->window / 16 + 2;
    const DecodePlan plan = plan_ranges(pool, B, seen);
    const size_t n = (size_t)B * pool->desc.num_q_heads * plan.nsplit, need = plan.nsplit > 1 ? parts_bytes(pool, n) : 0;
    st = check_workspace(who, workspace, workspace_bytes, need);
    if (st != EKV_OK) return st;
    ext::Params p;
    fill_ext(p, pool, q, out, block_tables, max_blocks_per_seq, seq_lens, plan);
    p.part_ml = (float2 *)workspace;
    p.part_o = (float *)((uint8_t *)workspace + align256(n * sizeof(float2)));
    p.slopes = scores->slopes, p.prefix_lens = scores->prefix_lens, p.window = scores->window;
    const bool cap = scores->cap > 0.f;
    p.scale_log2 = scale * kLog2e;
    if (cap) p.cap_scale = cap_scale_of(scale, scores->cap), p.cap_log2 = cap_log2_of(scores->cap);
    const cudaError_t e = pool->desc.head_dim == 128 ? scored_decode<128>(pool, layer, p, cap, B, (cudaStream_t)stream)
                                                     : scored_decode<64>(pool, layer, p, cap, B, (cudaStream_t)stream);
    return e == cudaSuccess ? EKV_OK : cuda_fail(e, "ekv_attn_decode_scored launch");
}

extern "C" size_t ekv_attn_prefill_scored_workspace_bytes(const ekv_pool_t *pool) {
    if (!pool || pool->host_only) return 0;
    return parts_bytes(pool, (size_t)pool->sm_count * rows::kItemRows);  // a call is cut only as long as all its items run at the same time
}

extern "C" ekv_status_t ekv_attn_prefill_chunk_scored(ekv_pool_t *pool, int32_t layer, const void *q, void *out, const int32_t *block_tables,
                                                      int32_t max_blocks_per_seq, const int32_t *cu_q_lens, const int32_t *cu_q_lens_host,
                                                      const int32_t *seq_lens, int32_t R, float scale, const ekv_scores_t *scores,
                                                      void *workspace, size_t workspace_bytes, void *stream) {
    static const char who[] = "ekv_attn_prefill_chunk_scored";
    ekv_status_t st = check_compute(pool, layer, who);
    if (st != EKV_OK) return st;
    if (R < 0 || max_blocks_per_seq < 1 || max_blocks_per_seq > (1 << 26) ||
        (R > 0 && (!q || !out || !block_tables || !cu_q_lens || !cu_q_lens_host || !seq_lens)) || (((uintptr_t)q | (uintptr_t)out) & 15)) {
        set_error("%s: bad argument (R=%d, max_blocks_per_seq=%d)", who, R, max_blocks_per_seq);
        return EKV_ERR_INVALID;
    }
    st = check_scores(who, pool, scores, scale);
    if (st != EKV_OK || R == 0) return st;
    if (cu_q_lens_host[0] != 0) {
        set_error("%s: cu_q_lens[0] must be 0", who);
        return EKV_ERR_INVALID;
    }
    rows::Params p;
    fill_rows(p, pool, q, out, block_tables, max_blocks_per_seq);
    long long tiles = 0;
    int longest = 0;
    for (int r = 0; r < R; ++r) {
        const int c = cu_q_lens_host[r + 1] - cu_q_lens_host[r];
        if (cu_q_lens_host[r + 1] < cu_q_lens_host[r]) {
            set_error("%s: cu_q_lens decreases at request %d", who, r);
            return EKV_ERR_INVALID;
        }
        if (c > longest) longest = c;
        if (R <= rows::kMaxGroups) p.tile_prefix[r] = (int)tiles;
        tiles += ((long long)c * p.group + rows::kItemRows - 1) / rows::kItemRows;
    }
    const long long T = cu_q_lens_host[R];
    if (T == 0) return EKV_OK;
    if (R > rows::kMaxGroups) tiles = T * p.group / rows::kItemRows + R;
    if (tiles > 65535 || T * p.num_q_heads >= (1LL << 31) || (long long)longest * p.group >= (1LL << 29)) {
        set_error("%s: too many rows (%lld)", who, T);
        return EKV_ERR_INVALID;
    }
    if (R <= rows::kMaxGroups) p.tile_prefix[R] = (int)tiles;
    p.parts = plan_parts(pool, tiles * p.num_kv_heads, max_blocks_per_seq, scores->window, scores->prefix_lens != nullptr,
                         longest < rows::kItemRows ? longest : rows::kItemRows);
    const size_t n = (size_t)T * p.num_q_heads * p.parts;
    st = check_workspace(who, workspace, workspace_bytes, p.parts > 1 ? parts_bytes(pool, n) : 0);
    if (st != EKV_OK) return st;
    p.part_ml = (float2 *)workspace;
    p.part_o = (float *)((uint8_t *)workspace + align256(n * sizeof(float2)));
    p.cu_q_lens = cu_q_lens, p.seq_lens = seq_lens, p.R = R, p.tiles = (int)tiles;
    p.slopes = scores->slopes, p.prefix_lens = scores->prefix_lens, p.window = scores->window;
    p.q_flip = scale < 0.f ? 0x80008000u : 0u;
    if (p.q_flip) p.q_tma = 0;
    const bool cap = scores->cap > 0.f;
    p.scale_log2 = fmaxf(fabsf(scale) * kLog2e, kSmallest);
    if (cap) {
        p.cap_scale = cap_scale_of(fabsf(scale), scores->cap), p.cap_log2 = cap_log2_of(scores->cap);
        // cap * log2 e * tanh(a s) for |a s| <= 1/2: a fitted polynomial in a s (6e-7), its powers of a in the coefficients
        const double a = p.cap_scale, c = p.scale_log2;
        p.near[0] = (float)(0.99999946 * c), p.near[1] = (float)(-0.33326319 * c * a * a);
        p.near[2] = (float)(0.13190296 * c * a * a * a * a), p.near[3] = (float)(-0.04440222 * c * a * a * a * a * a * a);
        p.near_limit = p.near[3] < -1e-36f && p.near[3] > -1e30f ? 0.5f / p.cap_scale : -1.f;  // (where a coefficient leaves fp32's range: `capped` alone)
    }
    const bool d128 = pool->desc.head_dim == 128;
    cudaError_t e = d128 ? scored_prefill<128>(pool, layer, p, cap, T, (cudaStream_t)stream) : scored_prefill<64>(pool, layer, p, cap, T, (cudaStream_t)stream);
    if (e == cudaSuccess && p.parts > 1) {
        const int all = (int)(T * p.num_q_heads);
        const dim3 grid((all + ext::kCombineWarps - 1) / ext::kCombineWarps);
        e = d128 ? launch(ext::combine_rows_kernel<128>, grid, ext::kCombineWarps * 32, 0, true, 1, (cudaStream_t)stream, (const float *)p.part_o,
                          (const float2 *)p.part_ml, p.out, cu_q_lens, R, p.num_q_heads, p.parts, all)
                 : launch(ext::combine_rows_kernel<64>, grid, ext::kCombineWarps * 32, 0, true, 1, (cudaStream_t)stream, (const float *)p.part_o,
                          (const float2 *)p.part_ml, p.out, cu_q_lens, R, p.num_q_heads, p.parts, all);
    }
    return e == cudaSuccess ? EKV_OK : cuda_fail(e, "ekv_attn_prefill_chunk_scored launch");
}

extern "C" size_t ekv_attn_decode_shared_workspace_bytes(const ekv_pool_t *pool, const int32_t *group_starts, const int32_t *shared_lens,
                                                         int32_t G, int32_t max_blocks_per_seq) {
    if (!pool || pool->host_only || G < 1 || check_groups("ekv_attn_decode_shared_workspace_bytes", pool, group_starts, shared_lens, G, max_blocks_per_seq, -1) != EKV_OK ||
        group_starts[G] < 1)
        return 0;
    const SharedPlan s = plan_shared(pool, group_starts, shared_lens, G, max_blocks_per_seq);
    return shared_need(pool, s, s.any ? plan_decode(pool, group_starts[G], s.own_blocks) : plan_ranges(pool, group_starts[G], s.own_blocks), group_starts[G]);
}

extern "C" ekv_status_t ekv_attn_decode_shared(ekv_pool_t *pool, int32_t layer, const void *q, void *out, const int32_t *block_tables,
                                               int32_t max_blocks_per_seq, const int32_t *seq_lens, int32_t B, const int32_t *group_starts,
                                               const int32_t *shared_lens, int32_t G, float scale, void *workspace, size_t workspace_bytes,
                                               void *stream) {
    static const char who[] = "ekv_attn_decode_shared";
    ekv_status_t st = check_compute(pool, layer, who);
    if (st == EKV_OK) st = check_decode(who, q, out, block_tables, max_blocks_per_seq, seq_lens, B);
    if (st != EKV_OK) return st;
    if (pool->e4m3() || !(scale > 0.f) || isinf(scale)) {
        set_error("%s: EKV_BF16 pools and positive scales only (scale=%g)", who, (double)scale);
        return EKV_ERR_INVALID;
    }
    st = check_groups(who, pool, group_starts, shared_lens, G, max_blocks_per_seq, B);
    if (st != EKV_OK || B == 0) return st;
    const SharedPlan s = plan_shared(pool, group_starts, shared_lens, G, max_blocks_per_seq);
    const DecodePlan plan = s.any ? plan_decode(pool, B, s.own_blocks) : plan_ranges(pool, B, s.own_blocks);
    st = check_workspace(who, workspace, workspace_bytes, shared_need(pool, s, plan, B));
    if (st != EKV_OK) return st;
    ext::Params p;
    rows::Params rp;
    fill_ext(p, pool, q, out, block_tables, max_blocks_per_seq, seq_lens, plan);
    fill_rows(rp, pool, q, out, block_tables, max_blocks_per_seq);
    const size_t head_rows = (size_t)B * p.num_q_heads;
    uint8_t *at = (uint8_t *)workspace;
    rp.part_ml = (float2 *)at;
    rp.part_o = (float *)(at + align256(head_rows * s.parts * sizeof(float2)));
    if (s.any) at += parts_bytes(pool, head_rows * s.parts);
    p.part_ml = (float2 *)at;
    p.part_o = (float *)(at + align256(head_rows * plan.nsplit * sizeof(float2)));
    p.shared_ml = rp.part_ml, p.shared_o = rp.part_o;
    p.parts = rp.parts = s.parts;
    p.G = rp.R = G;
    // Side by side, and added up by a launch of their own, unless there is next to nothing to read beside the shared keys (4 requests over 16384 shared
    // keys, up to 64 own ones: 22.4 us for 20.5).
    p.beside = s.any && (plan.nsplit > 1 || s.own_work > 32.);
    p.scale_log2 = rp.scale_log2 = scale * kLog2e;
    rp.chunk_tiles = s.chunk_tiles;
    int tiles = 0;
    for (int g = 0; g < G; ++g) {
        const int n = group_starts[g + 1] - group_starts[g];
        const bool takes = s.worth && takes_shared(n, shared_lens[g]);
        const int kt = (shared_lens[g] + rows::kBN - 1) / rows::kBN, mine = rows::part_tiles(s.chunk_tiles, (long long)n * p.group);
        const int ns = takes ? (kt + mine - 1) / mine : 0;
        p.start[g] = rp.start[g] = group_starts[g];
        p.shared[g] = shared_lens[g], rp.shared[g] = takes ? shared_lens[g] : 0;
        p.ns[g] = (uint8_t)ns;
        rp.tile_prefix[g] = tiles;
        tiles += (int)(((long long)n * p.group + rows::kItemRows - 1) / rows::kItemRows) * ns;
    }
    p.start[G] = rp.start[G] = B;
    rp.tile_prefix[G] = rp.tiles = tiles;
    const cudaError_t e = pool->desc.head_dim == 128 ? shared_decode<128>(pool, layer, rp, p, s.any, B, (cudaStream_t)stream)
                                                     : shared_decode<64>(pool, layer, rp, p, s.any, B, (cudaStream_t)stream);
    return e == cudaSuccess ? EKV_OK : cuda_fail(e, "ekv_attn_decode_shared launch");
}

// Attention of query rows over a bf16 pool on the 5th-generation tensor cores, for scores and masks that ekv_prefill_tc.cuh does not know:
//
//   x = scale * q.k;   x = cap * tanh(x / cap);   x -= slope[head] * |p - j|          (p: the row's position, j: the key's)
//   row p sees key j:  p - window < j <= p,  or  j < prefix                            out = sum_j softmax(x)_j v_j
//
// and, without any of that, for the keys that all requests of a group share (ekv_attn_decode_shared): every row sees every key, and
// partial results go to the workspace.
//
// A work item is 256 rows of ONE kv-head -- (position, head of the group) pairs in that order, in a shared pass (request, head) -- so all
// heads that share a K/V tile meet it in one place, whatever their number, and rows of many short requests fill a tile.  The CTA has two slots (S and O in
// TMEM, 128 columns each, and a softmax warpgroup with a thread a row) that take turns: the softmax of one runs beside the MMAs of the other.
// More than 128 rows: a slot for each half, both on every key tile.  Fewer: both slots hold the SAME rows and take every other key tile; their
// results meet in TMEM, where the first slot's warps can read the other's accumulator, row by row.
// Key tiles that no row of the item sees are not read: an item's tiles are those of the prefix and those of the window.
// A call of few items cuts each one's tiles into `parts`; (m, l, O) of each part go to the workspace.
//
//   warp 0        MMA issuer: S = Q K^T (both from shared memory), O += P V (P from TMEM, V MN-major), the slots by turns
//   warp 1        TMEM; TMA producer of V tiles
//   warp 2        item scheduler: the kernel is persistent, a CTA an SM, items by cluster launch control (no word of device memory that two
//                 launches or replays could share)
//   warp 3        barriers, before anything else
//   warps 4-7     softmax and write-out of slot 0: a thread a row
//   warps 8-11    of slot 1
//   warp 12       TMA producer of K tiles
//   warps 13-15   Q rows into shared memory (by TMA where the group divides a tile), and the care of V tiles that not every row sees whole: rows of V
//                 at keys nobody sees become 0; values that are not finite at keys that some rows see and others do not are taken out (a weight of 0
//                 does not stop a NaN) and given to the rows they belong to after the write-out
// All roles run on their own clocks through rings and barriers whose phases are counted over the CTA's whole life, so that an item's Q and
// first tiles are under way while the one before is finished.
//
// What bounds it is the chain of a slot: S ready, maximum, 128 weights a thread, P stored, P V issued; the tensor pipe is busy 43 to 54 % of a long
// item.  Measured, one B200, head_dim 128, back to back, us, without modifications / capped / with the distance bias:
//   2048 positions over 14001 keys, 32q/8kv   443 to 514 (980 to 1140 TFLOP/s), by the machine / 600 to 670, by the scores' size and the power cap / 560 to 603
//   a prompt of 8192, 32q/8kv                 465 to 524 / 655 to 682 / 593 to 627
//   24 prompts of up to 1500, 28q/4kv         202 to 215 / 283 to 313 / 229 to 253
//   64 positions over 8000 keys, 32q/8kv      27 to 31 / 32 to 35 / 30 to 32
// Scores mostly beyond half the cap, the first: 1200.  With a window of 257 keys the first takes 32 to 36.  256 requests' rows over 16384 shared keys, 32q/8kv:
// 76 = 904 TFLOP/s in 128 items, with next to no own keys; beside own keys the pass is cut into 96 items and takes 99, under the profiler.
// A thread a row: two threads a row halve the chain's exponentials but pay shuffles and twice the fixed work (754 -> 791 us for 2048 capped rows).
#pragma once
#include "ekv_prefill_tc.cuh"

namespace ekv {
namespace rows {

namespace cp = cuda::ptx;
using tc::fence_after;
using tc::fence_before;

static constexpr int kBM = 128, kBN = 128;
static constexpr int kItemRows = 2 * kBM;
static constexpr int kThreads = 512;
static constexpr int kRing = 4;
static constexpr int kHalfBytes = 128 * 128;  // [128 rows][64 channels], 128-byte swizzle
static constexpr int kMaxGroups = 256;
// setmaxnreg: warps 0-3 and 12-15 kRegsUtil, 4-11 kRegsSoftmax; the shares add up to what the CTA is launched with
static constexpr int kLaunchRegs = 128, kRegsUtil = 56, kRegsSoftmax = 200;
static_assert(256 * kRegsUtil + 256 * kRegsSoftmax <= kLaunchRegs * kThreads, "setmaxnreg split exceeds the CTA's registers");
static_assert(kRegsUtil == 56 && kRegsSoftmax == 200, "the setmaxnreg instructions in the kernel carry these numbers as literals");

struct Params {
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    const int *block_tables, *cu_q_lens, *seq_lens;
    const long long *live;
    unsigned *status;
    const float *slopes;        // of the distance bias, or null
    const int *prefix_lens;     // or null
    float *part_o;              // [T * num_q_heads * parts][D]
    float2 *part_ml;            // (m, l) beside them, m in units of log2
    int max_blocks, num_q_heads, num_kv_heads, group, R;
    int tiles;                  // items of the call per kv-head and part (an upper bound if R > kMaxGroups)
    int window;                 // 0: none
    int parts;                  // parts an item's keys are cut into (shared pass: the most that any group has)
    int chunk_tiles;            // shared pass: key tiles of a part (part_tiles)
    unsigned group_magic;       // ceil(2^32 / group)
    unsigned q_flip;            // 0x80008000 for a negative scale
    int q_tma;                  // Q tiles come by TMA
    float scale_log2;           // |scale| * log2 e
    float cap_scale, cap_log2;  // with a cap: |scale| / cap, cap * log2 e (both within fp32's normal range)
    float near_limit;           // scores q.k up to there take the short polynomial s * (near[0] + near[1] s^2 + near[2] s^4 + near[3] s^6), in units of log2
    float near[4];
    int tile_prefix[kMaxGroups + 1];  // items of requests (or groups) before r, if R <= kMaxGroups
    int start[kMaxGroups + 1];        // shared pass: first request of a group ...
    int shared[kMaxGroups];           // ... and its shared keys (a multiple of 16; 0: none are taken here)
};

enum Mode { kScored = 0, kShared = 1 };

// Shared pass: key tiles of a part, for a group of so many rows.  Up to 128 of them take half the time for a tile (the slots share the tiles out).
__host__ __device__ __forceinline__ int part_tiles(int chunk, long long rows) { return rows > kBM ? chunk : 2 * chunk; }

template <int D>
struct Geo {
    static constexpr int kHalves = D / 64;
    static constexpr int kStages = D == 64 ? 4 : 2;  // of K, and of V
    static constexpr int kTileBytes = kHalves * kHalfBytes;
    static constexpr int kOffQ = 0;
    static constexpr int kOffK = 2 * kTileBytes;
    static constexpr int kOffV = kOffK + kStages * kTileBytes;
    static constexpr int kOffStage = kOffV + kStages * kTileBytes;  // of the write-out: [32 rows][128 B] a warp
    static constexpr int kStageBytes = 32 * 128;
    static constexpr int kOffBar = kOffStage + 8 * kStageBytes;
    enum Bar { Q_FULL = 0, Q_EMPTY = 1, K_FULL = 2, K_EMPTY = K_FULL + kStages, V_RAW = K_EMPTY + kStages, V_FULL = V_RAW + kStages, V_EMPTY = V_FULL + kStages,
               S_READY = V_EMPTY + kStages, P_PART = S_READY + 2, P_READY = P_PART + 2, O_READY = P_READY + 2, O_FREE = O_READY + 2, MERGE = O_FREE + 2,
               ITEM_FULL = MERGE + 1, ITEM_EMPTY = ITEM_FULL + kRing, WANT = ITEM_EMPTY + kRing, NEXT, DRAIN, NBAR };
    __device__ static __forceinline__ uint32_t arrivals(int bar) {
        if (bar == Q_FULL || (bar >= V_FULL && bar < V_EMPTY)) return 3;               // warps 13-15
        if ((bar >= P_PART && bar < O_READY) || (bar >= O_FREE && bar <= MERGE)) return 4;  // a slot's warps
        if (bar >= ITEM_EMPTY && bar < WANT) return 14;                                      // every warp that reads items
        return 1;
    }
    static constexpr int kOffFlags = kOffBar + 8 * NBAR;                  // abort flag, TMEM address, two rings of 8 masks of invalid blocks
    static constexpr int kOffNext = (kOffFlags + 72 + 15) / 16 * 16;      // answer of the launch control
    static constexpr int kOffItems = kOffNext + 16;                        // kRing slots of 16 numbers
    static constexpr int kOffMerge = kOffItems + kRing * 64;               // (m, l) of slot 1's rows
    static constexpr int kSmemBytes = kOffMerge + 128 * 8 + 1024;          // + alignment slack
    static_assert(kSmemBytes <= 232448, "shared memory");
    static constexpr uint32_t kIdescQK = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
    static constexpr uint32_t kIdescPV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);
};

template <int D>
struct Smem {
    using G = Geo<D>;
    uint32_t base;
    uint8_t *ptr;
    __device__ __forceinline__ uint32_t bar(int i) const { return base + G::kOffBar + 8 * i; }
    __device__ __forceinline__ volatile int *abort_flag() const { return (volatile int *)(ptr + G::kOffFlags); }
    __device__ __forceinline__ uint32_t *tmem_slot() const { return (uint32_t *)(ptr + G::kOffFlags + 4); }
    // Invalid blocks of a key tile, from the producer of K (for the softmax) and from that of V (for its care).  Rings of 8: a producer writes tile
    // t + 8's entry after the MMAs of tile t + 8 - kStages have read its stage, for which everything of tile t + 6 - kStages is done.
    __device__ __forceinline__ volatile int *bad_mask(int kv, uint32_t t) const { return (volatile int *)(ptr + G::kOffFlags + 8 + 32 * kv + 4 * (t & 7)); }
    __device__ __forceinline__ uint4 *response() const { return (uint4 *)(ptr + G::kOffNext); }
    __device__ __forceinline__ volatile int *item(uint32_t n) const { return (volatile int *)(ptr + G::kOffItems) + 16 * (n % kRing); }
    __device__ __forceinline__ float2 *merge() const { return (float2 *)(ptr + G::kOffMerge); }
};

// Bounded wait of a whole warp, as in ekv_prefill_tc.cuh: one poll and a vote, then a small polling loop.
template <int D>
__device__ __forceinline__ bool wait_warp(const Smem<D> &sh, int bar, uint32_t parity) {
    if (__all_sync(0xffffffffu, mbar_try_wait(sh.bar(bar), parity & 1u))) return true;
    return __all_sync(0xffffffffu, mbar_wait_polls(sh.bar(bar), parity & 1u, sh.base + Geo<D>::kOffFlags, tc::kPollLimit));
}
// keeps the compiler from making a copy of a loop for each value of a condition that the loop does not change
__device__ __forceinline__ int opaque(int v) {
    asm volatile("" : "+r"(v));
    return v;
}

// An item as its roles see it: 14 numbers in a slot of the ring.
struct Item {
    int req;          // row of the block table
    int g;            // kv-head
    int row0, rows;   // first of the request's (position, head) rows, and how many
    int q0;           // the request's first query row
    int past;         // position of its first query
    int pre;          // keys below this are seen by every row
    int kv_end;       // keys that any row of the item sees lie below this
    int tile0, n_tiles;  // this part's tiles, counted over those that are read: ...
    int n_pre, skip;  // ... tile t of them is tile t of the keys below n_pre, t + skip from there on
    int part;
};
static constexpr int kItemNan = 15;  // word of the slot: a value that is not finite was taken out of a V tile

__device__ __forceinline__ bool read_item(const volatile int *s, Item &it) {
    if (s[0] == 0) return false;
    it.req = s[1], it.g = s[2], it.row0 = s[3], it.rows = s[4], it.q0 = s[5], it.past = s[6], it.pre = s[7], it.kv_end = s[8];
    it.tile0 = s[9], it.n_tiles = s[10], it.n_pre = s[11], it.skip = s[12], it.part = s[13];
    return true;
}

// Request of a call with more than kMaxGroups requests: request r's items begin at floor(first row / 256) + r, which leaves room for all of
// them (and a few empty ones) and can be searched for in cu_q_lens itself, 32 places at a time.
__device__ __forceinline__ long long spread_first(const Params &p, int r) { return (long long)p.cu_q_lens[r] * p.group / kItemRows + r; }
__device__ __forceinline__ int spread_request(const Params &p, int idx) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = p.R;  // first(lo) <= idx < first(hi)
#pragma unroll 1
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, at = min(lo + (lane + 1) * step, hi);
        const unsigned below = __ballot_sync(0xffffffffu, at < hi && spread_first(p, at) <= idx);
        const int n = __popc(below);  // monotone: the first n places are
        hi = min(lo + (n + 1) * step, hi);
        lo += n * step;
    }
    return lo;
}

// cap * tanh(v a) of two scores v for |v a| <= 1, in units of the score: v * (1 + u Q(u)) with u = (v a)^2, fitted (by reweighted least squares) to
// the relative error, 8e-7 in fp32.  What is left of 1 and what is left of the cap go with u, so a cap far above the scores leaves them as they are.
static constexpr float kTanhFast = 1.f;
__device__ __forceinline__ float2 capped2_fast(float2 v, float2 a) {
    auto two = [](float c) { return make_float2(c, c); };
    const float2 y = __fmul2_rn(v, a), u = __fmul2_rn(y, y);
    float2 r = __ffma2_rn(two(-0.00312658f), u, two(0.01690641f));
    r = __ffma2_rn(r, u, two(-0.05176829f));
    r = __ffma2_rn(r, u, two(0.1328849f));
    r = __ffma2_rn(r, u, two(-0.3333028f));
    r = __ffma2_rn(r, u, two(1.f));
    return __fmul2_rn(r, v);
}
// 1 - 2 / (e^2y + 1): absolute error of some 2^-23; +-1 at +-infinity
__device__ __forceinline__ float tanh_any(float y) {
    const float e = fast_exp2(y * 2.8853900817779268f);
    return 1.f - __fdividef(2.f, e + 1.f);
}
// A capped score in units of log2, for v = q.k of any size: c v (1 + u Q(u)), the same kind of fit (relative error 2e-7), as far as 1 - 2 / (e^2y + 1) would lose
// the score's own accuracy; from there on that, whose 2^-22 is then 2^-21 of the result.  (That form alone is off by 2^-23 of the CAP at every score: by 0.13 at a cap of 10^6.)
static constexpr float kTanhOwn = 0.625f;
__device__ __forceinline__ float capped(float v, float a, float c, float top) {  // a: scale / cap, c: scale * log2 e, top: cap * log2 e
    const float y = v * a, u = y * y;
    float r = fmaf(0.01519537f, u, -0.0519479f);
    r = fmaf(r, u, 0.13308175f);
    r = fmaf(r, u, -0.33332341f);
    const float own = v * c * fmaf(r, u, 1.f), far = top * tanh_any(y);
    return fabsf(y) <= kTanhOwn ? own : far;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// bits 0 .. k - 1 (k in any range)
__device__ __forceinline__ unsigned below(int k) { return k >= 32 ? 0xffffffffu : k <= 0 ? 0u : (1u << k) - 1u; }

// Values that are not finite at keys that not all rows of the item see: those of the keys a row does see are added to its result (weights are
// positive: an infinity stays one, NaN and opposite infinities give NaN).  A thread a row; hardly ever called.
template <int D, typename Add>
__device__ __noinline__ void add_nonfinite(const Params &p, const uint8_t *cache, long long block_stride, const Item &it, int from, int to, int lo, int lim, Add add) {
    const long long live = *p.live;
    const int *bt = p.block_tables + (size_t)it.req * p.max_blocks;
#pragma unroll 1
    for (int key = max(from, lo); key < min(to, lim + 1); ++key) {
        const int id = bt[key >> 4];
        if (id < 0 || (long long)id >= live) continue;
        const uint32_t *v = reinterpret_cast<const uint32_t *>(cache + (long long)id * block_stride + ((long long)(p.num_kv_heads + it.g) * 16 + (key & 15)) * (2 * D));
#pragma unroll 1
        for (int c = 0; c < D / 2; ++c) {
            const uint32_t w = v[c];
            if ((w & 0x7f80u) == 0x7f80u) add(2 * c, __uint_as_float(w << 16));
            if ((w & 0x7f800000u) == 0x7f800000u) add(2 * c + 1, __uint_as_float(w & 0xffff0000u));
        }
    }
}

template <int D, int kMode, bool kCap, bool kBias>
__global__ void __launch_bounds__(kThreads, 1)
rows_kernel(const __grid_constant__ CUtensorMap kvmap, const __grid_constant__ CUtensorMap qmap, const __grid_constant__ Params p, const uint8_t *cache, long long block_stride) {
    using G = Geo<D>;
    extern __shared__ uint8_t smem_raw[];
    Smem<D> sh;
    {
        const uint32_t raw = smem_u32(smem_raw);
        sh.base = (raw + 1023u) & ~1023u;
        sh.ptr = smem_raw + (sh.base - raw);
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = p.group;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // a launch that reads the parts comes up in the tail of this one
    // Set-up, side by side: barriers, TMEM, and the first item.
    if (warp == 3) {
        if (lane == 0) {
            prefetch_tensormap(&kvmap);
            if (p.q_tma) prefetch_tensormap(&qmap);
            *sh.abort_flag() = 0;
        }
        for (int i = lane; i < G::NBAR; i += 32) mbar_init(sh.bar(i), G::arrivals(i));
        mbar_fence_init();
    }
    if (warp == 1) {
        cp::tcgen05_alloc(cp::cta_group_1, sh.tmem_slot(), 512);
        cp::tcgen05_relinquish_alloc_permit(cp::cta_group_1);
    }
    auto by_group = [&](int r) { return group == 1 ? r : (int)__umulhi((unsigned)r, p.group_magic); };
    auto low_of = [&](int pos) { return p.window > 0 ? max(0, pos - p.window + 1) : 0; };  // first key of a row's window
    int in = blockIdx.x;  // scheduler: kv-head and part of the item; its rank is the other coordinate of the grid
    // Items are listed heaviest (latest) first, the kv-heads and parts of one next to each other.  false: nothing to post for this number
    auto post = [&](int rank, volatile int *slot) {
        const int idx = p.tiles - 1 - rank;
        int g = in, part = 0, req, q0, next_q0, first, L = 0, prefix = 0;
        if (kMode == kScored && p.parts > 1) part = in / p.num_kv_heads, g = in - part * p.num_kv_heads;
        if (kMode == kShared || p.R <= kMaxGroups) {
            int lo = 0, hi = p.R;
#pragma unroll 1
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (p.tile_prefix[mid] <= idx) lo = mid;
                else hi = mid;
            }
            req = lo, first = p.tile_prefix[lo];
        } else {
            req = spread_request(p, idx);
            first = (int)spread_first(p, req);
        }
        if (kMode == kShared) {
            q0 = p.start[req], next_q0 = p.start[req + 1];
        } else {  // all loads at once
            q0 = p.cu_q_lens[req], next_q0 = p.cu_q_lens[req + 1], L = p.seq_lens[req];
            if (p.prefix_lens) prefix = p.prefix_lens[req];
        }
        const int c_r = next_q0 - q0;
        int row0, past, pre, kv_end, n_pre, skip, tile0, n_tiles;
        if (kMode == kShared) {
            const int chunk = part_tiles(p.chunk_tiles, c_r * group);
            const int all = (p.shared[req] + kBN - 1) / kBN, ns = (all + chunk - 1) / chunk, tile = (idx - first) / ns;
            part = (idx - first) - tile * ns;
            row0 = tile * kItemRows;
            past = 0, pre = kv_end = p.shared[req], n_pre = all, skip = 0;
            tile0 = part * chunk;
            n_tiles = min(chunk, all - tile0);
            req = q0;  // the first request's table names the shared blocks
        } else {
            row0 = (idx - first) * kItemRows;
        }
        const int rows = min(kItemRows, c_r * group - row0);
        if (rows <= 0) return false;
        if (kMode == kScored) {
            L = min(L, p.max_blocks * 16);
            past = L - c_r;
            if (past < 0) {  // malformed request: zero rows, latch
                if (lane == 0) atomicOr(p.status, EKV_DEV_FLAG_OOB);
                for (int r = 0; r < rows; ++r) {
                    const int pos = by_group(row0 + r);
                    const size_t at = (size_t)(q0 + pos) * p.num_q_heads + (size_t)(g * group + row0 + r - pos * group);
                    if (p.parts > 1) {
                        if (lane == 0) p.part_ml[at * p.parts + part] = make_float2(-INFINITY, 0.f);
                    } else if (lane < D / 8) {
                        reinterpret_cast<uint4 *>(p.out + at * D)[lane] = make_uint4(0u, 0u, 0u, 0u);
                    }
                }
                return false;
            }
            const int p0 = past + by_group(row0), p1 = past + by_group(row0 + rows - 1);
            pre = max(0, min(prefix, L));
            kv_end = max(p1 + 1, pre);
            n_pre = (pre + kBN - 1) / kBN;
            skip = max(0, low_of(p0) / kBN - n_pre);
            const int n = (kv_end + kBN - 1) / kBN - skip;
            tile0 = (int)((long long)n * part / p.parts);
            n_tiles = (int)((long long)n * (part + 1) / p.parts) - tile0;
        }
        if (lane == 0) {
            slot[1] = req, slot[2] = g, slot[3] = row0, slot[4] = rows, slot[5] = q0, slot[6] = past, slot[7] = pre, slot[8] = kv_end;
            slot[9] = tile0, slot[10] = n_tiles, slot[11] = n_pre, slot[12] = skip, slot[13] = part, slot[kItemNan] = 0;
        }
        return true;
    };
    bool first_posted = false;
    if (warp == 2) first_posted = post(blockIdx.y, sh.item(0));
    // One place for all warps, and the register split right behind it: every warp of a warpgroup has to execute the same setmaxnreg.
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *sh.tmem_slot();

    auto wait = [&](int bar, uint32_t parity) { return wait_warp<D>(sh, bar, parity); };
    // the CTA's n-th item, 1 = to work on, 0 = the list has ended, -1 = given up
    auto fetch = [&](uint32_t n, Item &it) {
        if (!wait(G::ITEM_FULL + (int)(n % kRing), n / kRing)) return -1;
        return read_item(sh.item(n), it) ? 1 : 0;
    };
    auto release = [&](uint32_t n) {  // this warp will not look at the item's slot again
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.bar(G::ITEM_EMPTY + (int)(n % kRing)));
    };
    auto first_key = [&](const Item &it, int t) {  // of the part's tile t
        const int l = it.tile0 + t;
        return (l < it.n_pre ? l : l + it.skip) * kBN;
    };
    uint32_t issued = 0;  // producers: tiles under way or done (Q: items)

    if (warp < 4 || warp >= 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 2) {
        // =========================== item scheduler ===========================
        bool may_draw = true;
        uint32_t draws = 0;
        auto draw = [&]() {  // rank (and kv-head, part) of a CTA that will not start now, or -1
            if (!may_draw) return -1;
            if (lane == 0) {
                mbar_expect_tx(sh.bar(G::NEXT), 16);
                cp::clusterlaunchcontrol_try_cancel(sh.response(), (uint64_t *)(sh.ptr + G::kOffBar + 8 * G::NEXT));
            }
            __syncwarp();
            // (given up or not: an answer under way must not land in the shared memory of a CTA that has left)
            if (!__all_sync(0xffffffffu, mbar_wait(sh.bar(G::NEXT), draws++ & 1u))) {
                *sh.abort_flag() = 2;
                may_draw = false;
                return -1;
            }
            const uint4 response = *sh.response();
            fence_proxy_async_smem();  // read before the next answer is written there
            __syncwarp();
            may_draw = cp::clusterlaunchcontrol_query_cancel_is_canceled(response);  // nothing left: no further question is allowed
            in = may_draw ? cp::clusterlaunchcontrol_query_cancel_get_first_ctaid_x<int>(response) : 0;
            return may_draw ? cp::clusterlaunchcontrol_query_cancel_get_first_ctaid_y<int>(response) : -1;
        };
        int item = blockIdx.y;
        bool posted = first_posted;
#pragma unroll 1
        for (uint32_t n = 0;; ++n) {
            volatile int *slot = sh.item(n);
            // not before the producer has come to the last four tiles of the item before: an item drawn earlier would wait for this CTA while another
            // stands idle (drawing and decoding one takes some 4000 cycles)
            if (n > 0) (void)wait(G::WANT, n - 1);
            if (n >= kRing) (void)wait(G::ITEM_EMPTY + (int)(n % kRing), n / kRing - 1);
            while (!posted) {
                item = draw();
                // (a wait ran out: the CTAs that have not started, and would wait as long, are not to; the list ends when all are drawn)
                posted = item < 0 || (!*sh.abort_flag() && post(item, slot));
            }
            posted = false;
            if (lane == 0) {
                slot[0] = item >= 0;
                __threadfence_block();
                mbar_arrive(sh.bar(G::ITEM_FULL + (int)(n % kRing)));
            }
            __syncwarp();
            if (item < 0) break;
        }
    } else if (warp == 0) {
        // =========================== MMA issuer ===========================
        constexpr uint64_t kHi = (uint64_t)tc::kDescHi << 32;
        const uint64_t q_d = kHi | tc::desc_lo(sh.base + G::kOffQ, 16), k_d = kHi | tc::desc_lo(sh.base + G::kOffK, 16),
                       v_d = kHi | tc::desc_lo(sh.base + G::kOffV, kHalfBytes);
        uint32_t t0 = 0;                 // key tiles of the items before
        uint32_t cs[2] = {0, 0};         // ... and those that each slot saw
        uint32_t co[2] = {0, 0};         // items in which a slot saw any
        bool ok = true;
#pragma unroll 1
        for (uint32_t n = 0; ok; ++n) {
            Item it;
            if (fetch(n, it) <= 0) break;
            const int n_tiles = it.n_tiles;
            const int sh2 = opaque(it.rows > kBM ? 1 : 0);  // steps a tile takes: one for each slot, or one
            release(n);
            ok = wait(G::Q_FULL, n);
            if (!ok) break;
            // Steps alternate between the slots, so that the softmax of one runs beside the MMAs of the other: step u is P V of slot x = u & 1 on
            // its key tile number i = u >> 1, and Q K^T for the slot's next one; steps -2 and -1 only bring the first scores.
            const int step_max = n_tiles << sh2;
#pragma unroll 1
            for (int u = -2; u < step_max && ok; ++u) {
                const int x = u & 1, i = u >> 1;
                const int j = u >> sh2, jn = (u + 2) >> sh2;  // the part's key tiles of the two
                const uint32_t s = (t0 + (uint32_t)j) % G::kStages, s1 = (t0 + (uint32_t)jn) % G::kStages;
                const int pv = opaque(u >= 0), more = opaque(jn < n_tiles), closes = opaque(x >= sh2), opens = opaque(x == 0 || sh2 == 0);  // the last and the first slot to read these stages
                const uint32_t t_s = tmem + 128 * x, t_o = tmem + 256 + 128 * x;
                const uint64_t vd = v_d + s * (G::kTileBytes >> 4);
                if (!pv && !more) continue;
                // (what comes early is waited for first, and once: a wait takes some 300 cycles beside busy special functions)
                if (more && opens) ok = wait(G::K_FULL + (int)s1, (t0 + (uint32_t)jn) / G::kStages);
                if (pv) {
                    if (ok && opens) ok = wait(G::V_FULL + (int)s, (t0 + (uint32_t)j) / G::kStages);
                    // the slot's accumulator of the item before has been read
                    if (ok && i == 0 && co[x] > 0) ok = wait(G::O_FREE + x, co[x] - 1);
                    if (ok) ok = wait(G::P_PART + x, cs[x] + (uint32_t)i);
                    if (!ok) break;
                    fence_after();
                    if (tc::elect_one()) {  // keys 0..95 while the softmax warps finish the rest
#pragma unroll
                        for (int k = 0; k < tc::kPartSteps; ++k) tc::mma_ts(t_o, t_s + 8 * k, vd + ((k * 2048) >> 4), G::kIdescPV, (i > 0 || k > 0) ? 1u : 0u);
                    }
                    __syncwarp();
                    ok = wait(G::P_READY + x, cs[x] + (uint32_t)i);
                }
                if (!ok) break;
                fence_after();
                if (tc::elect_one()) {
                    if (pv) {
#pragma unroll
                        for (int k = tc::kPartSteps; k < kBN / 16; ++k) tc::mma_ts(t_o, t_s + 8 * k, vd + ((k * 2048) >> 4), G::kIdescPV, 1u);
                        if (closes) tc::mma_commit_one(sh.bar(G::V_EMPTY + (int)s));
                        if (!more) tc::mma_commit_one(sh.bar(G::O_READY + x));
                    }
                    if (more) {
                        const uint64_t qd = q_d + (uint32_t)(x & sh2) * (G::kTileBytes >> 4), kd = k_d + s1 * (G::kTileBytes >> 4);
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const uint32_t off = ((k >> 2) * kHalfBytes + (k & 3) * 32) >> 4;
                            tc::mma_ss(t_s, qd + off, kd + off, G::kIdescQK, k > 0 ? 1u : 0u);
                        }
                        tc::mma_commit_one(sh.bar(G::S_READY + x));  // the slot's next scores, and its O up to this tile
                        if (closes) tc::mma_commit_one(sh.bar(G::K_EMPTY + (int)s1));
                        if (closes && jn + 1 == n_tiles) tc::mma_commit_one(sh.bar(G::Q_EMPTY));  // the item's last scores
                    }
                }
                __syncwarp();
            }
            if (ok && n_tiles == 0) tc::mma_commit(sh.bar(G::Q_EMPTY));
            t0 += (uint32_t)n_tiles;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint32_t mine = sh2 ? (uint32_t)n_tiles : (uint32_t)(n_tiles - x + 1) >> 1;
                cs[x] += mine;
                co[x] += mine > 0 ? 1u : 0u;
            }
        }
        // every MMA this thread issued must be finished before TMEM is released
        tc::mma_commit(sh.bar(G::DRAIN));
        (void)wait(G::DRAIN, 0);
    } else if (warp == 12 || warp == 1) {
        // =========================== TMA producers: K tiles, V tiles ===========================
        // (One for each: a V tile waits for P V two tiles before, and the K tile after it must not wait with it.)
        const int kv = warp == 1;
        const int full = kv ? G::V_RAW : G::K_FULL, empty = kv ? G::V_EMPTY : G::K_EMPTY;
        const uint32_t to = sh.base + (kv ? G::kOffV : G::kOffK);
        const long long live = *p.live;
        bool ok = true;
#pragma unroll 1
        for (uint32_t n = 0; ok; ++n) {
            Item it;
            if (fetch(n, it) <= 0) break;
            release(n);
            const int *bt = p.block_tables + (size_t)it.req * p.max_blocks;
            // Keys between the prefix and the first row's window are seen by no row of the item: what the table names for blocks of nothing else does not
            // matter (they may have been given back since the window passed them).
            const int past_by = kMode == kShared ? 0 : low_of(it.past + by_group(it.row0));
            auto load_id = [&](int t) {  // lane l: id of block l % 8 of the part's tile t (-1 nothing to load, -2 invalid)
                int id = -1;
                const int bi = (first_key(it, t) >> 4) + (lane & 7);
                if (t < it.n_tiles && bi * 16 < it.kv_end) {
                    id = bt[bi];
                    if (id < 0 || (long long)id >= live) id = bi * 16 < it.pre || bi * 16 + 16 > past_by ? -2 : -1;
                }
                return id;
            };
            int id_next = load_id(0);
            if (it.n_tiles == 0 && lane == 0 && !kv) mbar_arrive(sh.bar(G::WANT));
#pragma unroll 1
            for (int j = 0; j < it.n_tiles; ++j) {
                const int id_raw = id_next;
                id_next = load_id(j + 1);
                const unsigned oob = __ballot_sync(0xffffffffu, id_raw == -2) & 0xffu;
                const unsigned bad = __ballot_sync(0xffffffffu, id_raw < 0) & 0xffu;
                const int id = id_raw < 0 ? 0 : id_raw;  // masked later; block 0 is always mapped
                const int b = lane & (8 * G::kHalves - 1), blk = b / G::kHalves, half = b % G::kHalves;
                const int my_id = __shfl_sync(0xffffffffu, id, blk);
                const uint32_t s = issued % G::kStages;
                if (j == max(0, it.n_tiles - 4) && lane == 0 && !kv) mbar_arrive(sh.bar(G::WANT));
                if (issued >= G::kStages && !(ok = wait(empty + (int)s, issued / G::kStages - 1))) break;
                if (lane == 0) {
                    if (oob && !kv) atomicOr(p.status, EKV_DEV_FLAG_OOB);
                    *sh.bad_mask(kv, issued) = (int)bad;
                    mbar_expect_tx(sh.bar(full + (int)s), G::kTileBytes);
                }
                __syncwarp();
                if (lane < 8 * G::kHalves)
                    tma_load_3d(to + s * G::kTileBytes + half * kHalfBytes + blk * 2048, &kvmap, 64 * half, (it.g + (kv ? p.num_kv_heads : 0)) * 16, my_id,
                                sh.bar(full + (int)s));
                ++issued;
            }
        }
    } else if (warp >= 13) {
        // =========================== Q rows, and the care of V tiles ===========================
        constexpr int kPieces = D / 8;  // 16-byte pieces of a row
        const int ct = threadIdx.x - 13 * 32;  // of 96
        uint32_t t = 0;
        bool ok = true;
        auto load_q = [&](const Item &it) {
            const int pos0 = by_group(it.row0), tiles = it.rows > kBM ? 2 : 1;
            if (p.q_tma) {  // (rows behind the item's last one are some other request's: nobody looks at their results)
                if (lane == 0 && warp == 13) mbar_expect_tx(sh.bar(G::Q_FULL), tiles * G::kTileBytes);
                else if (lane == 0) mbar_arrive(sh.bar(G::Q_FULL));
                __syncwarp();
                if (warp == 13 && lane < tiles * G::kHalves) {
                    const int x = lane / G::kHalves, half = lane % G::kHalves;
                    tma_load_3d(sh.base + G::kOffQ + x * G::kTileBytes + half * kHalfBytes, &qmap, 64 * half, it.g * group, it.q0 + pos0 + x * (kBM / group),
                                sh.bar(G::Q_FULL));
                }
                return;
            }
            const int head0 = it.row0 - pos0 * group;
            const __nv_bfloat16 *src = p.q + ((size_t)(it.q0 + pos0) * p.num_q_heads + (size_t)it.g * group) * D;
            auto place = [&](int i) {  // of piece i of the tiles
                const int r = i / kPieces, c = i % kPieces;
                return sh.base + G::kOffQ + (r >> 7) * G::kTileBytes + (c >> 3) * kHalfBytes + (r & 127) * 128 + (((c ^ r) & 7) << 4);
            };
#pragma unroll 2
            for (int i = ct; i < tiles * kBM * kPieces; i += 96) {
                const int r = i / kPieces, c = i % kPieces;
                const bool there = r < it.rows;
                const int h = head0 + (there ? r : 0);
                cp_async_16(place(i), src + (size_t)(by_group(h) * (p.num_q_heads - group) + h) * D + c * 8, there ? 16u : 0u);
            }
            cp_async_commit();
            cp_async_wait_all();
            if (p.q_flip) {  // a negative scale: its sign goes into Q
#pragma unroll 1
                for (int i = ct; i < tiles * kBM * kPieces; i += 96) {
                    const uint4 v = lds_16(place(i));
                    sts_16(place(i), make_uint4(v.x ^ p.q_flip, v.y ^ p.q_flip, v.z ^ p.q_flip, v.w ^ p.q_flip));
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(sh.bar(G::Q_FULL));
        };
#pragma unroll 1
        for (uint32_t n = 0; ok; ++n) {
            Item it;
            if (fetch(n, it) <= 0) break;
            if (n > 0 && !wait(G::Q_EMPTY, n - 1)) break;
            load_q(it);
            if (p.q_tma) ++issued;
            const int p0 = it.past + by_group(it.row0), p1 = it.past + by_group(it.row0 + it.rows - 1);
            const int lo1 = kMode == kShared ? 0 : low_of(p1);
#pragma unroll 1
            for (int j = 0; j < it.n_tiles && ok; ++j, ++t) {
                const uint32_t s = t % G::kStages;
                ok = wait(G::V_RAW + (int)s, t / G::kStages);
                if (!ok) break;
                const int key0 = first_key(it, j), bad = *sh.bad_mask(1, t);
                uint8_t *tile = sh.ptr + G::kOffV + s * G::kTileBytes;
                auto piece = [&](int i) { return reinterpret_cast<uint4 *>(tile + (i % kPieces >> 3) * kHalfBytes + (i / kPieces) * 128 + (i & 7) * 16); };
                bool touched = false;
                if (kMode == kScored && !(key0 + kBN <= it.pre || (key0 + kBN - 1 <= p0 && key0 >= lo1))) {
                    // keys that some rows see and others do not: at the window's lower edge, and from the first row's position on
                    bool seen_nan = false;
                    const int upper = max(p0 + 1, max(lo1, it.pre));
#pragma unroll 1
                    for (int edge = 0; edge < 2; ++edge) {
                        const int from = max(0, (edge ? upper : it.pre) - key0), to = min(kBN, (edge ? it.kv_end : lo1) - key0);  // rows of the tile
#pragma unroll 2
                        for (int i = from * kPieces + ct; i < to * kPieces; i += 96) {
                            const uint4 v = *piece(i);
                            uint32_t w[4] = {v.x, v.y, v.z, v.w}, any = 0;
#pragma unroll
                            for (int k = 0; k < 4; ++k) any |= ((w[k] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
                            if (any) {
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    if ((w[k] & 0x7f80u) == 0x7f80u) w[k] &= 0xffff0000u;
                                    if ((w[k] & 0x7f800000u) == 0x7f800000u) w[k] &= 0x0000ffffu;
                                }
                                *piece(i) = make_uint4(w[0], w[1], w[2], w[3]);
                                seen_nan = true;
                            }
                        }
                    }
                    if (seen_nan) sh.item(n)[kItemNan] = 1;
                    touched = true;
                }
                if (key0 + kBN > it.kv_end || bad) {  // keys that nobody sees: a slot that was never written may hold anything
                    const int end = max(0, it.kv_end - key0);
#pragma unroll 2
                    for (int i = (bad ? 0 : end * kPieces) + ct; i < kBN * kPieces; i += 96) {
                        const int r = i / kPieces;
                        if (r >= end || ((bad >> (r >> 4)) & 1)) *piece(i) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    touched = true;
                }
                if (touched) fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(sh.bar(G::V_FULL + (int)s));
            }
            release(n);
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        // =========================== softmax + write-out of one slot ===========================
        const int x = (warp - 4) >> 2;
        const int wrow0 = (warp & 3) << 5;    // TMEM lanes wrow0 .. +31 belong to this warp
        const int row = wrow0 | lane;         // row of the tile = TMEM lane
        const uint32_t t_s = tmem + ((uint32_t)wrow0 << 16) + 128 * x;
        const uint32_t t_o = tmem + ((uint32_t)wrow0 << 16) + 256 + 128 * x;
        uint32_t t0 = 0, cs = 0, co = 0, cm = 0;  // tiles of the items before, those of this slot, items in which it had any, merges
        bool ok = true;
        auto publish = [&](int bar) {  // this warp's rows of P are in TMEM
            cp::tcgen05_wait_st();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(sh.bar(bar));
        };
#pragma unroll 1
        for (uint32_t n = 0; ok; ++n) {
            Item it;
            if (fetch(n, it) <= 0) break;
            const bool by_rows = it.rows > kBM;
            const int rx = by_rows ? x : 0;                                    // its row tile
            const int n_it = by_rows ? it.n_tiles : (it.n_tiles - x + 1) >> 1;  // its key tiles
            const int dj = opaque(by_rows ? 0 : 1), j0 = opaque(by_rows ? 0 : x);  // the i-th of them is the part's tile (i << dj) + j0
            const int r_item = min(rx * kBM + row, it.rows - 1);
            const int pos_in = by_group(it.row0 + r_item);
            const int lim = it.past + pos_in, lo = kMode == kShared ? 0 : low_of(lim);  // the row's window: keys lo .. lim
            // tiles that every row of the slot sees whole take no mask
            const int lim_all = it.past + by_group(it.row0 + rx * kBM);
            const int lo_all = kMode == kShared ? 0 : low_of(it.past + by_group(it.row0 + min(rx * kBM + kBM, it.rows) - 1));
            const float slope = kBias ? p.slopes[it.g * group + it.row0 + r_item - pos_in * group] * 1.4426950408889634f : 0.f;
            float m_run = -INFINITY, l_run = 0.f;
#pragma unroll 1
            for (int i = 0; i < n_it && ok; ++i) {
                ok = wait(G::S_READY + x, cs + (uint32_t)i);
                if (!ok) break;
                fence_after();
                const int j = (i << dj) + j0;
                const int key0 = first_key(it, j);
                const int bad = *sh.bad_mask(0, t0 + (uint32_t)j);
                float sv[128];
                uint32_t(&raw)[128] = reinterpret_cast<uint32_t(&)[128]>(sv);
                auto load_s = [&]() {
                    cp::tcgen05_ld_32x32b(reinterpret_cast<uint32_t(&)[32]>(raw[0]), t_s);
                    cp::tcgen05_ld_32x32b(reinterpret_cast<uint32_t(&)[32]>(raw[32]), t_s + 32);
                    cp::tcgen05_ld_32x32b(reinterpret_cast<uint32_t(&)[32]>(raw[64]), t_s + 64);
                    cp::tcgen05_ld_32x32b(reinterpret_cast<uint32_t(&)[32]>(raw[96]), t_s + 96);
                    cp::tcgen05_wait_ld();
                };
                load_s();
                auto seen = [&](int cc) {  // which of keys 32 cc .. + 31 of the tile the row sees
                    const int c0 = key0 + 32 * cc;
                    const unsigned b2 = ((unsigned)bad >> (2 * cc)) & 3u;
                    const unsigned broken = ((b2 & 1u) ? 0x0000ffffu : 0u) | ((b2 & 2u) ? 0xffff0000u : 0u);
                    unsigned vis = below(it.pre - c0);
                    if (kMode == kScored) vis |= below(lim + 1 - c0) & ~below(lo - c0);
                    return vis & ~broken;
                };
                const bool whole = (key0 + kBN <= it.pre || (kMode == kScored && key0 + kBN - 1 <= lim_all && key0 >= lo_all)) && bad == 0;
                // ---- the cap.  Small scores that every row sees wait for the exponential, whose code has the polynomial in it; with a bias, up to the
                // cap, they are worked on in place; the rest goes through TMEM in a small loop, score by score as large as it is.
                constexpr bool kNear = kCap && !kBias;
                auto near_score = [&](float v) { return v * (p.near[0] + v * v * (p.near[1] + v * v * (p.near[2] + v * v * p.near[3]))); };
                bool near = false;
                float mul = p.scale_log2;
                if (kCap) {
                    float b0 = 0.f, b1 = 0.f;
#pragma unroll
                    for (int c = 0; c < 128; c += 4) b0 = max3(b0, fabsf(sv[c]), fabsf(sv[c + 1])), b1 = max3(b1, fabsf(sv[c + 2]), fabsf(sv[c + 3]));
                    const float far = fmaxf(b0, b1);
                    // (where rows do not see all of the tile, what they do not see may be anything, and no bit of the result is to depend on it)
                    const bool small = __all_sync(0xffffffffu, whole && (kNear ? far <= p.near_limit : far * p.cap_scale <= kTanhFast));
                    near = kNear && small;
                    if (kBias && small) {
                        const float2 a = make_float2(p.cap_scale, p.cap_scale);
#pragma unroll
                        for (int c = 0; c < 128; c += 2) {
                            const float2 v = capped2_fast(make_float2(sv[c], sv[c + 1]), a);
                            sv[c] = v.x, sv[c + 1] = v.y;
                        }
                    } else if (!near) {
                        mul = 1.f;
#pragma unroll 1
                        for (int cc = 0; cc < 4; ++cc) {
                            float v[32];
                            tc::tmem_ld32(v, t_s + 32 * cc);
#pragma unroll
                            for (int c = 0; c < 32; ++c) v[c] = capped(v[c], p.cap_scale, p.scale_log2, p.cap_log2);
                            tc::tmem_st32(t_s + 32 * cc, v);
                        }
                        cp::tcgen05_wait_st();
                        load_s();
                    }
                }
                if (kBias) {  // sv becomes the whole score in units of log2
                    const float2 sc = make_float2(mul, mul);
                    if (key0 + kBN - 1 <= lim_all) {  // keys behind every row: |p - j| = p - j
                        const float first = -slope * (float)(lim - key0);
                        const float2 sl = make_float2(slope, slope), f2 = make_float2(first, first);
#pragma unroll
                        for (int c = 0; c < 128; c += 2) {
                            const float2 b = __ffma2_rn(make_float2((float)c, (float)(c + 1)), sl, f2);
                            const float2 v = __ffma2_rn(make_float2(sv[c], sv[c + 1]), sc, b);
                            sv[c] = v.x, sv[c + 1] = v.y;
                        }
                    } else {
                        const float d0 = (float)(lim - key0);
#pragma unroll
                        for (int c = 0; c < 128; ++c) sv[c] = fmaf(sv[c], mul, -slope * fabsf(d0 - (float)c));
                    }
                    mul = 1.f;
                }
                if (!whole) {
#pragma unroll
                    for (int cc = 0; cc < 4; ++cc) {
                        const unsigned vis = seen(cc);
                        if (vis != 0xffffffffu) {
#pragma unroll
                            for (int c = 0; c < 32; ++c)
                                if (!((vis >> c) & 1u)) sv[32 * cc + c] = -INFINITY;
                        }
                    }
                }
                float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
                for (int c = 0; c < 128; c += 4) {
                    mx0 = fmaxf(mx0, sv[c]);
                    mx1 = fmaxf(mx1, sv[c + 1]);
                    mx2 = fmaxf(mx2, sv[c + 2]);
                    mx3 = fmaxf(mx3, sv[c + 3]);
                }
                float m_tile = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3));
                m_tile = near ? near_score(m_tile) : m_tile * mul;  // (tanh grows with its argument)
                // ---- lazy rescale: raise the reference max only when it is far behind
                const bool raise = m_tile > m_run + tc::kRescaleThreshold;  // also true for the first finite tile
                if (__any_sync(0xffffffffu, raise)) {
                    const float m_new = raise ? m_tile : m_run;
                    const float alpha = (raise && m_run > -INFINITY) ? fast_exp2(m_run - m_new) : (raise ? 0.f : 1.f);
                    m_run = m_new;
                    l_run *= alpha;
                    if (i > 0) {  // O holds the sum over earlier tiles and no MMA touches it right now
#pragma unroll 1
                        for (int cc = 0; cc < D / 32; ++cc) {
                            float ov[32];
                            tc::tmem_ld32(ov, t_o + 32 * cc);
#pragma unroll
                            for (int c = 0; c < 32; ++c) ov[c] *= alpha;
                            tc::tmem_st32(t_o + 32 * cc, ov);
                        }
                    }
                }
                const float m_use = m_run > -INFINITY ? m_run : 0.f;
                // ---- P = exp2(x - m) (a masked -inf gives 0), row sum in fp32, bf16 pairs into the S columns.  bf16 because both operands of an MMA have one type and
                // V is bf16: a weight is off by up to 2^-8 of itself, the sum that divides is not.  (Two bf16 a weight would double the P V MMAs.)  Against
                // 64 bits relative errors are 0.0019 to 0.0023 (2048 over 14001 keys 0.0021), of which 0.0017 is the result's own rounding.
                float2 acc_a = make_float2(0.f, 0.f), acc_b = make_float2(0.f, 0.f);
                const float2 sc2 = make_float2(mul, mul), nm2 = make_float2(-m_use, -m_use);
                auto weights = [&](auto score) {  // score(v): x - m of two keys
    #pragma unroll
                    for (int cc = 0; cc < 4; ++cc) {
                        uint32_t pk[16];
#pragma unroll
                        for (int c = 0; c < 32; c += 4) {
                            const float2 xa = score(make_float2(sv[32 * cc + c], sv[32 * cc + c + 1]));
                            const float2 xb = score(make_float2(sv[32 * cc + c + 2], sv[32 * cc + c + 3]));
                            const float2 pa = make_float2(fast_exp2(xa.x), fast_exp2(xa.y));
                            const float2 pb = make_float2(fast_exp2(xb.x), fast_exp2(xb.y));
                            acc_a = __fadd2_rn(acc_a, pa);
                            acc_b = __fadd2_rn(acc_b, pb);
                            pk[c >> 1] = pack_bf16x2(pa.x, pa.y);
                            pk[(c >> 1) + 1] = pack_bf16x2(pb.x, pb.y);
                        }
                        cp::tcgen05_st_32x32b(t_s + 16 * cc, pk);
                        if (cc == tc::kPartSteps / 2 - 1) publish(G::P_PART + x);  // 96 keys stored
                    }
                };
                if (kNear && near) {
                    const float2 c0 = make_float2(p.near[0], p.near[0]), c1 = make_float2(p.near[1], p.near[1]), c2 = make_float2(p.near[2], p.near[2]), c3 = make_float2(p.near[3], p.near[3]);
                    weights([&](float2 v) {
                        const float2 u = __fmul2_rn(v, v);
                        return __ffma2_rn(v, __ffma2_rn(u, __ffma2_rn(u, __ffma2_rn(u, c3, c2), c1), c0), nm2);
                    });
                } else {
                    weights([&](float2 v) { return __ffma2_rn(v, sc2, nm2); });
                }
                l_run += (acc_a.x + acc_a.y) + (acc_b.x + acc_b.y);
                publish(G::P_READY + x);
            }
            if (!ok) break;
            t0 += (uint32_t)it.n_tiles;
            cs += (uint32_t)n_it;
            if (n_it > 0 && !(ok = wait(G::O_READY + x, co))) break;
            if (n_it > 0) ++co;
            fence_after();  // every MMA that wrote the slot's O has completed

            // ---- slots that share rows: the second one leaves its (m, l) in shared memory, the first one takes both accumulators
            const int merge = opaque(!by_rows && it.n_tiles > 1);
            float w0 = 1.f, w1 = 0.f;
            if (merge) {
                if (x == 1) {
                    sh.merge()[row] = make_float2(m_run, l_run);
                    fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(sh.bar(G::MERGE));
                } else {
                    if (!(ok = wait(G::MERGE, cm))) break;
                    fence_after();
                    const float2 o = sh.merge()[row];
                    const float m_new = fmaxf(m_run, o.x);
                    w0 = m_run > -INFINITY ? fast_exp2(m_run - m_new) : 0.f;
                    w1 = o.x > -INFINITY ? fast_exp2(o.x - m_new) : 0.f;
                    l_run = l_run * w0 + o.y * w1;  // (a slot whose scores were all NaN has no maximum, but its sum is NaN, and stays so times 0)
                    m_run = m_new;
                }
                ++cm;
            }
            if (by_rows || x == 0) {
                const bool there = rx * kBM + row < it.rows;
                const size_t at = (size_t)(it.q0 + pos_in) * p.num_q_heads + (size_t)(it.g * group + it.row0 + r_item - pos_in * group);
                const int to_parts = opaque(kMode == kShared || p.parts > 1);
                const float inv = to_parts ? 1.f : (l_run == 0.f ? 0.f : 1.f / l_run);
                w0 *= inv, w1 *= inv;
                __nv_bfloat16 *out = p.out + at * D;
                float *part_o = p.part_o + (at * p.parts + it.part) * D;
                // 128 bytes of a row at a time -- 64 channels of bf16, or 32 of a part's fp32 -- go through shared memory, so that eight lanes write
                // a row's 128 bytes together.  (A thread a row, straight from the registers, took four times as long.)
                uint8_t *stage = sh.ptr + G::kOffStage + (warp - 4) * G::kStageBytes;
                const int piece = lane & 7, sub = lane >> 3;
                uint8_t *const to = to_parts ? reinterpret_cast<uint8_t *>(p.part_o) : reinterpret_cast<uint8_t *>(p.out);
                const int row_bytes = to_parts ? 4 * D : 2 * D, out_parts = to_parts ? p.parts : 1, out_part = to_parts ? it.part : 0;
                auto put = [&](int i, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
                    *reinterpret_cast<uint4 *>(stage + lane * 128 + ((i ^ (lane & 7)) << 4)) = make_uint4(a, b, c, d);
                };
                const int chunks = n_it > 0 ? D / 32 : 0;
#pragma unroll 1
                for (int ch = 0; ch < chunks; ++ch) {  // 32 channels of the result
                    float ov[32];
                    tc::tmem_ld32(ov, t_o + 32 * ch);
                    if (merge) {
                        float o1[32];
                        tc::tmem_ld32(o1, t_o + 128 + 32 * ch);
#pragma unroll
                        for (int c = 0; c < 32; ++c) ov[c] = ov[c] * w0 + o1[c] * w1;
                    } else {
#pragma unroll
                        for (int c = 0; c < 32; ++c) ov[c] *= w0;
                    }
                    if (ch == chunks - 1) {  // the accumulator has been read
                        fence_before();
                        __syncwarp();
                        if (lane == 0) {
                            mbar_arrive(sh.bar(G::O_FREE + x));
                            if (merge) mbar_arrive(sh.bar(G::O_FREE + 1));
                        }
                    }
                    if (to_parts) {
                        uint32_t(&w)[32] = reinterpret_cast<uint32_t(&)[32]>(ov);
#pragma unroll
                        for (int i = 0; i < 8; ++i) put(i, w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            put((ch & 1) * 4 + i, pack_bf16x2(ov[8 * i], ov[8 * i + 1]), pack_bf16x2(ov[8 * i + 2], ov[8 * i + 3]),
                                pack_bf16x2(ov[8 * i + 4], ov[8 * i + 5]), pack_bf16x2(ov[8 * i + 6], ov[8 * i + 7]));
                        if ((ch & 1) == 0) continue;
                    }
                    __syncwarp();
                    uint4 v[8];  // all reads at once: one takes some 300 cycles beside busy special functions
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = *reinterpret_cast<const uint4 *>(stage + (4 * k + sub) * 128 + ((piece ^ ((4 * k + sub) & 7)) << 4));
                    uint8_t *const at_piece = to + (to_parts ? ch : ch >> 1) * 128 + piece * 16;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int rr = rx * kBM + wrow0 + 4 * k + sub;
                        const int pos = by_group(it.row0 + rr);
                        const int i = (it.q0 + pos) * p.num_q_heads + it.g * group + it.row0 + rr - pos * group;  // (T * heads < 2^31)
                        if (rr < it.rows) *reinterpret_cast<uint4 *>(at_piece + ((size_t)i * out_parts + out_part) * row_bytes) = v[k];
                    }
                    __syncwarp();
                }
                if (n_it == 0 && there && !to_parts)
                    for (int c = 0; c < D / 8; ++c) reinterpret_cast<uint4 *>(out)[c] = make_uint4(0u, 0u, 0u, 0u);
                if (there && to_parts) p.part_ml[at * p.parts + it.part] = make_float2(n_it > 0 ? m_run : -INFINITY, n_it > 0 ? l_run : 0.f);
                if (kMode == kScored && sh.item(n)[kItemNan] && there) {
                    const int p0 = it.past + by_group(it.row0), lo1 = low_of(it.past + by_group(it.row0 + it.rows - 1));
                    auto add = [&](int c, float v) {
                        if (to_parts) part_o[c] += v;
                        else out[c] = __float2bfloat16_rn(__bfloat162float(out[c]) + v);
                    };
                    // keys that not every row sees, in this part's tiles: those of the window's lower edge, and those from the first row's position on
#pragma unroll 1
                    for (int t = 0; t < it.n_tiles; ++t) {
                        const int k0 = first_key(it, t);
                        const int upper = max(p0 + 1, max(lo1, it.pre));
                        add_nonfinite<D>(p, cache, block_stride, it, max(k0, it.pre), min(k0 + kBN, lo1), lo, lim, add);
                        add_nonfinite<D>(p, cache, block_stride, it, max(k0, upper), min(k0 + kBN, it.kv_end), lo, lim, add);
                    }
                }
            }
            release(n);
        }
    }

    // ---- teardown: everybody meets, copies in flight get a bounded chance to land, TMEM goes back
    fence_before();
    __syncthreads();
    fence_after();
    if (*sh.abort_flag()) {
        if (warp == 12 || warp == 1)
            for (uint32_t t = issued > G::kStages ? issued - G::kStages : 0; t < issued; ++t)
                (void)mbar_wait(sh.bar((warp == 1 ? G::V_RAW : G::K_FULL) + (int)(t % G::kStages)), (t / G::kStages) & 1u, 100000000ull);
        if (warp == 13 && issued > 0)  // (the other two warps may have given up in front of it, without arriving: then the limit is the chance)
            (void)mbar_wait(sh.bar(G::Q_FULL), (issued - 1) & 1u, 100000000ull);
        if (threadIdx.x == 0) atomicOr(p.status, EKV_DEV_FLAG_TIMEOUT);  // a wait ran out
    }
    __syncthreads();
    if (warp == 1) cp::tcgen05_dealloc(cp::cta_group_1, tmem, 512);
}

}  // namespace rows
}  // namespace ekv

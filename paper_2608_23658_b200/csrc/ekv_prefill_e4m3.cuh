// ekv_attn_prefill_chunk over an 8-bit pool, on the 5th-generation tensor cores.
//
//   S = (Q K_code^T) * s_K(block),   P = exp2(S - m),   O = sum P (V_code * s_V(block)) / sum P,   keys 0 .. position of the row
//
// tcgen05 takes no operand pair of bf16 and e4m3, and Q or P rounded to e4m3 would lose half their bits, so the codes become
// 16-bit operands on their way into shared memory.  That costs instructions for every key the CTA reads, and the whole shape
// of the kernel follows from spreading them over as many query rows as one SM can hold:
//   - A work item is 256 rows of ONE kv-head: rows are (position, head of the group) pairs in that order, so all query heads
//     that share the kv-head read the converted tile, whatever their number (groups of seven as well as of eight), and a
//     few drafted tokens of a request fill a tile that would be 128 times one head's few rows otherwise.
//   - The CTA has two slots (S and O in TMEM, a softmax warpgroup) that take turns: the softmax of one runs beside the MMAs of
//     the other.  More than 128 rows: a slot for each half, both on every key tile.  Fewer: both slots hold the SAME rows and
//     take every other key tile, so that a few rows do not run at the latency of one slot's chain.
//   - A call with too few items to fill the machine evenly cuts each item's keys into 2 .. 16 ranges, one for each CTA of a
//     cluster.  Slots and CTAs that share rows leave (m, l, O) in shared memory when they are through, and the CTAs of the
//     cluster merge a share of the rows each, out of all their shared memories.  No workspace, and the same bits every time.
//   - K goes to f16: one conversion instruction for two codes and nothing else, as its scale is applied to the scores, where
//     a multiplication by the softmax scale stands anyway.  Q becomes f16 with each row brought to a maximum in
//     [2^13, 2^14) by a power of two, as in decode (what f16 then drops lies 2^-37 below the row's largest element).
//   - V goes to bf16 with its scale multiplied in (exact, a power of two), since only bf16 has the scales' range; P is bf16.
// Measured, 32q/8kv, d128: 2048 positions over 14001 keys 480 to 523 us by how far the part is at its power cap, 965 to 1050 TFLOP/s,
// 0.60 to 0.65 of cuBLAS' burst (469 at best); a prompt of 8192 484 to 493 us, 1114 to 1136; 64 prompts of 512 304 us, 256 of 128 220 us.  What bounds it: a key tile's chain through one head's scores, softmax and P V (3500
// cycles a pair of tiles, as in the other tcgen05 kernels) plus a tenth for the conversion; 256 items on 148 SMs are two rounds for
// 1.73; and an item costs some 9000 cycles besides its tiles, which is most of a short prompt: Q on its way and to f16, the first scores,
// the write-out (whose rows go through the idle Q tile: straight from the registers, a thread a row, they took 224 us for 218).
//
//   warp 0        MMA issuer: S = Q K^T (both from shared memory) and O += P V (P from TMEM, V MN-major)
//   warp 1        TMEM allocation; warp 2: item scheduler (the kernel is persistent, a CTA an SM: set-up and instruction caches
//                 are paid for once, and the next item is decoded beside the current one); warp 3 completes the warpgroup
//   warps 4-7     rows 0-127: Q into shared memory, softmax (a thread a row), write-out
//   warps 8-11    rows 128-255
//   warps 12-15   converters: codes come through the block table by 16-byte asynchronous copies into places of shared memory
//                 that belong to the copying thread (so a thread waits for its own copies and for nobody), each place being
//                 refilled for the next tile as soon as it has been read; conversion, swizzled stores.  Keys past the item's
//                 last visible one become zero rows of V, so nothing a slot that was never written holds can reach a sum
//                 (0 * NaN), and no code is needed for that elsewhere.
// NaN codes of V at keys that some rows of the item see and others do not (the tiles that the causal boundary cuts) must reach the
// former and not the latter, whose weight of 0 does not stop them.  The converters look for them in those tiles alone (no time that
// could be measured), put zeros in their place and leave word; the CTA then takes no further item, and gives the rows their NaN from the
// codes themselves when all is written.  64 prompts of 512 take 304 us, 320 with one such value, 751 with one in every token and head.
// Softmax: online with lazy rescaling, as in the other tcgen05 kernels.  The sign of the scale is folded into Q.
// The loops are kept rolled wherever that costs no registers: all roles of a quarter of the SM share an instruction cache
// of about 32 KB (see ekv_prefill_tc.cuh), and with the converters' and the mask's loops unrolled (106 KB in all) every role ran at
// 4 to 6 cycles an instruction.
#pragma once
#include <cuda_fp16.h>

#include "e4m3.cuh"
#include "ekv_prefill_tc.cuh"

namespace ekv {
namespace tc8 {

namespace cp = cuda::ptx;
using tc::fence_after;
using tc::fence_before;

static constexpr int kBM = 128, kBN = 128;
static constexpr int kItemRows = 2 * kBM;
static constexpr int kMaxClusterLog = 4, kMaxCluster = 1 << kMaxClusterLog;
static constexpr int kThreads = 512;
static constexpr int kHalfBytes = 128 * 128;  // [128 rows][64 16-bit channels], 128-byte swizzle
static constexpr int kStages = 2;
// setmaxnreg: warps 0-3 kRegsUtil, 4-11 kRegsSoftmax, 12-15 kRegsConv; the shares add up to what the CTA is launched with
static constexpr int kLaunchRegs = 128, kRegsUtil = 40, kRegsSoftmax = 200, kRegsConv = 72;
static_assert(128 * (kRegsUtil + kRegsConv) + 256 * kRegsSoftmax <= kLaunchRegs * kThreads, "setmaxnreg split exceeds the CTA's registers");
static_assert(kRegsUtil == 40 && kRegsSoftmax == 200 && kRegsConv == 72, "the setmaxnreg instructions in the kernel carry these numbers as literals");

struct Params {
    PrefillParams p;  // q_tiles, tile_prefix: in items of kItemRows rows per kv-head; scale_log2 >= 0
    const uint8_t *cache;
    const float *scales;
    long long block_stride;
    unsigned group_magic;  // ceil(2^32 / group): a division by the group (2 or more) is one multiplication, exact below 2^29
    int few_rows;  // requests of at most this many rows are another kernel's (ekv_prefill_e4m3_few.cuh)
    int cluster, cluster_log;  // CTAs that share an item's keys: 2^cluster_log
    float q_sign;  // -1 for a negative scale; 0 for a scale of 0
};

template <int D>
struct Geo {
    static constexpr int kHalves = D / 64;
    static constexpr int kTileBytes = kHalves * kHalfBytes;
    static constexpr int kOffQ = 0;
    static constexpr int kOffK = 2 * kTileBytes;
    static constexpr int kOffV = kOffK + kStages * kTileBytes;
    static constexpr int kRawBytes = 128 * D;  // a tile of codes
    static constexpr int kOffRaw = kOffV + kStages * kTileBytes;  // one of K, one of V
    static constexpr int kOffBar = kOffRaw + 2 * kRawBytes;
    enum Bar { Q_READY = 0, K_FULL = 2, K_EMPTY = 4, V_FULL = 6, V_EMPTY = 8, S_READY = 10, P_PART = 12, P_READY = 14, DRAIN = 16, NEXT = 17, NBAR = 18 };
    __device__ static __forceinline__ uint32_t arrivals(int bar) {  // warps for Q, K and V tiles, threads for P, a commit for the others
        return bar >= P_PART && bar < DRAIN ? 128u : (bar < K_EMPTY || (bar >= V_FULL && bar < V_EMPTY)) ? 4u : 1u;
    }
    static constexpr int kOffFlags = kOffBar + 8 * NBAR;       // abort flag, TMEM address, 4 masks of invalid blocks
    static constexpr int kOffKScale = kOffBar + 192;           // [4 tiles][8 blocks] floats
    static constexpr int kOffQInv = kOffKScale + 128;          // [256 rows] floats
    static constexpr int kOffPart = 0;                         // merge: O of [2 slots][128 rows][D] floats, over the tiles ...
    static constexpr int kOffPartML = 2 * kBM * D * 4;         // ... and (m, l) of [2][128]
    static constexpr int kOffPartW = kOffPartML + 2 * kBM * 8;  // the CTA's own weights of its rows' partials: at most 512
    static_assert(kOffPartW + 512 * 4 <= kOffRaw, "merge area");
    static constexpr int kOffItem = kOffQInv + 1024;           // two slots of the scheduler: state and seven numbers; then progress, response, nan_seen
    static constexpr int kSmemBytes = kOffItem + 128 + 1024;    // + alignment slack
    static_assert(kOffFlags + 24 <= kOffKScale && kOffItem % 16 == 0 && kSmemBytes <= 232448, "shared memory");
    // kind::f16 instruction descriptors, D = f32, M = 128: QK with f16 operands, PV with bf16 ones and V MN-major
    static constexpr uint32_t kIdescQK = (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
    static constexpr uint32_t kIdescPV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);
};

template <int D>
struct Smem {
    uint32_t base;
    uint8_t *ptr;
    __device__ __forceinline__ uint32_t bar(int i) const { return base + Geo<D>::kOffBar + 8 * i; }
    __device__ __forceinline__ volatile int *abort_flag() const { return (volatile int *)(ptr + Geo<D>::kOffFlags); }
    __device__ __forceinline__ uint32_t *tmem_slot() const { return (uint32_t *)(ptr + Geo<D>::kOffFlags + 4); }
    // rings of 4 by key tile: the converters start on tile j + 3 only after the MMAs of tile j + 1's scores, i.e. after the
    // softmax of tile j has read its entry
    __device__ __forceinline__ volatile int *bad_mask(int tile) const { return (volatile int *)(ptr + Geo<D>::kOffFlags + 8 + 4 * (tile & 3)); }
    __device__ __forceinline__ float *k_scale(int tile) const { return (float *)(ptr + Geo<D>::kOffKScale) + 8 * (tile & 3); }
    __device__ __forceinline__ volatile int *progress() const { return (volatile int *)(ptr + Geo<D>::kOffItem + 64); }  // tile that the converters are at
    __device__ __forceinline__ uint4 *response() const { return (uint4 *)(ptr + Geo<D>::kOffItem + 80); }  // the launch's next CTA, if any
    __device__ __forceinline__ volatile int *nan_seen(int n) const { return (volatile int *)(ptr + Geo<D>::kOffItem + 96) + (n & 1); }  // by item
    __device__ __forceinline__ int *item(int n) const { return (int *)(ptr + Geo<D>::kOffItem) + 8 * (n & 1); }
    __device__ __forceinline__ float *q_inv() const { return (float *)(ptr + Geo<D>::kOffQInv); }
};

// Bounded wait of a whole warp, as in the two-head kernel: one poll and a vote, then a polling loop of a dozen instructions that
// gives up when another role has, or after tc::kPollLimit polls (it leaves 2 in the abort flag; the teardown reports it).
template <int D>
__device__ __forceinline__ bool wait_warp(const Smem<D> &sh, int bar, uint32_t parity) {
    if (__all_sync(0xffffffffu, mbar_try_wait(sh.bar(bar), parity))) return true;
    return __all_sync(0xffffffffu, mbar_wait_polls(sh.bar(bar), parity, sh.base + Geo<D>::kOffFlags, tc::kPollLimit));
}

// Which request owns item `idx` (items of kItemRows (position, head) rows, requests in order)?  Beyond the offsets that the launch carries, a
// walk from the first request on, in every item: 257 prompts of 128 take 514 us for the 219 of 256, 1024 take 6.5 ms.
__device__ __forceinline__ bool find_item(const PrefillParams &p, int few_rows, int idx, int &req, int &first, int &q0, int &c_r) {
    if (p.n_prefix) return find_request(p, idx, kItemRows, req, first, q0, c_r);
    int acc = 0;
    for (req = 0; req < p.R; ++req) {
        q0 = p.cu_q_lens[req];
        c_r = p.cu_q_lens[req + 1] - q0;
        const int n = (long long)c_r * p.group > few_rows ? (int)(((long long)c_r * p.group + kItemRows - 1) / kItemRows) : 0;
        if (idx < acc + n) {
            first = acc;
            return true;
        }
        acc += n;
    }
    return false;
}

// A warp gives rows from, from + step, ... < to their NaN: channels of V that are NaN in a key from `key0` (a block's first) on up to the last
// one that the row sees (keys before have had theirs from the sum).  row(r, lim, at): that key and where the row is in `out`.
template <int D, typename Row>
__device__ __forceinline__ void nan_values(const Params &pp, int g, const int *bt, int key0, int kv_end, int from, int to, int step, Row row) {
    const int c0 = 4 * (threadIdx.x & 31), num_kv_heads = pp.p.num_kv_heads;  // four channels a lane
    if (c0 >= D) return;
    const long long live = *pp.p.live;
    int first[4] = {kv_end, kv_end, kv_end, kv_end};  // the first key of which a channel is NaN
#pragma unroll 1
    for (int t0 = key0; t0 < kv_end; t0 += 16) {
        const int id = bt[t0 >> 4];
        if (id < 0 || (long long)id >= live || !(pp.scales[((long long)id * 2 + 1) * num_kv_heads + g] > 0.f)) continue;
        const uint8_t *codes = pp.cache + (long long)id * pp.block_stride + (long long)(num_kv_heads + g) * (16 * D) + c0;
#pragma unroll 8
        for (int t = 0; t < 16; ++t) {
            const uint32_t nan = nan_codes(*reinterpret_cast<const uint32_t *>(codes + t * D));
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((nan >> (8 * i)) & 0x80u) first[i] = min(first[i], t0 + t);
        }
    }
#pragma unroll 1
    for (int r = from; r < to; r += step) {
        int lim;
        __nv_bfloat16 *at;
        row(r, lim, at);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (first[i] <= lim && first[i] < kv_end) at[c0 + i] = __ushort_as_bfloat16(0x7fff);
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) prefill8_kernel(const __grid_constant__ Params pp) {
    using G = Geo<D>;
    const PrefillParams &p = pp.p;
    constexpr int kPieces = D / 8;              // 16-byte pieces of a row of Q / O
    constexpr int kRowsPerInst = 32 / kPieces;  // rows one warp-wide 16-byte access covers
    extern __shared__ uint8_t smem_raw[];
    Smem<D> sh;
    {
        const uint32_t raw = smem_u32(smem_raw);
        sh.base = (raw + 1023u) & ~1023u;
        sh.ptr = smem_raw + (sh.base - raw);
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cluster = pp.cluster, part = blockIdx.x % cluster;  // CTAs that share an item's keys; which of them this is

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the call's other kernel, if it has one, may use what falls free
    if (threadIdx.x == 64) {
#pragma unroll 1
        for (int i = 0; i < G::NBAR; ++i) mbar_init(sh.bar(i), G::arrivals(i));
        mbar_fence_init();
        *sh.abort_flag() = 0;
        *sh.nan_seen(0) = *sh.nan_seen(1) = 0;
    }
    if (warp == 1) {
        cp::tcgen05_alloc(cp::cta_group_1, sh.tmem_slot(), 512);
        cp::tcgen05_relinquish_alloc_permit(cp::cta_group_1);
    }
    const int group = p.group;
    auto by_group = [&](int r) { return group == 1 ? r : (int)__umulhi((unsigned)r, pp.group_magic); };

    // ---- the scheduler (warp 2): which (request, rows, kv-head) is next?  Items are listed heaviest (latest) first, all kv-heads of
    // one next to each other, and the launch has a CTA for each.  A CTA starts with the one of its own number and then takes the
    // place of CTAs that have not started (cluster launch control), each while it works on the item before: no word of device memory
    // that two launches, or two replays of captured ones, could share.  Rows that have no keys to see are dealt with here.  (The CTAs of a cluster have one item.)
    bool may_draw = cluster == 1;
    uint32_t draws = 0;
    auto draw = [&]() {  // number of a CTA that will not start now, or -1
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
        return may_draw ? cp::clusterlaunchcontrol_query_cancel_get_first_ctaid_x<int>(response) : -1;
    };
    auto post = [&](int item, int n) {
        int *slot = sh.item(n);
        for (;; item = -1) {
            // (the last item for a CTA that has NaN values to give: the slots keep the numbers of two items)
            if (item < 0) item = __any_sync(0xffffffffu, *sh.nan_seen(0) | *sh.nan_seen(1)) ? -1 : draw();
            const bool over = item < 0;
            const int rank = item / p.num_kv_heads, g = item - rank * p.num_kv_heads, idx = p.q_tiles - 1 - rank;
            int req = 0, first = 0, c_r = 0, q0 = 0;
            if (!over && !find_item(p, pp.few_rows, idx, req, first, q0, c_r)) continue;
            const int row0 = (idx - first) * kItemRows;  // first of the request's c_r * group rows
            const int rows_here = min(kItemRows, c_r * group - row0);
            const int L = over ? 0 : min(p.seq_lens[req], p.max_blocks * 16);
            if (!over && rows_here <= 0) continue;  // the device's offsets say less than the host's
            if (!over && L < c_r) {  // malformed request: zero rows, latch
                if (lane == 0) atomicOr(p.status, EKV_DEV_FLAG_OOB);
                for (int r = 0; r < rows_here && part == 0; ++r) {
                    const int pos = by_group(row0 + r), hg = row0 + r - pos * group;
                    if (lane < kPieces) reinterpret_cast<uint4 *>(p.out + ((size_t)(q0 + pos) * p.num_q_heads + (size_t)(g * group + hg)) * D)[lane] = make_uint4(0u, 0u, 0u, 0u);
                }
                continue;
            }
            if (lane == 0) slot[0] = over ? 0 : 1;  // (the numbers of the item there before may still be needed)
            if (lane == 0 && !over) slot[1] = req, slot[2] = g, slot[3] = row0, slot[4] = rows_here, slot[5] = q0, slot[6] = L, slot[7] = L - c_r;
            break;
        }
        __syncwarp();
    };
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *sh.tmem_slot();

    // ---- the current item, as each role reads it from the scheduler's slot
    int req, g, row0, rows_here, q0, prefix, kv_end, tile0, n_tiles, n_blocks;
    bool by_rows, merge;
    int pos0, head0;    // the item's first row: its position in the request and its head of the group
    size_t first_head;  // offset in q and out of the first head of the group, at that position
    auto position = [&](int r) { return pos0 + by_group(head0 + r); };
    // offset of a row of the item behind that: 32 bits hold it (256 rows)
    auto row_offset = [&](int r) { return (by_group(head0 + r) * (p.num_q_heads - group) + head0 + r) * D; };
    // Barriers live as long as the CTA; an item's waits count phases from 0, on top of what earlier items left in bit `bar` of this.
    uint32_t phases = 0;
    auto wait = [&](int bar, uint32_t parity) { return wait_warp<D>(sh, bar, (parity ^ (phases >> bar)) & 1u); };
    auto count_phases = [&](int n) {
        if (n > 0) {  // completions of the item before, by barrier
            const uint32_t t[2] = {(uint32_t)(n_tiles + 1) >> 1, (uint32_t)n_tiles >> 1};
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint32_t of_slot = by_rows ? (uint32_t)n_tiles : t[x];
                phases ^= (x == 0 || by_rows ? 1u : 0u) << (G::Q_READY + x);
                phases ^= (t[x] & 1u) * (1u << (G::K_FULL + x) | 1u << (G::K_EMPTY + x) | 1u << (G::V_FULL + x) | 1u << (G::V_EMPTY + x));
                phases ^= (of_slot & 1u) * (1u << (G::P_PART + x) | 1u << (G::P_READY + x)) ^ ((of_slot + 1u) & 1u) << (G::S_READY + x);
            }
            phases ^= 1u << G::DRAIN;
        }
    };
    auto meet_items = [&]() {  // all roles are through with the item before (its shared memory and TMEM), and the next one's slot is posted
        fence_before();
        __syncwarp();
        asm volatile("bar.sync 3, 512;" ::: "memory");
        fence_after();
    };
    auto read_item = [&](int n) {
        const volatile int *slot = sh.item(n);
        if (slot[0] == 0) return false;
        req = slot[1], g = slot[2], row0 = slot[3], rows_here = slot[4], q0 = slot[5], prefix = slot[7];
        pos0 = by_group(row0);
        head0 = row0 - pos0 * group;
        first_head = ((size_t)(q0 + pos0) * p.num_q_heads + (size_t)g * group) * D;
        kv_end = min(slot[6], prefix + position(rows_here - 1) + 1);  // keys any row of the item may see
        const int all_tiles = (kv_end + kBN - 1) / kBN;
        tile0 = (all_tiles * part) >> pp.cluster_log;  // this CTA's key tiles: tile0 .. tile0 + n_tiles - 1 (possibly none)
        n_tiles = ((all_tiles * (part + 1)) >> pp.cluster_log) - tile0;
        n_blocks = (kv_end + 15) >> 4;
        // by_rows: slot x holds rows 128 x .. and sees every key tile j.  Else both hold rows 0 .. and slot x sees tiles x, x + 2, ...
        by_rows = rows_here > kBM;
        merge = cluster > 1 || !by_rows;
        return true;
    };
    auto next_item = [&](int n) {
        count_phases(n);
        meet_items();
        return !*sh.abort_flag() && read_item(n);
    };

    // The merge: all roles meet when the CTA's tiles are no longer needed, again when the partial results of the cluster are in
    // place, and (clusters) once more when they have been read.  Hardware barriers; every role comes here, given up or not.
    auto meet_all = [&]() { asm volatile("bar.sync 1, 512;" ::: "memory"); };
    auto meet_cluster = [&]() {
        if (cluster > 1) cluster_barrier();
        else meet_all();
    };
    auto merge_barriers = [&]() {
        __syncwarp();
        meet_all();
        meet_cluster();
        if (cluster > 1) cluster_barrier();
    };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 2) {
            // =========================== item scheduler ===========================
            int item = blockIdx.x / cluster;
#pragma unroll 1
            for (int n = 0;; ++n) {
                if (n > 0 && cluster == 1) {
                    // Not before the converters have come to the item's last tile, some 6000 cycles from its end: an item drawn at the
                    // start of the one before would wait for this CTA while another stands idle.  (A plain word, since a phase parity
                    // cannot tell "not yet" from "two phases ago"; bounded like every wait.)
                    const uint64_t t0 = global_timer_ns();
                    while (*sh.progress() < n_tiles - 1 && !*sh.abort_flag()) {
                        __nanosleep(200);
                        if (global_timer_ns() - t0 > 2000000000ull) *sh.abort_flag() = 2;
                    }
                }
                post(item, n);  // beside the end of the work on item n - 1
                asm volatile("bar.arrive 4, 160;" ::: "memory");  // the converters may look at it
                if (n > 0 && cluster == 1) {  // its Q rows into L2, while the item before takes its time
                    const volatile int *slot = sh.item(n);
                    if (slot[0]) {
                        const int at = slot[3] - by_group(slot[3]) * group, lines = slot[4] * (D / 64);
                        const __nv_bfloat16 *from = p.q + ((size_t)(slot[5] + by_group(slot[3])) * p.num_q_heads + (size_t)slot[2] * group) * D;
#pragma unroll 1
                        for (int i = lane; i < lines; i += 32) {
                            const int r = at + i / (D / 64);
                            asm volatile("prefetch.global.L2 [%0];" ::"l"(from + (by_group(r) * (p.num_q_heads - group) + r) * D + i % (D / 64) * 64));
                        }
                    }
                }
                item = -1;
                if (n > 0 && merge) merge_barriers();
                if (lane == 0) *sh.progress() = -1;
                if (!next_item(n)) break;
            }
            if (*sh.abort_flag())  // a wait ran out: the CTAs that have not started, and would wait as long, are not to
                while (draw() >= 0) {}
        } else {
#pragma unroll 1
        for (int n = 0; next_item(n); ++n) {
        if (warp == 0) {
            // =========================== MMA issuer ===========================
            constexpr uint64_t kHi = (uint64_t)tc::kDescHi << 32;
            const uint64_t q_d = kHi | tc::desc_lo(sh.base + G::kOffQ, 16), k_d = kHi | tc::desc_lo(sh.base + G::kOffK, 16),
                           v_d = kHi | tc::desc_lo(sh.base + G::kOffV, kHalfBytes);
            // Steps alternate between the slots: step u is P V of slot x = u & 1 on its key tile number i = u >> 1, and Q K^T for the
            // slot's next one; steps -2 and -1 only bring the first scores.  One elected lane issues a step in one go: the last
            // quarter of PV, QK^T, the commits.
            bool ok = true;
            int sh2 = by_rows ? 1 : 0;  // (through an empty asm, here and below: one copy of the loop, not one for each case)
            asm volatile("" : "+r"(sh2));
            const int step_max = n_tiles > 0 ? n_tiles << sh2 : -2;
#pragma unroll 1
            for (int u = -2; u < step_max && ok; ++u) {
                const int x = u & 1, i = u >> 1;
                const int j = u >> sh2, jn = (u + 2) >> sh2;  // the CTA's key tiles of the two
                const int s = j & 1, s1 = jn & 1;
                int pv = u >= 0, more = jn < n_tiles, closes = x >= sh2;  // closes: the last slot to read these stages
                asm volatile("" : "+r"(pv), "+r"(more), "+r"(closes));
                const uint32_t t_s = tmem + 128 * x, t_o = tmem + 256 + 128 * x;
                const uint64_t vd = v_d + (uint32_t)s * (G::kTileBytes >> 4);
                if (pv) {
                    ok = wait(G::V_FULL + s, (uint32_t)((j >> 1) & 1));
                    if (ok) ok = wait(G::P_PART + x, (uint32_t)(i & 1));
                    if (!ok) break;
                    fence_after();
                    if (tc::elect_one()) {  // keys 0..95 while the softmax warps finish the rest
#pragma unroll
                        for (int k = 0; k < tc::kPartSteps; ++k)
                            tc::mma_ts(t_o, t_s + 8 * k, vd + ((k * 2048) >> 4), G::kIdescPV, (i > 0 || k > 0) ? 1u : 0u);
                    }
                    __syncwarp();
                    ok = wait(G::P_READY + x, (uint32_t)(i & 1));
                } else {
                    ok = wait(G::Q_READY + (x & sh2), 0);
                }
                if (ok && more) ok = wait(G::K_FULL + s1, (uint32_t)((jn >> 1) & 1));
                if (!ok) break;
                fence_after();
                if (tc::elect_one()) {
                    if (pv) {
#pragma unroll
                        for (int k = tc::kPartSteps; k < kBN / 16; ++k) tc::mma_ts(t_o, t_s + 8 * k, vd + ((k * 2048) >> 4), G::kIdescPV, 1u);
                        if (closes) tc::mma_commit_one(sh.bar(G::V_EMPTY + s));
                    }
                    if (more) {
                        const uint64_t qd = q_d + (uint32_t)(x & sh2) * (G::kTileBytes >> 4), kd = k_d + (uint32_t)s1 * (G::kTileBytes >> 4);
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const uint32_t off = ((k >> 2) * kHalfBytes + (k & 3) * 32) >> 4;
                            tc::mma_ss(t_s, qd + off, kd + off, G::kIdescQK, k > 0 ? 1u : 0u);
                        }
                        if (closes) tc::mma_commit_one(sh.bar(G::K_EMPTY + s1));
                    }
                    tc::mma_commit_one(sh.bar(G::S_READY + x));  // the slot's next scores, and its O up to this tile
                }
                __syncwarp();
            }
            // every MMA this thread issued must be finished before TMEM is released
            tc::mma_commit(sh.bar(G::DRAIN));
            (void)wait(G::DRAIN, 0);
        }
        if (merge) merge_barriers();
        }
        }
    } else if (warp >= 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        // =========================== converters ===========================
        constexpr int kIts = D / 16;                       // 16-byte pieces of codes a thread takes of a tile
        constexpr int kBlocksPerIt = 128 * 16 / (16 * D);  // blocks the 128 threads cover at once: 1, or 2 at head_dim 64
        const int ct = threadIdx.x - 384;
        // Which 16 bytes of a block: eight neighbouring lanes take four pieces of two rows, so that their stores into the
        // 128-byte swizzled tile (two chunks a piece) never meet in a bank.
        const int in_block = ct % D;                       // 16 * D bytes of a block are D pieces
        const int rowb = D == 128 ? (in_block >> 5 << 2) | ((in_block >> 3) & 2) | ((in_block >> 2) & 1) : in_block >> 2;
        const int piece = D == 128 ? ((in_block >> 1) & 4) | (in_block & 3) : in_block & 3;
        const int first_block = kBlocksPerIt > 1 ? ct / D : 0;
        const long long live = *p.live;
        const int *bt;
        const uint8_t *src;
        const long long v_off = (long long)p.num_kv_heads * (16 * D);
        const uint32_t raw = sh.base + G::kOffRaw + ct * 16;  // this thread's places: one every 2048 bytes
        // lane l: id of block 8j + l % 8 of tile j (-1 past the end, -2 invalid)
        auto load_id = [&](int j) {
            int id = -1;
            const int bi = 8 * (tile0 + j) + (lane & 7);
            if (j < n_tiles && bi < n_blocks) {
                id = bt[bi];
                if (id < 0 || (long long)id >= live) id = -2;
            }
            return id;
        };
        auto load_scale = [&](int ids, int kv) { return ids >= 0 ? __ldg(pp.scales + ((long long)ids * 2 + kv) * p.num_kv_heads + g) : 0.f; };
        auto copy = [&](int it, int ids, int kv) {  // piece `it` of this thread; an invalid block's codes read as 0
            const int id = __shfl_sync(0xffffffffu, ids, it * kBlocksPerIt + first_block);
            cp_async_16(raw + kv * G::kRawBytes + it * 2048, src + (long long)max(id, 0) * pp.block_stride + (kv ? v_off : 0), id >= 0 ? 16u : 0u);
        };
        // 16 values of one row -> two 16-byte chunks of the tile.  The place inside a block's 16 rows is the same for every block.
        uint8_t *const store_at = sh.ptr + (piece >> 2) * kHalfBytes + (first_block * 16 + rowb) * 128;
        const int c0 = ((2 * (piece & 3)) ^ (rowb & 7)) << 4, c1 = c0 ^ 16;
        auto store = [&](uint32_t tile_off, int it, const uint32_t (&w)[8]) {
            uint8_t *to = store_at + tile_off + it * (kBlocksPerIt * 2048);
            *reinterpret_cast<uint4 *>(to + c0) = make_uint4(w[0], w[1], w[2], w[3]);
            *reinterpret_cast<uint4 *>(to + c1) = make_uint4(w[4], w[5], w[6], w[7]);
        };
        auto put_k = [&](int s, int it, const uint4 &v) {  // f16
            const uint32_t c[4] = {v.x, v.y, v.z, v.w};
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[2 * i] = e4m3_lo(c[i]);
                w[2 * i + 1] = e4m3_hi(c[i]);
            }
            store(G::kOffK + s * G::kTileBytes, it, w);
        };
        auto put_v = [&](int s, int it, const uint4 &v, float scale) {  // bf16 with the scale in it
            const uint32_t c[4] = {v.x, v.y, v.z, v.w};
            const __nv_bfloat162 s2 = __float2bfloat162_rn(scale);
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 a = f16x2_to_float2(e4m3_lo(c[i])), b = f16x2_to_float2(e4m3_hi(c[i]));
                const __nv_bfloat162 x = __hmul2(__floats2bfloat162_rn(a.x, a.y), s2), y = __hmul2(__floats2bfloat162_rn(b.x, b.y), s2);
                w[2 * i] = *reinterpret_cast<const uint32_t *>(&x);
                w[2 * i + 1] = *reinterpret_cast<const uint32_t *>(&y);
            }
            store(G::kOffV + s * G::kTileBytes, it, w);
        };
        const uint4 zeros = make_uint4(0u, 0u, 0u, 0u);
        auto publish = [&](int bar) {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(sh.bar(bar));
        };
        // An item's first tile of codes is on its way before the item before is finished by the other roles: the places are free.
        int ids, ids_next;
        float ks, vs;
        auto start_item = [&](int n) {
            asm volatile("bar.sync 4, 160;" ::: "memory");  // posted
            if (!read_item(n)) return false;
            bt = p.block_tables + (size_t)req * p.max_blocks;
            src = pp.cache + (long long)g * (16 * D) + rowb * D + piece * 16;
            ids = load_id(0);
            ks = load_scale(ids, 0), vs = load_scale(ids, 1);
#pragma unroll 1
            for (int kv = 0; kv < 2; ++kv) {
#pragma unroll 2
                for (int it = 0; it < kIts; ++it) copy(it, ids, kv);
                cp_async_commit();
            }
            ids_next = load_id(1);
            return true;
        };
        bool more = start_item(0);
        meet_items();
#pragma unroll 1
        for (int n = 0; more && !*sh.abort_flag(); ++n) {
        bool ok = true;
#pragma unroll 1
        for (int j = 0; j < n_tiles; ++j) {
            const int s = j & 1;
            const uint32_t ph = (uint32_t)(((j >> 1) - 1) & 1);
            const int ids_after = load_id(j + 2);
            const float ks_next = load_scale(ids_next, 0), vs_next = load_scale(ids_next, 1);
            int reports = warp == 12;  // for all four warps
            asm volatile("" : "+r"(reports));  // (one copy of the loop)
            if (reports && lane == 0) *sh.progress() = j;
            // Rows that are to be 0 whatever their codes: of blocks that were never written (no scale) or do not exist, and V's past
            // the last visible key.  A tile without any takes no notice.
            const bool some_zero = __any_sync(0xffffffffu, !(ks > 0.f) || !(vs > 0.f)) || (tile0 + j + 1) * kBN > kv_end;
            // ---- K, with its scales beside it
            cp_async_wait_1();
            ok = j < kStages || wait(G::K_EMPTY + s, ph);
            if (!ok) break;
            if (reports) {
                const unsigned bad = __ballot_sync(0xffffffffu, ids < 0) & 0xffu;  // invalid, or past the last visible key
                const unsigned oob = __ballot_sync(0xffffffffu, ids == -2) & 0xffu;
                if (lane < 8) sh.k_scale(j)[lane] = ks > 0.f ? ks : 1.f;
                if (lane == 0) {
                    *sh.bad_mask(j) = (int)bad;
                    if (oob) atomicOr(p.status, EKV_DEV_FLAG_OOB);
                }
            }
            if (some_zero) {
#pragma unroll 1
                for (int it = 0; it < kIts; ++it) {
                    const uint4 v = lds_16(raw + it * 2048);
                    copy(it, ids_next, 0);
                    put_k(s, it, __shfl_sync(0xffffffffu, ks, it * kBlocksPerIt + first_block) > 0.f ? v : zeros);
                }
            } else {
#pragma unroll 1
                for (int it = 0; it < kIts; it += 4) {  // four pieces side by side: one alone is a chain of some 180 cycles
                    uint4 v[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) v[u] = lds_16(raw + (it + u) * 2048);
#pragma unroll
                    for (int u = 0; u < 4; ++u) copy(it + u, ids_next, 0);  // the places are free: the next tile's codes
#pragma unroll
                    for (int u = 0; u < 4; ++u) put_k(s, it + u, v[u]);
                }
            }
            cp_async_commit();
            publish(G::K_FULL + s);
            // ---- V
            cp_async_wait_1();
            if ((tile0 + j + 1) * kBN > prefix + pos0 + 1) {  // not every row sees all of the tile: no NaN codes into it
#pragma unroll 1
                for (int it = 0; it < kIts; it += 4) {
                    const uint32_t at = raw + G::kRawBytes + it * 2048;
                    uint4 v[4];
                    uint32_t any = 0;
#pragma unroll
                    for (int u = 0; u < 4; ++u) v[u] = lds_16(at + u * 2048);
#pragma unroll
                    for (int u = 0; u < 4; ++u) any |= nan_codes(v[u].x) | nan_codes(v[u].y) | nan_codes(v[u].z) | nan_codes(v[u].w);
                    if (any) {
#pragma unroll 1
                        for (int u = 0; u < 4; ++u) {
                            const uint4 w = lds_16(at + u * 2048), clean = without_nan_codes(w);
                            sts_16(at + u * 2048, clean);
                            // (those past the last visible key, slots not written yet, are nobody's)
                            if ((w.x != clean.x || w.y != clean.y || w.z != clean.z || w.w != clean.w) &&
                                (tile0 + j) * kBN + ((it + u) * kBlocksPerIt + first_block) * 16 + rowb < kv_end)
                                *sh.nan_seen(n) = 1;
                        }
                    }
                }
            }
            ok = j < kStages || wait(G::V_EMPTY + s, ph);
            if (!ok) break;
            if (some_zero) {
#pragma unroll 1
                for (int it = 0; it < kIts; ++it) {
                    const uint4 v = lds_16(raw + G::kRawBytes + it * 2048);
                    copy(it, ids_next, 1);
                    const int blk = it * kBlocksPerIt + first_block;
                    const float scale = __shfl_sync(0xffffffffu, vs, blk);
                    put_v(s, it, scale > 0.f && (tile0 + j) * kBN + blk * 16 + rowb < kv_end ? v : zeros, scale);
                }
            } else {
#pragma unroll 1
                for (int it = 0; it < kIts; it += 4) {
                    uint4 v[4];
                    float scale[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) v[u] = lds_16(raw + G::kRawBytes + (it + u) * 2048);
#pragma unroll
                    for (int u = 0; u < 4; ++u) copy(it + u, ids_next, 1);
#pragma unroll
                    for (int u = 0; u < 4; ++u) scale[u] = __shfl_sync(0xffffffffu, vs, (it + u) * kBlocksPerIt + first_block);
#pragma unroll
                    for (int u = 0; u < 4; ++u) put_v(s, it + u, v[u], scale[u]);
                }
            }
            cp_async_commit();
            publish(G::V_FULL + s);
            ids = ids_next;
            ids_next = ids_after;
            ks = ks_next;
            vs = vs_next;
        }
        cp_async_wait_all();  // what was started for a tile that does not come (or after a wait that was given up)
        const bool merges = merge;
        count_phases(n + 1);
        more = start_item(n + 1);
        if (merges) merge_barriers();
        meet_items();
        }
        cp_async_wait_all();
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        // =========================== softmax + write-out ===========================
#pragma unroll 1
        for (int n = 0; next_item(n); ++n) {
        const int x = (warp - 4) >> 2;        // slot
        const int rx = by_rows ? x : 0;       // its row tile
        const int n_it = by_rows ? n_tiles : (n_tiles - x + 1) >> 1;  // its key tiles
        const int wrow0 = (warp & 3) << 5;    // TMEM lanes wrow0 .. +31 belong to this warp
        const int row = wrow0 | lane;         // row of the tile = TMEM lane
        const uint32_t t_s = tmem + ((uint32_t)wrow0 << 16) + 128 * x;
        const uint32_t t_o = tmem + ((uint32_t)wrow0 << 16) + 256 + 128 * x;
        uint8_t *q_tile = sh.ptr + G::kOffQ + rx * G::kTileBytes;
        const int piece = lane % kPieces, sub = lane / kPieces;
        if (by_rows || x == 0) {
            // ---- Q rows of this warp: all of them on their way at once, straight to where they belong in the 128-byte swizzled
            // tile, then bf16 -> f16 in place with a row's largest magnitude in [2^13, 2^14); rows past the end are 0.  A warp-wide
            // access covers kRowsPerInst rows; four of them come back to the same place of the swizzle.
            constexpr int kBatch = 4, kBatchRows = kBatch * kRowsPerInst;
            static_assert(kBatchRows % 8 == 0, "swizzle period");
            uint32_t place[kBatch];  // of this lane's piece in the rows of a batch
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int r = kRowsPerInst * u + sub;
                place[u] = G::kOffQ + x * G::kTileBytes + (piece >> 3) * kHalfBytes + (wrow0 + r) * 128 + (((piece & 7) ^ (r & 7)) << 4);
            }
            const __nv_bfloat16 *q_src = p.q + first_head + piece * 8;
            const int first_row = x * kBM + wrow0 + sub;
#pragma unroll 1
            for (int b = 0; b < 32 / kBatchRows; ++b) {
#pragma unroll
                for (int u = 0; u < kBatch; ++u) {
                    const int in_item = first_row + b * kBatchRows + kRowsPerInst * u;
                    const bool there = in_item < rows_here;
                    cp_async_16(sh.base + place[u] + b * (kBatchRows * 128), q_src + row_offset(there ? in_item : 0), there ? 16u : 0u);
                }
            }
            cp_async_commit();
            cp_async_wait_all();
            __syncwarp();
            // a thread a row from here: the maximum takes no shuffles, and eight rows' chunks at the same place lie in all banks
            uint8_t *const mine = sh.ptr + G::kOffQ + x * G::kTileBytes + row * 128;
            auto chunk = [&](int c) { return mine + (c >> 3) * kHalfBytes + (((c ^ row) & 7) << 4); };
            uint32_t top = 0;
#pragma unroll 1
            for (int c = 0; c < kPieces; c += 4) {
                uint4 v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const uint4 *>(chunk(c + u));
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    top = __vmaxu2(top, __vmaxu2(__vmaxu2(v[u].x & 0x7fff7fffu, v[u].y & 0x7fff7fffu), __vmaxu2(v[u].z & 0x7fff7fffu, v[u].w & 0x7fff7fffu)));
            }
            const float up = to_f16_range(__uint_as_float(max(top & 0xffffu, top >> 16) << 16)), f = up * pp.q_sign;
            sh.q_inv()[x * kBM + row] = pow2_inverse(up);
#pragma unroll 1
            for (int c = 0; c < kPieces; c += 4) {
                uint4 v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const uint4 *>(chunk(c + u));
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
                    uint32_t h[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) h[i] = pack_f16x2(__uint_as_float(w[i] << 16) * f, __uint_as_float(w[i] & 0xffff0000u) * f);
                    *reinterpret_cast<uint4 *>(chunk(c + u)) = make_uint4(h[0], h[1], h[2], h[3]);
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(sh.bar(G::Q_READY + x));
        }
        bool ok = true;
        if (!by_rows && x == 1 && n_it > 0) ok = wait(G::S_READY + 1, 0);  // the other slot's warps have been through Q
        const float row_scale = p.scale_log2 * (n_it > 0 ? sh.q_inv()[rx * kBM + row] : 1.f);

        const int first_lim = prefix + position(rx * kBM);                          // last key the tile's first row may see
        const int lim = prefix + position(min(rx * kBM + row, rows_here - 1));      // ... and this row
        int dj = by_rows ? 0 : 1, j0 = by_rows ? 0 : x;
        asm volatile("" : "+r"(dj), "+r"(j0));
        float m_run = -INFINITY, l_run = 0.f;
        auto publish = [&](int bar) {  // this thread's row of P is in TMEM
            cp::tcgen05_wait_st();
            fence_before();
            mbar_arrive(sh.bar(bar));
        };
#pragma unroll 1
        for (int i = 0; i < n_it && ok; ++i) {
            ok = wait(G::S_READY + x, (uint32_t)(i & 1));
            if (!ok) break;
            fence_after();
            const int j = (i << dj) + j0;  // the CTA's key tile
            const int key0 = (tile0 + j) * kBN;
            const int bad = *sh.bad_mask(j);
            // ---- a tile that the causal boundary cuts, or that holds a block the table does not name, first gets its hidden
            // scores overwritten with -inf in TMEM, and then runs through the same code as every other one
            if (key0 + kBN - 1 > first_lim || bad != 0) {
                const int rel = lim - key0;  // this row sees columns 0..rel
                const int rel_min = __reduce_min_sync(0xffffffffu, rel);
#pragma unroll 1
                for (int cc = 0; cc < 4; ++cc) {
                    const unsigned b2 = ((unsigned)bad >> (2 * cc)) & 3u;
                    if (32 * cc + 31 <= rel_min && b2 == 0u) continue;
                    const int r = rel - 32 * cc;
                    const unsigned past = r >= 31 ? 0u : (r < 0 ? 0xffffffffu : 0xfffffffeu << r);
                    const unsigned hid = past | ((b2 & 1u) ? 0x0000ffffu : 0u) | ((b2 & 2u) ? 0xffff0000u : 0u);
                    float v[32];
                    tc::tmem_ld32(v, t_s + 32 * cc);
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = ((hid >> i) & 1u) ? -INFINITY : v[i];
                    tc::tmem_st32(t_s + 32 * cc, v);
                }
                cp::tcgen05_wait_st();
            }
            float sv[128];
            {
                uint32_t(&r)[128] = reinterpret_cast<uint32_t(&)[128]>(sv);
                cp::tcgen05_ld_32x32b(reinterpret_cast<uint32_t(&)[32]>(r[0]), t_s);
                cp::tcgen05_ld_32x32b(reinterpret_cast<uint32_t(&)[32]>(r[32]), t_s + 32);
                cp::tcgen05_ld_32x32b(reinterpret_cast<uint32_t(&)[32]>(r[64]), t_s + 64);
                cp::tcgen05_ld_32x32b(reinterpret_cast<uint32_t(&)[32]>(r[96]), t_s + 96);
                cp::tcgen05_wait_ld();
            }
            float ks[8];
            {
                const float4 a = *reinterpret_cast<const float4 *>(sh.k_scale(j)), b = *reinterpret_cast<const float4 *>(sh.k_scale(j) + 4);
                const float e[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) ks[i] = fmaxf(e[i] * row_scale, 1.17549435e-38f);  // not 0: a masked score times it stays -inf
            }
            float m_tile = -INFINITY;  // scaled: a block at a time
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                float m0 = sv[16 * b], m1 = sv[16 * b + 1];
#pragma unroll
                for (int i = 2; i < 16; i += 2) {
                    m0 = fmaxf(m0, sv[16 * b + i]);
                    m1 = fmaxf(m1, sv[16 * b + i + 1]);
                }
                m_tile = fmaxf(m_tile, fmaxf(m0, m1) * ks[b]);
            }
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
            // ---- P = exp2(S*scale - m) (a masked -inf gives 0), row sum, bf16 pairs into the S columns
            float2 acc_a = make_float2(0.f, 0.f), acc_b = make_float2(0.f, 0.f);
            const float2 nm2 = make_float2(-m_use, -m_use);
#pragma unroll
            for (int cc = 0; cc < 4; ++cc) {
                uint32_t pk[16];
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    const float2 sc2 = make_float2(ks[2 * cc + (i >> 4)], ks[2 * cc + (i >> 4)]);
                    const float2 xa = __ffma2_rn(make_float2(sv[32 * cc + i], sv[32 * cc + i + 1]), sc2, nm2);
                    const float2 xb = __ffma2_rn(make_float2(sv[32 * cc + i + 2], sv[32 * cc + i + 3]), sc2, nm2);
                    const float2 pa = make_float2(fast_exp2(xa.x), fast_exp2(xa.y));
                    const float2 pb = make_float2(fast_exp2(xb.x), fast_exp2(xb.y));
                    acc_a = __fadd2_rn(acc_a, pa);
                    acc_b = __fadd2_rn(acc_b, pb);
                    pk[i >> 1] = pack_bf16x2(pa.x, pa.y);
                    pk[(i >> 1) + 1] = pack_bf16x2(pb.x, pb.y);
                }
                cp::tcgen05_st_32x32b(t_s + 16 * cc, pk);
                if (cc == tc::kPartSteps / 2 - 1) publish(G::P_PART + x);  // 96 keys stored
            }
            l_run += (acc_a.x + acc_a.y) + (acc_b.x + acc_b.y);
            publish(G::P_READY + x);
        }

        if (ok && n_it > 0) ok = wait(G::S_READY + x, (uint32_t)(n_it & 1));
        fence_after();  // every MMA that read the slot's Q tile or wrote its O has completed (the commit covers all earlier ones)
        if (!merge) {
            // ---- write-out: O / l -> bf16 -> the (now idle) Q tile in shared memory -> global, whole rows per instruction.
            // Only the warp that wrote a row reads it: __syncwarp suffices.
            if (ok) {
                const float inv = l_run > 0.f ? 1.f / l_run : 0.f;
#pragma unroll 1
                for (int cc = 0; cc < D / 32; ++cc) {
                    float ov[32];
                    tc::tmem_ld32(ov, t_o + 32 * cc);
#pragma unroll
                    for (int i = 0; i < 32; i += 8) {
                        uint4 v;
                        v.x = pack_bf16x2(ov[i] * inv, ov[i + 1] * inv);
                        v.y = pack_bf16x2(ov[i + 2] * inv, ov[i + 3] * inv);
                        v.z = pack_bf16x2(ov[i + 4] * inv, ov[i + 5] * inv);
                        v.w = pack_bf16x2(ov[i + 6] * inv, ov[i + 7] * inv);
                        const int c16 = cc * 4 + (i >> 3);
                        *reinterpret_cast<uint4 *>(q_tile + row * (D * 2) + ((c16 ^ (row & (kPieces - 1))) << 4)) = v;
                    }
                }
                __syncwarp();
                __nv_bfloat16 *to = p.out + first_head + piece * 8;
#pragma unroll 1
                for (int it = 0; it < 32 / kRowsPerInst; it += 4) {
                    uint4 v[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int rr = wrow0 + kRowsPerInst * (it + u) + sub;
                        v[u] = *reinterpret_cast<const uint4 *>(q_tile + rr * (D * 2) + ((piece ^ (rr & (kPieces - 1))) << 4));
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int in_item = rx * kBM + wrow0 + kRowsPerInst * (it + u) + sub;
                        if (in_item < rows_here) *reinterpret_cast<uint4 *>(to + row_offset(in_item)) = v[u];
                    }
                }
            }
        } else {
            // ---- partial results into shared memory, in place of the tiles, once every role is through with those.  Chunks of 16
            // bytes are XORed with the row, so that the 32 rows of a warp do not meet in a bank.
            constexpr int kChunks = D / 4;
            meet_all();
            const bool none = !ok || n_it == 0;
            if (rx * kBM + wrow0 < rows_here) {
#pragma unroll 1
                for (int cc = 0; cc < D / 32; ++cc) {
                    float ov[32];
                    tc::tmem_ld32(ov, t_o + 32 * cc);
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const float4 v = none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(ov[4 * c], ov[4 * c + 1], ov[4 * c + 2], ov[4 * c + 3]);
                        *reinterpret_cast<float4 *>(sh.ptr + G::kOffPart + ((x * kBM + row) * kChunks + ((8 * cc + c) ^ (row & (kChunks - 1)))) * 16) = v;
                    }
                }
                *reinterpret_cast<float2 *>(sh.ptr + G::kOffPartML + (x * kBM + row) * 8) = none ? make_float2(-INFINITY, 0.f) : make_float2(m_run, l_run);
            }
            meet_cluster();
            // ---- this CTA's share of the rows (part, part + cluster, ...), out of the shared memories of all of the cluster.  A read
            // of another SM's shared memory takes most of a microsecond, so it is done wide: first a thread a row for the weights,
            // then a warp for four rows (kChunks lanes a row) at a time.
            const int parts = by_rows ? cluster : 2 * cluster;
            const int n_rows = (rows_here - part + cluster - 1) / cluster;
            float *weights = (float *)(sh.ptr + G::kOffPartW);
            auto source = [&](int i, int r, uint32_t &slot_row) {  // partial i of row r: a CTA's, or a CTA's slot's
                slot_row = (uint32_t)((by_rows ? r >> 7 : i & 1) * kBM + (r & (kBM - 1)));
                return cluster > 1 ? map_to_cta(sh.base, by_rows ? i : i >> 1) : sh.base;
            };
            for (int k = threadIdx.x - 128; k < n_rows; k += 256) {
                float m = -INFINITY, l = 0.f;
#pragma unroll 4
                for (int i = 0; i < parts; ++i) {
                    uint32_t sr;
                    const uint32_t base = source(i, part + cluster * k, sr);
                    const float2 v = ld_cluster_f2(base + G::kOffPartML + sr * 8);
                    const float m_new = fmaxf(m, v.x);
                    if (m_new > -INFINITY) l = l * fast_exp2(m - m_new) + v.y * fast_exp2(v.x - m_new);
                    m = m_new;
                }
                const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll 4
                for (int i = 0; i < parts; ++i) {
                    uint32_t sr;
                    const uint32_t base = source(i, part + cluster * k, sr);
                    const float mi = ld_cluster_f2(base + G::kOffPartML + sr * 8).x;
                    weights[k * parts + i] = mi > -INFINITY ? fast_exp2(mi - m) * inv : 0.f;
                }
            }
            asm volatile("bar.sync 2, 256;" ::: "memory");
            constexpr int kRowsAtOnce = 4, kRowsPerWarp = 32 / kChunks;
            const int chunk = lane & (kChunks - 1);
#pragma unroll 1
            for (int k0 = (warp - 4) * kRowsPerWarp * kRowsAtOnce + lane / kChunks; k0 < n_rows; k0 += 8 * kRowsPerWarp * kRowsAtOnce) {
                float4 acc[kRowsAtOnce];
#pragma unroll
                for (int u = 0; u < kRowsAtOnce; ++u) acc[u] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
                for (int i = 0; i < parts; ++i) {
#pragma unroll
                    for (int u = 0; u < kRowsAtOnce; ++u) {
                        const int k = min(k0 + u * kRowsPerWarp, n_rows - 1), r = part + cluster * k;
                        uint32_t sr;
                        const uint32_t base = source(i, r, sr);
                        const float4 o = ld_cluster_f4(base + G::kOffPart + (sr * kChunks + (chunk ^ (r & (kChunks - 1)))) * 16);
                        const float w = weights[k * parts + i];
                        acc[u].x += w * o.x, acc[u].y += w * o.y, acc[u].z += w * o.z, acc[u].w += w * o.w;
                    }
                }
#pragma unroll
                for (int u = 0; u < kRowsAtOnce; ++u) {
                    const int k = k0 + u * kRowsPerWarp;
                    if (k < n_rows)
                        *reinterpret_cast<uint2 *>(p.out + first_head + row_offset(part + cluster * k) + chunk * 4) =
                            make_uint2(pack_bf16x2(acc[u].x, acc[u].y), pack_bf16x2(acc[u].z, acc[u].w));
                }
            }
            if (cluster > 1) cluster_barrier();  // nobody leaves while another may read its shared memory
        }
        }
    }

    // ---- teardown: everybody meets, TMEM goes back
    fence_before();
    __syncthreads();
    fence_after();
    if (threadIdx.x == 0 && *sh.abort_flag()) atomicOr(p.status, EKV_DEV_FLAG_TIMEOUT);  // a wait ran out
    if (warp == 1) cp::tcgen05_dealloc(cp::cta_group_1, tmem, 512);

    // ---- NaN values: of the last item or the one before it, whose rows have been written and whose numbers are still in their slots.  (By
    // warps that have the registers; behind everything else, since in any other place this code cost calls without NaN up to 4 %.)
    if (warp < 4 || warp >= 12 || *sh.abort_flag()) return;
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
        if (!*sh.nan_seen(k)) continue;
        const volatile int *slot = sh.item(k);
        const int kv_head = slot[2], from = slot[3], q_first = slot[5], before = slot[7];
        nan_values<D>(pp, kv_head, p.block_tables + (size_t)slot[1] * p.max_blocks, (before + by_group(from) + 1) / kBN * kBN,
                      min(slot[6], before + by_group(from + slot[4] - 1) + 1), warp - 4, slot[4], 8, [&](int r, int &last, __nv_bfloat16 *&at) {
                          const int pos = by_group(from + r);
                          last = before + pos;
                          at = p.out + ((size_t)(q_first + pos) * p.num_q_heads + (size_t)(kv_head * group + from + r - pos * group)) * D;
                      });
    }
}

// fit[i] = clusters of 2^i CTAs of the kernel that run at the same time on the current device (0: none do)
static void clusters_that_fit(const void *kernel, cudaLaunchConfig_t cfg, int *fit) {
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    for (int i = kMaxClusterLog; i >= 0; --i) {
        attr.val.clusterDim.x = 1u << i;
        cfg.gridDim = dim3(1u << i);
        if (cudaOccupancyMaxActiveClusters(&fit[i], kernel, &cfg) != cudaSuccess) {
            fit[i] = 0;
            (void)cudaGetLastError();
        }
    }
    if (fit[0] < 1) fit[0] = 1;  // asked
}

// log2 of the CTAs that an item's keys are cut over: as many as let all items run at the same time, while a part keeps two key
// tiles of the longest sequence that the table can hold.  fit[i]: clusters of 2^i CTAs that run at the same time.  Never more than
// one round of the machine: a part costs 10 to 15 us beyond its tiles (a cold start and the merge).  Measured, 32q/8kv, us with 1 / 2
// / 4 / 8 / 16 CTAs an item: 64 positions over 30000 keys (8 items) 460 243 134 81 104; 128 over 8000 (16) 136 80 50 70 89; 512 over
// 8000 (64) 143 85 100 176 296; 1024 over 8000 (128) 151 163 198 319 566.  (Clusters stay inside a GPC: of a B200's 148 SMs, 7
// clusters of 16, 15 of 8, 33 of 4 run at a time.)
// Depends on the call's shape arguments alone.
static int plan_cluster(long long items, int max_blocks, const int *fit) {
    const long long max_tiles = ((long long)max_blocks * 16 + kBN - 1) / kBN;
    int c = 0;
    while (c < kMaxClusterLog && items <= fit[c + 1] && (4ll << c) <= max_tiles) ++c;
    return c;
}

template <int D>
static ekv_status_t launch_prefill8(ekv_pool *pool, Params &pp, cudaStream_t stream) {
    static int fits[64][kMaxClusterLog + 1] = {};  // per device: clusters of 2^i CTAs that run at the same time; [..][0] 0: not asked yet
    const int dev = pool->desc.device;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Geo<D>::kSmemBytes;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int asked[kMaxClusterLog + 1] = {}, *fit = dev < 64 ? fits[dev] : asked;
    if (fit[0] == 0) {
        cudaError_t e = cudaFuncSetAttribute(prefill8_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Geo<D>::kSmemBytes);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(prefill8_kernel<D>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return cuda_fail(e, "ekv_attn_prefill_chunk: kernel attributes");
        clusters_that_fit((const void *)prefill8_kernel<D>, cfg, fit);
    }
    const long long items = (long long)pp.p.q_tiles * pp.p.num_kv_heads;
    pp.cluster_log = plan_cluster(items, pp.p.max_blocks, fit);
    pp.cluster = 1 << pp.cluster_log;
    attr.val.clusterDim.x = (unsigned)pp.cluster;
    cfg.gridDim = dim3((unsigned)(items * pp.cluster));
    cfg.stream = stream;
    cudaError_t e = cudaLaunchKernelEx(&cfg, prefill8_kernel<D>, pp);
    if (e != cudaSuccess) return cuda_fail(e, "ekv_attn_prefill_chunk: launch");
    return EKV_OK;
}

}  // namespace tc8
}  // namespace ekv

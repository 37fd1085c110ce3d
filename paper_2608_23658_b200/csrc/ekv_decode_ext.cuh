// Decode attention for the scores and masks of ekv_rows.cuh, and for the keys of a request behind those that its group shares.
//
// The split pass of ekv_decode.cu -- a CTA per (sequence, kv-head, range of keys), each warp a ring of TMA loads for every fourth block of 16
// keys, the heads of the group as the rows of mma.m16n8k16, partial (m, l, O) per range -- over those blocks alone that the sequence sees:
// of its prefix and of its window, or from the end of the shared keys on.  Bound by the bytes of these: 64 sequences of up to 16000 keys, 32q/8kv, 1.04 GB
// in 158 to 166 us = 6.3 to 6.6 TB/s.  Where a sequence has a single range (many do, where the tables are wider than the sequences long) the CTA
// writes the final rows itself.  Up to sixteen ranges whose CTAs are all there at once are a cluster and add themselves up out of each other's shared
// memory (5 sequences of up to 1000 keys, 4q/2kv d64: 5.5 us on the device for 6.6 with a second launch; one of 4000 6.5 for 11.2); for more,
// combine_ext_kernel does, a warp a (sequence, head).
// In a shared call this launch comes up beside the rows kernel's, which takes an SM for an item and is cut so that SMs are left, and fills the rest as its
// items end; combine_ext_kernel adds the parts of both.  256 requests of 17..700 own keys behind 16384 shared ones: 114 us, one after the other
// 130; nine groups of 28q/4kv 37 for 48.  Only the last CTA waits for the rows kernel, so that the launch behind this one finds both done.
// With next to no own keys each CTA waits and takes the shared keys' parts along instead, which saves a launch.
#pragma once
#include "ekv_rows.cuh"

namespace ekv {
namespace ext {

using rows::kMaxGroups;

static constexpr int kWarps = 4;
static constexpr int kStages = 2;  // of a warp; 64 KB in all, so that three CTAs fit an SM: with three stages and two CTAs, own parts of 256 requests took 88 us for 75
static constexpr int kBoxBytes = 16 * 128;  // 16 tokens x 64 channels
static constexpr int kCluster = 16;         // ranges of a sequence that are a cluster, at most
static constexpr int kMaxParts = 64;        // that the rows kernel cuts shared keys into

struct Params {
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    const int *block_tables, *seq_lens;
    const long long *live;
    unsigned *status;
    const float *slopes;      // or null
    const int *prefix_lens;   // or null
    float *part_o;            // [B * Hq * nsplit][D], own ranges
    float2 *part_ml;
    const float *shared_o;    // [B * Hq * parts][D], of the shared keys
    const float2 *shared_ml;
    int max_blocks, num_q_heads, num_kv_heads, group;
    int chunk_tokens, nsplit;
    int window;
    int parts, G;
    int cluster;              // a sequence's ranges are a cluster, which adds them up itself
    int beside;               // shared call: the two passes run side by side, and combine_ext_kernel adds the shared keys' parts
    float scale_log2;           // scale * log2 e
    float cap_scale, cap_log2;  // with a cap: scale / cap, cap * log2 e (both within fp32's normal range)
    int start[kMaxGroups + 1];     // shared call: first request of a group,
    int shared[kMaxGroups];        // its shared keys
    uint8_t ns[kMaxGroups];        // and the parts that the rows kernel cut them into; 0: it did not, every request reads its own
};

// What of a sequence is to be read: blocks 0 .. n_pre - 1 and those from n_pre + skip on, `tokens` of them counted up to the last key.
struct Span {
    int L, lo, pre;       // keys lo .. L-1 and those below pre are seen
    int n_pre, skip, tokens;
    int parts;            // of the shared keys
    int first, common;    // blocks below `common` are named by the table of request `first`
    bool invalid;
};

template <bool kShared>
__device__ __forceinline__ Span span_of(const Params &p, int b) {
    Span s;
    s.L = max(0, min(p.seq_lens[b], p.max_blocks * 16));
    s.parts = 0;
    s.invalid = false;
    s.lo = s.pre = s.n_pre = s.skip = s.common = 0;
    s.first = b;
    if (kShared) {
        int g = 0, hi = p.G;
#pragma unroll 1
        while (hi - g > 1) {
            const int mid = (g + hi) >> 1;
            if (p.start[mid] <= b) g = mid;
            else hi = mid;
        }
        s.invalid = s.L > 0 && s.L < p.shared[g];
        s.first = p.start[g], s.common = p.shared[g] / 16;
        if (s.invalid) s.L = 0;
        s.parts = s.L > 0 ? p.ns[g] : 0;
        if (s.parts > 0) s.lo = p.shared[g], s.skip = s.lo / 16;
    } else {
        s.lo = p.window > 0 ? max(0, s.L - p.window) : 0;
        s.pre = p.prefix_lens ? max(0, min(p.prefix_lens[b], s.L)) : 0;
        s.n_pre = (s.pre + 15) / 16;
        s.skip = max(0, s.lo / 16 - s.n_pre);
    }
    s.tokens = s.L - s.skip * 16;
    return s;
}

__device__ __forceinline__ float finish(float acc, float l) { return l == 0.f ? 0.f : acc / l; }

template <int D, bool kShared, bool kCap, bool kBias>
__global__ void __launch_bounds__(kWarps * 32, 3) decode_ext_kernel(const __grid_constant__ CUtensorMap kvmap, const __grid_constant__ Params p) {
    constexpr int BOXES = D / 64;
    constexpr int TILE_BYTES = BOXES * kBoxBytes;
    constexpr int STAGE_BYTES = 2 * TILE_BYTES;
    constexpr int KSTEPS = D / 16;
    constexpr unsigned FULL = 0xffffffffu;

    const int split = blockIdx.x, g = blockIdx.y, b = blockIdx.z;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r = lane >> 2, c = lane & 3;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the combine pass comes up in the tail of this one
    const Span sp = span_of<kShared>(p, b);
    const int t_begin = split * p.chunk_tokens;
    const bool is_last = split == (int)gridDim.x - 1 && g == (int)gridDim.y - 1 && b == (int)gridDim.z - 1;
    // Ranges of a cluster meet at its end if there are several: those without keys then stay.
    const bool meet = p.cluster && sp.tokens > p.chunk_tokens;
    if (split > 0 && t_begin >= sp.tokens && !meet) {  // whole CTA leaves before any barrier exists
        if (kShared && (!p.beside || is_last)) asm volatile("griddepcontrol.wait;" ::: "memory");  // this launch is not over before the one it came up beside
        return;
    }
    if (kShared && sp.invalid && split == 0 && g == 0 && threadIdx.x == 0) atomicOr(p.status, EKV_DEV_FLAG_OOB);
    const int t_end = min(sp.tokens, t_begin + p.chunk_tokens);  // counted over what is read
    const int nblk = (max(t_end - t_begin, 0) + 15) >> 4;
    const int nw = max(0, (nblk - warp + kWarps - 1) / kWarps);  // blocks this warp owns (<= 32)
    auto block_of = [&](int i) {  // the warp's i-th block, in the sequence
        const int l = (t_begin >> 4) + warp + kWarps * i;
        return l < sp.n_pre ? l : l + sp.skip;
    };

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_u32 = smem_u32(smem_raw);
    const uint32_t base_u32 = (raw_u32 + 1023u) & ~1023u;
    uint8_t *base_ptr = smem_raw + (base_u32 - raw_u32);
    const uint32_t my_stages = base_u32 + warp * kStages * STAGE_BYTES;
    const uint32_t my_bars = base_u32 + kWarps * kStages * STAGE_BYTES + warp * kStages * 8;
    if (lane == 0) {
        prefetch_tensormap(&kvmap);
        for (int s = 0; s < kStages; ++s) mbar_init(my_bars + 8 * s, 1);
        mbar_fence_init();
    }
    __syncwarp();

    // Block ids of this warp's blocks: lane i holds the id of its i-th block.
    const long long live = *p.live;
    const int my_block = block_of(lane);
    const int my_id = (lane < nw) ? p.block_tables[(size_t)(my_block < sp.common ? sp.first : b) * p.max_blocks + my_block] : 0;
    const bool my_ok = (lane < nw) && my_id >= 0 && (long long)my_id < live;
    const unsigned valid_mask = __ballot_sync(FULL, my_ok);
    if (lane < nw && !my_ok) atomicOr(p.status, EKV_DEV_FLAG_OOB);

    const uint64_t policy = policy_evict_first();
    auto issue = [&](int i) {
        const int id = __shfl_sync(FULL, my_id, i);
        if (lane == 0 && ((valid_mask >> i) & 1u)) {
            const int stage = i % kStages;
            const uint32_t bar = my_bars + 8 * stage;
            const uint32_t dst = my_stages + stage * STAGE_BYTES;
            const int row_k = g * 16, row_v = row_k + p.num_kv_heads * 16;  // row inside the block: (K|V, kv-head, token)
            mbar_expect_tx(bar, STAGE_BYTES);
#pragma unroll
            for (int x = 0; x < BOXES; ++x) {
                tma_load_3d_hint(dst + x * kBoxBytes, &kvmap, 64 * x, row_k, id, bar, policy);
                tma_load_3d_hint(dst + TILE_BYTES + x * kBoxBytes, &kvmap, 64 * x, row_v, id, bar, policy);
            }
        }
    };
    for (int s = 0; s < kStages && s < nw; ++s) issue(s);

    // Q fragments (A operand): rows = heads of the group (r < group), zero above.
    uint32_t qa[KSTEPS][2];
    {
        const __nv_bfloat16 *qrow = p.q + ((size_t)b * p.num_q_heads + (size_t)g * p.group + r) * D;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
            qa[ks][0] = (r < p.group) ? *reinterpret_cast<const uint32_t *>(qrow + 16 * ks + 2 * c) : 0u;
            qa[ks][1] = (r < p.group) ? *reinterpret_cast<const uint32_t *>(qrow + 16 * ks + 8 + 2 * c) : 0u;
        }
    }
    const float slope = kBias && r < p.group ? p.slopes[g * p.group + r] * 1.4426950408889634f : 0.f;

    // ldmatrix lane addressing inside one swizzled tile: matrix mi = lane/8, row rr = lane%8.
    const int mi = lane >> 3, rr = lane & 7;
    const uint32_t lane_row_off = (8 * (mi >> 1) + rr) * 128;
    const int lane_par = mi & 1;

    float o[KSTEPS][4];
#pragma unroll
    for (int mt = 0; mt < KSTEPS; ++mt) o[mt][0] = o[mt][1] = o[mt][2] = o[mt][3] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    bool failed = false;

    uint32_t stage_parity = 0;  // of the copies that really went through a stage
    int i = 0;
    for (; i < nw; ++i) {
        const int stage = i % kStages;
        if ((valid_mask >> i) & 1u) {
            const bool got = mbar_wait(my_bars + 8 * stage, (stage_parity >> stage) & 1u);
            stage_parity ^= 1u << stage;
            if (__any_sync(FULL, !got)) {
                failed = true;
                break;
            }
            const uint32_t kbase = my_stages + stage * STAGE_BYTES;
            const uint32_t vbase = kbase + TILE_BYTES;
            const int tok0 = block_of(i) * 16;
            const bool partial = tok0 + 16 > sp.L || (tok0 < sp.lo && tok0 + 16 > sp.pre);

            float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks) {
                const int chunk = 2 * ks + lane_par;
                const uint32_t addr = kbase + (chunk >> 3) * kBoxBytes + lane_row_off + (((chunk & 7) ^ rr) << 4);
                uint32_t k0, k1, k2, k3;
                ldmatrix_x4(addr, k0, k1, k2, k3);
                mma_bf16_16816(s0, qa[ks][0], 0u, qa[ks][1], 0u, k0, k1);
                mma_bf16_16816(s1, qa[ks][0], 0u, qa[ks][1], 0u, k2, k3);
            }
            const int t = tok0 + 2 * c;  // this lane's keys: t, t + 1, t + 8, t + 9
            float x[4] = {s0[0], s0[1], s1[0], s1[1]};
            uint32_t mask_lo = 0xffffffffu, mask_hi = 0xffffffffu;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (kCap) x[e] = rows::capped(x[e], p.cap_scale, p.scale_log2, p.cap_log2);
                else x[e] *= p.scale_log2;
                if (kBias) x[e] -= slope * (float)(sp.L - 1 - (t + (e & 1) + 8 * (e >> 1)));
            }
            if (partial) {
                auto seen = [&](int key) { return key < sp.L && (key >= sp.lo || key < sp.pre); };
                const bool v0 = seen(t), v1 = seen(t + 1), v2 = seen(t + 8), v3 = seen(t + 9);
                if (!v0) x[0] = -INFINITY;
                if (!v1) x[1] = -INFINITY;
                if (!v2) x[2] = -INFINITY;
                if (!v3) x[3] = -INFINITY;
                mask_lo = (v0 ? 0x0000ffffu : 0u) | (v1 ? 0xffff0000u : 0u);
                mask_hi = (v2 ? 0x0000ffffu : 0u) | (v3 ? 0xffff0000u : 0u);
            }
            float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
            mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, 2));
            const float m_new = fmaxf(m_run, mx);
            const float m_use = m_new > -INFINITY ? m_new : 0.f;  // (scores of -infinity, as infinite keys give them, weigh nothing)
            const float alpha = fast_exp2(m_run - m_use);
            const float p0 = fast_exp2(x[0] - m_use), p1 = fast_exp2(x[1] - m_use);
            const float p2 = fast_exp2(x[2] - m_use), p3 = fast_exp2(x[3] - m_use);
            l_run = l_run * alpha + ((p0 + p1) + (p2 + p3));
            m_run = m_new;
            if (__any_sync(FULL, alpha != 1.f)) {
                const float a_lo = __shfl_sync(FULL, alpha, 8 * c);
                const float a_hi = __shfl_sync(FULL, alpha, 8 * c + 4);
#pragma unroll
                for (int mt = 0; mt < KSTEPS; ++mt) {
                    o[mt][0] *= a_lo;
                    o[mt][1] *= a_hi;
                    o[mt][2] *= a_lo;
                    o[mt][3] *= a_hi;
                }
            }
            const uint32_t pb0 = pack_bf16x2(p0, p1), pb1 = pack_bf16x2(p2, p3);  // weights in bf16, V's type, as the MMA wants: off by up to 2^-8 of themselves
#pragma unroll
            for (int mt = 0; mt < KSTEPS; ++mt) {
                const int chunk = 2 * mt + lane_par;
                const uint32_t addr = vbase + (chunk >> 3) * kBoxBytes + lane_row_off + (((chunk & 7) ^ rr) << 4);
                uint32_t v0, v1, v2, v3;
                ldmatrix_x4_trans(addr, v0, v1, v2, v3);
                if (partial) {  // values at keys that are not seen may be anything: 0 * NaN must not reach O
                    v0 &= mask_lo;
                    v1 &= mask_lo;
                    v2 &= mask_hi;
                    v3 &= mask_hi;
                }
                mma_bf16_16816(o[mt], v0, v1, v2, v3, pb0, pb1);
            }
        }
        __syncwarp();  // every lane is done reading the stage before it is refilled
        if (i + kStages < nw) issue(i + kStages);
    }

    if (failed) {
        // A copy barrier never completed.  Latch the error, give copies still in flight a bounded chance to land (their destination
        // must stay allocated), and contribute nothing.
        if (lane == 0) atomicOr(p.status, EKV_DEV_FLAG_TIMEOUT);
        stage_parity ^= 1u << (i % kStages);  // the wait that failed belongs to a copy still outstanding
        for (int j = i; j < nw && j < i + kStages; ++j)
            if ((valid_mask >> j) & 1u)
                (void)mbar_wait(my_bars + 8 * (j % kStages), (stage_parity >> (j % kStages)) & 1u, 200000000ull);
        m_run = -INFINITY;
        l_run = 0.f;
#pragma unroll
        for (int mt = 0; mt < KSTEPS; ++mt) o[mt][0] = o[mt][1] = o[mt][2] = o[mt][3] = 0.f;
    }

    l_run += __shfl_xor_sync(FULL, l_run, 1);
    l_run += __shfl_xor_sync(FULL, l_run, 2);

    // Merge the 4 warps through shared memory (each warp reuses its own, now idle, first stage).
    float *wo = reinterpret_cast<float *>(base_ptr + warp * kStages * STAGE_BYTES);  // [8][D]
    float *wm = wo + 8 * D;                                                          // [8] m, [8] l
#pragma unroll
    for (int mt = 0; mt < KSTEPS; ++mt) {
        wo[(2 * c) * D + 16 * mt + r] = o[mt][0];
        wo[(2 * c + 1) * D + 16 * mt + r] = o[mt][1];
        wo[(2 * c) * D + 16 * mt + 8 + r] = o[mt][2];
        wo[(2 * c + 1) * D + 16 * mt + 8 + r] = o[mt][3];
    }
    if (c == 0) {
        wm[r] = m_run;
        wm[8 + r] = l_run;
    }
    __syncthreads();
    if (kShared && (!p.beside || is_last)) asm volatile("griddepcontrol.wait;" ::: "memory");  // the shared keys' parts are complete
    // The weights of what a head's row is made of -- the four warps' results and, where the sequence ends here, the shared keys' parts -- once a
    // head, by a warp; then a thread a channel.  (In warp 0's second stage: idle, too.)
    constexpr int kTerms = kWarps + kMaxParts;
    const bool last = sp.tokens <= p.chunk_tokens && !(kShared && p.beside && sp.parts > 0);  // the sequence's only range: finish here
    const int n_parts = kShared && last ? sp.parts : 0;
    float *weights = reinterpret_cast<float *>(base_ptr + STAGE_BYTES);  // [8][kTerms]
    float *rowsum = weights + 8 * kTerms;                                // [8] l, [8] m
    float *result = reinterpret_cast<float *>(base_ptr + (kStages + 1) * STAGE_BYTES);  // [8][D], in warp 1's second stage
    static_assert((8 * kTerms + 16) * 4 <= STAGE_BYTES && (8 * D + 16) * 4 <= STAGE_BYTES, "merge area");
    for (int h = warp; h < p.group; h += kWarps) {
        const size_t row = (size_t)b * p.num_q_heads + (size_t)g * p.group + h;
        float2 ml[kTerms / 32 + 1];
        float mstar = -INFINITY;
#pragma unroll
        for (int k = 0; k <= kTerms / 32; ++k) {
            const int i = 32 * k + lane;
            const float *own = reinterpret_cast<const float *>(base_ptr + (i & (kWarps - 1)) * kStages * STAGE_BYTES) + 8 * D;
            ml[k] = i < kWarps ? make_float2(own[h], own[8 + h]) : i - kWarps < n_parts ? p.shared_ml[row * p.parts + i - kWarps] : make_float2(-INFINITY, 0.f);
            mstar = fmaxf(mstar, ml[k].x);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) mstar = fmaxf(mstar, __shfl_xor_sync(FULL, mstar, d));
        float lsum = 0.f;
#pragma unroll
        for (int k = 0; k <= kTerms / 32; ++k) {  // (a term without a maximum holds zeros, or NaN if its scores were NaN: either counts)
            const float w = ml[k].x > -INFINITY ? fast_exp2(ml[k].x - mstar) : 0.f;
            lsum += w * ml[k].y;
            if (32 * k + lane < kTerms) weights[h * kTerms + 32 * k + lane] = w;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) lsum += __shfl_xor_sync(FULL, lsum, d);
        if (lane == 0) rowsum[h] = lsum, rowsum[8 + h] = mstar;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.group * D; e += kWarps * 32) {
        const int h = e / D, ch = e % D;
        const size_t row = (size_t)b * p.num_q_heads + (size_t)g * p.group + h;
        float acc = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) acc += weights[h * kTerms + w] * reinterpret_cast<const float *>(base_ptr + w * kStages * STAGE_BYTES)[h * D + ch];
        const float *part = p.shared_o + (row * p.parts) * D + ch;
        for (int s = 0; s < n_parts; s += 4) {  // four loads under way, whatever their number
            float w[4], o[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                w[u] = s + u < n_parts ? weights[h * kTerms + kWarps + s + u] : 0.f;
                o[u] = w[u] != 0.f ? part[(size_t)(s + u) * D] : 0.f;  // (0: nothing may have been written for it)
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) acc += w[u] * o[u];
        }
        if (last) {
            p.out[row * D + ch] = __float2bfloat16_rn(finish(acc, rowsum[h]));
        } else if (meet) {
            result[e] = acc;
        } else {
            const size_t slot = row * p.nsplit + split;
            p.part_o[slot * D + ch] = acc;
            if (ch == 0) p.part_ml[slot] = make_float2(rowsum[8 + h], rowsum[h]);
        }
    }
    if (!meet) return;
    // ---- ranges: each CTA adds up a share of the elements out of the shared memories of all of the cluster
    cluster_barrier();
    const uint32_t result_at = base_u32 + (uint32_t)((uint8_t *)result - base_ptr), rowsum_at = base_u32 + (uint32_t)((uint8_t *)rowsum - base_ptr);
    for (int e = split * kWarps * 32 + threadIdx.x; e < p.group * D; e += p.nsplit * kWarps * 32) {
        const int h = e / D;
        float l[kCluster], m[kCluster], mstar = -INFINITY;
#pragma unroll
        for (int i = 0; i < kCluster; ++i) {
            if (i == 8 && p.nsplit <= 8) break;
            const uint32_t at = map_to_cta(rowsum_at + 4 * h, min(i, p.nsplit - 1));
            l[i] = i < p.nsplit ? ld_cluster_f1(at) : 0.f;
            m[i] = i < p.nsplit ? ld_cluster_f1(at + 32) : -INFINITY;
            mstar = fmaxf(mstar, m[i]);
        }
        float acc = 0.f, lsum = 0.f;
#pragma unroll
        for (int i = 0; i < kCluster; ++i) {  // (a range without a maximum has a sum of 0, or NaN if its scores were NaN)
            if (i == 8 && p.nsplit <= 8) break;
            const float w = m[i] > -INFINITY ? fast_exp2(m[i] - mstar) : 0.f;
            lsum += w * l[i];
            if (w != 0.f) acc += w * ld_cluster_f1(map_to_cta(result_at + 4 * e, i));
        }
        p.out[((size_t)b * p.num_q_heads + (size_t)g * p.group) * D + e] = __float2bfloat16_rn(finish(acc, lsum));
    }
    cluster_barrier();  // nobody leaves while its shared memory is read
}

// Adds the parts of a row, a list at a time: a warp a row, D / 32 channels a lane, eight parts' loads under way.
template <int D>
struct RowSum {
    static constexpr int kC = D / 32;
    float acc[kC], m = -INFINITY, l = 0.f;
    __device__ __forceinline__ RowSum() {
#pragma unroll
        for (int c = 0; c < kC; ++c) acc[c] = 0.f;
    }
    __device__ __forceinline__ void add(const float *o, const float2 *ml, int n) {
        const int lane = threadIdx.x & 31;
        for (int s0 = 0; s0 < n; s0 += 32) {
            const float2 v = s0 + lane < n ? ml[s0 + lane] : make_float2(-INFINITY, 0.f);
            float top = v.x;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            const float m_new = fmaxf(m, top), alpha = m > -INFINITY ? fast_exp2(m - m_new) : 1.f;  // (nothing added yet, or NaN)
            const float w = v.x > -INFINITY ? fast_exp2(v.x - m_new) : 0.f;
            float sum = w * v.y;  // (a part whose scores were NaN has no maximum and a sum of NaN, which 0 leaves NaN)
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            l = l * alpha + sum;
#pragma unroll
            for (int c = 0; c < kC; ++c) acc[c] *= alpha;
            m = m_new;
            const int here = min(32, n - s0);
#pragma unroll 8
            for (int s = 0; s < here; ++s) {
                const float ws = __shfl_sync(0xffffffffu, w, s);
                const float ms = __shfl_sync(0xffffffffu, v.x, s);
                if (!(ms > -INFINITY)) continue;  // nothing was written for it
                const float *src = o + (size_t)(s0 + s) * D + lane * kC;
                if (kC == 4) {
                    const float4 x = *reinterpret_cast<const float4 *>(src);
                    acc[0] += ws * x.x, acc[1] += ws * x.y, acc[kC - 2] += ws * x.z, acc[kC - 1] += ws * x.w;
                } else {
                    const float2 x = *reinterpret_cast<const float2 *>(src);
                    acc[0] += ws * x.x, acc[kC - 1] += ws * x.y;
                }
            }
        }
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *out) const {
        const int lane = threadIdx.x & 31;
        uint32_t w[kC / 2];
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int c = 0; c < kC; c += 2) w[c / 2] = pack_bf16x2(acc[c] * inv, acc[c + 1] * inv);
        if (kC == 4) *reinterpret_cast<uint2 *>(out + lane * kC) = make_uint2(w[0], w[kC / 2 - 1]);
        else *reinterpret_cast<uint32_t *>(out + lane * kC) = w[0];
    }
};

static constexpr int kCombineWarps = 4;

template <int D, bool kShared>
__global__ void __launch_bounds__(kCombineWarps * 32) combine_ext_kernel(const __grid_constant__ Params p, int rows) {
    const int row = blockIdx.x * kCombineWarps + (threadIdx.x >> 5);
    if (row >= rows) {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        return;
    }
    const Span sp = span_of<kShared>(p, row / p.num_q_heads);  // (lengths and offsets were there before the split pass)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (sp.tokens <= p.chunk_tokens && !(kShared && p.beside && sp.parts > 0)) return;  // finished by the split pass
    RowSum<D> sum;
    if (kShared) sum.add(p.shared_o + (size_t)row * p.parts * D, p.shared_ml + (size_t)row * p.parts, sp.parts);
    sum.add(p.part_o + (size_t)row * p.nsplit * D, p.part_ml + (size_t)row * p.nsplit, (sp.tokens + p.chunk_tokens - 1) / p.chunk_tokens);
    sum.store(p.out + (size_t)row * D);
}

// The parts of prefill rows: every row of a request has as many.
template <int D>
__global__ void __launch_bounds__(kCombineWarps * 32) combine_rows_kernel(const float *part_o, const float2 *part_ml, __nv_bfloat16 *out, const int *cu_q_lens, int R,
                                                                          int num_q_heads, int parts, int rows) {
    const int row = blockIdx.x * kCombineWarps + (threadIdx.x >> 5);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (row >= rows || row / num_q_heads >= cu_q_lens[R]) return;
    RowSum<D> sum;
    sum.add(part_o + (size_t)row * parts * D, part_ml + (size_t)row * parts, parts);
    sum.store(out + (size_t)row * D);
}

}  // namespace ext
}  // namespace ekv

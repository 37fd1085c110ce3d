// ekv_attn_prefill_chunk over an 8-bit pool for requests of FEW query rows (drafted tokens to be checked, a decode row in a
// mixed batch): at most 32 (position, head of the group) rows per kv-head.
//
// Such a request is bound by reading its keys and values once, like decode, and the tensor instruction of 128 rows would be
// mostly empty behind a conversion of every tile into shared memory.  So this is decode's split pass (ekv_decode_e4m3.cuh has
// the fragments and why the codes get there without shuffles) with a full 16-row tile as the A operand of the scores and two 8-row
// tiles as the B operand of O^T += V^T P^T.
//   ring         one warp, or two for a request of more than 16 rows, read the same TMA stages, so that a block crosses from device
//                memory once whatever the rows; each converts it for itself (sharing the conversion too would take the registers
//                of two row tiles in one warp, and with them the warps that hide its latency; it was slower)
//   CTA          8 warps = 8 or 4 rings; ring k takes every 8th or 4th block of the CTA's key range
//   cluster      up to 16 CTAs share a (request, kv-head)'s keys and merge (m, l, O) through distributed shared memory: the call
//                has no workspace.  Rings first, then CTAs, each in a fixed order: the same bits every time.
// Measured, 32q/8kv, d128, us here and on the tensor instruction's kernel: 128 requests over 2000..8000 keys, 16 rows 282 (4.6 TB/s)
// and 613, 32 rows 569 and 615; one of 32 rows over 30000 62 and 97; 32 of 32 rows over 500 35 and 34.  More than 32 rows would take
// four warps a ring, each converting what it reads: half the rate again, and slower than the 615.
// Rows differ in the last key they see, so a block can be hidden from a row altogether: its references may stay at the value that
// stands for none.
// NaN codes of V at keys that some rows see and others do not must reach the former and not the latter, whose weight of 0 does not
// stop them.  Those keys lie in the last three blocks at most; their codes come into shared memory beside the loop and are looked at behind
// it.  If there are any, the item is done again by a second instantiation, which takes NaN codes out of its tiles, and its rows get
// their NaN after the write-out (tc8::nan_values): 128 requests of 4 rows over 4000 keys take 213 us, 577 if all have such values.  (The same in the one loop, however it was put, cost calls without NaN 2 to 7 %: the loop
// has no register left.)
#pragma once
#include "ekv_prefill_e4m3.cuh"

namespace ekv {
namespace few8 {

static constexpr int kWarps = 8;
static constexpr int kThreads = 32 * kWarps;
static constexpr int kMaxRows = 32;
static constexpr int kMaxClusterLog = tc8::kMaxClusterLog;

template <int D>
struct Geo {
    static constexpr int kTileBytes = 16 * D;
    static constexpr int kStageBytes = 2 * kTileBytes;
    static constexpr int kStages = D == 128 ? 2 : 4;                  // of a ring of one warp; one of two warps has twice as many
    static constexpr int kOffBar = kWarps * kStages * kStageBytes;    // in front: the rings, later O of each ring's rows
    static constexpr int kOffML = kOffBar + 8 * kWarps * kStages;     // (m, l) of each ring's rows (8 x 16 or 4 x 32), then of the CTA's
    static constexpr int kCutBlocks = 3;                              // blocks that some rows see and others do not: of at most 31 keys
    static constexpr int kOffCut = kOffML + (kWarps * 16 + kMaxRows) * 8;
    static constexpr int kOffBarAgain = kOffCut + kCutBlocks * kTileBytes;
    static constexpr int kSmemBytes = kOffBarAgain + 8 * kWarps * kStages + 1024;
    static_assert(kWarps * 16 * D * 4 <= kOffBar, "merge area");
    static_assert(2 * (kSmemBytes + 1024) <= 233472, "two CTAs an SM");
};

// kTwo: 1 for rings of two warps.  kClean: the item's second time, with NaN codes taken out.  Returns whether there has to be one.
template <int D, int kTwo, bool kClean>
__device__ __forceinline__ bool few8_item(const CUtensorMap &kvmap, const tc8::Params &pp) {
    using G = Geo<D>;
    const PrefillParams &p = pp.p;
    constexpr int KSTEPS = D / 16;
    constexpr unsigned FULL = 0xffffffffu;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r = lane >> 2, c = lane & 3;
    const int cluster = pp.cluster, part = blockIdx.x % cluster, item = blockIdx.x / cluster;
    const int req = item / p.num_kv_heads, g = item - req * p.num_kv_heads;

    const int q0 = p.cu_q_lens[req], c_r = p.cu_q_lens[req + 1] - q0;
    const int group = p.group, rows = c_r * group;
    constexpr int rings = kWarps >> kTwo, stages = G::kStages << kTwo, ring_rows = 16 << kTwo;
    const int ring = warp >> kTwo, tile = warp & kTwo;  // this warp's stages, and which 16 rows it computes
    const int L = min(p.seq_lens[req], p.max_blocks * 16);
    const int prefix = L - c_r;
    auto row_offset = [&](int i) {
        const int pos = i / group;
        return ((size_t)(q0 + pos) * p.num_q_heads + (size_t)(g * group + i - pos * group)) * D;
    };
    if (prefix < 0) {  // malformed request: zero rows, latch
        if (threadIdx.x == 0) atomicOr(p.status, EKV_DEV_FLAG_OOB);
        for (int e = threadIdx.x; e < rows * (D / 8) && part == 0; e += kThreads)
            *reinterpret_cast<uint4 *>(p.out + row_offset(e / (D / 8)) + (e % (D / 8)) * 8) = make_uint4(0u, 0u, 0u, 0u);
        return false;
    }
    const int all_blocks = (L + 15) >> 4;
    const int blk0 = (int)((long long)all_blocks * part >> pp.cluster_log), blk1 = (int)((long long)all_blocks * (part + 1) >> pp.cluster_log);
    const int nw = max(0, (blk1 - blk0 - ring + rings - 1) / rings);  // blocks of this ring
    const bool busy = 16 * tile < rows;  // a warp without rows only keeps step

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_u32 = smem_u32(smem_raw);
    const uint32_t base = (raw_u32 + 1023u) & ~1023u;
    uint8_t *ptr = smem_raw + (base - raw_u32);
    const uint32_t my_stages = base + ring * stages * G::kStageBytes;
    const uint32_t my_bars = base + (kClean ? G::kOffBarAgain : G::kOffBar) + ring * stages * 8;
    const bool leads = tile == 0;  // ... the ring's other warps and issues its copies
    auto ring_sync = [&]() {
        if (kTwo) asm volatile("bar.sync %0, 64;" ::"r"(1 + ring) : "memory");
        else __syncwarp();
    };
    if (lane == 0 && leads) {
        prefetch_tensormap(&kvmap);
        for (int s = 0; s < stages; ++s) mbar_init(my_bars + 8 * s, 1);
        mbar_fence_init();
    }
    ring_sync();

    // Lane l holds the id (-1: invalid, skipped) and the scales of the ring's block 32 k + l, and of block 32 (k + 1) + l.
    const long long live = *p.live;
    const int *bt = p.block_tables + (size_t)req * p.max_blocks + blk0 + ring;
    auto load_ids = [&](int first, int &id, float &sk, float &sv) {
        const int i = first + lane;
        id = -1;
        sk = sv = 0.f;
        if (i < nw) {
            id = bt[i * rings];
            if (id < 0 || (long long)id >= live) {
                id = -1;
                if (leads) atomicOr(p.status, EKV_DEV_FLAG_OOB);
            } else {
                const float *at = pp.scales + (long long)id * 2 * p.num_kv_heads + g;
                sk = at[0];
                sv = at[p.num_kv_heads];
            }
        }
    };
    int id_a, id_b;
    float sk_a, sv_a, sk_b, sv_b;
    load_ids(0, id_a, sk_a, sv_a);
    load_ids(32, id_b, sk_b, sv_b);
    const uint64_t policy = policy_evict_first();
    auto issue = [&](int i, int i0) {  // block i of the ring, i0 = first block that id_a holds
        const int id = __shfl_sync(FULL, i - i0 < 32 ? id_a : id_b, (i - i0) & 31);
        if (lane == 0 && leads && id >= 0) {
            const int stage = i & (stages - 1);
            const uint32_t bar = my_bars + 8 * stage, dst = my_stages + stage * G::kStageBytes;
            mbar_expect_tx(bar, G::kStageBytes);
            tma_load_3d_hint(dst, &kvmap, 0, g * 16, id, bar, policy);
            tma_load_3d_hint(dst + G::kTileBytes, &kvmap, 0, (p.num_kv_heads + g) * 16, id, bar, policy);
        }
    };
    for (int s = 0; s < stages && s < nw; ++s) issue(s, 0);
    const int cut = (prefix + 1) >> 4;  // the first block that not every row sees all of
    const bool looks = !kClean && warp < G::kCutBlocks && 16 * (cut + warp) < L && c_r > 1;
    const int cut_id = looks ? p.block_tables[(size_t)req * p.max_blocks + cut + warp] : -1;
    if (looks) {  // (invalid: zeros)
        const bool valid = cut_id >= 0 && (long long)cut_id < live;
        const uint8_t *codes = pp.cache + (long long)(valid ? cut_id : 0) * pp.block_stride + (long long)(p.num_kv_heads + g) * G::kTileBytes;
#pragma unroll 1
        for (int at = lane * 16; at < G::kTileBytes; at += 512) cp_async_16(base + G::kOffCut + warp * G::kTileBytes + at, codes + at, valid ? 16u : 0u);
    }

    // Q fragments: rows r and r + 8 of the warp's tile, f16 with the row's largest magnitude in [2^13, 2^14)
    uint32_t qa[KSTEPS][4];
    float row_scale[2];
    int lim[2];  // last key the row sees; -1 for rows that do not exist
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
        const int i = 16 * tile + 8 * hi + r;
        const bool there = i < rows;
        const uint2 *src = reinterpret_cast<const uint2 *>(p.q + row_offset(there ? i : 0));
        uint2 raw[KSTEPS];
        uint32_t top = 0;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
            raw[ks] = there ? src[4 * ks + c] : make_uint2(0u, 0u);
            top = __vmaxu2(top, __vmaxu2(raw[ks].x & 0x7fff7fffu, raw[ks].y & 0x7fff7fffu));
        }
        top = max(top & 0xffffu, top >> 16);
        top = max(top, __shfl_xor_sync(FULL, top, 1));
        top = max(top, __shfl_xor_sync(FULL, top, 2));
        const float up = to_f16_range(__uint_as_float(top << 16));
        const float f = up * pp.q_sign;
        row_scale[hi] = p.scale_log2 * pow2_inverse(up);
        lim[hi] = there ? prefix + i / group : -1;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
            const __half2 a = __floats2half2_rn(__uint_as_float(raw[ks].x << 16) * f, __uint_as_float(raw[ks].x & 0xffff0000u) * f);
            const __half2 b = __floats2half2_rn(__uint_as_float(raw[ks].y << 16) * f, __uint_as_float(raw[ks].y & 0xffff0000u) * f);
            qa[ks][hi] = *reinterpret_cast<const uint32_t *>(&a);
            qa[ks][2 + hi] = *reinterpret_cast<const uint32_t *>(&b);
        }
    }

    // ldmatrix lane addressing (matrix mi = lane / 8: tokens 8 (mi >> 1) .. + 7, 16-byte chunk step + (mi & 1); the TMA swizzle
    // spans one row): chunk `step` of a tile is at (tile + lane_at) ^ (step << 4) for even steps
    const int mi = lane >> 3, lane_row = 8 * (mi >> 1) + (lane & 7);
    const uint32_t lane_at = D == 128 ? lane_row * 128 + (((mi & 1) ^ (lane_row & 7)) << 4) : lane_row * 64 + (((mi & 1) ^ ((lane_row >> 1) & 3)) << 4);

    float o[KSTEPS][2][4];  // O^T: channels x rows 8 n .. 8 n + 7 of the tile
#pragma unroll
    for (int i = 0; i < KSTEPS; ++i)
#pragma unroll
        for (int n = 0; n < 2; ++n) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.f;
    RowRef ref[2] = {{kNoRef, kNoRef, 0.f}, {kNoRef, kNoRef, 0.f}};  // of rows 8 n + r

    bool failed = false;
    uint32_t stage_parity = 0;  // advances with the copies that went through a stage (skipped blocks have none)
    int i = 0, i0 = 0;
#pragma unroll 1
    for (; i < nw; ++i) {
        if (i - i0 == 32) {
            i0 = i;
            id_a = id_b, sk_a = sk_b, sv_a = sv_b;
            load_ids(i0 + 32, id_b, sk_b, sv_b);
        }
        const int stage = i & (stages - 1);
        const int tok0 = (blk0 + ring + rings * i) * 16;
        if (__shfl_sync(FULL, id_a, i - i0) >= 0) {
            const bool got = mbar_wait(my_bars + 8 * stage, (stage_parity >> stage) & 1u, failed ? 1000000ull : 2000000000ull);
            stage_parity ^= 1u << stage;
            if (__any_sync(FULL, !got)) failed = true;  // goes on in step with the ring's other warps, but computes no more
            if (kClean && tok0 + 15 > prefix) {  // (a ring's two warps both do this, each before it reads: what they write is the same)
#pragma unroll 1
                for (int at = lane * 16; at < G::kTileBytes; at += 512) {
                    const uint32_t to = my_stages + stage * G::kStageBytes + G::kTileBytes + at;
                    sts_16(to, without_nan_codes(lds_16(to)));
                }
                fence_proxy_async_smem();  // before the stage's next copy
                __syncwarp();
            }
        }
        if (busy && !failed && __shfl_sync(FULL, id_a, i - i0) >= 0) {
            const uint32_t kbase = my_stages + stage * G::kStageBytes + lane_at, vbase = kbase + G::kTileBytes;
            const float xs = __shfl_sync(FULL, sk_a, i - i0), sv = __shfl_sync(FULL, sv_a, i - i0);
            const float e_v = scale_exponent(sv);

            float s[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) s[h][0] = s[h][1] = s[h][2] = s[h][3] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ks += 2) {
                uint32_t k[4];  // tokens 0-7: steps ks, ks + 1; tokens 8-15: the same
                ldmatrix_x4(kbase ^ (ks << 4), k[0], k[1], k[2], k[3]);
#pragma unroll
                for (int u = 0; u < 4; ++u) mma_f16(s[u >> 1], qa[ks + (u & 1)], e4m3_lo(k[u]), e4m3_hi(k[u]));
            }
            if (!(xs > 0.f)) {  // never written: the keys are 0, whatever the codes
#pragma unroll
                for (int h = 0; h < 2; ++h) s[h][0] = s[h][1] = s[h][2] = s[h][3] = 0.f;
            }
            const float f0 = row_scale[0] * xs, f1 = row_scale[1] * xs;
            if (tok0 + 15 > prefix) {  // some row does not see all of the block (or it ends here)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int t = tok0 + 8 * h + 2 * c + (e & 1);
                        s[h][e] = t > lim[e >> 1] ? -INFINITY : s[h][e] * (e < 2 ? f0 : f1);
                    }
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) s[h][0] *= f0, s[h][1] *= f0, s[h][2] *= f1, s[h][3] *= f1;
            }
            // A row's references are raised only when one of its scores is 2^8 above them: most blocks have no vote but this one.
            const float top0 = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1])), top1 = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
            if (__any_sync(FULL, top0 > fminf(ref[0].m, ref[0].M - e_v) + kLazy || top1 > fminf(ref[1].m, ref[1].M - e_v) + kLazy)) {
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    float top = n ? top1 : top0;
                    top = fmaxf(top, __shfl_xor_sync(FULL, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(FULL, top, 2));
                    const float m_new = fmaxf(ref[n].m, top), M_new = fmaxf(ref[n].M, top + e_v);
                    const float alpha = fast_exp2(ref[n].M - M_new);
                    ref[n].l *= fast_exp2(ref[n].m - m_new);
                    ref[n].m = m_new;
                    ref[n].M = M_new;
                    const float a_lo = __shfl_sync(FULL, alpha, 8 * c), a_hi = __shfl_sync(FULL, alpha, 8 * c + 4);
#pragma unroll
                    for (int mt = 0; mt < KSTEPS; ++mt) o[mt][n][0] *= a_lo, o[mt][n][1] *= a_hi, o[mt][n][2] *= a_lo, o[mt][n][3] *= a_hi;
                }
            }
            uint32_t pb[2][2];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const float m = ref[n].m, up = ref[n].p_factor(e_v);
                const float p0 = fast_exp2(s[0][2 * n] - m), p1 = fast_exp2(s[0][2 * n + 1] - m);
                const float p2 = fast_exp2(s[1][2 * n] - m), p3 = fast_exp2(s[1][2 * n + 1] - m);
                ref[n].l += (p0 + p1) + (p2 + p3);
                pb[n][0] = pack_f16x2(p0 * up, p1 * up);
                pb[n][1] = pack_f16x2(p2 * up, p3 * up);
            }
            uint32_t keep_lo = sv > 0.f ? 0xffffffffu : 0u, keep_hi = keep_lo;  // bytes of codes that count: tokens 2c in bytes 0 and 2, 2c + 1 in 1 and 3
            if (tok0 + 16 > L) {  // slots not written may hold NaN codes: 0 * NaN must not reach O
                const int t = tok0 + 2 * c;
                keep_lo &= (t < L ? 0x00ff00ffu : 0u) | (t + 1 < L ? 0xff00ff00u : 0u);
                keep_hi &= (t + 8 < L ? 0x00ff00ffu : 0u) | (t + 9 < L ? 0xff00ff00u : 0u);
            }
#pragma unroll
            for (int mt = 0; mt < KSTEPS; mt += 2) {
                uint32_t w[4];  // chunk mt: tokens 0-7, chunk mt + 1: tokens 0-7, and tokens 8-15 of both
                ldmatrix_x4_trans(vbase ^ (mt << 4), w[0], w[1], w[2], w[3]);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = __byte_perm(w[j], 0, 0x3120);  // (d 2r: tokens 2c, 2c + 1), (d 2r + 1: ...)
                w[0] &= keep_lo, w[1] &= keep_lo, w[2] &= keep_hi, w[3] &= keep_hi;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t va[4] = {e4m3_lo(w[j]), e4m3_hi(w[j]), e4m3_lo(w[j + 2]), e4m3_hi(w[j + 2])};
                    mma_f16(o[mt + j][0], va, pb[0][0], pb[0][1]);
                    mma_f16(o[mt + j][1], va, pb[1][0], pb[1][1]);
                }
            }
        }
        ring_sync();  // every warp is done reading the stage before it is refilled
        if (i + stages < nw) issue(i + stages, i0);
    }
    if (failed || !busy) {  // a copy never came: latched, contributes nothing (every copy has had its wait, so none is in flight)
        if (failed && lane == 0) atomicOr(p.status, EKV_DEV_FLAG_TIMEOUT);
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            ref[n] = {kNoRef, kNoRef, 0.f};
#pragma unroll
            for (int mt = 0; mt < KSTEPS; ++mt) o[mt][n][0] = o[mt][n][1] = o[mt][n][2] = o[mt][n][3] = 0.f;
        }
    }

    // ---- rings: (m, l, O) of each into shared memory (over the stages, once all are through), then one set for the CTA
    float2 *ml = reinterpret_cast<float2 *>(ptr + G::kOffML);  // [ring][row], then [row] of the CTA
    float *ow = reinterpret_cast<float *>(ptr);                // [ring][row][D]
    if (kClean) {
        __syncthreads();
    } else {  // all CTAs of a cluster look at the same codes, so they go on the same way
        cp_async_wait_all();
        __syncthreads();
        uint32_t nan = 0;
#pragma unroll 1
        for (int at = threadIdx.x * 16; at < G::kCutBlocks * G::kTileBytes; at += kThreads * 16) {
            const int t = 16 * cut + at / D;
            if (t <= prefix || t >= L) continue;
            const uint4 v = lds_16(base + G::kOffCut + at);
            nan |= nan_codes(v.x) | nan_codes(v.y) | nan_codes(v.z) | nan_codes(v.w);
        }
        if (__syncthreads_or((int)(nan != 0u))) return true;
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        float l = ref[n].l;
        l += __shfl_xor_sync(FULL, l, 1);
        l += __shfl_xor_sync(FULL, l, 2);
        if (c == 0) ml[ring * ring_rows + 16 * tile + 8 * n + r] = make_float2(ref[n].m, l);
        const float f = ref[n].o_factor(), f_lo = __shfl_sync(FULL, f, 8 * c), f_hi = __shfl_sync(FULL, f, 8 * c + 4);
        float *to = ow + ((size_t)ring * ring_rows + 16 * tile + 8 * n) * D + 2 * r;
#pragma unroll
        for (int mt = 0; mt < KSTEPS; ++mt) {  // row r of the fragment is channel 2r of the sixteen, row r + 8 channel 2r + 1
            *reinterpret_cast<float2 *>(to + (2 * c) * D + 16 * mt) = make_float2(o[mt][n][0] * f_lo, o[mt][n][2] * f_lo);
            *reinterpret_cast<float2 *>(to + (2 * c + 1) * D + 16 * mt) = make_float2(o[mt][n][1] * f_hi, o[mt][n][3] * f_hi);
        }
    }
    __syncthreads();
    constexpr int kQuads = D / 4;
    for (int e = threadIdx.x; e < rows * kQuads; e += kThreads) {
        const int row = e / kQuads, x = e % kQuads;
        float m = kNoRef, l = 0.f;
#pragma unroll 4
        for (int w = 0; w < rings; ++w) m = fmaxf(m, ml[w * ring_rows + row].x);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int w = 0; w < rings; ++w) {
            const float2 v = ml[w * ring_rows + row];
            const float wgt = fast_exp2(v.x - m);
            const float4 u = reinterpret_cast<const float4 *>(ow)[((size_t)w * ring_rows + row) * kQuads + x];
            l += wgt * v.y;
            acc.x += wgt * u.x, acc.y += wgt * u.y, acc.z += wgt * u.z, acc.w += wgt * u.w;
        }
        if (cluster == 1) {
            const float inv = l > 0.f ? 1.f / l : 0.f;
            *reinterpret_cast<uint2 *>(p.out + row_offset(row) + 4 * x) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
        } else {  // in place of ring 0's set: this thread alone reads and writes these four channels of it
            reinterpret_cast<float4 *>(ow)[(size_t)row * kQuads + x] = acc;
            if (x == 0) ml[rings * ring_rows + row] = make_float2(m, l);
        }
    }
    // ---- CTAs: each merges a share of the elements out of the shared memories of all of the cluster
    if (cluster > 1) cluster_barrier();
    for (int e = part * kThreads + threadIdx.x; e < rows * kQuads && cluster > 1; e += cluster * kThreads) {
        const int row = e / kQuads, x = e % kQuads;
        const uint32_t ml_at = base + G::kOffML + (rings * ring_rows + row) * 8, o_at = base + (row * kQuads + x) * 16;
        float m = kNoRef, l = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int i = 0; i < cluster; ++i) {
            const float2 v = ld_cluster_f2(map_to_cta(ml_at, i));
            const float4 u = ld_cluster_f4(map_to_cta(o_at, i));
            const float m_new = fmaxf(m, v.x), a = fast_exp2(m - m_new), b = fast_exp2(v.x - m_new);
            l = l * a + v.y * b;
            acc.x = acc.x * a + u.x * b, acc.y = acc.y * a + u.y * b, acc.z = acc.z * a + u.z * b, acc.w = acc.w * a + u.w * b;
            m = m_new;
        }
        const float inv = l > 0.f ? 1.f / l : 0.f;
        *reinterpret_cast<uint2 *>(p.out + row_offset(row) + 4 * x) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    }
    if (cluster > 1) cluster_barrier();  // nobody leaves while another may read its shared memory
    if (kClean) {
        if (cluster == 1) __syncthreads();
        tc8::nan_values<D>(pp, g, p.block_tables + (size_t)req * p.max_blocks, 16 * cut, L, warp, part == 0 ? rows : 0, kWarps, [&](int i, int &last, __nv_bfloat16 *&at) {
            last = prefix + i / group;
            at = p.out + row_offset(i);
        });
    }
    return false;
}

// Two CTAs an SM leave 128 registers a thread, and at head_dim 128 that is not enough: 420 bytes are spilled by the three instantiations of
// the item together (one CTA an SM would not spill, with half the warps to hide a block's chain).
template <int D>
__global__ void __launch_bounds__(kThreads, 2) few8_kernel(const __grid_constant__ CUtensorMap kvmap, const __grid_constant__ tc8::Params pp) {
    const int req = blockIdx.x / pp.cluster / pp.p.num_kv_heads;
    const long long rows = (long long)(pp.p.cu_q_lens[req + 1] - pp.p.cu_q_lens[req]) * pp.p.group;
    // Every reason to leave, here and in few8_item, is the same for all CTAs of a cluster.
    if (rows <= 0 || rows > kMaxRows) {}  // not one of this kernel's requests
    else if (rows > 16 ? few8_item<D, 1, false>(kvmap, pp) : few8_item<D, 0, false>(kvmap, pp)) (void)few8_item<D, 1, true>(kvmap, pp);
    // Beside the other kernel of the call, which it shares nothing with, but not through before it: what follows on the stream
    // waits for this launch alone.
    if (blockIdx.x == 0) asm volatile("griddepcontrol.wait;" ::: "memory");
}

template <int D>
static ekv_status_t launch(ekv_pool *pool, int layer, tc8::Params &pp, long long few, bool beside, cudaStream_t stream) {
    using G = Geo<D>;
    static int fits[64][kMaxClusterLog + 1] = {};  // per device: clusters of 2^i CTAs that run at the same time; [..][0] 0: not asked yet
    const int dev = pool->desc.device;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // from the tail of the launch before on, if that is the call's own
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = G::kSmemBytes;
    int asked[kMaxClusterLog + 1] = {}, *fit = dev < 64 ? fits[dev] : asked;
    if (fit[0] == 0) {
        cudaError_t e = cudaFuncSetAttribute(few8_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, G::kSmemBytes);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(few8_kernel<D>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return cuda_fail(e, "ekv_attn_prefill_chunk: kernel attributes");
        tc8::clusters_that_fit((const void *)few8_kernel<D>, cfg, fit);
    }
    // Parts: as many as let the items run at the same time, or nearly so (slack[i] quarters of that for 2^i CTAs), while a part has
    // eight blocks, one a ring, of the longest sequence that the table can hold -- 64 if the items take turns, as a cluster takes longer
    // to start than a CTA, and 128 if they take more than two.  Measured, requests of 16 rows, us with 1 / 2 / 4 / 8 / 16 CTAs an item: one
    // over 30000 keys (8 items) 292 152 83 47 38; over 1000..8000 keys 2 requests 50 31 21 20 29; 4: 65 39 25 22 42; 10: 83 48 37 48 83;
    // 16: 83 50 59 72 129; 20: 85 58 64 85 157; 48: 131 119; 64: 169 159 180 265 498; 72: 171 175; 64 over 1200..2100 67 81; 32 of 4 to 20
    // rows over 1000..4100 101 75 83 119 219; over 400 keys 1: 13 13 11 11 15, 8: 13 13 15 24 57, 32: 17 28 44 84 193.  (14 clusters of 16
    // run at a time, 33 of 8, 71 of 4, 148 of 2.)  Depends on the call's shape arguments alone.
    const long long items = few * pool->desc.num_kv_heads;  // (those of the other requests leave at once)
    static constexpr int slack[kMaxClusterLog + 1] = {0, 14, 5, 5, 4};
    int c = 0;
    while (c < kMaxClusterLog && 4ll * items <= (long long)slack[c + 1] * fit[c + 1]) {
        const long long part_blocks = items <= fit[c + 1] ? 8 : items <= 2ll * fit[c + 1] ? 64 : 128;
        if (pp.p.max_blocks < part_blocks << (c + 1)) break;
        ++c;
    }
    pp.cluster_log = c;
    pp.cluster = 1 << c;
    attr[0].val.clusterDim.x = (unsigned)pp.cluster;
    cfg.attrs = attr;
    cfg.numAttrs = beside ? 2 : 1;
    cfg.gridDim = dim3((unsigned)((long long)pp.p.R * pool->desc.num_kv_heads * pp.cluster));
    cfg.stream = stream;
    cudaError_t e = cudaLaunchKernelEx(&cfg, few8_kernel<D>, pool->kv_map[layer], (const tc8::Params &)pp);
    if (e != cudaSuccess) return cuda_fail(e, "ekv_attn_prefill_chunk: launch");
    return EKV_OK;
}

}  // namespace few8
}  // namespace ekv

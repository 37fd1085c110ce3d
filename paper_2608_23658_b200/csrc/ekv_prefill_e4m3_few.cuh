// ekv_attn_prefill_chunk over an 8-bit pool for requests of FEW query rows (drafted tokens to be checked, a decode row in a
// mixed batch): at most 64 (position, head of the group) rows per kv-head.
//
// Such a request is bound by reading its keys and values once, like decode, and the tensor instruction of 128 rows would be
// mostly empty behind a conversion of every tile into shared memory.  So this is decode's split pass (ekv_decode_e4m3.cuh has
// the fragments and why the codes get there without shuffles) with a full 16-row tile as the A operand of the scores and two 8-row
// tiles as the B operand of O^T += V^T P^T.
//   ring         NT = 1, 2 or 4 warps, one for each 16 rows, read the same TMA stages, so that a block crosses from device memory
//                once whatever the rows; each converts it for itself (sharing the conversion too would take the registers of
//                several row tiles in one warp, and with them the warps that hide its latency: two tiles a warp ran at 0.6 of this)
//   CTA          8 warps = 8 / NT rings; ring k takes every (8 / NT)-th block of the CTA's key range
//   cluster      up to 16 CTAs share a (request, kv-head)'s keys and merge (m, l, O) through distributed shared memory: the call
//                has no workspace.  Rings first, then CTAs, each in a fixed order: the same bits every time.
// Rows differ in the last key they see, so a block can be hidden from a row altogether: its running maximum may stay -inf.
#pragma once
#include "ekv_prefill_e4m3.cuh"

namespace ekv {
namespace few8 {

static constexpr int kWarps = 8;
static constexpr int kThreads = 32 * kWarps;
static constexpr int kMaxRows = 64;
static constexpr int kMaxCluster = 16;

template <int D, int NT>
struct Geo {
    static constexpr int kRows = 16 * NT;
    static constexpr int kRings = kWarps / NT;
    static constexpr int kTileBytes = 16 * D;
    static constexpr int kStageBytes = 2 * kTileBytes;
    static constexpr int kStages = (D == 128 ? 2 : 4) * NT;
    static constexpr int kOffBar = kRings * kStages * kStageBytes;    // in front: the rings, later O of each ring's rows
    static constexpr int kOffML = kOffBar + 8 * kRings * kStages;     // (m, l) of each ring's rows, then of the CTA's
    static constexpr int kSmemBytes = kOffML + (kRings + 1) * kRows * 8 + 1024;
    static_assert(kRings * kRows * D * 4 <= kOffBar && kStages <= 32, "merge area; one parity bit a stage");
    static_assert(2 * (kSmemBytes + 1024) <= 233472, "two CTAs an SM");
};

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, 2) few8_kernel(const __grid_constant__ CUtensorMap kvmap, const __grid_constant__ tc8::Params pp) {
    using G = Geo<D, NT>;
    const PrefillParams &p = pp.p;
    constexpr int KSTEPS = D / 16;
    constexpr unsigned FULL = 0xffffffffu;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r = lane >> 2, c = lane & 3;
    const int ring = warp / NT, tile = warp % NT;  // this warp's stages, and which 16 rows it computes
    const int cluster = pp.cluster, part = blockIdx.x % cluster, item = blockIdx.x / cluster;
    const int req = item / p.num_kv_heads, g = item - req * p.num_kv_heads;

    // Every reason to leave here is the same for all CTAs of the cluster.
    const int q0 = p.cu_q_lens[req], c_r = p.cu_q_lens[req + 1] - q0;
    const int group = p.group, rows = c_r * group;
    if (c_r <= 0 || rows > G::kRows) return;  // not one of this kernel's requests
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
        return;
    }
    const int all_blocks = (L + 15) >> 4;
    const int blk0 = (int)((long long)all_blocks * part / cluster), blk1 = (int)((long long)all_blocks * (part + 1) / cluster);
    const int nw = max(0, (blk1 - blk0 - ring + G::kRings - 1) / G::kRings);  // blocks of this ring
    const bool busy = 16 * tile < rows;  // a warp without rows only keeps step

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_u32 = smem_u32(smem_raw);
    const uint32_t base = (raw_u32 + 1023u) & ~1023u;
    uint8_t *ptr = smem_raw + (base - raw_u32);
    const uint32_t my_stages = base + ring * G::kStages * G::kStageBytes;
    const uint32_t my_bars = base + G::kOffBar + ring * G::kStages * 8;
    const bool leads = tile == 0;  // ... the ring's other warps and issues its copies
    auto ring_sync = [&]() {
        if (NT == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + ring), "n"(32 * NT) : "memory");
    };
    if (lane == 0 && leads) {
        prefetch_tensormap(&kvmap);
        for (int s = 0; s < G::kStages; ++s) mbar_init(my_bars + 8 * s, 1);
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
            id = bt[i * G::kRings];
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
            const int stage = i % G::kStages;
            const uint32_t bar = my_bars + 8 * stage, dst = my_stages + stage * G::kStageBytes;
            mbar_expect_tx(bar, G::kStageBytes);
            tma_load_3d_hint(dst, &kvmap, 0, g * 16, id, bar, policy);
            tma_load_3d_hint(dst + G::kTileBytes, &kvmap, 0, (p.num_kv_heads + g) * 16, id, bar, policy);
        }
    };
    for (int s = 0; s < G::kStages && s < nw; ++s) issue(s, 0);

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

    const int mi = lane >> 3, rr = lane & 7;
    const int lane_row = 8 * (mi >> 1) + rr, lane_par = mi & 1;
    auto chunk_addr = [&](uint32_t at, int chunk) {  // the TMA swizzle spans one row: 128 bytes, or 64
        if (D == 128) return at + lane_row * 128 + ((chunk ^ (lane_row & 7)) << 4);
        return at + lane_row * 64 + ((chunk ^ ((lane_row >> 1) & 3)) << 4);
    };

    float o[KSTEPS][2][4];  // O^T: channels x rows 8 n .. 8 n + 7
#pragma unroll
    for (int i = 0; i < KSTEPS; ++i)
#pragma unroll
        for (int n = 0; n < 2; ++n) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.f;
    float m_run[2], l_run[2];  // of rows 8 n + r
#pragma unroll
    for (int n = 0; n < 2; ++n) m_run[n] = -INFINITY, l_run[n] = 0.f;

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
        const int stage = i % G::kStages;
        const int tok0 = (blk0 + ring + G::kRings * i) * 16;
        if (__shfl_sync(FULL, id_a, i - i0) >= 0) {
            const bool got = mbar_wait(my_bars + 8 * stage, (stage_parity >> stage) & 1u, failed ? 1000000ull : 2000000000ull);
            stage_parity ^= 1u << stage;
            if (__any_sync(FULL, !got)) failed = true;  // goes on in step with the ring's other warps, but computes no more
        }
        if (busy && !failed && __shfl_sync(FULL, id_a, i - i0) >= 0) {
            const uint32_t kbase = my_stages + stage * G::kStageBytes, vbase = kbase + G::kTileBytes;
            const bool partial = tok0 + 15 > prefix;  // some row does not see all of the block (or it ends here)
            const float xs = __shfl_sync(FULL, sk_a, i - i0), sv = __shfl_sync(FULL, sv_a, i - i0);

            float s[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) s[h][0] = s[h][1] = s[h][2] = s[h][3] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ks += 2) {
                uint32_t k[4];  // tokens 0-7: steps ks, ks + 1; tokens 8-15: the same
                ldmatrix_x4(chunk_addr(kbase, ks + lane_par), k[0], k[1], k[2], k[3]);
#pragma unroll
                for (int u = 0; u < 4; ++u) mma_f16(s[u >> 1], qa[ks + (u & 1)], e4m3_lo(k[u]), e4m3_hi(k[u]));
            }
            uint32_t pb[2][2];
            bool rescale = false;
            float alpha[2];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const float f = row_scale[n] * xs;
                float x0 = s[0][2 * n] * f, x1 = s[0][2 * n + 1] * f, x2 = s[1][2 * n] * f, x3 = s[1][2 * n + 1] * f;
                if (partial) {
                    const int t = tok0 + 2 * c, last = lim[n];
                    if (t > last) x0 = -INFINITY;
                    if (t + 1 > last) x1 = -INFINITY;
                    if (t + 8 > last) x2 = -INFINITY;
                    if (t + 9 > last) x3 = -INFINITY;
                }
                float mx = fmaxf(fmaxf(x0, x1), fmaxf(x2, x3));
                mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, 2));
                const float m_new = fmaxf(m_run[n], mx), m_use = m_new > -INFINITY ? m_new : 0.f;
                alpha[n] = fast_exp2(m_run[n] - m_use);
                const float p0 = fast_exp2(x0 - m_use), p1 = fast_exp2(x1 - m_use), p2 = fast_exp2(x2 - m_use), p3 = fast_exp2(x3 - m_use);
                l_run[n] = l_run[n] * alpha[n] + ((p0 + p1) + (p2 + p3));
                rescale |= m_new > m_run[n];
                m_run[n] = m_new;
                pb[n][0] = pack_bf16x2(p0 * sv, p1 * sv);
                pb[n][1] = pack_bf16x2(p2 * sv, p3 * sv);
            }
            if (__any_sync(FULL, rescale)) {
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const float a_lo = __shfl_sync(FULL, alpha[n], 8 * c), a_hi = __shfl_sync(FULL, alpha[n], 8 * c + 4);
#pragma unroll
                    for (int mt = 0; mt < KSTEPS; ++mt) o[mt][n][0] *= a_lo, o[mt][n][1] *= a_hi, o[mt][n][2] *= a_lo, o[mt][n][3] *= a_hi;
                }
            }
            uint32_t mask_lo = 0xffffffffu, mask_hi = 0xffffffffu;
            if (tok0 + 16 > L) {  // slots not written may hold NaN codes: 0 * NaN must not reach O
                const int t = tok0 + 2 * c;
                mask_lo = (t < L ? 0x0000ffffu : 0u) | (t + 1 < L ? 0xffff0000u : 0u);
                mask_hi = (t + 8 < L ? 0x0000ffffu : 0u) | (t + 9 < L ? 0xffff0000u : 0u);
            }
#pragma unroll
            for (int mt = 0; mt < KSTEPS; mt += 2) {
                uint32_t w[4];  // chunk mt: tokens 0-7, chunk mt + 1: tokens 0-7, and tokens 8-15 of both
                ldmatrix_x4_trans(chunk_addr(vbase, mt + lane_par), w[0], w[1], w[2], w[3]);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = __byte_perm(w[j], 0, 0x3120);  // (d 2r: tokens 2c, 2c + 1), (d 2r + 1: ...)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t v0 = f16x2_to_bf16x2(e4m3_lo(w[j])) & mask_lo, v1 = f16x2_to_bf16x2(e4m3_hi(w[j])) & mask_lo;
                    const uint32_t v2 = f16x2_to_bf16x2(e4m3_lo(w[j + 2])) & mask_hi, v3 = f16x2_to_bf16x2(e4m3_hi(w[j + 2])) & mask_hi;
#pragma unroll
                    for (int n = 0; n < 2; ++n) mma_bf16_16816(o[mt + j][n], v0, v1, v2, v3, pb[n][0], pb[n][1]);
                }
            }
        }
        ring_sync();  // every warp is done reading the stage before it is refilled
        if (i + G::kStages < nw) issue(i + G::kStages, i0);
    }
    if (failed || !busy) {  // a copy never came: latched, contributes nothing (every copy has had its wait, so none is in flight)
        if (failed && lane == 0) atomicOr(p.status, EKV_DEV_FLAG_TIMEOUT);
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            m_run[n] = -INFINITY, l_run[n] = 0.f;
#pragma unroll
            for (int mt = 0; mt < KSTEPS; ++mt) o[mt][n][0] = o[mt][n][1] = o[mt][n][2] = o[mt][n][3] = 0.f;
        }
    }

    // ---- rings: (m, l, O) of each into shared memory (over the stages, once all are through), then one set for the CTA
    float2 *ml = reinterpret_cast<float2 *>(ptr + G::kOffML);  // [ring][row], then [row] of the CTA
    float *ow = reinterpret_cast<float *>(ptr);                // [ring][row][D]
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        l_run[n] += __shfl_xor_sync(FULL, l_run[n], 1);
        l_run[n] += __shfl_xor_sync(FULL, l_run[n], 2);
        if (c == 0) ml[ring * G::kRows + 16 * tile + 8 * n + r] = make_float2(m_run[n], l_run[n]);
        float *to = ow + ((size_t)ring * G::kRows + 16 * tile + 8 * n) * D + 2 * r;
#pragma unroll
        for (int mt = 0; mt < KSTEPS; ++mt) {  // row r of the fragment is channel 2r of the sixteen, row r + 8 channel 2r + 1
            *reinterpret_cast<float2 *>(to + (2 * c) * D + 16 * mt) = make_float2(o[mt][n][0], o[mt][n][2]);
            *reinterpret_cast<float2 *>(to + (2 * c + 1) * D + 16 * mt) = make_float2(o[mt][n][1], o[mt][n][3]);
        }
    }
    __syncthreads();
    constexpr int kQuads = D / 4;
    for (int e = threadIdx.x; e < rows * kQuads; e += kThreads) {
        const int row = e / kQuads, x = e % kQuads;
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int w = 0; w < G::kRings; ++w) m = fmaxf(m, ml[w * G::kRows + row].x);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < G::kRings; ++w) {
            const float2 v = ml[w * G::kRows + row];
            const float wgt = v.x > -INFINITY ? fast_exp2(v.x - m) : 0.f;
            const float4 u = reinterpret_cast<const float4 *>(ow)[((size_t)w * G::kRows + row) * kQuads + x];
            l += wgt * v.y;
            acc.x += wgt * u.x, acc.y += wgt * u.y, acc.z += wgt * u.z, acc.w += wgt * u.w;
        }
        if (cluster == 1) {
            const float inv = l > 0.f ? 1.f / l : 0.f;
            *reinterpret_cast<uint2 *>(p.out + row_offset(row) + 4 * x) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
        } else {  // in place of ring 0's set: this thread alone reads and writes these four channels of it
            reinterpret_cast<float4 *>(ow)[(size_t)row * kQuads + x] = acc;
            if (x == 0) ml[G::kRings * G::kRows + row] = make_float2(m, l);
        }
    }
    if (cluster == 1) return;

    // ---- CTAs: each merges a share of the elements out of the shared memories of all of the cluster
    cluster_barrier();
    for (int e = part * kThreads + threadIdx.x; e < rows * kQuads; e += cluster * kThreads) {
        const int row = e / kQuads, x = e % kQuads;
        const uint32_t ml_at = base + G::kOffML + (G::kRings * G::kRows + row) * 8, o_at = base + (row * kQuads + x) * 16;
        float m = -INFINITY, l = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int i = 0; i < cluster; ++i) {
            const float2 v = ld_cluster_f2(map_to_cta(ml_at, i));
            const float4 u = ld_cluster_f4(map_to_cta(o_at, i));
            const float m_new = fmaxf(m, v.x);
            if (m_new > -INFINITY) {
                const float a = fast_exp2(m - m_new), b = fast_exp2(v.x - m_new);
                l = l * a + v.y * b;
                acc.x = acc.x * a + u.x * b, acc.y = acc.y * a + u.y * b, acc.z = acc.z * a + u.z * b, acc.w = acc.w * a + u.w * b;
            }
            m = m_new;
        }
        const float inv = l > 0.f ? 1.f / l : 0.f;
        *reinterpret_cast<uint2 *>(p.out + row_offset(row) + 4 * x) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    }
    cluster_barrier();  // nobody leaves while another may read its shared memory
}

template <int D, int NT>
static ekv_status_t launch(ekv_pool *pool, int layer, tc8::Params &pp, int items, cudaStream_t stream) {
    using G = Geo<D, NT>;
    static int max_cluster[64] = {0};  // 0: not asked yet
    const int dev = pool->desc.device;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = G::kSmemBytes;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int most = dev < 64 ? max_cluster[dev] : 0;
    if (most == 0) {
        cudaError_t e = cudaFuncSetAttribute(few8_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, G::kSmemBytes);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(few8_kernel<D, NT>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return cuda_fail(e, "ekv_attn_prefill_chunk: kernel attributes");
        for (most = kMaxCluster; most > 8; most /= 2) {  // more than 8 is for the device to allow
            int fit = 0;
            attr.val.clusterDim.x = (unsigned)most;
            cfg.gridDim = dim3((unsigned)most);
            if (cudaOccupancyMaxActiveClusters(&fit, few8_kernel<D, NT>, &cfg) == cudaSuccess && fit > 0) break;
            (void)cudaGetLastError();
        }
        if (dev < 64) max_cluster[dev] = most;
    }
    // Parts: about two rounds of the machine, while a ring keeps two blocks of the longest sequence that the table can hold.  Depends
    // on the call's shape arguments alone.
    pp.cluster = 1;
    while (pp.cluster < most && (long long)items * pp.cluster < 4ll * pool->sm_count && pp.p.max_blocks / (2 * pp.cluster) >= 2 * G::kRings) pp.cluster *= 2;
    attr.val.clusterDim.x = (unsigned)pp.cluster;
    cfg.gridDim = dim3((unsigned)((long long)items * pp.cluster));
    cfg.stream = stream;
    cudaError_t e = cudaLaunchKernelEx(&cfg, few8_kernel<D, NT>, pool->kv_map[layer], (const tc8::Params &)pp);
    if (e != cudaSuccess) return cuda_fail(e, "ekv_attn_prefill_chunk: launch");
    return EKV_OK;
}

}  // namespace few8
}  // namespace ekv

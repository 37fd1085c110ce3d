// ekv_attn_decode's split pass over an 8-bit pool (the combine pass is the bf16 pool's).
//
//   S[head, t] = s_K(block of t) * (Q . code_K[t]),   O^T[d, head] += code_V[t, d] * (P[head, t] * s_V(block of t))
//
// The plan, the key ranges, the four warps with rings of TMA stages and the merge are those of decode_split_kernel; a block's
// K and V tiles are 16 x head_dim BYTES here.  What differs is the way from a code to a tensor operand:
//   - ldmatrix moves 16-bit units, so one 8x8 matrix is 8 tokens x 16 codes, and a lane gets four neighbouring codes of one
//     token.  The order of channels inside a dot product is free: codes (4c, 4c+1) stand for the columns (2c, 2c+1) of the
//     B fragment and (4c+2, 4c+3) for (2c+8, 2c+9), and Q is loaded in the same order.  No shuffles.
//   - ldmatrix.trans gives V's codes as (token 2c: d 2r, 2r+1; token 2c+1: d 2r, 2r+1): one byte permute makes the pairs
//     (d 2r; tokens 2c, 2c+1) and (d 2r+1; ...), i.e. rows r and r+8 of the A fragment with channels 2r and 2r+1 in them.
//   - Codes convert in pairs to f16, exactly, and K is used as f16.  Q becomes f16 too: a row is first brought to a
//     maximum in [2^13, 2^14) by a power of two (undone with the scale of the scores), so bf16's 8 bits fit, and
//     what falls below 2^-24 there is 2^-37 of the row's largest element, less than the fp32 sum resolves.
//   - V goes on to bf16 (exact as well): P takes the block's s_V before its rounding, and only bf16 has the range for
//     that.  Scaling by a power of two does not change what P's rounding loses.
#pragma once
#include "e4m3.cuh"
#include "ekv_internal.h"
#include "ptx.cuh"

namespace ekv {

// Four CTAs share an SM, with rings of 4 to 8 KiB a warp (64 to 128 KiB in flight per SM).  The bf16 kernel's two CTAs with
// rings three times as deep leave this kernel at 0.72 of the copy rate: converting makes a block's chain of instructions long,
// and it takes four warps a scheduler to hide it (256 sequences of 2048..8192 keys, 32q/8kv: 2 CTAs x 6 stages 540 us, 3 x 4
// 429, 4 x 3 416, 4 x 2 411, 5 x 2 427, 6 x 2 505 -- registers are spilled from 5 on).
static constexpr int kDecode8Ctas = 4;
template <int D>
constexpr int kDecode8Stages = D == 128 ? 2 : 4;

__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int D>
__global__ void __launch_bounds__(kDecodeWarps * 32, kDecode8Ctas)
decode8_split_kernel(const __grid_constant__ CUtensorMap kvmap, const DecodeParams p, const float *__restrict__ scales) {
    constexpr int STAGES = kDecode8Stages<D>;
    constexpr int TILE_BYTES = 16 * D;  // 16 tokens of K (or V) of one head
    constexpr int STAGE_BYTES = 2 * TILE_BYTES;
    constexpr int KSTEPS = D / 16;
    constexpr unsigned FULL = 0xffffffffu;

    const int split = blockIdx.x, g = blockIdx.y, b = blockIdx.z;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r = lane >> 2, c = lane & 3;

    int L = p.seq_lens[b];
    L = max(0, min(L, p.max_blocks * 16));
    const int t_begin = split * p.chunk_tokens;
    if (t_begin >= L) {  // whole CTA leaves before any barrier exists
        if (p.nsplit == 1)  // no combine pass will run: an empty sequence gets its zero rows here
            for (int e = threadIdx.x; e < p.group * D; e += kDecodeWarps * 32)
                p.out[((size_t)b * p.num_q_heads + (size_t)g * p.group) * D + e] = __float2bfloat16_rn(0.f);
        return;
    }
    const int t_end = min(L, t_begin + p.chunk_tokens);
    const int nblk = (t_end - t_begin + 15) >> 4;
    const int nw = max(0, (nblk - warp + kDecodeWarps - 1) / kDecodeWarps);  // blocks this warp owns (<= 32)

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_u32 = smem_u32(smem_raw);
    const uint32_t base_u32 = (raw_u32 + 1023u) & ~1023u;
    uint8_t *base_ptr = smem_raw + (base_u32 - raw_u32);
    const uint32_t my_stages = base_u32 + warp * STAGES * STAGE_BYTES;
    const uint32_t my_bars = base_u32 + kDecodeWarps * STAGES * STAGE_BYTES + warp * STAGES * 8;

    if (lane == 0) {
        prefetch_tensormap(&kvmap);
        for (int s = 0; s < STAGES; ++s) mbar_init(my_bars + 8 * s, 1);
        mbar_fence_init();
    }
    __syncwarp();

    // Block ids of this warp's blocks: lane i holds the id of its i-th block, and the scales of its K and V tile.
    const long long live = *p.live;
    const int *bt = p.block_tables + (size_t)b * p.max_blocks + (t_begin >> 4) + warp;
    const int my_id = (lane < nw) ? bt[lane * kDecodeWarps] : 0;
    const bool my_ok = (lane < nw) && my_id >= 0 && (long long)my_id < live;
    const unsigned valid_mask = __ballot_sync(FULL, my_ok);
    if (lane < nw && !my_ok) atomicOr(p.status, EKV_DEV_FLAG_OOB);

    const uint64_t policy = policy_evict_first();
    auto issue = [&](int i) {
        const int id = __shfl_sync(FULL, my_id, i);
        if (lane == 0 && ((valid_mask >> i) & 1u)) {
            const int stage = i % STAGES;
            const uint32_t bar = my_bars + 8 * stage;
            const uint32_t dst = my_stages + stage * STAGE_BYTES;
            mbar_expect_tx(bar, STAGE_BYTES);
            tma_load_3d_hint(dst, &kvmap, 0, g * 16, id, bar, policy);
            tma_load_3d_hint(dst + TILE_BYTES, &kvmap, 0, (p.num_kv_heads + g) * 16, id, bar, policy);
        }
    };
    for (int s = 0; s < STAGES && s < nw; ++s) issue(s);
    float my_sk = 0.f, my_sv = 0.f;
    if (my_ok) {
        const float *at = scales + (size_t)my_id * 2 * p.num_kv_heads + g;
        my_sk = at[0];
        my_sv = at[p.num_kv_heads];
    }

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the combine pass may take its place on the SMs (and waits there)

    // Q fragments (A operand, f16): rows = heads of the group (r < group), zero above; channels in the order of K's codes.
    uint32_t qa[KSTEPS][2];
    float score_scale;
    {
        const uint2 *qrow = reinterpret_cast<const uint2 *>(p.q + ((size_t)b * p.num_q_heads + (size_t)g * p.group + r) * D);
        uint2 raw[KSTEPS];
        uint32_t top = 0;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
            raw[ks] = (r < p.group) ? qrow[4 * ks + c] : make_uint2(0u, 0u);
            top = __vmaxu2(top, __vmaxu2(raw[ks].x & 0x7fff7fffu, raw[ks].y & 0x7fff7fffu));
        }
        top = max(top & 0xffffu, top >> 16);
        top = max(top, __shfl_xor_sync(FULL, top, 1));
        top = max(top, __shfl_xor_sync(FULL, top, 2));
        const float up = to_f16_range(__uint_as_float(top << 16));
        score_scale = p.scale_log2 * pow2_inverse(up);
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
            const __half2 lo = __floats2half2_rn(__uint_as_float(raw[ks].x << 16) * up, __uint_as_float(raw[ks].x & 0xffff0000u) * up);
            const __half2 hi = __floats2half2_rn(__uint_as_float(raw[ks].y << 16) * up, __uint_as_float(raw[ks].y & 0xffff0000u) * up);
            qa[ks][0] = *reinterpret_cast<const uint32_t *>(&lo);
            qa[ks][1] = *reinterpret_cast<const uint32_t *>(&hi);
        }
    }

    // ldmatrix lane addressing: matrix mi = lane/8 is (tokens 8*(mi>>1)..+7) x (16-byte chunk 2*step + (mi&1)), row rr = lane%8
    const int mi = lane >> 3, rr = lane & 7;
    const int lane_row = 8 * (mi >> 1) + rr;
    const int lane_par = mi & 1;
    auto chunk_addr = [&](uint32_t tile, int chunk) {  // the TMA swizzle spans one row: 128 bytes, or 64
        if (D == 128) return tile + lane_row * 128 + ((chunk ^ (lane_row & 7)) << 4);
        return tile + lane_row * 64 + ((chunk ^ ((lane_row >> 1) & 3)) << 4);
    };

    float o[KSTEPS][4];
#pragma unroll
    for (int mt = 0; mt < KSTEPS; ++mt) o[mt][0] = o[mt][1] = o[mt][2] = o[mt][3] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    bool failed = false;

    // Phase parity per stage.  A skipped (invalid) block neither issues a copy nor waits, so the parity of a
    // stage advances only with the copies that really went through it, not with the iteration count.
    uint32_t stage_parity = 0;
    int i = 0;
    for (; i < nw; ++i) {
        const int stage = i % STAGES;
        if ((valid_mask >> i) & 1u) {
            const bool got = mbar_wait(my_bars + 8 * stage, (stage_parity >> stage) & 1u);
            stage_parity ^= 1u << stage;
            if (__any_sync(FULL, !got)) {
                failed = true;
                break;
            }
            const uint32_t kbase = my_stages + stage * STAGE_BYTES;
            const uint32_t vbase = kbase + TILE_BYTES;
            const int tok0 = t_begin + (warp + kDecodeWarps * i) * 16;
            const bool partial = tok0 + 16 > L;
            const float xs = score_scale * __shfl_sync(FULL, my_sk, i);
            const float sv = __shfl_sync(FULL, my_sv, i);

            float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ks += 2) {
                uint32_t k0, k1, k2, k3;  // tokens 0-7: steps ks, ks+1; tokens 8-15: steps ks, ks+1
                ldmatrix_x4(chunk_addr(kbase, ks + lane_par), k0, k1, k2, k3);
                mma_f16_16816(s0, qa[ks][0], 0u, qa[ks][1], 0u, e4m3_lo(k0), e4m3_hi(k0));
                mma_f16_16816(s1, qa[ks][0], 0u, qa[ks][1], 0u, e4m3_lo(k2), e4m3_hi(k2));
                mma_f16_16816(s0, qa[ks + 1][0], 0u, qa[ks + 1][1], 0u, e4m3_lo(k1), e4m3_hi(k1));
                mma_f16_16816(s1, qa[ks + 1][0], 0u, qa[ks + 1][1], 0u, e4m3_lo(k3), e4m3_hi(k3));
            }
            float x0 = s0[0] * xs, x1 = s0[1] * xs;
            float x2 = s1[0] * xs, x3 = s1[1] * xs;
            uint32_t mask_lo = 0xffffffffu, mask_hi = 0xffffffffu;
            if (partial) {
                const int t = tok0 + 2 * c;
                if (t >= L) x0 = -INFINITY;
                if (t + 1 >= L) x1 = -INFINITY;
                if (t + 8 >= L) x2 = -INFINITY;
                if (t + 9 >= L) x3 = -INFINITY;
                mask_lo = (t < L ? 0x0000ffffu : 0u) | (t + 1 < L ? 0xffff0000u : 0u);
                mask_hi = (t + 8 < L ? 0x0000ffffu : 0u) | (t + 9 < L ? 0xffff0000u : 0u);
            }
            float mx = fmaxf(fmaxf(x0, x1), fmaxf(x2, x3));
            mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, 2));
            const float m_new = fmaxf(m_run, mx);  // finite: token tok0 < L is never masked
            const float alpha = fast_exp2(m_run - m_new);
            const float p0 = fast_exp2(x0 - m_new), p1 = fast_exp2(x1 - m_new);
            const float p2 = fast_exp2(x2 - m_new), p3 = fast_exp2(x3 - m_new);
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
            const uint32_t pb0 = pack_bf16x2(p0 * sv, p1 * sv), pb1 = pack_bf16x2(p2 * sv, p3 * sv);
#pragma unroll
            for (int mt = 0; mt < KSTEPS; mt += 2) {
                uint32_t w[4];  // chunk mt: tokens 0-7, chunk mt+1: tokens 0-7, and tokens 8-15 of both
                ldmatrix_x4_trans(chunk_addr(vbase, mt + lane_par), w[0], w[1], w[2], w[3]);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = __byte_perm(w[j], 0, 0x3120);  // (d 2r: tokens 2c, 2c+1), (d 2r+1: ...)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uint32_t v0 = f16x2_to_bf16x2(e4m3_lo(w[j])), v1 = f16x2_to_bf16x2(e4m3_hi(w[j]));
                    uint32_t v2 = f16x2_to_bf16x2(e4m3_lo(w[j + 2])), v3 = f16x2_to_bf16x2(e4m3_hi(w[j + 2]));
                    if (partial) {  // slots not written may hold NaN codes: 0 * NaN must not reach O
                        v0 &= mask_lo;
                        v1 &= mask_lo;
                        v2 &= mask_hi;
                        v3 &= mask_hi;
                    }
                    mma_bf16_16816(o[mt + j], v0, v1, v2, v3, pb0, pb1);
                }
            }
        }
        __syncwarp();  // every lane is done reading the stage before it is refilled
        if (i + STAGES < nw) issue(i + STAGES);
    }

    if (failed) {
        // A copy barrier never completed.  Latch the error, give copies still in flight a bounded
        // chance to land (their destination must stay allocated), and contribute nothing.
        if (lane == 0) atomicOr(p.status, EKV_DEV_FLAG_TIMEOUT);
        stage_parity ^= 1u << (i % STAGES);  // the wait that failed belongs to a copy still outstanding
        for (int j = i; j < nw && j < i + STAGES; ++j)
            if ((valid_mask >> j) & 1u)
                (void)mbar_wait(my_bars + 8 * (j % STAGES), (stage_parity >> (j % STAGES)) & 1u, 200000000ull);
        m_run = -INFINITY;
        l_run = 0.f;
#pragma unroll
        for (int mt = 0; mt < KSTEPS; ++mt) o[mt][0] = o[mt][1] = o[mt][2] = o[mt][3] = 0.f;
    }

    l_run += __shfl_xor_sync(FULL, l_run, 1);
    l_run += __shfl_xor_sync(FULL, l_run, 2);

    // Merge the 4 warps through shared memory (each warp reuses its own, now idle, stages).
    float *wo = reinterpret_cast<float *>(base_ptr + warp * STAGES * STAGE_BYTES);  // [8][D]
    float *wm = wo + 8 * D;                                                                 // [8] m, [8] l
    static_assert((8 * D + 16) * 4 <= STAGES * STAGE_BYTES, "merge area");
#pragma unroll
    for (int mt = 0; mt < KSTEPS; ++mt) {  // row r of the fragment is channel 2r of the sixteen, row r+8 channel 2r+1
        *reinterpret_cast<float2 *>(wo + (2 * c) * D + 16 * mt + 2 * r) = make_float2(o[mt][0], o[mt][2]);
        *reinterpret_cast<float2 *>(wo + (2 * c + 1) * D + 16 * mt + 2 * r) = make_float2(o[mt][1], o[mt][3]);
    }
    if (c == 0) {
        wm[r] = m_run;
        wm[8 + r] = l_run;
    }
    __syncthreads();

    for (int e = threadIdx.x; e < p.group * D; e += kDecodeWarps * 32) {
        const int h = e / D, x = e % D;
        float mw[kDecodeWarps], mstar = -INFINITY;
#pragma unroll
        for (int w = 0; w < kDecodeWarps; ++w) {
            mw[w] = reinterpret_cast<const float *>(base_ptr + w * STAGES * STAGE_BYTES)[8 * D + h];
            mstar = fmaxf(mstar, mw[w]);
        }
        float acc = 0.f, lsum = 0.f;
        if (mstar > -INFINITY) {
#pragma unroll
            for (int w = 0; w < kDecodeWarps; ++w) {
                const float *src = reinterpret_cast<const float *>(base_ptr + w * STAGES * STAGE_BYTES);
                const float wgt = (mw[w] > -INFINITY) ? fast_exp2(mw[w] - mstar) : 0.f;
                acc += wgt * src[h * D + x];
                lsum += wgt * src[8 * D + 8 + h];
            }
        }
        const size_t slot = ((size_t)b * p.num_q_heads + (size_t)g * p.group + h) * p.nsplit + split;
        if (p.nsplit == 1) {  // the only split of every sequence: finish here, no partials, no combine pass
            p.out[slot * D + x] = __float2bfloat16_rn(lsum > 0.f ? acc / lsum : 0.f);
        } else {
            p.part_o[slot * D + x] = acc;
            if (x == 0) p.part_ml[slot] = make_float2(mstar, lsum);
        }
    }
}

}  // namespace ekv

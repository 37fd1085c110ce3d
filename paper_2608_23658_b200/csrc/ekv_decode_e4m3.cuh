// ekv_attn_decode's split pass over an 8-bit pool (the combine pass is the bf16 pool's).
//
//   S[head, t] = s_K(block of t) * (Q . code_K[t]),   O^T[d, head] += code_V[t, d] * P[head, t],   P = 2^(scale log2(e) S + e_V(block of t) - M)
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
//   - V is used as f16 as well, and its scale goes into the exponent of P (e4m3.cuh has how, and what f16 keeps of P).
#pragma once
#include "e4m3.cuh"
#include "ekv_internal.h"
#include "ptx.cuh"

namespace ekv {

// Four CTAs share an SM, with rings of 4 to 8 KiB a warp (64 to 128 KiB in flight per SM).  The bf16 kernel's two CTAs with
// rings three times as deep leave this kernel at 0.87 of the copy rate: converting makes a block's chain of instructions long,
// and it takes three or four warps a scheduler to hide it.  Measured on one machine and one set of inputs (others: 404 to 449 for
// the 399), us: 256 sequences of 2048..8192 keys, 32q/8kv, d128 (2.68 GB; at
// the copy rate 411) 2 CTAs x 6 stages 458, 3 x 4 399, 4 x 3 400, 4 x 2 399 = 6.7 TB/s, 5 x 2 416 (registers are spilled from 5 on);
// 64 sequences of 8000..30000, 16q/2kv, d64 (0.33 GB) 101, 83, 92, 77, 83.
static constexpr int kDecode8Ctas = 4;
template <int D>
constexpr int kDecode8Stages = D == 128 ? 2 : 4;

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
    uint32_t qa[KSTEPS][4];
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
            qa[ks][2] = *reinterpret_cast<const uint32_t *>(&hi);
            qa[ks][1] = qa[ks][3] = 0u;  // rows 8-15
        }
    }

    // ldmatrix lane addressing (matrix mi = lane / 8: tokens 8 (mi >> 1) .. + 7, 16-byte chunk step + (mi & 1); the TMA swizzle
    // spans one row, 128 bytes or 64): chunk `step` of a tile is at (tile + lane_at) ^ (step << 4) for even steps
    const int mi = lane >> 3, lane_row = 8 * (mi >> 1) + (lane & 7);
    const uint32_t lane_at = D == 128 ? lane_row * 128 + (((mi & 1) ^ (lane_row & 7)) << 4) : lane_row * 64 + (((mi & 1) ^ ((lane_row >> 1) & 3)) << 4);

    float o[KSTEPS][4];
#pragma unroll
    for (int mt = 0; mt < KSTEPS; ++mt) o[mt][0] = o[mt][1] = o[mt][2] = o[mt][3] = 0.f;
    RowRef ref = {kNoRef, kNoRef, 0.f};  // of head r
    bool failed = false;

    // Phase parity per stage.  A skipped (invalid) block neither issues a copy nor waits, so the parity of a
    // stage advances only with the copies that really went through it, not with the iteration count.
    uint32_t stage_parity = 0;
    int i = 0;
#pragma unroll 1
    for (; i < nw; ++i) {
        const int stage = i % STAGES;
        if ((valid_mask >> i) & 1u) {
            const bool got = mbar_wait(my_bars + 8 * stage, (stage_parity >> stage) & 1u);
            stage_parity ^= 1u << stage;
            if (__any_sync(FULL, !got)) {
                failed = true;
                break;
            }
            const uint32_t kbase = my_stages + stage * STAGE_BYTES + lane_at, vbase = kbase + TILE_BYTES;
            const int tok0 = t_begin + (warp + kDecodeWarps * i) * 16;
            const bool partial = tok0 + 16 > L;
            const float xs = __shfl_sync(FULL, my_sk, i), sv = __shfl_sync(FULL, my_sv, i);
            const float e_v = scale_exponent(sv);

            float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ks += 2) {
                uint32_t k0, k1, k2, k3;  // tokens 0-7: steps ks, ks+1; tokens 8-15: steps ks, ks+1
                ldmatrix_x4(kbase ^ (ks << 4), k0, k1, k2, k3);
                mma_f16(s0, qa[ks], e4m3_lo(k0), e4m3_hi(k0));
                mma_f16(s1, qa[ks], e4m3_lo(k2), e4m3_hi(k2));
                mma_f16(s0, qa[ks + 1], e4m3_lo(k1), e4m3_hi(k1));
                mma_f16(s1, qa[ks + 1], e4m3_lo(k3), e4m3_hi(k3));
            }
            if (!(xs > 0.f)) s0[0] = s0[1] = s1[0] = s1[1] = 0.f;  // never written: the keys are 0, whatever the codes
            const float f = score_scale * xs;
            float x0 = s0[0] * f, x1 = s0[1] * f, x2 = s1[0] * f, x3 = s1[1] * f;
            uint32_t keep_lo = sv > 0.f ? 0xffffffffu : 0u, keep_hi = keep_lo;  // bytes of codes that count: tokens 2c in bytes 0 and 2, 2c + 1 in 1 and 3
            if (partial) {
                const int t = tok0 + 2 * c;
                if (t >= L) x0 = -INFINITY;
                if (t + 1 >= L) x1 = -INFINITY;
                if (t + 8 >= L) x2 = -INFINITY;
                if (t + 9 >= L) x3 = -INFINITY;
                // slots not written may hold NaN codes: 0 * NaN must not reach O
                keep_lo &= (t < L ? 0x00ff00ffu : 0u) | (t + 1 < L ? 0xff00ff00u : 0u);
                keep_hi &= (t + 8 < L ? 0x00ff00ffu : 0u) | (t + 9 < L ? 0xff00ff00u : 0u);
            }
            // the references are raised only when a score is 2^8 above one of them: most blocks take no vote but this one
            float top = fmaxf(fmaxf(x0, x1), fmaxf(x2, x3));
            if (__any_sync(FULL, top > fminf(ref.m, ref.M - e_v) + kLazy)) {
                top = fmaxf(top, __shfl_xor_sync(FULL, top, 1));
                top = fmaxf(top, __shfl_xor_sync(FULL, top, 2));
                const float m_new = fmaxf(ref.m, top), M_new = fmaxf(ref.M, top + e_v), alpha = fast_exp2(ref.M - M_new);
                ref.l *= fast_exp2(ref.m - m_new);
                ref.m = m_new;
                ref.M = M_new;
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
            const float up = ref.p_factor(e_v);
            const float p0 = fast_exp2(x0 - ref.m), p1 = fast_exp2(x1 - ref.m), p2 = fast_exp2(x2 - ref.m), p3 = fast_exp2(x3 - ref.m);
            ref.l += (p0 + p1) + (p2 + p3);
            const uint32_t pb0 = pack_f16x2(p0 * up, p1 * up), pb1 = pack_f16x2(p2 * up, p3 * up);
#pragma unroll
            for (int mt = 0; mt < KSTEPS; mt += 2) {
                uint32_t w[4];  // chunk mt: tokens 0-7, chunk mt+1: tokens 0-7, and tokens 8-15 of both
                ldmatrix_x4_trans(vbase ^ (mt << 4), w[0], w[1], w[2], w[3]);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = __byte_perm(w[j], 0, 0x3120);  // (d 2r: tokens 2c, 2c+1), (d 2r+1: ...)
                w[0] &= keep_lo, w[1] &= keep_lo, w[2] &= keep_hi, w[3] &= keep_hi;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t va[4] = {e4m3_lo(w[j]), e4m3_hi(w[j]), e4m3_lo(w[j + 2]), e4m3_hi(w[j + 2])};
                    mma_f16(o[mt + j], va, pb0, pb1);
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
        ref = {kNoRef, kNoRef, 0.f};
#pragma unroll
        for (int mt = 0; mt < KSTEPS; ++mt) o[mt][0] = o[mt][1] = o[mt][2] = o[mt][3] = 0.f;
    }

    ref.l += __shfl_xor_sync(FULL, ref.l, 1);
    ref.l += __shfl_xor_sync(FULL, ref.l, 2);
    const float f = ref.o_factor(), f_lo = __shfl_sync(FULL, f, 8 * c), f_hi = __shfl_sync(FULL, f, 8 * c + 4);

    // Merge the 4 warps through shared memory (each warp reuses its own, now idle, stages).
    float *wo = reinterpret_cast<float *>(base_ptr + warp * STAGES * STAGE_BYTES);  // [8][D]
    float *wm = wo + 8 * D;                                                                 // [8] m, [8] l
    static_assert((8 * D + 16) * 4 <= STAGES * STAGE_BYTES, "merge area");
#pragma unroll
    for (int mt = 0; mt < KSTEPS; ++mt) {  // row r of the fragment is channel 2r of the sixteen, row r+8 channel 2r+1
        *reinterpret_cast<float2 *>(wo + (2 * c) * D + 16 * mt + 2 * r) = make_float2(o[mt][0] * f_lo, o[mt][2] * f_lo);
        *reinterpret_cast<float2 *>(wo + (2 * c + 1) * D + 16 * mt + 2 * r) = make_float2(o[mt][1] * f_hi, o[mt][3] * f_hi);
    }
    if (c == 0) {
        wm[r] = ref.m;
        wm[8 + r] = ref.l;
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
#pragma unroll
        for (int w = 0; w < kDecodeWarps; ++w) {  // (a warp without keys has kNoRef and zeros)
            const float *src = reinterpret_cast<const float *>(base_ptr + w * STAGES * STAGE_BYTES);
            const float wgt = fast_exp2(mw[w] - mstar);
            acc += wgt * src[h * D + x];
            lsum += wgt * src[8 * D + 8 + h];
        }
        const size_t slot = ((size_t)b * p.num_q_heads + (size_t)g * p.group + h) * p.nsplit + split;
        if (p.nsplit == 1) {  // the only split of every sequence: finish here, no partials, no combine pass
            p.out[slot * D + x] = __float2bfloat16_rn(finish_row(acc, lsum));
        } else {
            p.part_o[slot * D + x] = acc;
            if (x == 0) p.part_ml[slot] = make_float2(mstar, lsum);
        }
    }
}

}  // namespace ekv

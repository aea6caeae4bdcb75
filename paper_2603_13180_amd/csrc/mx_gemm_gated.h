// mx_gemm_gated.h -- the output of the gated product: H = act(G) U from a
// wave's gate products G and up products U (mx_gemm.h describes the tile), as
// float, bf16 or MX codes, and the products themselves where a backward pass
// will need them.
//
// In accumulator layout lane (g, qd) of tile i holds row qd, columns 16 i + 4 g
// .. + 3, and a wave holds 32 output columns: the two tiles of a row are one MX
// block over four lanes, so its absmax is two lane swaps away and nothing
// passes through LDS.
#pragma once

#include "gate.h"
#include "mx_gemm.h"
#include "norm_cast.h"

namespace mxg {

// The tiles v0, v1 of one row group as 32 bf16 columns: as in store_tile, lane
// row g stores 8 adjacent columns of tile g & 1 from column 8 (g >> 1), a row 64
// bytes.  Where those straddle two lines of 64 (N not a multiple of 32) the
// stores must meet their neighbours' in the caches: 3793 x 13872 x 1024, E4M3
// 122 us by ordinary stores and 157 past the caches, with gate and up 210 and
// 302; but at 13856 columns 122 and 119, 197 and 157.
__device__ __forceinline__ void store_row_bf16(__amdgpu_buffer_rsrc_t rs, const v4f &v0, const v4f &v1,
                                               uint32_t off, bool in, bool lines)
{
    const auto sl = __builtin_amdgcn_permlane16_swap(pack_bf16(v0[0], v0[1]), pack_bf16(v1[0], v1[1]),
                                                     false, false);
    const auto sh = __builtin_amdgcn_permlane16_swap(pack_bf16(v0[2], v0[3]), pack_bf16(v1[2], v1[3]),
                                                     false, false);
    const u32x4 v = {sl[0], sh[0], sl[1], sh[1]};
    if (in) {
        if (lines)
            __builtin_amdgcn_raw_buffer_store_b128(v, rs, (int)off, 0, kStorePolicy);
        else
            __builtin_amdgcn_raw_buffer_store_b128(v, rs, (int)off, 0, 0);
    }
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(void *p, int64_t byte)
{
    return __builtin_amdgcn_make_buffer_rsrc(static_cast<uint8_t *>(p) + byte, 0, 0x7FFFFFFF, 0x00020000);
}

// The codes of two row groups from mr as gated_rows leaves them: lane rows 0 and
// 1 store 16 columns each of the first group's rows, lane rows 2 and 3 of the
// second's.  One row group at a time, 8 columns a lane: E2M1 [8192, 14336] over
// K 4096 500 us instead of 491, with gate and up 580 instead of 551.
// Ordinary stores, since a product reads the codes next; beside gate and up,
// five times their size in E4M3, the codes would lose their place in the caches
// anyway, and non-temporal stores make [8192, 14336] 874 us instead of 926,
// [16384, 14336] 1743 instead of 2031 (E2M1: 551 instead of 513 for the codes
// alone, so ordinary).
template <int ELEM>
__device__ __forceinline__ void store_codes(const GatedArgs &A, const uint32_t (&c0)[2],
                                            const uint32_t (&c1)[2], int64_t mr, int64_t nc, int g, int qd)
{
    const int r = 16 * (g >> 1) + qd;
    const int64_t n = nc + 16 * (g & 1);
    const bool in = mr + r < A.M && n < A.N;
    const uint32_t off = (uint32_t)(r * A.N + n);
    const auto x = __builtin_amdgcn_permlane32_swap(c0[0], c1[0], false, false);
    if constexpr (ELEM == MX_ELEM_E4M3) {
        const auto y = __builtin_amdgcn_permlane32_swap(c0[1], c1[1], false, false);
        const __amdgpu_buffer_rsrc_t rs = rows_rsrc(A.out, mr * A.N);
        const u32x4 v = {x[0], y[0], x[1], y[1]};
        if (in) {
            if (A.gu)
                __builtin_amdgcn_raw_buffer_store_b128(v, rs, (int)off, 0, mxk::kBufNT);
            else
                __builtin_amdgcn_raw_buffer_store_b128(v, rs, (int)off, 0, 0);
        }
    } else {
        if (in)
            __builtin_amdgcn_raw_buffer_store_b64(mxk::u32x2_t{x[0], x[1]},
                                                  rows_rsrc(A.out, mr * (A.N / 2)), (int)(off / 2), 0, 0);
    }
}

// 16 rows from mr, 32 output columns from nc: gate products p[0], p[1], up
// products p[2], p[3].  MX_OUT_CODES: returns the block's E8M0 byte, the same in
// the four lanes of a row, and in `codes` the codes of this lane's 8 columns
// (E2M1: in codes[0]); the other outputs are stored.
template <int ELEM, int OUT, int ACT>
__device__ __forceinline__ uint32_t gated_rows(const GatedArgs &A, const v4f (&p)[4], int64_t mr,
                                               int64_t nc, int g, int qd, uint32_t (&codes)[2])
{
    constexpr int O = OUT - kGate;
    const bool lines = O == MX_OUT_CODES || A.N % 32 == 0;
    const bool row = mr + qd < A.M;
    const int64_t n8 = nc + 16 * (g & 1) + 8 * (g >> 1); // this lane's 8 columns
    const bool in8 = row && n8 < A.N;                    // N is a multiple of 16
    if (A.gu) {
        const __amdgpu_buffer_rsrc_t rs = rows_rsrc(A.gu, mr * A.N * 4);
        const uint32_t off = (uint32_t)(qd * A.N) * 4 + (uint32_t)n8 * 2;
        store_row_bf16(rs, p[0], p[1], off, in8, lines);
        store_row_bf16(rs, p[2], p[3], off + (uint32_t)A.N * 2, in8, lines);
    }
    v4f h[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            h[i][e] = p[i][e] * mxk::gate_sigma<ACT>(p[i][e]) * p[i + 2][e];

    if constexpr (O == MX_OUT_F32) {
        const __amdgpu_buffer_rsrc_t rs = rows_rsrc(A.out, mr * A.N * 4);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t n = nc + 16 * i + 4 * g;
            if (row && n < A.N)
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, h[i]), rs,
                                                       (int)((uint32_t)(qd * A.N + n) * 4), 0,
                                                       kStorePolicy);
        }
        return 0;
    } else if constexpr (O == MX_OUT_BF16) {
        store_row_bf16(rows_rsrc(A.out, mr * A.N * 2), h[0], h[1], (uint32_t)(qd * A.N + n8) * 2, in8, lines);
        return 0;
    } else {
        // The MX cast of the float values (no rounding to bf16 in between).
        // The block's absmax as the integer maximum of the magnitudes (NaN
        // above infinity): a lane's 8 values, then lanes 16 and 32 away.
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                m = max(m, __float_as_uint(h[i][e]) & 0x7FFFFFFFu);
        const auto m16 = __builtin_amdgcn_permlane16_swap(m, m, false, false);
        m = max(m16[0], m16[1]);
        const auto m32 = __builtin_amdgcn_permlane32_swap(m, m, false, false);
        m = max(m32[0], m32[1]);
        const float a = __uint_as_float(m);
        uint32_t q[2];
        uint32_t byte;
        if constexpr (ELEM == MX_ELEM_E4M3) {
            byte = mxk::e8m0_byte<false>(a, A.mode);
            if (A.mode == MX_SCALE_FLOOR) { // RCEIL never exceeds 448 * 2^e
                const float lim = __uint_as_float(((byte + 8u) << 23) | 0x600000u);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        h[i][e] = __builtin_amdgcn_fmed3f(h[i][e], -lim, lim);
            }
            const float scale = __uint_as_float(byte << 23);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                q[i] = mxk::e4m3x4_hw(h[i][0], h[i][1], h[i][2], h[i][3], scale);
        } else {
            byte = mxk::e8m0_byte<true>(a, A.mode);
            const float scale = __uint_as_float(byte << 23);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, h[i][0], h[i][1], scale, 0);
                q[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q[i], h[i][2], h[i][3], scale, 1);
            }
        }
        if (__builtin_amdgcn_ballot_w64(byte == 0xFFu)) { // rare: non-finite values
            if (byte == 0xFFu) { // their signs, all-ones magnitudes
                constexpr int W = ELEM == MX_ELEM_E4M3 ? 8 : 4;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    q[i] = ELEM == MX_ELEM_E4M3 ? 0x7F7F7F7Fu : 0x7777u;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        q[i] |= (__float_as_uint(h[i][e]) >> 31) << (W * e + W - 1);
                }
            }
        }
        const auto s = __builtin_amdgcn_permlane16_swap(q[0], q[1], false, false);
        codes[0] = ELEM == MX_ELEM_E4M3 ? s[0] : s[0] | (s[1] << 16);
        codes[1] = s[1];
        return byte;
    }
}

template <int ELEM, int OUT, int ACT, int FM>
__device__ __forceinline__ void store_gated_act(const GatedArgs &A, const v4f (&acc)[4][FM], int64_t m,
                                                int64_t nc, int g, int qd)
{
    static_assert(FM == 1 || FM % 2 == 0, "codes are stored by two row groups");
    uint32_t byte[FM], codes[2][2];
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const v4f p[4] = {acc[0][j], acc[1][j], acc[2][j], acc[3][j]};
        byte[j] = gated_rows<ELEM, OUT, ACT>(A, p, m + 16 * j, nc, g, qd, codes[j & 1]);
        if constexpr (OUT - kGate == MX_OUT_CODES) {
            if (j & 1)
                store_codes<ELEM>(A, codes[0], codes[1], m + 16 * (j - 1), nc, g, qd);
        }
    }
    if constexpr (OUT - kGate == MX_OUT_CODES) {
        if constexpr (FM == 1) {
            const int64_t n8 = nc + 16 * (g & 1) + 8 * (g >> 1);
            if (m + qd < A.M && n8 < A.N) {
                uint8_t *dst = static_cast<uint8_t *>(A.out) +
                               ((m + qd) * A.N + n8) / (ELEM == MX_ELEM_E4M3 ? 1 : 2);
                if constexpr (ELEM == MX_ELEM_E4M3)
                    *reinterpret_cast<uint2 *>(dst) = make_uint2(codes[0][0], codes[0][1]);
                else
                    *reinterpret_cast<uint32_t *>(dst) = codes[0][0];
            }
        }
        // lane row g stores the scales of row groups g, 4 + g, ...
#pragma unroll
        for (int j = 0; j < FM; j += 4) {
            uint32_t b = byte[j];
#pragma unroll
            for (int k = 1; k < 4 && j + k < FM; ++k)
                b = g == k ? byte[j + k] : b;
            const int64_t r = m + 16 * (j + g) + qd;
            if (j + g < FM && r < A.M && nc < A.N)
                A.hs[r * (A.N / 32) + nc / 32] = (uint8_t)b;
        }
    }
}

template <int ELEM, int OUT, int FM, int FN>
__device__ __forceinline__ void store_gated(const GatedArgs &A, const v4f (&acc)[FN][FM], int64_t m0,
                                            int64_t n0, int wm, int wn, int g, int qd)
{
    static_assert(FN == 4, "a wave's output columns are one MX block");
    if (A.act == MX_ACT_SILU)
        store_gated_act<ELEM, OUT, MX_ACT_SILU, FM>(A, acc, m0 + wm, n0 + wn, g, qd);
    else
        store_gated_act<ELEM, OUT, MX_ACT_GELU_TANH, FM>(A, acc, m0 + wm, n0 + wn, g, qd);
}

} // namespace mxg

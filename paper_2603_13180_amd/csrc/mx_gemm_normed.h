// mx_gemm_normed.h -- MXNorm of a few rows within the product that reads them.
//
// A decoding step's norm is 8 KB a row and 4 us of launch, against 20 us for
// its product's weights.  A K-split tile (mx_gemm_ksplit.h) of so few rows can
// instead form their codes itself: a wave needs the codes of its own K steps
// only, and of the other waves one sum per row.  Every workgroup does this
// again, out of L2 and while its first weights are on their way from HBM.
// Measured in graphs, bf16 out, cycling through 600 MB of weights, in two
// launches -> here: F = 14336, d = 4096, one row E4M3 27.8 -> 23.4 us, E2M1 18.2
// -> 15.4, four rows 29.5 -> 27.6 and 18.8 -> 16.5; F = 8192, d = 2048, one row
// 12.2 -> 8.9 and 9.1 -> 6.5.  From Python it also saves a launch, 2 us.  What
// it costs grows with the rows, a sum over the wave for each: four of d = 768
// 6.4 -> 6.1 us, but eight 7.1 -> 8.1 (F = 2048), of d = 1024 7.9 -> 8.5 (F =
// 4096); so at most four.
//   1. the wave's x of its steps into LDS, ahead of its first weights (the loads
//      return in order, and a wait can leave the later ones in flight), and from
//      there into registers
//   2. block absmaxes, and their sum over the wave's steps (Alg. 2)
//   3. the waves' sums meet in LDS; rho~ as in norm_cast_kernel: the sums are
//      exact in double (short of absmaxes 2^15 apart), so their order is free
//   4. codes and scales into LDS in the fragment reads' layout
// The matrix core's 16 rows beyond the last one repeat it.
#pragma once

#include "mx_gemm.h"
#include "norm_cast.h"

namespace mxg {

struct NormedArgs : GatedArgs {
    const uint16_t *x; // bf16 [M, K], in place of a and as
    float *rho;        // [M] or NULL
    int p;
    float coef, eps;
};

// NCH: chunks of x per lane, at most.  4: x passes through the second slot of the
// wave's ring, which then takes weights, so that two steps' are on their way
// during the norm (one row of d = 4096, E4M3: 25.3 us with one slot, 23.4 with
// two).  8: LDS has no room for that slot beside the codes, not at two workgroups
// a compute unit.
template <int ELEM, int NW, int NCH_> struct Normed {
    static constexpr int SB = kSB<ELEM>;
    static constexpr int CPS = ELEM == MX_ELEM_E2M1 ? 32 : 16; // 16-byte chunks of x per row and step
    static constexpr int PER = 64 / CPS;                       // steps a wave takes at a time
    static constexpr int NCH = NCH_, ROWS = 4;
    static constexpr int S = NCH == 4 ? 2 : 1; // slots of the ring
    static constexpr int SCALES = NCH * PER * KB, CODES = SCALES + NCH * PER * SB;
    static constexpr int AREA = S == 2 ? CODES : NCH * 1024; // of LDS per wave: codes, x before
    static_assert(CODES <= AREA, "codes replace x");

    // times that a wave takes PER steps of one row
    __host__ __device__ static int rounds(int steps)
    {
        return ((steps + NW - 1) / NW + PER - 1) / PER;
    }
    static bool fits(int64_t M, int steps) { return M <= ROWS && M * rounds(steps) <= NCH; }

    // 1: chunk i of lane l is chunk l % CPS of step l / CPS of a round; steps
    // past the last one read the row's start
    __device__ static __forceinline__ void load(const NormedArgs &A, uint32_t slot, int w, int l)
    {
        const int rounds_ = rounds(A.steps);
        int row = 0, t = 0;
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            if (row >= (int)A.M)
                break;
            const int k = w + NW * (t * PER + l / CPS);
            const uint32_t at = (uint32_t)(row * A.steps + (k < A.steps ? k : 0)) * CPS + l % CPS;
            lds_load16(A.x, 16 * at, slot + 1024 * i);
            if (++t == rounds_) {
                t = 0;
                ++row;
            }
        }
    }

    // after the loads' wait; the slot is free when it returns
    __device__ static __forceinline__ void read(const LDS_AS uint8_t *slot, int l, uint4 (&v)[NCH])
    {
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const u32x4 x = *reinterpret_cast<const LDS_AS u32x4 *>(slot + 1024 * i + 16 * l);
            v[i] = make_uint4(x[0], x[1], x[2], x[3]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int i = 0; i < NCH; ++i)
            asm volatile("" : "+v"(v[i].x), "+v"(v[i].y), "+v"(v[i].z), "+v"(v[i].w));
    }

    // 2 to 4.  red: [NW][ROWS]; first: this workgroup stores rho~.
    __device__ static __forceinline__ void cast(const NormedArgs &A, const uint4 (&v)[NCH],
                                                LDS_AS uint8_t *area, LDS_AS double *red, bool first,
                                                int w, int l)
    {
        constexpr bool FP4 = ELEM == MX_ELEM_E2M1;
        const int rounds_ = rounds(A.steps), rows = (int)A.M;
        uint32_t mb[NCH];
        double s = 0.0;
        int row = 0, t = 0;
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            if (row >= rows)
                break;
            const bool in = w + NW * (t * PER + l / CPS) < A.steps;
            const uint32_t m = mxk::block_max<4>(mxk::chunk_absmax_bits(v[i]));
            mb[i] = m;
            const double md = in ? (double)__uint_as_float(m << 16) : 0.0;
            s += A.p == 1 ? md : md * md; // by each of the block's four lanes
            if (++t == rounds_) {
                s = mxk::team_sum<64>(s, nullptr, l);
                if (l == 0)
                    red[w * ROWS + row] = s;
                s = 0.0;
                t = 0;
                ++row;
            }
        }
        barrier();
        const int r = min(l, rows - 1);
        double S = 0.0;
#pragma unroll
        for (int u = 0; u < NW; ++u)
            S += red[u * ROWS + r];
        // lane r: rho~ of row r
        const float rhos = mxk::rho_estimate(S * 0.25, (int)A.rs, A.p, A.coef, A.eps);
        if (first && w == 0 && l < rows && A.rho)
            A.rho[l] = rhos;
        row = t = 0;
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            if (row >= rows)
                break;
            const float rho = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(rhos), row));
            uint32_t lo, hi;
            const uint32_t byte = mxk::cast_chunk<FP4>(v[i], rho, mb[i], A.mode, lo, hi);
            const int p = t * PER + l / CPS, c = l % CPS;
            if (w + NW * p < A.steps) {
                LDS_AS uint8_t *codes = area + (p * rows + row) * KB;
                if constexpr (FP4)
                    *reinterpret_cast<LDS_AS uint32_t *>(codes + 16 * ((c >> 2) ^ row) + 4 * (c & 3)) = lo;
                else
                    *reinterpret_cast<LDS_AS mxk::u32x2_t *>(codes + 16 * ((c >> 1) ^ row) + 8 * (c & 1)) =
                        mxk::u32x2_t{lo, hi};
                if ((c & 3) == 0)
                    area[SCALES + (p * rows + row) * SB + (c >> 2)] = (uint8_t)byte;
            }
            if (++t == rounds_) {
                t = 0;
                ++row;
            }
        }
    }

    // the fragment of the wave's step p
    __device__ static __forceinline__ Frag frag(const NormedArgs &A, const LDS_AS uint8_t *area, int p,
                                                int g, int qd)
    {
        const int rows = (int)A.M, row = min(qd, rows - 1);
        const LDS_AS uint8_t *codes = area + (p * rows + row) * KB;
        const LDS_AS uint8_t *scales = area + SCALES + (p * rows + row) * SB;
        Frag f;
        f.v = join(*reinterpret_cast<const LDS_AS u32x4 *>(codes + 16 * (g ^ row)),
                   *reinterpret_cast<const LDS_AS u32x4 *>(codes + 16 * ((4 + g) ^ row)));
        f.s0 = scales[g];
        f.s1 = ELEM == MX_ELEM_E2M1 ? (int)scales[4 + g] : 0;
        return f;
    }
};

} // namespace mxg

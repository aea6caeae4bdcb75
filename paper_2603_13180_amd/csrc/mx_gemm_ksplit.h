// mx_gemm_ksplit.h -- the MX product for outputs of few small tiles: one
// BM x BN tile per workgroup, its K steps dealt to the NW waves.
//
// What bounds it: the serial chain of a tile's K steps.  With the waves on
// different parts of one tile every step costs a barrier and an LDS round
// trip (0.4 us at 64 x 64); here wave w multiplies the whole tile for steps w,
// w + NW, ... from a ring of S steps of LDS that only this wave loads and
// reads.  Nothing synchronises the waves until their NW partial sums meet in
// LDS, where they are added in wave order.  Per compute unit the operand
// stream then runs at its limit of about 55 GB/s.  Measured (E4M3, K = 4096):
// 16 x 6144 47.7 us on 256 x 256 tiles, 12.5 us as a ring of 64 x 64 tiles,
// 6.8 us here with 16 x 32 tiles; 1024 x 768 x 2304 31.2 -> 8.7 us with
// 64 x 64.
#pragma once

#include "mx_gemm.h"
#include "mx_gemm_normed.h"

namespace mxg {

template <int BM_, int BN_, int NW_, int S_> struct KSplit {
    static constexpr int BM = BM_, BN = BN_, NW = NW_, S = S_, NT = 64 * NW;
    static constexpr int FM = BM / 16, FN = BN / 16;
};

// NORM > 0: A's rows are normed and cast here (mx_gemm_normed.h: NORM chunks), not
// loaded; the ring's slots are then B's rows alone.
template <class C, int ELEM, int NORM> struct KSplitOp {
    using R = Normed<ELEM, C::NW, NORM>;
    static constexpr int SB = kSB<ELEM>;
    static constexpr int AR = NORM ? 0 : C::BM, ROWS = AR + C::BN; // rows of a slot: A's, then B's
    static constexpr int S = NORM ? R::S : C::S;
    static constexpr int LC = ROWS / 8;                 // code loads per step
    static constexpr int LS = (ROWS * SB + 255) / 256; // scale loads per step
    static constexpr int L = LC + LS;
    static constexpr int SLOT = ROWS * KB + LS * 256;
    static_assert((S - 1) * L <= 63, "vmcnt range");
    // a wave's part of LDS: its ring, then its partial sums
    static constexpr int PART = S * SLOT > C::FM * C::FN * 1024 ? S * SLOT : C::FM * C::FN * 1024;
    static_assert(C::NW * PART <= 160 * 1024, "LDS");
};

template <int OUT, int NORM> using KSplitArgs = std::conditional_t<(NORM > 0), NormedArgs, ArgsOf<OUT>>;

// Tile v of the launch on this workgroup.  lds: NW PART bytes; NORM: act, NW AREA
// bytes, and red, NW ROWS sums.
template <int ELEM, int OUT, class C, int NORM>
__device__ __forceinline__ void ksplit_tile(const KSplitArgs<OUT, NORM> &A, LDS_AS uint8_t *lds,
                                            LDS_AS uint8_t *act, LDS_AS double *red, int v)
{
    using O = KSplitOp<C, ELEM, NORM>;
    using R = typename O::R;
    static_assert(!NORM || (C::FM == 1 && R::ROWS <= C::BM && R::NCH * 1024 <= O::SLOT), "normed rows");
    constexpr bool GATED = kGated<OUT>;
    constexpr int CN = kCols<OUT>(C::BN); // output columns of a tile
    constexpr int SB = O::SB, DW = SB / 4, AR = O::AR;

    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l = threadIdx.x & 63;
    const int g = l >> 4, qd = l & 15;
    int64_t m0, n0;
    tile_of(A, C::BM, CN, v, m0, n0);
    if (m0 >= A.M || n0 >= A.N) // a part of a cell that lies outside H
        return;

    // Lane offsets of the rows this lane loads (A's BM rows, then B's; 8 rows
    // x 128 bytes per instruction, swizzled as in the fragment reads; scale
    // dword 64 t + l of the step).  Rows past M or N read the last row: their
    // results are never stored.
    // Gated: the second half of B's rows are up rows, N rows further on.
    const uint8_t *ta = A.a + m0 * A.rb, *tb = A.b + n0 * A.rb;
    const uint8_t *tb2 = GATED ? tb + A.N * A.rb : tb;
    auto brow = [](int r) { return GATED ? (r - AR) % (C::BN / 2) : r - AR; };
    const int rr = l >> 3, ch = (l & 7) ^ rr;
    uint32_t code[O::LC];
#pragma unroll
    for (int t = 0; t < O::LC; ++t) {
        const int r = 8 * t;
        const int64_t off = r < AR ? min(m0 + r + rr, A.M - 1) - m0
                                      : min(n0 + brow(r) + rr, A.N - 1) - n0;
        code[t] = (uint32_t)(off * A.rb) + 16 * ch;
    }
    const uint8_t *sc[O::LS];
#pragma unroll
    for (int t = 0; t < O::LS; ++t) {
        const int dw = 64 * t + l, r = min(dw / DW, O::ROWS - 1);
        sc[t] = (r < AR ? A.as + min(m0 + r, A.M - 1) * A.rs
                           : A.bs + (min(n0 + brow(r), A.N - 1) +
                                     (GATED && r >= AR + CN ? A.N : 0)) * A.rs) + 4 * (dw % DW);
    }

    LDS_AS uint8_t *ring = lds + w * O::PART;
    const uint32_t ring_addr = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)ring);
    auto issue = [&](int k, int slot) {
        const uint32_t st = ring_addr + slot * O::SLOT;
        auto codes = [&](auto nt) {
#pragma unroll
            for (int t = 0; t < O::LC; ++t) {
                const uint8_t *base = 8 * t < AR ? ta : 8 * t < AR + CN ? tb : tb2;
                if (decltype(nt)::value && 8 * t >= AR)
                    lds_load16_nt(base, code[t] + (uint32_t)k * KB, st + 8 * t * KB);
                else
                    lds_load16(base, code[t] + (uint32_t)k * KB, st + 8 * t * KB);
            }
        };
        if constexpr (GATED) {
            if (A.once)
                codes(std::true_type{});
            else
                codes(std::false_type{});
        } else {
            codes(std::false_type{});
        }
#pragma unroll
        for (int t = 0; t < O::LS; ++t)
            lds_load4(sc[t] + (uint32_t)k * SB, st + O::ROWS * KB + 256 * t);
    };
    const FragBase ba = frag_base<ELEM>(0, O::ROWS * KB, 0, qd, g);
    const FragBase bb = frag_base<ELEM>(AR * KB, O::ROWS * KB + AR * SB, 0, qd, g);

    v4f acc[C::FM][C::FN];
#pragma unroll
    for (int j = 0; j < C::FM; ++j)
#pragma unroll
        for (int i = 0; i < C::FN; ++i)
            acc[j][i] = v4f{0.f, 0.f, 0.f, 0.f};
    const int mine = w < A.steps ? (A.steps - w - 1) / C::NW + 1 : 0; // this wave's steps
    LDS_AS uint8_t *area = act + w * R::AREA;
    if constexpr (NORM > 0) {
        LDS_AS uint8_t *xs = O::S == 2 ? ring + O::SLOT : area;
        R::load(A, __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)xs), w, l);
        if (mine > 0) {
            issue(w, 0);
            wait_vmcnt<O::L>();
        } else {
            wait_vmcnt<0>();
        }
        uint4 x[R::NCH];
        R::read(xs, l, x);
        if (O::S == 2 && mine > 1)
            issue(w + C::NW, 1);
        R::cast(A, x, area, red, n0 == 0, w, l);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    } else {
#pragma unroll 1
        for (int p = 0; p < O::S && p < mine; ++p)
            issue(w + p * C::NW, p);
    }
    int slot = 0;
#pragma unroll 1
    for (int p = 0; p < mine; ++p) {
        wait_steps<O::L, O::S - 1>(mine - 1 - p);
        const LDS_AS uint8_t *st = ring + slot * O::SLOT;
        Frag fa[C::FM], fb[C::FN];
        read_frags<ELEM, GATED ? CN : 0>(fb, st, bb, std::make_integer_sequence<int, C::FN>{});
        if constexpr (NORM > 0)
            fa[0] = R::frag(A, area, p, g, qd);
        else
            read_frags<ELEM, 0>(fa, st, ba, std::make_integer_sequence<int, C::FM>{});
        // the slot is in registers: its next step may land in it
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (p + O::S < mine)
            issue(w + (p + O::S) * C::NW, slot);
#pragma unroll
        for (int j = 0; j < C::FM; ++j)
            mma_column<ELEM, C::FN>(acc[j], fb, fa[j]);
        slot = slot + 1 == O::S ? 0 : slot + 1;
    }

    // partial sums, each wave's in its own ring
    LDS_AS v4f *sum = reinterpret_cast<LDS_AS v4f *>(ring);
#pragma unroll
    for (int j = 0; j < C::FM; ++j)
#pragma unroll
        for (int i = 0; i < C::FN; ++i)
            sum[(j * C::FN + i) * 64 + l] = acc[j][i];
    barrier();
    auto total = [&](int f) {
        v4f v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < C::NW; ++u)
            v += reinterpret_cast<const LDS_AS v4f *>(lds + u * O::PART)[f * 64 + l];
        return v;
    };
    if constexpr (GATED) {
        // a wave takes the rows of one tile row: its columns' MX block is whole
        for (int j = w; j < C::FM; j += C::NW) {
            v4f at[C::FN][1];
#pragma unroll
            for (int i = 0; i < C::FN; ++i)
                at[i][0] = total(j * C::FN + i);
            store_gated<ELEM, OUT, 1, C::FN>(A, at, m0, n0, 16 * j, 0, g, qd);
        }
        return;
    }
    for (int f = w; f < C::FM * C::FN; f += C::NW) {
        v4f v = total(f);
        // lane (g, qd) of tile (j, i) holds H[m0 + 16 j + qd][n0 + 16 i + 4 g .. +3]
        const int64_t m = m0 + 16 * (f / C::FN) + qd, n = n0 + 16 * (f % C::FN) + 4 * g;
        if (m < A.M && n < A.N) { // N is a multiple of 16
            if (A.bgain) {
                const uint2 gw = *reinterpret_cast<const uint2 *>(A.bgain + n);
                v[0] = v[0] * __uint_as_float(gw.x << 16);
                v[1] = v[1] * __uint_as_float(gw.x & 0xFFFF0000u);
                v[2] = v[2] * __uint_as_float(gw.y << 16);
                v[3] = v[3] * __uint_as_float(gw.y & 0xFFFF0000u);
            }
            if constexpr (OUT == MX_OUT_F32)
                *reinterpret_cast<v4f *>(static_cast<float *>(A.out) + m * A.N + n) = v;
            else
                *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(A.out) + m * A.N + n) =
                    make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
        }
    }
}

template <int ELEM, int OUT, class C, int NORM>
__global__ void __launch_bounds__(C::NT) mx_gemm_ksplit_kernel(KSplitArgs<OUT, NORM> A)
{
    using O = KSplitOp<C, ELEM, NORM>;
    __shared__ __attribute__((aligned(16))) uint8_t lds[C::NW * O::PART];
    if constexpr (NORM > 0) {
        __shared__ __attribute__((aligned(16))) uint8_t act[C::NW * O::R::AREA];
        __shared__ double red[C::NW * O::R::ROWS];
        ksplit_tile<ELEM, OUT, C, NORM>(A, (LDS_AS uint8_t *)lds, (LDS_AS uint8_t *)act, (LDS_AS double *)red,
                                        blockIdx.x);
    } else {
        ksplit_tile<ELEM, OUT, C, 0>(A, (LDS_AS uint8_t *)lds, nullptr, nullptr, blockIdx.x);
    }
}

template <int ELEM, int OUT, class C, int NORM = 0>
hipError_t launch_ksplit(const KSplitArgs<OUT, NORM> &A, hipStream_t stream)
{
    hipLaunchKernelGGL((mx_gemm_ksplit_kernel<ELEM, OUT, C, NORM>), dim3((unsigned)(A.cells * A.sub_m * A.sub_n)),
                       dim3(C::NT), 0, stream, A);
    return hipGetLastError();
}

} // namespace mxg

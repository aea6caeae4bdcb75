// mx_gemm_256.h -- the MX product on 256 x 256 tiles, one persistent workgroup
// per compute unit.
//
// Tiling: a workgroup of 8 waves (two per SIMD) computes a 256 (M) x 256 (N)
// output tile; wave w owns the 128 x 64 quarter-column (w & 1, w >> 1) as
// 8 x 4 matrix-core tiles of 16 x 16, 128 accumulator registers.  Two waves
// per SIMD are what lets the matrix core run while the other wave waits on
// LDS or a barrier: with one wave per SIMD the E2M1 instruction issues at
// about half its rate.  The K loop moves 128 bytes of every row per step
// (128 E4M3 or 256 E2M1 elements) from global memory straight into LDS
// (16-byte global_load_lds, no staging registers) into two stages of 66 KB;
// each step reads its four B fragments into registers and streams the eight
// A fragments two ahead of the matrix core.  In LDS, 16-byte chunk c of row r
// lives at chunk c ^ (r & 7) of the row, so the fragment reads of 8
// consecutive rows hit distinct banks.
//
// What bounds it: at 256 x 256 the operand stream is 64 KB per K step per
// workgroup, about 10 TB/s of L2 requests at half the fp8 peak.  Two stages
// fill LDS, so the DMA runs one step ahead of the products and each step
// waits for it; the tile's stores slow the operand stream (the non-temporal
// policy below halves that); and after each step's barrier every wave reads
// fragments before its first product.  The eight waves' accumulators fill
// half the register file, which leaves no room for a third stage in
// registers.
#pragma once

#include <type_traits>

#include "mx_gemm.h"

namespace mxg {

constexpr int BM = 256;    // tile rows of A (M)
constexpr int BN = 256;    // tile rows of B (N)
constexpr int NT = 512;    // threads: 8 waves, two per SIMD
constexpr int WTM = 128;   // wave tile along M
constexpr int WTN = 64;    // wave tile along N
constexpr int FM = WTM / 16, FN = WTN / 16;

// Tile v of a launch whose cells are 256 x CN (fewer divisions than tile_of:
// they stand between two tiles' loads).
template <int CN = BN>
__device__ __forceinline__ void whole_tile(const Args &A, int v, int64_t &m0, int64_t &n0)
{
    int cm, cn;
    cell_of(A, xcd_range(v, A.cells), cm, cn);
    m0 = (int64_t)cm * BM;
    n0 = (int64_t)cn * CN;
}

template <int ELEM> struct Op {
    static constexpr int SB = kSB<ELEM>;
    static constexpr int STAGE = (BM + BN) * KB + (BM + BN) * SB;
};

// Per-lane part of the DMA addresses, fixed for the whole K loop: byte
// offsets, relative to the tile's first row, of the rows this lane moves.
// Wave w moves code rows 32w .. 32w+31 of both tiles (4 instructions of
// 8 rows x 128 bytes each: lane l fills LDS slot l % 8 of row l / 8 of its
// group, which holds source chunk (l % 8) ^ (l / 8)); waves 0-3 move the
// scale bytes of A's rows 64w .. 64w+63, waves 4-7 those of B's rows
// 64(w-4) .. 64(w-4)+63 (lane i of scale instruction u moves dword
// i % (SB/4) of row u (64 / (SB/4)) + i / (SB/4)).  Rows past M or N read
// row M-1 or N-1: their results are never stored.  Gated: B's rows 0 .. 127 are
// gate rows, which waves 0-3 (scales: 4-5) move, the others up rows; the
// offsets are relative to the tile's first gate or up row.
template <int ELEM> struct Rows {
    uint32_t a[4], b[4];
    uint32_t s[Op<ELEM>::SB / 4];
};

template <int ELEM, bool GATED = false>
__device__ __forceinline__ Rows<ELEM> lane_rows(const Args &A, int64_t m0, int64_t n0, int w,
                                                int l)
{
    constexpr int DW = Op<ELEM>::SB / 4;
    Rows<ELEM> R;
    const int rr = l >> 3;       // row within the 8-row group
    const int ch = (l & 7) ^ rr; // source chunk for this LDS slot (the swizzle)
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int r = 32 * w + 8 * t + rr;
        const int rb = GATED ? r & (BN / 2 - 1) : r;
        R.a[t] = (uint32_t)((min(m0 + r, A.M - 1) - m0) * A.rb) + 16 * ch;
        R.b[t] = (uint32_t)((min(n0 + rb, A.N - 1) - n0) * A.rb) + 16 * ch;
    }
    const bool on_a = w < 4;
    const int64_t base = on_a ? m0 : n0, lim = on_a ? A.M : A.N;
#pragma unroll
    for (int u = 0; u < DW; ++u) {
        const int r = 64 * (GATED && !on_a ? w & 1 : w & 3) + u * (64 / DW) + l / DW;
        R.s[u] = (uint32_t)((min(base + r, lim - 1) - base) * A.rs) + 4 * (l % DW);
    }
    return R;
}

// Issue this wave's loads of K step s into one LDS stage, laid out as
// [A codes 256 x 128][B codes 256 x 128][A scales 256 x SB][B scales 256 x SB].
template <int ELEM>
__device__ __forceinline__ void issue_step(const uint8_t *ta, const uint8_t *tb,
                                           const uint8_t *tsa, const uint8_t *tsb,
                                           const Rows<ELEM> &R, int s, uint32_t stage, int w)
{
    constexpr int SB = Op<ELEM>::SB;
    constexpr int DW = SB / 4;
    const uint32_t xa = stage;
    const uint32_t xb = stage + BM * KB;
    const uint32_t kc = (uint32_t)s * KB, ks = (uint32_t)s * SB;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        lds_load16(ta, R.a[t] + kc, xa + (32 * w + 8 * t) * KB);
        lds_load16(tb, R.b[t] + kc, xb + (32 * w + 8 * t) * KB);
    }
    const uint8_t *ts = w < 4 ? tsa : tsb;
    const uint32_t xs = stage + (BM + BN) * KB + (w < 4 ? 0 : BM * SB) + 64 * (w & 3) * SB;
#pragma unroll
    for (int u = 0; u < DW; ++u)
        lds_load4(ts, R.s[u] + ks, xs + u * (64 / DW) * SB);
}

// The products of one K step from the stage at st: the step's four B
// fragments held in registers, the eight A fragments streamed, each requested
// two ahead of the products that use it.
// UP: the distance of the up rows from the gate rows of a gated product's B.
template <int ELEM, int UP = 0>
__device__ __forceinline__ void step_products(v4f (&acc)[FN][FM], const LDS_AS uint8_t *st,
                                              const FragBase &ba, const FragBase &bb)
{
    if constexpr (ELEM == MX_ELEM_E2M1) {
        // Whole fragments, read in the E4M3 order below (the lane's low and
        // high 16-byte chunks each feed one instruction: E2M1 blocks g and
        // 4 + g of the step).  Per column, the four tiles' products of the
        // low halves, then those of the high halves: an accumulator's two
        // instructions sit four apart, not back to back (where the second
        // waits for the first's result), in the same order of additions.
        // (Two passes over the 32 tiles, every low half and then every high
        // half from half-fragment reads, were 1.5-3% slower at the QKV and
        // gate+up shapes.)
        Frag fb[FN], fa[FM];
        fb[0] = read_frag_at<ELEM, frag_row<FN, UP>(0)>(st, bb);
        fb[1] = read_frag_at<ELEM, frag_row<FN, UP>(1)>(st, bb);
        fa[0] = read_frag<ELEM, 0>(st, ba);
        __builtin_amdgcn_sched_barrier(0);
        fb[2] = read_frag_at<ELEM, frag_row<FN, UP>(2)>(st, bb);
        fb[3] = read_frag_at<ELEM, frag_row<FN, UP>(3)>(st, bb);
        fa[1] = read_frag<ELEM, 1>(st, ba);
        __builtin_amdgcn_sched_barrier(0);
        auto column = [&](auto jc) {
            constexpr int j = decltype(jc)::value;
            if constexpr (j + 2 < FM)
                fa[j + 2] = read_frag<ELEM, j + 2>(st, ba);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < FN; ++i)
                mma_e2m1_lo(acc[i][j], fb[i], fa[j]);
#pragma unroll
            for (int i = 0; i < FN; ++i)
                mma_e2m1_hi(acc[i][j], fb[i], fa[j]);
            __builtin_amdgcn_sched_barrier(0);
        };
        column(std::integral_constant<int, 0>{});
        column(std::integral_constant<int, 1>{});
        column(std::integral_constant<int, 2>{});
        column(std::integral_constant<int, 3>{});
        column(std::integral_constant<int, 4>{});
        column(std::integral_constant<int, 5>{});
        column(std::integral_constant<int, 6>{});
        column(std::integral_constant<int, 7>{});
        return;
    }
    // The step starts with every wave reading fragments after the barrier:
    // B0, B1 and A0 first, so that the first two products wait for three
    // fragments, not six (QKV shape: 1-3% faster).
    Frag fb[FN], fa[FM];
    fb[0] = read_frag_at<ELEM, frag_row<FN, UP>(0)>(st, bb);
    fb[1] = read_frag_at<ELEM, frag_row<FN, UP>(1)>(st, bb);
    fa[0] = read_frag<ELEM, 0>(st, ba);
    __builtin_amdgcn_sched_barrier(0);
    fb[2] = read_frag_at<ELEM, frag_row<FN, UP>(2)>(st, bb);
    fb[3] = read_frag_at<ELEM, frag_row<FN, UP>(3)>(st, bb);
    fa[1] = read_frag<ELEM, 1>(st, ba);
    __builtin_amdgcn_sched_barrier(0);
    fa[2] = read_frag<ELEM, 2>(st, ba);
    __builtin_amdgcn_sched_barrier(0);
    mma_e4m3(acc[0][0], fb[0], fa[0]);
    mma_e4m3(acc[1][0], fb[1], fa[0]);
    __builtin_amdgcn_sched_barrier(0);
    mma_e4m3(acc[2][0], fb[2], fa[0]);
    mma_e4m3(acc[3][0], fb[3], fa[0]);
    __builtin_amdgcn_sched_barrier(0);
    auto column = [&](auto jc) {
        constexpr int j = decltype(jc)::value;
        if constexpr (j + 2 < FM)
            fa[j + 2] = read_frag<ELEM, j + 2>(st, ba);
        // keep the read ahead of this fragment's products
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < FN; ++i)
            mma_e4m3(acc[i][j], fb[i], fa[j]);
        __builtin_amdgcn_sched_barrier(0);
    };
    column(std::integral_constant<int, 1>{});
    column(std::integral_constant<int, 2>{});
    column(std::integral_constant<int, 3>{});
    column(std::integral_constant<int, 4>{});
    column(std::integral_constant<int, 5>{});
    column(std::integral_constant<int, 6>{});
    column(std::integral_constant<int, 7>{});
}

template <int ELEM, int OUT>
__global__ void __launch_bounds__(NT) mx_gemm_kernel(ArgsOf<OUT> A)
{
    constexpr bool GATED = kGated<OUT>;
    constexpr int CN = kCols<OUT>(BN); // output columns of a tile
    constexpr int SB = Op<ELEM>::SB;
    constexpr int STAGE = Op<ELEM>::STAGE;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * STAGE];

    // The grid is at most one workgroup per compute unit, and workgroup b
    // takes tiles v = b, b + grid, b + 2 grid, ...
    const int G = A.cells;

    const int tid = threadIdx.x;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6); // wave-uniform
    const int l = tid & 63;
    const int g = l >> 4, qd = l & 15; // lane group (K block / output row quad), row in fragment
    const int wm = (w & 1) * WTM, wn = (w >> 1) * kCols<OUT>(WTN);

    LDS_AS uint8_t *st0 = (LDS_AS uint8_t *)lds;
    const uint32_t st0_addr = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)st0);
    const FragBase ba = frag_base<ELEM>(0, (BM + BN) * KB, wm, qd, g);
    const FragBase bb = frag_base<ELEM>(BM * KB, (BM + BN) * KB + BM * SB, wn, qd, g);
    // the B operand as this wave moves it: its codes and its scales
    const uint8_t *wb = A.b, *wbs = A.bs;
    if constexpr (GATED) {
        wb += w >= 4 ? A.N * A.rb : 0;
        wbs += w >= 6 ? A.N * A.rs : 0;
    }

    int v = blockIdx.x;
    int64_t m0, n0;
    whole_tile<CN>(A, v, m0, n0);
    Rows<ELEM> R = lane_rows<ELEM, GATED>(A, m0, n0, w, l);

    // Pipeline, one barrier per K step.  At the top of a step every wave has
    // its own DMA of the step landed (vmcnt) and, past the barrier, so has
    // every other wave, and no wave still reads the other stage (the previous
    // step): the DMA of the next step goes there, and after a tile's last
    // step the DMA of the next tile's first step, which then runs under that
    // last step's products and the tile's stores.
    issue_step<ELEM>(A.a + m0 * A.rb, wb + n0 * A.rb, A.as + m0 * A.rs, wbs + n0 * A.rs, R, 0,
                     st0_addr, w);
    bool prev_full = false; // the previous tile lies inside H (all its stores ran)
    for (int gs = 0;;) {
        v4f acc[FN][FM];
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j)
                acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
        const int nv = v + (int)gridDim.x;
        int64_t m1 = 0, n1 = 0;
        for (int s = 0; s < A.steps; ++s, ++gs) {
            const int cur = gs & 1;
            // this step's DMA has landed.  In a tile's first step the
            // previous tile's stores, issued after this DMA, need not have
            // completed: operations complete in order, so at most that many
            // may remain (a partial tile ran fewer stores: wait for all).
            if constexpr (GATED) {
                constexpr int H = kGatedStores<OUT, FM>;
                if (s == 0 && prev_full && A.gu)
                    wait_vmcnt<H + kKeptStores<FM>>();
                else if (s == 0 && prev_full)
                    wait_vmcnt<H>();
                else
                    wait_vmcnt<0>();
            } else {
                if (s == 0 && prev_full)
                    wait_vmcnt<kTileStores<OUT, FM, FN>>();
                else
                    wait_vmcnt<0>();
            }
            barrier();
            const uint32_t nxt = st0_addr + (cur ^ 1) * STAGE;
            if (s + 1 < A.steps) {
                issue_step<ELEM>(A.a + m0 * A.rb, wb + n0 * A.rb, A.as + m0 * A.rs,
                                 wbs + n0 * A.rs, R, s + 1, nxt, w);
            } else if (nv < G) {
                whole_tile<CN>(A, nv, m1, n1);
                R = lane_rows<ELEM, GATED>(A, m1, n1, w, l);
                issue_step<ELEM>(A.a + m1 * A.rb, wb + n1 * A.rb, A.as + m1 * A.rs,
                                 wbs + n1 * A.rs, R, 0, nxt, w);
            }
            step_products<ELEM, GATED ? CN : 0>(acc, st0 + cur * STAGE, ba, bb);
        }
        if constexpr (GATED)
            store_gated<ELEM, OUT, FM, FN>(A, acc, m0, n0, wm, wn, g, qd);
        else
            store_tile<OUT, FM, FN>(A, acc, m0, n0, wm, wn, g, qd);
        prev_full = m0 + BM <= A.M && n0 + CN <= A.N;
        if (nv >= G)
            break;
        v = nv;
        m0 = m1;
        n0 = n1;
    }
}

template <int ELEM, int OUT>
hipError_t launch(const ArgsOf<OUT> &A, hipStream_t stream)
{
    const int G = A.cells;
    const int grid = G < A.grid_max ? G : A.grid_max;
    hipLaunchKernelGGL((mx_gemm_kernel<ELEM, OUT>), dim3((unsigned)grid), dim3(NT), 0, stream, A);
    return hipGetLastError();
}

} // namespace mxg

// mx_gemm_plan.h -- the tile shapes of the MX product's kernels, what each
// costs, and the choice between them.
#pragma once

#include <algorithm>

#include "mx_gemm.h"
#include "mx_gemm_256.h"
#include "mx_gemm_ksplit.h"
#include "mx_gemm_ring.h"
#include "products.h"

namespace mxg {

// Ring tiles: 4 waves, two workgroups per compute unit.
using R64x128 = Ring<64, 128, 2, 2, 3>;
using R128x128 = Ring<128, 128, 2, 2, 2>;
// K-split tiles: 8 waves, one workgroup per compute unit.
using K16x32 = KSplit<16, 32, 8, 3>;
using K32x32 = KSplit<32, 32, 8, 2>;
using K32x64 = KSplit<32, 64, 8, 1>;
using K64x64 = KSplit<64, 64, 8, 1>;
// K-split tiles of gated products, whose waves hold a whole MX block: 4 waves,
// two or three workgroups per compute unit.  A decoding step's tiles are then
// resident at once instead of in two uneven rounds (1 to 16 rows, 448 tiles of
// 14336 x 4096: E4M3 28.0 -> 26.7 us, E2M1 15.4 -> 13.1 against 8 waves; where
// they are one a unit anyhow, 8192 x 8192, 28.9 -> 29.7 and 14.2 -> 14.1).
using G16x64 = KSplit<16, 64, 4, 1>;
using G32x64 = KSplit<32, 64, 4, 1>;
using G64x64 = KSplit<64, 64, 4, 1>;

enum Shape { S_K16x32, S_K32x32, S_K32x64, S_K64x64, S_R64x128, S_R128x128, S_256x256, S_COUNT };
constexpr int S_G16x64 = S_COUNT, S_G32x64 = S_COUNT + 1, S_G64x64 = S_COUNT + 2;
constexpr int S_ALL = S_COUNT + 3;

// What a launch of each tile shape costs on MI355X, fitted to times at K =
// 512 .. 8192 and 64 to 3400 tiles: us once per launch, per round of tiles
// (their stores, and for the K-split kernel the start of a tile's loads, which
// nothing overlaps) and per K step of a round.  Below 256 x 256 the time per
// step is the tile's operand bytes at about 55 GB/s per compute unit, so a
// larger tile does more products per byte and a smaller one leaves fewer
// compute units idle.
//
// With few K steps a smaller tile's latency is not covered (a ring waits for
// the stores of the tile before, a K-split tile for its only step): many
// rounds take `few` + steps * `few_step` each at least.  At one K step, bf16,
// 128 x 128 tiles then take 2.3-2.5 us a round, not 1.4, and lose to 256 x
// 256: 9526 x 22336 129 against 106 us, 142102 x 1152 97 against 70.  Counted
// from the ninth round on for the rings (with fewer rounds 256 x 256 tiles do
// not reach their pace either: two K steps, 3 to 8 rounds, the rings are 1.05
// to 1.4 times as fast in the median of each output type), from the first if N leaves half of the
// 64 x 128 tile empty (63697 x 48 10.5 against 8.0), and for the K-split tiles
// beyond two rounds.  Over 1000 sizes of 1 to 4 steps and 1e6 to 2e8 outputs
// the choice was more than 3% slower than 256 x 256 tiles at 106, by up to 28%,
// and is now at 35, 32 of them of one step, by up to 16%; on average it is
// 1.15 times as fast as those.
//
// An estimate ranks the shapes; it does not predict the time.  It has no term
// for operands that come from HBM rather than L2, nor for the output's type:
// 61 x 28672 x 4096 is put at 17 us in E4M3 and takes 34, and at 10 in E2M1
// and takes 14.
struct Cost {
    int bm, bn;
    float once, round, step, few, few_step;
};
constexpr Cost kCost[S_ALL] = {
    {16, 32, 1.3f, 1.0f, 0.14f, 1.6f, 0.0f},   {32, 32, 1.4f, 1.1f, 0.14f, 1.9f, 0.0f},
    {32, 64, 2.2f, 0.7f, 0.19f, 2.15f, 0.0f},  {64, 64, 0.4f, 2.6f, 0.275f, 2.9f, 0.2f},
    {64, 128, 3.1f, 0.4f, 0.425f, 1.1f, 0.3f}, {128, 128, 4.1f, 0.8f, 0.59f, 1.8f, 0.45f},
    {256, 256, 1.2f, 4.0f, 1.75f, 0.0f, 0.0f},
    // (gated: ranked against times at 1 to 128 rows, F = 1024 .. 14336)
    {16, 64, 2.2f, 0.7f, 0.17f, 2.15f, 0.0f},
    {32, 64, 2.2f, 0.7f, 0.24f, 2.15f, 0.0f},
    {64, 64, 0.4f, 2.6f, 0.275f, 2.9f, 0.2f},
};

// us a launch over `cells` outputs of cm x cn takes on `cus` compute units
inline double launch_cost(int shape, int64_t cells, int64_t cm, int64_t cn, int steps, int cus)
{
    const Cost &c = kCost[shape];
    const int64_t tiles = cells * ((cm + c.bm - 1) / c.bm) * ((cn + c.bn - 1) / c.bn);
    const int64_t rounds = (tiles + cus - 1) / cus;
    const double per = c.round + (double)steps * c.step;
    const double few = std::max(per, (double)c.few + (double)steps * c.few_step);
    if (shape <= S_K64x64 || shape >= S_COUNT)
        return c.once + (double)rounds * (rounds > 2 ? few : per);
    double us = (double)rounds * per + (double)std::max<int64_t>(0, rounds - 8) * (few - per);
    if (shape == S_R64x128 && cn <= 64 && rounds > 2)
        us = std::max(us, (double)rounds * (1.3 + 0.3 * (double)steps));
    return c.once + us;
}

// How one product is computed: the whole output in tiles of `shape`; or, where
// that is at least 5% cheaper, its first `whole` cells of 256 x 256 (whole
// rounds of them) in one launch and the cells left in tiles of `tail` in a
// second.
struct Plan {
    int shape;
    int whole, tail; // whole = 0: one launch
    double us;
};

// The tile shapes smaller than 256 x 256 that a product may take.
constexpr int kPlainShapes[] = {S_K16x32, S_K32x32, S_K32x64, S_K64x64, S_R64x128, S_R128x128};
constexpr int kGatedShapes[] = {S_G16x64, S_G32x64, S_G64x64, S_R64x128, S_R128x128};

template <size_t NS>
inline Plan plan_among(const int (&shapes)[NS], int64_t M, int64_t N, int steps, int cus)
{
    Plan P{S_256x256, 0, 0, launch_cost(S_256x256, 1, M, N, steps, cus)};
    for (const int s : shapes) {
        const double c = launch_cost(s, 1, M, N, steps, cus);
        if (c < P.us) {
            P.us = c;
            P.shape = s;
        }
    }
    const int64_t cells = ((M + BM - 1) / BM) * ((N + BN - 1) / BN);
    const int64_t whole = cells / cus * cus, left = cells - whole;
    if (whole && left) {
        int tail = shapes[0];
        double tcost = launch_cost(tail, left, BM, BN, steps, cus);
        for (const int s : shapes) {
            const double c = launch_cost(s, left, BM, BN, steps, cus);
            if (c < tcost) {
                tcost = c;
                tail = s;
            }
        }
        const double two = launch_cost(S_256x256, whole, BM, BN, steps, cus) + tcost;
        if (two < 0.95 * P.us)
            P = Plan{S_256x256, (int)whole, tail, two};
    }
    return P;
}

inline Plan plan_product(int64_t M, int64_t N, int steps, int cus)
{
    return plan_among(kPlainShapes, M, N, steps, cus);
}

// N columns of H: a tile of bn B rows gives bn / 2 of them.
inline Plan plan_gated(int64_t M, int64_t N, int steps, int cus)
{
    return plan_among(kGatedShapes, M, 2 * N, steps, cus);
}

template <int ELEM, int OUT>
hipError_t launch_shape(int shape, const ArgsOf<OUT> &A, hipStream_t stream)
{
    if constexpr (kGated<OUT>) {
        switch (shape) {
        case S_G16x64: return launch_ksplit<ELEM, OUT, G16x64>(A, stream);
        case S_G32x64: return launch_ksplit<ELEM, OUT, G32x64>(A, stream);
        case S_G64x64: return launch_ksplit<ELEM, OUT, G64x64>(A, stream);
        case S_R64x128: return launch_ring<ELEM, OUT, R64x128>(A, stream);
        case S_R128x128: return launch_ring<ELEM, OUT, R128x128>(A, stream);
        default: return launch<ELEM, OUT>(A, stream);
        }
    } else {
        switch (shape) {
        case S_K16x32: return launch_ksplit<ELEM, OUT, K16x32>(A, stream);
        case S_K32x32: return launch_ksplit<ELEM, OUT, K32x32>(A, stream);
        case S_K32x64: return launch_ksplit<ELEM, OUT, K32x64>(A, stream);
        case S_K64x64: return launch_ksplit<ELEM, OUT, K64x64>(A, stream);
        case S_R64x128: return launch_ring<ELEM, OUT, R64x128>(A, stream);
        case S_R128x128: return launch_ring<ELEM, OUT, R128x128>(A, stream);
        default: return launch<ELEM, OUT>(A, stream);
        }
    }
}

// A weight of this many bytes that a launch reads once (one row of its tiles) is
// loaded past the caches' normal allocation: no later call finds it there.
// Cycling through 550 to 600 MB of weights at 1 to 61 rows: 117 MB (E4M3) 26.7
// -> 24.7 and 32.1 -> 30.4 us (and 29.5 with the rings' K steps in turn), 134 MB
// 28.9 -> 25.7; but 62 MB (E2M1) 13.1 ->
// 12.9 and 16.8 -> 16.7, 67 MB 14.2 -> 15.4, 17 MB (E4M3) 10.1 -> 11.1.
// A tail's smaller tiles, several rows of them over the same weights, share their
// loads in the caches: 200 rows, F = 36096 123 -> 117 us, 49152 169 -> 157.
constexpr int64_t kOnceBytes = 96 << 20;
inline bool read_once(const GatedArgs &A, int shape)
{
    return A.M <= kCost[shape].bm && 2 * A.N * A.rb >= kOnceBytes;
}

template <int ELEM, int OUT>
hipError_t multiply_as(const Plan &P, ArgsOf<OUT> A, hipStream_t stream)
{
    set_tiles(A, kCost[P.shape].bm, kCols<OUT>(kCost[P.shape].bn), 1024);
    if constexpr (kGated<OUT>)
        A.once = read_once(A, P.shape);
    if (!P.whole)
        return launch_shape<ELEM, OUT>(P.shape, A, stream);
    const int left = A.cells - P.whole;
    A.cells = P.whole;
    const hipError_t e = launch<ELEM, OUT>(A, stream);
    if (e != hipSuccess)
        return e;
    A.pid0 = P.whole;
    A.cells = left;
    A.sub_m = BM / kCost[P.tail].bm;
    A.sub_n = BN / kCost[P.tail].bn;
    if constexpr (kGated<OUT>)
        A.once = read_once(A, P.tail);
    return launch_shape<ELEM, OUT>(P.tail, A, stream);
}

template <int ELEM, int OUT> hipError_t multiply(const ArgsOf<OUT> &A, hipStream_t stream)
{
    if constexpr (kGated<OUT>)
        return multiply_as<ELEM, OUT>(plan_gated(A.M, A.N, A.steps, A.grid_max), A, stream);
    else
        return multiply_as<ELEM, OUT>(plan_product(A.M, A.N, A.steps, A.grid_max), A, stream);
}

// A checked product's kernel arguments (without tiles).
void product_args(Args &A, const Product &P, int elem, hipStream_t stream);

} // namespace mxg

// MX matrix product H = dec(A) dec(B)^T on the gfx950 block-scaled matrix
// cores (Sec. 3.7 eq. (mx-matmul): the product MXNormLinear takes of MXNorm's
// output and the gain-folded weight cast; the implementation appendix's
// mx_norm_linear_forward ends in this product).
//
// A [M, K] (activations, MXNorm codes) and B [N, K] (weights) are both blocked
// along K with one E8M0 scale per 32 elements; elements are E4M3 (one byte)
// or E2M1 (two per byte, element 2j in the low nibble).  The hardware
// instruction v_mfma_scale_f32_16x16x128_f8f6f4 multiplies a 16x128 tile of
// each operand with one scale byte per row and 32-element block applied
// exactly, accumulating in fp32.
//
// mx_gemm_256.h, mx_gemm_ring.h and mx_gemm_ksplit.h hold the kernels,
// mx_gemm_plan.h the choice between them; here are two products in one launch
// and the entry point.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "mx_gemm.h"
#include "mx_gemm_plan.h"
#include "mxnorm.h"
#include "products.h"
#include "status.h"
#include "testing.h"

namespace mxg {

// ------------------------------------------------- two products, one launch --

// Two products in one persistent launch, so that the last, partly empty round
// of one is filled with tiles of the other (the weight gradient's 384 tiles
// on 256 compute units leave half of them idle for a round of 256 K steps).
// A step takes about 2 us whether all compute units or half of them run, so
// the fullest workgroup's load is the time.  Measured against the two
// launches: 6144 x 4096 x 32768 with 32768 x 4096 x 6144 (E4M3) 1795 -> 1690
// us, 6144 x 4096 x 4096 with 4096 x 4096 x 6144 142 -> 130 us (E2M1) and 216
// -> 199 us (E4M3).
// Workgroup b is of class b >= split; a workgroup of class c takes n[c][0]
// tiles of product 0 (output OUT0), then n[c][1] of product 1 (bf16 output).
struct PairArgs {
    Args p[2];
    int split; // workgroups of class 0
    int n[2][2];
};

// Product i's tile that is number j of workgroup b's share: the shares both
// classes have in whole rounds over the grid, the rest in rounds over the
// class that has more.  Past the product's last tile: -1.
__device__ __forceinline__ int pair_tile(const PairArgs &W, int i, int j, int b, int grid)
{
    const int c = b >= W.split;
    const int both = min(W.n[0][i], W.n[1][i]);
    const int first = c ? W.split : 0, size = c ? grid - W.split : W.split;
    const int v = j < both ? j * grid + b : both * grid + (j - both) * size + (b - first);
    return j < W.n[c][i] && v < W.p[i].cells ? v : -1;
}

template <int ELEM, int OUT0>
__global__ void __launch_bounds__(NT) mx_gemm_pair_kernel(PairArgs W)
{
    constexpr int SB = Op<ELEM>::SB;
    constexpr int STAGE = Op<ELEM>::STAGE;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * STAGE];

    const int tid = threadIdx.x;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6); // wave-uniform
    const int l = tid & 63;
    const int g = l >> 4, qd = l & 15;
    const int wm = (w & 1) * WTM, wn = (w >> 1) * WTN;
    const int b = blockIdx.x, grid = gridDim.x;

    LDS_AS uint8_t *st0 = (LDS_AS uint8_t *)lds;
    const uint32_t st0_addr = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)st0);
    const FragBase ba = frag_base<ELEM>(0, (BM + BN) * KB, wm, qd, g);
    const FragBase bb = frag_base<ELEM>(BM * KB, (BM + BN) * KB + BM * SB, wn, qd, g);

    // tile number j of product i, and the one after it
    int i = 0, j = 0, v = pair_tile(W, 0, 0, b, grid);
    if (v < 0) {
        i = 1;
        v = pair_tile(W, 1, 0, b, grid);
        if (v < 0)
            return;
    }
    int64_t m0, n0;
    whole_tile(W.p[i], v, m0, n0);
    Rows<ELEM> R = lane_rows<ELEM>(W.p[i], m0, n0, w, l);
    const uint8_t *ta = W.p[i].a + m0 * W.p[i].rb, *tb = W.p[i].b + n0 * W.p[i].rb;
    const uint8_t *tsa = W.p[i].as + m0 * W.p[i].rs, *tsb = W.p[i].bs + n0 * W.p[i].rs;

    // the pipeline of mx_gemm_kernel
    issue_step<ELEM>(ta, tb, tsa, tsb, R, 0, st0_addr, w);
    int stores = 0; // stores of the previous tile, if it lies inside its H
    for (int gs = 0;;) {
        v4f acc[FN][FM];
#pragma unroll
        for (int n = 0; n < FN; ++n)
#pragma unroll
            for (int m = 0; m < FM; ++m)
                acc[n][m] = v4f{0.f, 0.f, 0.f, 0.f};
        int ni = i, nj = j + 1, nv = pair_tile(W, i, nj, b, grid);
        if (nv < 0 && i == 0) {
            ni = 1;
            nj = 0;
            nv = pair_tile(W, 1, 0, b, grid);
        }
        int64_t m1 = 0, n1 = 0;
        const int steps = W.p[i].steps;
        for (int s = 0; s < steps; ++s, ++gs) {
            const int cur = gs & 1;
            if (s == 0 && stores == kTileStores<OUT0, FM, FN>)
                wait_vmcnt<kTileStores<OUT0, FM, FN>>();
            else if (s == 0 && stores == kTileStores<MX_OUT_BF16, FM, FN>)
                wait_vmcnt<kTileStores<MX_OUT_BF16, FM, FN>>();
            else
                wait_vmcnt<0>();
            barrier();
            const uint32_t nxt = st0_addr + (cur ^ 1) * STAGE;
            if (s + 1 < steps) {
                issue_step<ELEM>(ta, tb, tsa, tsb, R, s + 1, nxt, w);
            } else if (nv >= 0) {
                const Args &A = W.p[ni];
                whole_tile(A, nv, m1, n1);
                R = lane_rows<ELEM>(A, m1, n1, w, l);
                ta = A.a + m1 * A.rb;
                tb = A.b + n1 * A.rb;
                tsa = A.as + m1 * A.rs;
                tsb = A.bs + n1 * A.rs;
                issue_step<ELEM>(ta, tb, tsa, tsb, R, 0, nxt, w);
            }
            step_products<ELEM>(acc, st0 + cur * STAGE, ba, bb);
        }
        const bool full = m0 + BM <= W.p[i].M && n0 + BN <= W.p[i].N;
        if (i == 0) {
            store_tile<OUT0, FM, FN>(W.p[0], acc, m0, n0, wm, wn, g, qd);
            stores = full ? kTileStores<OUT0, FM, FN> : 0;
        } else {
            store_tile<MX_OUT_BF16, FM, FN>(W.p[1], acc, m0, n0, wm, wn, g, qd);
            stores = full ? kTileStores<MX_OUT_BF16, FM, FN> : 0;
        }
        if (nv < 0)
            break;
        i = ni;
        j = nj;
        v = nv;
        m0 = m1;
        n0 = n1;
    }
}

// Shares of the two products' tiles for `cus` workgroups that make the
// fullest workgroup's load, in steps, as small as two classes of workgroups
// can: class 0 takes n0 tiles of product 0, class 1 takes n1 > n0, and both
// fill what the load leaves with tiles of product 1.  A tile costs its K
// steps and about two steps' time for its stores.  Returns the load, or 0 if
// the products have too many tiles to search.
inline int64_t pair_plan(PairArgs &W, int cus)
{
    constexpr int kTileSteps = 2;
    const int64_t g0 = W.p[0].cells, g1 = W.p[1].cells;
    const int64_t c0 = W.p[0].steps + kTileSteps, c1 = W.p[1].steps + kTileSteps;
    const int64_t q = g0 / cus;
    if (q > 16 || g1 / cus > 4096)
        return 0;
    const int64_t lower = (g0 * c0 + g1 * c1 + cus - 1) / cus;
    int64_t best = 0;
    // the load of some workgroup is a * c0 + b * c1: for each a and pair of
    // shares, the smallest such load that holds both products
    for (int64_t lo = 0; lo <= q; ++lo)
        for (int64_t hi = q + 1; hi <= q + 3; ++hi) {
            // workgroups of class 1: the fewest that take the rest of product
            // 0, in eights, so that a tile number keeps its workgroup's XCD
            const int64_t k =
                std::max<int64_t>(0, (g0 - lo * cus + (hi - lo) - 1) / (hi - lo) + 7) / 8 * 8;
            if (k > cus)
                continue;
            for (int side = 0; side < 2; ++side) {
                const int64_t a = side ? hi : lo;
                int64_t b = lower > a * c0 ? (lower - a * c0 + c1 - 1) / c1 : 0;
                for (int t = 0; t < 4; ++t, ++b) {
                    const int64_t load = a * c0 + b * c1;
                    if (load < (k ? hi : lo) * c0 || (best && load >= best))
                        continue;
                    const int64_t b0 = (load - lo * c0) / c1, b1 = k ? (load - hi * c0) / c1 : 0;
                    if ((cus - k) * b0 + k * b1 < g1)
                        continue;
                    best = load;
                    W.split = (int)(cus - k);
                    W.n[0][0] = (int)lo;
                    W.n[0][1] = (int)b0;
                    W.n[1][0] = (int)hi;
                    W.n[1][1] = (int)b1;
                }
            }
        }
    return best;
}

// As mx_gemm_ring_pair_kernel, but product 1 on 64 x 64 tiles with K split over
// four waves: where it has few tiles and many steps (a gated backward's grad_Z,
// whose K is 2F), its workgroups' chains of steps are the launch's time, and here a
// quarter as long.  W.second_first: its tiles come first.
template <int ELEM, int OUT0>
__global__ void __launch_bounds__(R64x128::NT) mx_gemm_split_pair_kernel(RingPair W)
{
    using O = KSplitOp<G64x64, ELEM, 0>;
    static_assert(R64x128::NT == G64x64::NT, "one launch");
    constexpr int RING = R64x128::S * RingOp<R64x128, ELEM>::STAGE, PARTS = G64x64::NW * O::PART;
    __shared__ __attribute__((aligned(16))) uint8_t lds[RING > PARTS ? RING : PARTS];
    const int b = blockIdx.x;
    const int first = W.second_first ? W.n1 : W.n0;
    if ((b < first) == (W.second_first != 0))
        ksplit_tile<ELEM, MX_OUT_BF16, G64x64, 0>(W.p[1], (LDS_AS uint8_t *)lds, nullptr, nullptr,
                                                  W.second_first ? b : b - first);
    else
        ring_tiles<ELEM, OUT0, R64x128>(W.p[0], (LDS_AS uint8_t *)lds, W.second_first ? b - first : b, W.n0);
}

// How two products are computed: one launch each, or in one launch on 256 x
// 256 tiles shared out by load or on 64 x 128 tiles that are all resident at
// once, where that is 3% cheaper; or (where the caller allows sums in the order of
// K-split tiles) on 64 x 128 and K-split tiles.
enum PairMode { PAIR_APART, PAIR_LARGE, PAIR_SMALL, PAIR_SPLIT };
struct PairPlan {
    int mode;
    bool can_large;             // the shares of the large tiles were found
    double apart, large, small, split; // us; large, small or split = apart: not possible
    PairArgs W;
    RingPair Q, K; // small, split
};

inline void plan_pair(PairPlan &P, const Args &A0, const Args &A1, bool may_split)
{
    const int cus = A0.grid_max;
    P.apart = plan_product(A0.M, A0.N, A0.steps, cus).us + plan_product(A1.M, A1.N, A1.steps, cus).us;
    P.W.p[0] = A0;
    P.W.p[1] = A1;
    set_tiles(P.W.p[0], BM, BN, 1024);
    set_tiles(P.W.p[1], BM, BN, 1024);
    const int64_t load = pair_plan(P.W, cus);
    P.can_large = load != 0;
    P.large = load ? kCost[S_256x256].once + (double)load * kCost[S_256x256].step : P.apart;

    // two workgroups of 64 x 128 tiles per compute unit
    constexpr Cost c = kCost[S_R64x128];
    P.Q.p[0] = A0;
    P.Q.p[1] = A1;
    set_tiles(P.Q.p[0], c.bm, c.bn, 1024);
    set_tiles(P.Q.p[1], c.bm, c.bn, 1024);
    P.Q.n0 = P.Q.p[0].cells;
    P.Q.n1 = P.Q.p[1].cells;
    P.Q.second_first = A1.steps > A0.steps;
    P.small = P.apart;
    if ((int64_t)P.Q.n0 + P.Q.n1 <= 2 * (int64_t)cus) {
        const double steps = std::max((double)std::max(A0.steps, A1.steps),
                                      ((double)P.Q.n0 * A0.steps + (double)P.Q.n1 * A1.steps) / cus);
        P.small = c.once + c.round + 1.2 * steps * c.step; // two loads share the step
    }
    P.mode = P.small <= P.large && P.small < 0.97 * P.apart ? PAIR_SMALL
             : P.large < 0.97 * P.apart                     ? PAIR_LARGE
                                                            : PAIR_APART;

    // Product 1 on K-split tiles.  us of a compute unit: 0.45 and 0.3 for the
    // operands of a step of either tile at 55 GB/s, 0.6 of which the longer chain
    // of steps does not cover (1 us a step of a K-split wave, 0.5 of a ring).
    // On 56 sizes of T = 50 .. 3000, F = 512 .. 6144, d = 384 .. 3328 that it was not
    // fitted to the choice is 1.2% slower than the faster one on average and 12% at
    // most; without this launch 5.7% and 42%.  (With more than six tiles a compute
    // unit up to 25%.)  F = 2048, d = 768, E4M3, T = 1024: 23.8 -> 19.4 us; F = d =
    // 2048, T = 128 19.5 -> 15.9.
    P.K = P.Q;
    set_tiles(P.K.p[1], G64x64::BM, G64x64::BN, 1024);
    P.K.n1 = P.K.p[1].cells;
    const double own = (A1.steps + G64x64::NW - 1) / G64x64::NW, ring = 0.5 * A0.steps;
    P.K.second_first = own >= ring;
    const double bytes = (0.45 * P.K.n0 * A0.steps + 0.3 * P.K.n1 * A1.steps) / cus;
    P.split = 3.0 + 0.6 * bytes + std::max(own, ring);
    const double now = P.mode == PAIR_SMALL ? P.small : P.mode == PAIR_LARGE ? P.large : P.apart;
    if (may_split && (int64_t)P.K.n0 + P.K.n1 <= 6 * (int64_t)cus && P.split < now)
        P.mode = PAIR_SPLIT;
}

// Products 0 (output OUT0) and 1 (bf16 output) on one stream.
template <int ELEM, int OUT0>
hipError_t multiply_pair_as(const PairPlan &P, const Args &A0, const Args &A1, hipStream_t stream)
{
    if (P.mode == PAIR_SMALL) {
        hipLaunchKernelGGL((mx_gemm_ring_pair_kernel<ELEM, OUT0, R64x128>),
                           dim3((unsigned)(P.Q.n0 + P.Q.n1)), dim3(R64x128::NT), 0, stream, P.Q);
        return hipGetLastError();
    }
    if (P.mode == PAIR_SPLIT) {
        hipLaunchKernelGGL((mx_gemm_split_pair_kernel<ELEM, OUT0>), dim3((unsigned)(P.K.n0 + P.K.n1)),
                           dim3(R64x128::NT), 0, stream, P.K);
        return hipGetLastError();
    }
    if (P.mode == PAIR_LARGE) {
        hipLaunchKernelGGL((mx_gemm_pair_kernel<ELEM, OUT0>), dim3((unsigned)A0.grid_max), dim3(NT), 0,
                           stream, P.W);
        return hipGetLastError();
    }
    const hipError_t e = multiply<ELEM, MX_OUT_BF16>(A1, stream);
    return e != hipSuccess ? e : multiply<ELEM, OUT0>(A0, stream);
}

template <int ELEM, int OUT0>
hipError_t multiply_pair(const Args &A0, const Args &A1, bool may_split, hipStream_t stream)
{
    PairPlan P;
    plan_pair(P, A0, A1, may_split);
    return multiply_pair_as<ELEM, OUT0>(P, A0, A1, stream);
}

} // namespace mxg

// host side -------------------------------------------------------------------

namespace {

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// Compute units of the device `stream` runs on (the current device for the
// null stream), looked up once per device; 0 if unknown.
int compute_units(hipStream_t stream)
{
    static std::atomic<int> cache[64];
    int dev = -1;
    if (stream) {
        hipDevice_t hd;
        if (hipStreamGetDevice(static_cast<hipStream_t>(stream), &hd) != hipSuccess)
            return 0;
        dev = (int)hd;
    } else if (hipGetDevice(&dev) != hipSuccess) {
        return 0;
    }
    if (dev < 0 || dev >= 64)
        return 0;
    int n = cache[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
            n <= 0)
            return 0;
        cache[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

} // namespace

namespace mxg {

mx_status check_product(const Product &P, int block, int elem, int out_dtype)
{
    if (P.M < 0 || P.N < 0 || P.K <= 0)
        return mxk::fail(MX_EINVAL, "M and N must be >= 0 and K > 0");
    if (elem != MX_ELEM_E4M3 && elem != MX_ELEM_E2M1)
        return mxk::fail(MX_EINVAL, "elem must be MX_ELEM_E4M3 or MX_ELEM_E2M1");
    if (out_dtype != MX_OUT_F32 && out_dtype != MX_OUT_BF16)
        return mxk::fail(MX_EINVAL, "out_dtype must be MX_OUT_F32 or MX_OUT_BF16");
    if (block != 32)
        return mxk::fail(MX_EUNSUPPORTED, "the matrix cores apply one scale per 32 elements: block must be 32");
    const int64_t kstep = elem == MX_ELEM_E2M1 ? 256 : 128;
    if (P.K % kstep != 0)
        return mxk::fail(MX_EUNSUPPORTED, "K must be a multiple of 128 (E4M3) or 256 (E2M1)");
    if (P.N % 16 != 0)
        return mxk::fail(MX_EUNSUPPORTED, "N must be a multiple of 16");
    if (P.K > MX_MATMUL_MAX_K)
        return mxk::fail(MX_EUNSUPPORTED, "K exceeds %d", MX_MATMUL_MAX_K);
    if (P.M == 0 || P.N == 0)
        return MX_OK;
    if (!P.a || !P.as || !P.b || !P.bs || !P.out)
        return mxk::fail(MX_EINVAL, "NULL pointer");
    if (!aligned(P.a, 16) || !aligned(P.b, 16) || !aligned(P.as, 4) || !aligned(P.bs, 4) ||
        !aligned(P.out, 16) || (P.gain && !aligned(P.gain, 8)))
        return mxk::fail(MX_EINVAL, "codes and out must be 16-byte, scales 4-byte and b_gain "
                               "8-byte aligned");
    const int64_t tm = (P.M + BM - 1) / BM, tn = (P.N + BN - 1) / BN;
    if (tm * tn > INT32_MAX / 2 || P.M > INT32_MAX || P.N > MX_MATMUL_MAX_N)
        return mxk::fail(MX_EUNSUPPORTED, "problem too large (N at most %d)", MX_MATMUL_MAX_N);
    return MX_OK;
}

} // namespace mxg

namespace mxg {

void product_args(Args &A, const Product &P, int elem, hipStream_t stream)
{
    A.a = P.a;
    A.as = P.as;
    A.b = P.b;
    A.bs = P.bs;
    A.bgain = static_cast<const uint16_t *>(P.gain);
    A.out = P.out;
    A.M = P.M;
    A.N = P.N;
    A.rb = elem == MX_ELEM_E2M1 ? P.K / 2 : P.K;
    A.rs = P.K / 32;
    A.steps = (int)(A.rb / KB);
    const int cus = compute_units(stream);
    A.grid_max = cus > 0 ? cus : 256;
}

} // namespace mxg

extern "C" {

mx_status mx_matmul_fwd(const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *b_codes,
                        const uint8_t *b_scales, int64_t M, int64_t N, int64_t K, int block,
                        int elem, const void *b_gain, int out_dtype, void *out, hipStream_t stream)
{
    mxk::clear_error();
    const mxg::Product P{a_codes, a_scales, b_codes, b_scales, M, N, K, b_gain, out};
    const mx_status ok = mxg::check_product(P, block, elem, out_dtype);
    if (ok != MX_OK || M == 0 || N == 0)
        return ok;
    mxg::Args A;
    mxg::product_args(A, P, elem, stream);
    hipStream_t st = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (elem == MX_ELEM_E4M3)
        e = out_dtype == MX_OUT_F32 ? mxg::multiply<MX_ELEM_E4M3, MX_OUT_F32>(A, st)
                                         : mxg::multiply<MX_ELEM_E4M3, MX_OUT_BF16>(A, st);
    else
        e = out_dtype == MX_OUT_F32 ? mxg::multiply<MX_ELEM_E2M1, MX_OUT_F32>(A, st)
                                         : mxg::multiply<MX_ELEM_E2M1, MX_OUT_BF16>(A, st);
    if (e != hipSuccess)
        return mxk::fail(MX_EHIP, "kernel launch failed: %s", hipGetErrorString(e));
    return MX_OK;
}

} // extern "C"

namespace mxg {

mx_status matmul_pair(const Product &first, int out0, const Product &bf16, int elem, bool may_split,
                      hipStream_t stream)
{
    Args A0, A1;
    product_args(A0, first, elem, stream);
    product_args(A1, bf16, elem, stream);
    hipError_t e;
    if (elem == MX_ELEM_E4M3)
        e = out0 == MX_OUT_F32 ? multiply_pair<MX_ELEM_E4M3, MX_OUT_F32>(A0, A1, may_split, stream)
                               : multiply_pair<MX_ELEM_E4M3, MX_OUT_BF16>(A0, A1, may_split, stream);
    else
        e = out0 == MX_OUT_F32 ? multiply_pair<MX_ELEM_E2M1, MX_OUT_F32>(A0, A1, may_split, stream)
                               : multiply_pair<MX_ELEM_E2M1, MX_OUT_BF16>(A0, A1, may_split, stream);
    return e == hipSuccess ? MX_OK
                           : mxk::fail(MX_EHIP, "kernel launch failed: %s", hipGetErrorString(e));
}

} // namespace mxg

// ---------------------------------------------------- for the library's tests --

namespace {

bool known_shape(int s) { return s >= 0 && s < mxg::S_COUNT; }

template <int ELEM>
hipError_t multiply_as(const mxg::Plan &P, const mxg::Args &A, int out_dtype, hipStream_t stream)
{
    return out_dtype == MX_OUT_F32 ? mxg::multiply_as<ELEM, MX_OUT_F32>(P, A, stream)
                                   : mxg::multiply_as<ELEM, MX_OUT_BF16>(P, A, stream);
}

// M, N and the K steps alone: what the plans depend on.
bool plan_args(mxg::Args &A, int64_t M, int64_t N, int64_t K, int elem, int units)
{
    const int64_t rb = elem == MX_ELEM_E2M1 ? K / 2 : K;
    if (M <= 0 || N <= 0 || K <= 0 || rb % mxg::KB != 0 || units <= 0)
        return false;
    A = mxg::Args{};
    A.M = M;
    A.N = N;
    A.steps = (int)(rb / mxg::KB);
    A.grid_max = units;
    return true;
}

} // namespace

extern "C" {

int mxt_product_plan(int64_t M, int64_t N, int64_t K, int elem, int units, int *whole, int *tail,
                     double *us)
{
    mxg::Args A;
    if (!plan_args(A, M, N, K, elem, units))
        return -1;
    const mxg::Plan P = mxg::plan_product(M, N, A.steps, units);
    *whole = P.whole;
    *tail = P.tail;
    *us = P.us;
    return P.shape;
}

int mxt_gated_pair_plan(int64_t M0, int64_t N0, int64_t K0, int64_t M1, int64_t N1, int64_t K1,
                        int elem, int units)
{
    mxg::Args A0, A1;
    if (!plan_args(A0, M0, N0, K0, elem, units) || !plan_args(A1, M1, N1, K1, elem, units))
        return -1;
    mxg::PairPlan P;
    mxg::plan_pair(P, A0, A1, true);
    return P.mode;
}

int mxt_pair_plan(int64_t M0, int64_t N0, int64_t K0, int64_t M1, int64_t N1, int64_t K1, int elem,
                  int units, double *us)
{
    mxg::Args A0, A1;
    if (!plan_args(A0, M0, N0, K0, elem, units) || !plan_args(A1, M1, N1, K1, elem, units))
        return -1;
    mxg::PairPlan P;
    mxg::plan_pair(P, A0, A1, false);
    us[0] = P.apart;
    us[1] = P.large;
    us[2] = P.small;
    return P.mode;
}

mx_status mxt_matmul(const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *b_codes,
                     const uint8_t *b_scales, int64_t M, int64_t N, int64_t K, int elem,
                     const void *b_gain, int out_dtype, void *out, int shape, int whole, int units,
                     hipStream_t stream)
{
    mxk::clear_error();
    const mxg::Product P0{a_codes, a_scales, b_codes, b_scales, M, N, K, b_gain, out};
    const mx_status ok = mxg::check_product(P0, 32, elem, out_dtype);
    if (ok != MX_OK || M == 0 || N == 0)
        return ok;
    mxg::Args A;
    mxg::product_args(A, P0, elem, stream);
    const int64_t cells = ((M + mxg::BM - 1) / mxg::BM) * ((N + mxg::BN - 1) / mxg::BN);
    if (!known_shape(shape) || whole < 0 || whole >= cells || units < 0 || units > A.grid_max)
        return mxk::fail(MX_EINVAL, "no such tile shape, first launch or number of units");
    if (units)
        A.grid_max = units;
    const mxg::Plan P{whole ? (int)mxg::S_256x256 : shape, whole, shape, 0.0};
    const hipError_t e = elem == MX_ELEM_E4M3 ? multiply_as<MX_ELEM_E4M3>(P, A, out_dtype, stream)
                                              : multiply_as<MX_ELEM_E2M1>(P, A, out_dtype, stream);
    return e == hipSuccess ? MX_OK
                           : mxk::fail(MX_EHIP, "kernel launch failed: %s", hipGetErrorString(e));
}

mx_status mxt_matmul_pair(const MxtProduct *f32, const MxtProduct *bf16, int elem, int mode,
                          int units, hipStream_t stream)
{
    mxk::clear_error();
    const mxg::Product p0{f32->a, f32->as, f32->b, f32->bs, f32->M, f32->N, f32->K, f32->gain, f32->out};
    const mxg::Product p1{bf16->a, bf16->as, bf16->b, bf16->bs, bf16->M, bf16->N, bf16->K, bf16->gain,
                          bf16->out};
    mx_status ok = mxg::check_product(p0, 32, elem, MX_OUT_F32);
    if (ok == MX_OK)
        ok = mxg::check_product(p1, 32, elem, MX_OUT_BF16);
    if (ok != MX_OK)
        return ok;
    mxg::Args A0, A1;
    mxg::product_args(A0, p0, elem, stream);
    mxg::product_args(A1, p1, elem, stream);
    if (f32->M == 0 || f32->N == 0 || bf16->M == 0 || bf16->N == 0 || units < 0 ||
        units > A0.grid_max)
        return mxk::fail(MX_EINVAL, "empty product, or no such number of units");
    if (units)
        A0.grid_max = A1.grid_max = units;
    mxg::PairPlan P;
    mxg::plan_pair(P, A0, A1, false);
    if (mode < 0 || mode > mxg::PAIR_SPLIT || (mode == mxg::PAIR_LARGE && !P.can_large))
        return mxk::fail(MX_EINVAL, "no such pair launch");
    P.mode = mode;
    const hipError_t e = elem == MX_ELEM_E4M3
                             ? mxg::multiply_pair_as<MX_ELEM_E4M3, MX_OUT_F32>(P, A0, A1, stream)
                             : mxg::multiply_pair_as<MX_ELEM_E2M1, MX_OUT_F32>(P, A0, A1, stream);
    return e == hipSuccess ? MX_OK
                           : mxk::fail(MX_EHIP, "kernel launch failed: %s", hipGetErrorString(e));
}

} // extern "C"

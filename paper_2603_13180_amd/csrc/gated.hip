// gated.hip -- the gated feed-forward's first half (mx_gated_fwd): the two
// projections that share an operand, activation and product in one kernel.
//
// The gate and up products of a column are two columns of an ordinary MX
// product with W [2F, K].  A tile that takes its B rows half from the gate
// rows and half from the same up rows holds both products of its columns in
// one wave's accumulators, so the product kernels (mx_gemm_256.h, _ring.h,
// _ksplit.h) serve unchanged but for the rows they load and what they store
// (mx_gemm_gated.h).  The operand stream and the matrix instructions are those
// of the plain product; what is saved is G and U, 8 F bytes a row written and
// read again, or their rounding to bf16 and 4 F.  What bounds it is what bounds
// the product: 8192 x 2 14336 x 4096, bf16 out, E4M3 800 us against 807 for the
// plain product of as many columns, E2M1 486 against 522 (it writes twice as much);
// a decoding step's weights, 1 x 2 14336 x 4096 E4M3, 21 us with the norm, 5.7 TB/s.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "gate.h"
#include "mx_gemm_gated.h"
#include "mx_gemm_plan.h"
#include "mxnorm.h"
#include "products.h"
#include "status.h"
#include "testing.h"

namespace {

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

void gated_args(mxg::GatedArgs &A, const mxg::GatedProduct &P, int elem, hipStream_t stream)
{
    mxg::product_args(A, {P.a, P.as, P.w, P.ws, P.M, P.F, P.K, nullptr, P.out}, elem, stream);
    A.hs = P.out_scales;
    A.gu = static_cast<uint16_t *>(P.gu);
    A.act = P.act;
    A.mode = P.mode;
}

// f(ELEM, OUT of the kernels) for the call's types
template <class F> hipError_t by_type(int elem, int out_dtype, F f)
{
    using namespace mxg;
    auto out = [&](auto e) {
        switch (out_dtype) {
        case MX_OUT_F32: return f(e, std::integral_constant<int, kGate + MX_OUT_F32>{});
        case MX_OUT_BF16: return f(e, std::integral_constant<int, kGate + MX_OUT_BF16>{});
        default: return f(e, std::integral_constant<int, kGate + MX_OUT_CODES>{});
        }
    };
    return elem == MX_ELEM_E4M3 ? out(std::integral_constant<int, MX_ELEM_E4M3>{})
                                : out(std::integral_constant<int, MX_ELEM_E2M1>{});
}

mx_status launched(hipError_t e)
{
    return e == hipSuccess ? MX_OK
                           : mxk::fail(MX_EHIP, "kernel launch failed: %s", hipGetErrorString(e));
}

} // namespace

namespace mxg {

mx_status check_gated(const GatedProduct &P, int block, int elem)
{
    if (P.M < 0 || P.F < 0 || P.K <= 0)
        return mxk::fail(MX_EINVAL, "M and F must be >= 0 and K > 0");
    if (elem != MX_ELEM_E4M3 && elem != MX_ELEM_E2M1)
        return mxk::fail(MX_EINVAL, "elem must be MX_ELEM_E4M3 or MX_ELEM_E2M1");
    if (P.act != MX_ACT_SILU && P.act != MX_ACT_GELU_TANH)
        return mxk::fail(MX_EINVAL, "act must be MX_ACT_SILU or MX_ACT_GELU_TANH");
    if (P.out_dtype != MX_OUT_F32 && P.out_dtype != MX_OUT_BF16 && P.out_dtype != MX_OUT_CODES)
        return mxk::fail(MX_EINVAL, "out_dtype must be MX_OUT_F32, MX_OUT_BF16 or MX_OUT_CODES");
    if (P.mode != MX_SCALE_RCEIL && P.mode != MX_SCALE_FLOOR)
        return mxk::fail(MX_EINVAL, "unknown scale_mode %d", P.mode);
    if (block != 32)
        return mxk::fail(MX_EUNSUPPORTED, "the matrix cores apply one scale per 32 elements: block must be 32");
    if (P.K % (elem == MX_ELEM_E2M1 ? 256 : 128) != 0)
        return mxk::fail(MX_EUNSUPPORTED, "K must be a multiple of 128 (E4M3) or 256 (E2M1)");
    if (P.F % (P.out_dtype == MX_OUT_CODES ? 32 : 16) != 0)
        return mxk::fail(MX_EUNSUPPORTED, "F must be a multiple of 16, or of 32 for MX_OUT_CODES");
    if (P.K > MX_MATMUL_MAX_K)
        return mxk::fail(MX_EUNSUPPORTED, "K exceeds %d", MX_MATMUL_MAX_K);
    if (P.M == 0 || P.F == 0)
        return MX_OK;
    if (!P.a || !P.as || !P.w || !P.ws || !P.out)
        return mxk::fail(MX_EINVAL, "NULL pointer");
    if ((P.out_dtype == MX_OUT_CODES) != (P.out_scales != nullptr))
        return mxk::fail(MX_EINVAL, "out_scales goes with MX_OUT_CODES, and with it alone");
    if (!aligned(P.a, 16) || !aligned(P.w, 16) || !aligned(P.as, 4) || !aligned(P.ws, 4) ||
        !aligned(P.out, 16) || !aligned(P.gu, 16))
        return mxk::fail(MX_EINVAL, "codes, out and gu must be 16-byte, operand scales 4-byte aligned");
    if (P.M > INT32_MAX || P.F > MX_MATMUL_MAX_N / 2 ||
        ((P.M + BM - 1) / BM) * ((2 * P.F + BN - 1) / BN) > INT32_MAX / 2)
        return mxk::fail(MX_EUNSUPPORTED, "problem too large (F at most %d)", MX_MATMUL_MAX_N / 2);
    return MX_OK;
}

mx_status check_gated_bwd(const void *grad_h, const void *gu, int64_t T, int64_t F, int act,
                          const void *grad_gu)
{
    if (T < 0 || F < 0)
        return mxk::fail(MX_EINVAL, "T and F must be >= 0");
    if (act != MX_ACT_SILU && act != MX_ACT_GELU_TANH)
        return mxk::fail(MX_EINVAL, "act must be MX_ACT_SILU or MX_ACT_GELU_TANH");
    if (F % 8 != 0)
        return mxk::fail(MX_EINVAL, "F must be a multiple of 8");
    if (T > INT32_MAX || F > MX_MATMUL_MAX_N / 2)
        return mxk::fail(MX_EUNSUPPORTED, "matrix too large (F at most %d)", MX_MATMUL_MAX_N / 2);
    if (T == 0 || F == 0)
        return MX_OK;
    if (!grad_h || !gu || !grad_gu)
        return mxk::fail(MX_EINVAL, "grad_h, gu and grad_gu must be non-NULL");
    if (!aligned(grad_h, 16) || !aligned(gu, 16) || !aligned(grad_gu, 16))
        return mxk::fail(MX_EINVAL, "grad_h, gu and grad_gu must be 16-byte aligned");
    return MX_OK;
}

// The chunks a lane needs (4 or 8) if a product of M rows takes the tile that can
// norm them, and they fit; else 0.
static int fits_normed(int64_t M, int64_t F, int steps, int elem, int units)
{
    auto fits = [&](auto nch) {
        constexpr int N = decltype(nch)::value;
        return elem == MX_ELEM_E2M1 ? Normed<MX_ELEM_E2M1, G16x64::NW, N>::fits(M, steps)
                                    : Normed<MX_ELEM_E4M3, G16x64::NW, N>::fits(M, steps);
    };
    const int n = fits(std::integral_constant<int, 4>{}) ? 4 : fits(std::integral_constant<int, 8>{}) ? 8 : 0;
    if (n == 0)
        return 0;
    const Plan plan = plan_gated(M, F, steps, units);
    return plan.shape == S_G16x64 && !plan.whole ? n : 0;
}

bool normed_product(const GatedProduct &P, const RowNorm &n, int elem, hipStream_t stream, mx_status &st)
{
    NormedArgs A;
    gated_args(A, P, elem, stream);
    const int chunks = fits_normed(P.M, P.F, A.steps, elem, A.grid_max);
    if (chunks == 0)
        return false;
    A.x = static_cast<const uint16_t *>(n.x);
    A.rho = n.rho;
    A.p = n.p;
    A.coef = n.coef;
    A.eps = n.eps;
    set_tiles(A, G16x64::BM, G16x64::BN / 2, 1024);
    A.once = read_once(A, S_G16x64);
    st = launched(by_type(elem, P.out_dtype, [&](auto e, auto o) {
        constexpr int E = decltype(e)::value, O = decltype(o)::value;
        return chunks == 4 ? launch_ksplit<E, O, G16x64, 4>(A, stream) : launch_ksplit<E, O, G16x64, 8>(A, stream);
    }));
    return true;
}

// The gradients of both projections, bf16 [T, 2F] from grad_h [T, F] and the
// kept products [T, 2F]: a lane takes 8 columns of a row.  HBM bound: [8192, 14336]
// 183 us, 6.4 TB/s of its 10 bytes a column.
template <int ACT>
__global__ void __launch_bounds__(256) gated_bwd_kernel(const uint16_t *gh, const uint16_t *gu,
                                                        uint16_t *out, int64_t T, int64_t F)
{
    const int64_t per = F / 8, n = T * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / per, at = t * 2 * F + 8 * (i - t * per);
        const uint4 h = mxk::load_stream(reinterpret_cast<const uint4 *>(gh) + i);
        const uint4 g = mxk::load_stream(reinterpret_cast<const uint4 *>(gu + at));
        const uint4 u = mxk::load_stream(reinterpret_cast<const uint4 *>(gu + at + F));
        uint4 dg, du;
        mxk::gate_gradients<ACT>(g, u, h, dg, du);
        __builtin_nontemporal_store(mxk::u32x4_t{dg.x, dg.y, dg.z, dg.w},
                                    reinterpret_cast<mxk::u32x4_t *>(out + at));
        __builtin_nontemporal_store(mxk::u32x4_t{du.x, du.y, du.z, du.w},
                                    reinterpret_cast<mxk::u32x4_t *>(out + at + F));
    }
}

} // namespace mxg

extern "C" {

mx_status mx_gated_fwd(const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *w_codes,
                       const uint8_t *w_scales, int64_t M, int64_t F, int64_t K, int block,
                       int elem, int act, int scale_mode, int out_dtype, void *out,
                       uint8_t *out_scales, void *gu, hipStream_t stream)
{
    mxk::clear_error();
    const mxg::GatedProduct P{a_codes, a_scales, w_codes, w_scales,  M,   F,
                              K,       act,      scale_mode, out_dtype, out, out_scales, gu};
    const mx_status ok = mxg::check_gated(P, block, elem);
    if (ok != MX_OK || M == 0 || F == 0)
        return ok;
    mxg::GatedArgs A;
    gated_args(A, P, elem, stream);
    return launched(by_type(elem, out_dtype, [&](auto e, auto o) {
        return mxg::multiply<decltype(e)::value, decltype(o)::value>(A, stream);
    }));
}

mx_status mx_gated_bwd(const void *grad_h, const void *gu, int64_t T, int64_t F, int act,
                       void *grad_gu, hipStream_t stream)
{
    mxk::clear_error();
    const mx_status ok = mxg::check_gated_bwd(grad_h, gu, T, F, act, grad_gu);
    if (ok != MX_OK || T == 0 || F == 0)
        return ok;
    const unsigned grid = (unsigned)std::min<int64_t>((T * (F / 8) + 255) / 256, 1 << 20);
    const auto *h = static_cast<const uint16_t *>(grad_h), *p = static_cast<const uint16_t *>(gu);
    auto *o = static_cast<uint16_t *>(grad_gu);
    if (act == MX_ACT_SILU)
        hipLaunchKernelGGL((mxg::gated_bwd_kernel<MX_ACT_SILU>), dim3(grid), dim3(256), 0, stream, h, p, o, T, F);
    else
        hipLaunchKernelGGL((mxg::gated_bwd_kernel<MX_ACT_GELU_TANH>), dim3(grid), dim3(256), 0, stream, h, p, o,
                           T, F);
    return launched(hipGetLastError());
}

int mxt_gated_plan(int64_t M, int64_t F, int64_t K, int elem, int units, int *whole, int *tail,
                   double *us)
{
    const int64_t rb = elem == MX_ELEM_E2M1 ? K / 2 : K;
    if (M <= 0 || F <= 0 || K <= 0 || rb % mxg::KB != 0 || units <= 0)
        return -1;
    const mxg::Plan P = mxg::plan_gated(M, F, (int)(rb / mxg::KB), units);
    *whole = P.whole;
    *tail = P.tail;
    *us = P.us;
    return P.shape;
}

int mxt_gated_once(int64_t M, int64_t F, int64_t K, int elem, int units)
{
    if (M <= 0 || F <= 0 || K <= 0 || units <= 0)
        return -1;
    mxg::GatedArgs A{};
    A.M = M;
    A.N = F;
    A.rb = elem == MX_ELEM_E2M1 ? K / 2 : K;
    A.steps = (int)(A.rb / mxg::KB);
    const mxg::Plan P = mxg::plan_gated(M, F, A.steps, units);
    return mxg::read_once(A, P.shape) + (P.whole && mxg::read_once(A, P.tail) ? 2 : 0);
}

int mxt_gated_normed(int64_t M, int64_t F, int64_t K, int elem, int units)
{
    const int64_t rb = elem == MX_ELEM_E2M1 ? K / 2 : K;
    return M > 0 && F > 0 && K > 0 && units > 0 ? mxg::fits_normed(M, F, (int)(rb / mxg::KB), elem, units) : 0;
}

mx_status mxt_gated(const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *w_codes,
                    const uint8_t *w_scales, int64_t M, int64_t F, int64_t K, int elem, int act,
                    int scale_mode, int out_dtype, void *out, uint8_t *out_scales, void *gu,
                    int shape, int whole, int units, hipStream_t stream)
{
    mxk::clear_error();
    const mxg::GatedProduct P{a_codes, a_scales, w_codes, w_scales,  M,   F,
                              K,       act,      scale_mode, out_dtype, out, out_scales, gu};
    const mx_status ok = mxg::check_gated(P, 32, elem);
    if (ok != MX_OK || M == 0 || F == 0)
        return ok;
    mxg::GatedArgs A;
    gated_args(A, P, elem, stream);
    const int64_t cells = ((M + mxg::BM - 1) / mxg::BM) * ((2 * F + mxg::BN - 1) / mxg::BN);
    bool known = shape == mxg::S_256x256;
    for (const int s : mxg::kGatedShapes)
        known = known || s == shape;
    if (!known || whole < 0 || whole >= cells || (whole && shape == mxg::S_256x256) || units < 0 ||
        units > A.grid_max)
        return mxk::fail(MX_EINVAL, "no such tile shape, first launch or number of units");
    if (units)
        A.grid_max = units;
    const mxg::Plan plan{whole ? (int)mxg::S_256x256 : shape, whole, shape, 0.0};
    return launched(by_type(elem, out_dtype, [&](auto e, auto o) {
        return mxg::multiply_as<decltype(e)::value, decltype(o)::value>(plan, A, stream);
    }));
}

} // extern "C"

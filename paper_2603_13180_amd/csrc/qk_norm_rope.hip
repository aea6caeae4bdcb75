// qk_norm_rope.hip -- RMSNorm of every query and key head and the rotation of
// its first R elements by the token's position, forward and backward, straight
// from the fused projection's output.
//
// Per head x of D elements with gain gamma, r = ((1/D) sum x^2 + eps)^(-1/2):
//   n = (x r) gamma;  y = n with each pair (a, b) of the first R turned by the
//   angle t_i = pos inv_freq[i]:  (a cos t - b sin t, b cos t + a sin t).
// Backward, from the gradient of y: m = that gradient turned back,
//   v = gamma m,  u = sum v x,  grad_x = r v - (r^3 u / D) x,
//   grad_gamma = sum over tokens and heads of (r x) m.
//
// A lane holds the two 16-byte chunks of a head whose elements are paired
// (chunks l and l + R/16 of the rotated part, two chunks of the rest), so a
// pair never crosses lanes, and a head is a group of G = 4 .. 32 lanes; a wave
// takes 64 / G heads of one token.  An angle costs a double product and a
// sine, and every head of the token needs it: the workgroup computes its
// tokens' angles once into LDS.  HBM bound: 4 bytes an element forward, 6
// backward.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "mxnorm.h"
#include "norm_cast.h"
#include "status.h"

#pragma clang fp contract(off)

namespace mxq {

using namespace mxk;

constexpr int NT = 256, NW = NT / 64;
constexpr int MAX_D = 512;
constexpr int TOKENS = 4; // tokens whose angles a workgroup holds at once

struct Heads {
    const uint16_t *in;  // x
    const uint16_t *gy;  // backward: the gradient of the output
    uint16_t *out;       // y, or grad_x
    const uint16_t *gamma;
    int64_t in_t, in_h, gy_t, gy_h, out_t, out_h; // strides, elements
    int heads, blocks;   // blocks of 64 / G heads
};

struct Args {
    Heads q, k;
    const int64_t *pos;    // NULL: 0, 1, ...
    const float *inv_freq; // [R/2]
    float *part;           // backward: [workgroups][2][D] gain gradients, or NULL
    int64_t T;
    int D, R, tb;          // tb: tokens a workgroup takes at a time
    float eps;
    double inv_d; // 1 / D
};

// lanes that hold a head's chunks
__host__ __device__ inline int lanes_of(int D, int R) { return R / 16 + (D - R + 15) / 16; }

// The two chunks of lane l; the second may lie past the head (an odd number of
// chunks that do not turn).
__device__ __forceinline__ void chunks_of(int D, int R, int l, int &a, int &b)
{
    const int rot = R / 16;
    if (l < rot) {
        a = l;
        b = l + rot;
    } else {
        a = R / 8 + l - rot;
        b = a + (D - R + 15) / 16;
    }
}

// cos and sin of the workgroup's tokens' angles, eight a rotated lane: those
// of its elements 0 .. 7 (halves: element e of chunk a with element e of chunk
// b) or of the pairs (2i, 2i + 1) of chunk a, then of chunk b.  The angle in
// turns is formed in double, so that far positions keep their angle, and only
// its fraction is rounded to float.
template <bool INTER>
__device__ __forceinline__ void fill_angles(const Args &A, int64_t t0, int nt, float *cs, float *sn)
{
    const int half = A.R / 2;
    for (int i = threadIdx.x; i < nt * half; i += NT) {
        const int t = i / half, p = i - t * half; // p = 8 l + e
        const int l = p >> 3, e = p & 7;
        const int pair = !INTER ? p : e < 4 ? 4 * l + e : A.R / 4 + 4 * l + e - 4;
        const int64_t pos = A.pos ? A.pos[t0 + t] : t0 + t;
        const double turns = (double)pos * (double)A.inv_freq[pair] * 0.15915494309189535;
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        cs[i] = c;
        sn[i] = s;
    }
}

// Sum over the G lanes of a head, in every lane the same bits.
template <int G> __device__ __forceinline__ double head_sum(double s)
{
    s += dpp_f64<0xB1>(s);
    s += dpp_f64<0x4E>(s);
    if constexpr (G >= 8)
        s += dpp_f64<0x141>(s);
    if constexpr (G >= 16)
        s += dpp_f64<0x140>(s);
    if constexpr (G >= 32)
        s += __shfl_xor(s, 16);
    return s;
}

// (S / D + eps)^(-1/2), 0 for a radicand that is zero or infinite: the
// hardware's estimate and one Newton step in double, rounded to float.
__device__ __forceinline__ float inverse_rms(double S, double inv_d, float eps)
{
    const double u = S * inv_d + (double)eps;
    const double y = __builtin_amdgcn_rsq(u);
    const double z = __builtin_fma(y, __builtin_fma(-0.5 * u * y, y, 0.5), y);
    return u == 0.0 || u == INFINITY ? 0.0f : (float)z;
}

struct Chunk {
    float v[8];
};

__device__ __forceinline__ Chunk widen(uint4 w)
{
    return {{bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y), bf16_lo(w.z), bf16_hi(w.z),
             bf16_lo(w.w), bf16_hi(w.w)}};
}

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const __bf16 x = (__bf16)a, y = (__bf16)b;
    return (uint32_t)__builtin_bit_cast(uint16_t, x) | ((uint32_t)__builtin_bit_cast(uint16_t, y) << 16);
}

__device__ __forceinline__ uint4 narrow(const Chunk &c)
{
    return make_uint4(pack2(c.v[0], c.v[1]), pack2(c.v[2], c.v[3]), pack2(c.v[4], c.v[5]),
                      pack2(c.v[6], c.v[7]));
}

// Turn the lane's pairs by its angles, or (BACK) by their negatives.
template <bool INTER, bool BACK>
__device__ __forceinline__ void turn(Chunk &a, Chunk &b, const float *cs, const float *sn)
{
    auto one = [](float &x, float &y, float c, float s) {
        if (BACK)
            s = -s;
        const float t = __builtin_fmaf(x, c, -(y * s));
        y = __builtin_fmaf(y, c, x * s);
        x = t;
    };
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (!INTER)
            one(a.v[e], b.v[e], cs[e], sn[e]);
        else if (e < 4)
            one(a.v[2 * e], a.v[2 * e + 1], cs[e], sn[e]);
        else
            one(b.v[2 * e - 8], b.v[2 * e - 7], cs[e], sn[e]);
    }
}

__device__ __forceinline__ uint4 load16(const uint16_t *p, bool in)
{
    return in ? load_stream(reinterpret_cast<const uint4 *>(p)) : make_uint4(0, 0, 0, 0);
}

__device__ __forceinline__ void store16(uint16_t *p, const uint4 &v)
{
    __builtin_nontemporal_store(u32x4_t{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4_t *>(p));
}

// A lane's place in its head and the gains of its chunks.
template <int G> struct Lane {
    int l, sub, ca, cb;
    bool in_a, in_b, rot;
    __device__ Lane(const Args &A)
    {
        const int lane = threadIdx.x & 63;
        l = lane % G;
        sub = lane / G;
        chunks_of(A.D, A.R, l, ca, cb);
        in_a = l < lanes_of(A.D, A.R);
        in_b = in_a && 8 * cb < A.D;
        rot = l < A.R / 16;
    }
    __device__ void gains(const uint16_t *gamma, uint4 &ga, uint4 &gb) const
    {
        const uint32_t one = 0x3F803F80u;
        ga = gb = make_uint4(one, one, one, one);
        if (gamma && in_a)
            ga = *reinterpret_cast<const uint4 *>(gamma + 8 * ca);
        if (gamma && in_b)
            gb = *reinterpret_cast<const uint4 *>(gamma + 8 * cb);
    }
};

template <int G, bool INTER> __global__ void __launch_bounds__(NT) fwd_kernel(Args A)
{
    __shared__ float cs[TOKENS * MAX_D / 2], sn[TOKENS * MAX_D / 2];
    const int w = threadIdx.x >> 6, half = A.R / 2;
    const Lane<G> L(A);
    uint4 gq[2], gk[2];
    L.gains(A.q.gamma, gq[0], gq[1]);
    L.gains(A.k.gamma, gk[0], gk[1]);
    const int per = A.q.blocks + A.k.blocks;
    for (int64_t t0 = (int64_t)blockIdx.x * A.tb; t0 < A.T; t0 += (int64_t)gridDim.x * A.tb) {
        const int nt = (int)min((int64_t)A.tb, A.T - t0);
        __syncthreads(); // the angles of the tokens before are read
        fill_angles<INTER>(A, t0, nt, cs, sn);
        __syncthreads();
        for (int i = w; i < nt * per; i += NW) {
            const int t = i / per, blk = i - t * per;
            const bool key = blk >= A.q.blocks;
            const Heads &H = key ? A.k : A.q;
            const int h = (key ? blk - A.q.blocks : blk) * (64 / G) + L.sub;
            const bool on = h < H.heads;
            const uint16_t *x = H.in + (t0 + t) * H.in_t + h * H.in_h;
            Chunk a = widen(load16(x + 8 * L.ca, on && L.in_a));
            Chunk b = widen(load16(x + 8 * L.cb, on && L.in_b));
            double S = 0.0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                S = __builtin_fma((double)a.v[e], (double)a.v[e], S);
                S = __builtin_fma((double)b.v[e], (double)b.v[e], S);
            }
            const float r = inverse_rms(head_sum<G>(S), A.inv_d, A.eps);
            const Chunk ga = widen(key ? gk[0] : gq[0]), gb = widen(key ? gk[1] : gq[1]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                a.v[e] = a.v[e] * r * ga.v[e];
                b.v[e] = b.v[e] * r * gb.v[e];
            }
            if (L.rot)
                turn<INTER, false>(a, b, cs + t * half + 8 * L.l, sn + t * half + 8 * L.l);
            uint16_t *y = H.out + (t0 + t) * H.out_t + h * H.out_h;
            if (on && L.in_a)
                store16(y + 8 * L.ca, narrow(a));
            if (on && L.in_b)
                store16(y + 8 * L.cb, narrow(b));
        }
    }
}

// As the forward; each lane also keeps the gain gradients of its chunks, of
// queries and of keys, in float over its heads.  At the end the workgroup's
// lanes are added in a fixed order into its row of the partial sums.
template <int G, bool INTER> __global__ void __launch_bounds__(NT) bwd_kernel(Args A)
{
    __shared__ float cs[TOKENS * MAX_D / 2], sn[TOKENS * MAX_D / 2];
    __shared__ float red[NW * 64 / G][16 * G]; // D <= 16 G
    const int w = threadIdx.x >> 6, half = A.R / 2;
    const Lane<G> L(A);
    uint4 gq[2], gk[2];
    L.gains(A.q.gamma, gq[0], gq[1]);
    L.gains(A.k.gamma, gk[0], gk[1]);
    float sum[2][16] = {};
    const int per = A.q.blocks + A.k.blocks;
    for (int64_t t0 = (int64_t)blockIdx.x * A.tb; t0 < A.T; t0 += (int64_t)gridDim.x * A.tb) {
        const int nt = (int)min((int64_t)A.tb, A.T - t0);
        __syncthreads();
        fill_angles<INTER>(A, t0, nt, cs, sn);
        __syncthreads();
        for (int i = w; i < nt * per; i += NW) {
            const int t = i / per, blk = i - t * per;
            const bool key = blk >= A.q.blocks;
            const Heads &H = key ? A.k : A.q;
            const int h = (key ? blk - A.q.blocks : blk) * (64 / G) + L.sub;
            const bool on = h < H.heads;
            const uint16_t *x = H.in + (t0 + t) * H.in_t + h * H.in_h;
            const uint16_t *gy = H.gy + (t0 + t) * H.gy_t + h * H.gy_h;
            const Chunk a = widen(load16(x + 8 * L.ca, on && L.in_a));
            const Chunk b = widen(load16(x + 8 * L.cb, on && L.in_b));
            Chunk ma = widen(load16(gy + 8 * L.ca, on && L.in_a));
            Chunk mb = widen(load16(gy + 8 * L.cb, on && L.in_b));
            if (L.rot)
                turn<INTER, true>(ma, mb, cs + t * half + 8 * L.l, sn + t * half + 8 * L.l);
            const Chunk ga = widen(key ? gk[0] : gq[0]), gb = widen(key ? gk[1] : gq[1]);
            Chunk va, vb;
            double S = 0.0, u = 0.0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                va.v[e] = ma.v[e] * ga.v[e];
                vb.v[e] = mb.v[e] * gb.v[e];
                S = __builtin_fma((double)a.v[e], (double)a.v[e], S);
                S = __builtin_fma((double)b.v[e], (double)b.v[e], S);
                u = __builtin_fma((double)a.v[e], (double)va.v[e], u);
                u = __builtin_fma((double)b.v[e], (double)vb.v[e], u);
            }
            const float r = inverse_rms(head_sum<G>(S), A.inv_d, A.eps);
            const double rd = (double)r;
            const float c = (float)(rd * rd * rd * head_sum<G>(u) * A.inv_d);
            auto gain_terms = [&](float (&to)[16]) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    to[e] += a.v[e] * r * ma.v[e];
                    to[8 + e] += b.v[e] * r * mb.v[e];
                }
            };
            if (key) // the same for the whole wave
                gain_terms(sum[1]);
            else
                gain_terms(sum[0]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                va.v[e] = r * va.v[e] - c * a.v[e];
                vb.v[e] = r * vb.v[e] - c * b.v[e];
            }
            uint16_t *y = H.out + (t0 + t) * H.out_t + h * H.out_h;
            if (on && L.in_a)
                store16(y + 8 * L.ca, narrow(va));
            if (on && L.in_b)
                store16(y + 8 * L.cb, narrow(vb));
        }
    }
    if (!A.part)
        return;
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
        float *row = red[w * (64 / G) + L.sub];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (L.in_a)
                row[8 * L.ca + e] = sum[which][e];
            if (L.in_b)
                row[8 * L.cb + e] = sum[which][8 + e];
        }
        __syncthreads();
        for (int e = threadIdx.x; e < A.D; e += NT) {
            float s = 0.0f;
            for (int g = 0; g < NW * 64 / G; ++g)
                s += red[g][e];
            A.part[((int64_t)blockIdx.x * 2 + which) * A.D + e] = s;
        }
    }
}

// Gain gradients: the workgroups' partial rows [P][2][D] added in double in a
// fixed order.  Block (j, which) sums elements 8 j .. 8 j + 7 (D is a multiple
// of 8); thread (g, q) adds rows g, g + 512, ... of four of them, so that with
// 1024 rows a thread waits for two loads (64 elements a block and 64 loads one
// after the other took 20 us).
constexpr int GAIN_GROUPS = 512;
__global__ void __launch_bounds__(1024) gain_kernel(const float *part, int P, int D, float *gq, float *gk)
{
    __shared__ double red[16][8];
    const int q = threadIdx.x & 1, g = threadIdx.x >> 1, which = blockIdx.y;
    const int j = blockIdx.x * 8 + 4 * q;
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (int p = g; p < P; p += GAIN_GROUPS) {
        const float4 v = *reinterpret_cast<const float4 *>(part + ((int64_t)p * 2 + which) * D + j);
        s[0] += (double)v.x;
        s[1] += (double)v.y;
        s[2] += (double)v.z;
        s[3] += (double)v.w;
    }
    // the 32 rows of a wave, then the waves in order
#pragma unroll
    for (int m = 2; m < 64; m *= 2)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            s[e] += __shfl_xor(s[e], m);
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) < 2)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            red[w][4 * q + e] = s[e];
    __syncthreads();
    float *out = which ? gk : gq;
    if (threadIdx.x < 8 && out) {
        double t = 0.0;
        for (int i = 0; i < 16; ++i)
            t += red[i][threadIdx.x];
        out[blockIdx.x * 8 + threadIdx.x] = (float)t;
    }
}

// lanes of a head's group: a power of two from 4
inline int group_of(int D, int R)
{
    int g = 4;
    while (g < lanes_of(D, R))
        g *= 2;
    return g;
}

template <bool BWD, int G> void launch_group(const Args &A, bool inter, unsigned grid, hipStream_t st)
{
    if constexpr (BWD) {
        if (inter)
            hipLaunchKernelGGL((bwd_kernel<G, true>), dim3(grid), dim3(NT), 0, st, A);
        else
            hipLaunchKernelGGL((bwd_kernel<G, false>), dim3(grid), dim3(NT), 0, st, A);
    } else {
        if (inter)
            hipLaunchKernelGGL((fwd_kernel<G, true>), dim3(grid), dim3(NT), 0, st, A);
        else
            hipLaunchKernelGGL((fwd_kernel<G, false>), dim3(grid), dim3(NT), 0, st, A);
    }
}

template <bool BWD> void launch(const Args &A, bool inter, unsigned grid, hipStream_t st)
{
    switch (group_of(A.D, A.R)) {
    case 4: return launch_group<BWD, 4>(A, inter, grid, st);
    case 8: return launch_group<BWD, 8>(A, inter, grid, st);
    case 16: return launch_group<BWD, 16>(A, inter, grid, st);
    default: return launch_group<BWD, 32>(A, inter, grid, st);
    }
}

// tokens a workgroup takes at a time: one where that gives the chip no more
// than a few workgroups a compute unit
inline int tokens_at_once(int64_t T) { return T >= 4096 ? TOKENS : 1; }

inline unsigned workgroups(int64_t T, bool bwd)
{
    const int tb = tokens_at_once(T);
    return (unsigned)std::min<int64_t>((T + tb - 1) / tb, bwd ? 1024 : 1 << 20);
}

} // namespace mxq

namespace {

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// One tensor of heads: an input (any strides, 0 among them) or an output,
// whose heads must not share elements.
mx_status check_heads(const mx_heads *h, const char *name, int64_t T, int64_t D, int64_t heads, bool out)
{
    if (!h)
        return mxk::fail(MX_EINVAL, "%s is NULL", name);
    if (h->heads != heads)
        return mxk::fail(MX_EINVAL, "%s has %lld heads, not %lld", name, (long long)h->heads, (long long)heads);
    if (T == 0 || heads == 0)
        return MX_OK;
    const int64_t t = T > 1 ? h->token_stride : 0, s = heads > 1 ? h->head_stride : 0;
    if (!h->data || !aligned(h->data, 16) || t % 8 != 0 || s % 8 != 0)
        return mxk::fail(MX_EINVAL, "%s must be non-NULL, 16-byte aligned, its strides multiples of 8", name);
    if (t < 0 || s < 0 || t > INT64_MAX / 4 / T || s > INT64_MAX / 4 / heads)
        return mxk::fail(MX_EINVAL, "%s: bad strides", name);
    if (out) {
        const bool by_token = (heads == 1 || s >= D) && (T == 1 || t >= s * (heads - 1) + D);
        const bool by_head = (T == 1 || t >= D) && (heads == 1 || s >= t * (T - 1) + D);
        if (!by_token && !by_head)
            return mxk::fail(MX_EINVAL, "%s: its heads overlap", name);
    }
    return MX_OK;
}

mx_status check_common(const mx_heads *q, const mx_heads *k, const void *q_gamma, const void *k_gamma,
                       int64_t T, int64_t D, int64_t R, const int64_t *pos, const float *inv_freq,
                       float eps)
{
    if (T < 0)
        return mxk::fail(MX_EINVAL, "T must be >= 0");
    if (D <= 0 || D % 8 != 0)
        return mxk::fail(MX_EINVAL, "D must be a positive multiple of 8");
    if (R < 0 || R > D || R % 16 != 0)
        return mxk::fail(MX_EINVAL, "R must be a multiple of 16 from 0 to D");
    if (D > mxq::MAX_D)
        return mxk::fail(MX_EUNSUPPORTED, "D exceeds %d", mxq::MAX_D);
    if (!(eps >= 0.0f) || eps > 3.4e38f)
        return mxk::fail(MX_EINVAL, "eps must be finite and >= 0");
    if (!q || !k || q->heads < 0 || k->heads < 0)
        return mxk::fail(MX_EINVAL, "q and k must be given, with 0 heads or more");
    if (q->heads > 65536 || k->heads > 65536 || T > ((int64_t)1 << 40))
        return mxk::fail(MX_EUNSUPPORTED, "at most 65536 heads and 2^40 tokens");
    if (T > 0 && R > 0 && (!inv_freq || !aligned(inv_freq, 4) || !aligned(pos, 8)))
        return mxk::fail(MX_EINVAL, "inv_freq must be non-NULL and 4-byte, pos 8-byte aligned");
    if (!aligned(q_gamma, 16) || !aligned(k_gamma, 16))
        return mxk::fail(MX_EINVAL, "the gains must be 16-byte aligned");
    return MX_OK;
}

mxq::Heads heads_of(const mx_heads *in, const mx_heads *gy, const mx_heads *out, const void *gamma, int G)
{
    mxq::Heads H{};
    H.in = static_cast<const uint16_t *>(in->data);
    H.in_t = in->token_stride;
    H.in_h = in->head_stride;
    if (gy) {
        H.gy = static_cast<const uint16_t *>(gy->data);
        H.gy_t = gy->token_stride;
        H.gy_h = gy->head_stride;
    }
    H.out = static_cast<uint16_t *>(out->data);
    H.out_t = out->token_stride;
    H.out_h = out->head_stride;
    H.gamma = static_cast<const uint16_t *>(gamma);
    H.heads = (int)in->heads;
    H.blocks = (int)((in->heads + 64 / G - 1) / (64 / G));
    return H;
}

mx_status launched()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MX_OK : mxk::fail(MX_EHIP, "kernel launch failed: %s", hipGetErrorString(e));
}

} // namespace

extern "C" {

mx_status qk_norm_rope_fwd(const mx_heads *q, const mx_heads *k, const void *q_gamma, const void *k_gamma,
                           int64_t T, int64_t D, int64_t R, const int64_t *pos, const float *inv_freq,
                           int interleaved, float eps, const mx_heads *q_out, const mx_heads *k_out,
                           hipStream_t stream)
{
    mxk::clear_error();
    mx_status st = check_common(q, k, q_gamma, k_gamma, T, D, R, pos, inv_freq, eps);
    if (st != MX_OK || (st = check_heads(q, "q", T, D, q->heads, false)) != MX_OK ||
        (st = check_heads(k, "k", T, D, k->heads, false)) != MX_OK ||
        (st = check_heads(q_out, "q_out", T, D, q->heads, true)) != MX_OK ||
        (st = check_heads(k_out, "k_out", T, D, k->heads, true)) != MX_OK)
        return st;
    if (T == 0 || q->heads + k->heads == 0)
        return MX_OK;
    const int G = mxq::group_of((int)D, (int)R);
    mxq::Args A{};
    A.q = heads_of(q, nullptr, q_out, q_gamma, G);
    A.k = heads_of(k, nullptr, k_out, k_gamma, G);
    A.pos = pos;
    A.inv_freq = inv_freq;
    A.T = T;
    A.D = (int)D;
    A.R = (int)R;
    A.tb = mxq::tokens_at_once(T);
    A.eps = eps;
    A.inv_d = 1.0 / (double)D;
    mxq::launch<false>(A, interleaved != 0, mxq::workgroups(T, false), stream);
    return launched();
}

size_t qk_norm_rope_bwd_workspace_bytes(int64_t T, int64_t D)
{
    if (T <= 0 || D <= 0 || T > ((int64_t)1 << 40) || D > mxq::MAX_D)
        return 0;
    return (size_t)mxq::workgroups(T, true) * 2 * (size_t)D * sizeof(float);
}

mx_status qk_norm_rope_bwd(const mx_heads *grad_q_out, const mx_heads *grad_k_out, const mx_heads *q,
                           const mx_heads *k, const void *q_gamma, const void *k_gamma, int64_t T,
                           int64_t D, int64_t R, const int64_t *pos, const float *inv_freq,
                           int interleaved, float eps, const mx_heads *grad_q, const mx_heads *grad_k,
                           float *grad_q_gamma, float *grad_k_gamma, void *workspace,
                           size_t workspace_bytes, hipStream_t stream)
{
    mxk::clear_error();
    mx_status st = check_common(q, k, q_gamma, k_gamma, T, D, R, pos, inv_freq, eps);
    if (st != MX_OK || (st = check_heads(grad_q_out, "grad_q_out", T, D, q->heads, false)) != MX_OK ||
        (st = check_heads(grad_k_out, "grad_k_out", T, D, k->heads, false)) != MX_OK ||
        (st = check_heads(q, "q", T, D, q->heads, false)) != MX_OK ||
        (st = check_heads(k, "k", T, D, k->heads, false)) != MX_OK ||
        (st = check_heads(grad_q, "grad_q", T, D, q->heads, true)) != MX_OK ||
        (st = check_heads(grad_k, "grad_k", T, D, k->heads, true)) != MX_OK)
        return st;
    if (!aligned(grad_q_gamma, 4) || !aligned(grad_k_gamma, 4))
        return mxk::fail(MX_EINVAL, "the gain gradients must be 4-byte aligned");
    const bool gains = grad_q_gamma || grad_k_gamma;
    if (gains && T > 0 &&
        (!workspace || !aligned(workspace, 16) || workspace_bytes < qk_norm_rope_bwd_workspace_bytes(T, D)))
        return mxk::fail(MX_EINVAL, "the gain gradients need a 16-byte aligned workspace of %zu bytes",
                         qk_norm_rope_bwd_workspace_bytes(T, D));
    if (T == 0) { // the sums over no tokens
        if (!gains)
            return MX_OK;
        hipLaunchKernelGGL(mxq::gain_kernel, dim3((unsigned)(D / 8), 2), dim3(1024), 0, stream,
                           nullptr, 0, (int)D, grad_q_gamma, grad_k_gamma);
        return launched();
    }
    const int G = mxq::group_of((int)D, (int)R);
    mxq::Args A{};
    A.q = heads_of(q, grad_q_out, grad_q, q_gamma, G);
    A.k = heads_of(k, grad_k_out, grad_k, k_gamma, G);
    A.pos = pos;
    A.inv_freq = inv_freq;
    A.part = gains ? static_cast<float *>(workspace) : nullptr;
    A.T = T;
    A.D = (int)D;
    A.R = (int)R;
    A.tb = mxq::tokens_at_once(T);
    A.eps = eps;
    A.inv_d = 1.0 / (double)D;
    const unsigned grid = mxq::workgroups(T, true);
    mxq::launch<true>(A, interleaved != 0, grid, stream);
    if (gains)
        hipLaunchKernelGGL(mxq::gain_kernel, dim3((unsigned)(D / 8), 2), dim3(1024), 0, stream,
                           A.part, (int)grid, (int)D, grad_q_gamma, grad_k_gamma);
    return launched();
}

} // extern "C"

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
// takes 64 / G heads of one token, or several tokens' if they have so few, the
// next ones' loads in flight.  An angle costs a double product and a sine, and
// every head of the token needs it: the workgroup computes its tokens' angles
// once into LDS.
//
// What bounds it: HBM, 4 bytes an element forward and 6 backward.  32768 tokens
// of 32 + 8 heads of 128 out of a projection of 48: forward 118 us, 5.7 TB/s (a
// copy of as much 125 us); backward 187 us, 5.4 TB/s (an addition of as much
// 167); 15 us of the backward are for writing rows with gaps (the values' part
// of the projection's gradient).  There the angles cost nothing (left out: the
// same and 1% more).  With few heads a token they do, once for its queries and
// once for its keys: 26066 tokens of 2 + 1 heads of 128 18.0 us forward and 32.6
// backward, 14.7 and 25.8 without them; 8000 of 12 + 4 of 64 13.3 and 24.2, 12.4
// and 22.7.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "heads.h"
#include "mxnorm.h"
#include "norm_cast.h"
#include "status.h"

#pragma clang fp contract(off)

namespace mxq {

using namespace mxk;

constexpr int NT = 256, NW = NT / 64;
constexpr int MAX_D = 512;
constexpr int ANGLES = 1024; // angles a workgroup holds at once

struct Heads {
    const uint16_t *in;  // x
    const uint16_t *gy;  // backward: the gradient of the output
    uint16_t *out;       // y, or grad_x
    const uint16_t *gamma;
    int64_t in_t, in_h, gy_t, gy_h, out_t, out_h; // strides, elements
    int heads, blocks;   // blocks of 64 / G heads
    // Tokens of an item: as many as have room in a wave.  (One token an item:
    // 4831 tokens of 4 + 2 heads of 128 backward 23.1 us, so 17.8; 26066 of 2 + 1
    // forward 29.9, so 18.0.)
    int tpi;
    int tb;              // tokens a workgroup takes at a time
    int64_t steps;       // of tb tokens
};

struct Args {
    Heads q, k;
    const int64_t *pos;    // NULL: 0, 1, ...
    const float *inv_freq; // [R/2]
    float *part;           // backward: [2][workgroups][D] gain gradients, or NULL
    int64_t T;
    int D, R;
    float eps;
    double inv_d; // 1 / D
};

// lanes that hold a head's chunks
__host__ __device__ inline int lanes_of(int D, int R) { return R / 16 + (D - R + 15) / 16; }

// a / b for 0 <= a < 4096 and b > 0: (a + 1/2) / b is at least 1 / (2 b) from an
// integer, its rounding and the reciprocal's are below 2^-20 a / b.
__device__ __forceinline__ int quotient(int a, int b)
{
    return (int)(((float)a + 0.5f) * __builtin_amdgcn_rcpf((float)b));
}

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
    const int half = A.R / 2, n = nt * half;
    constexpr int UP = ANGLES / NT; // a lane's angles: their loads are in flight together
    float turn[UP];
#pragma unroll
    for (int k = 0; k < UP; ++k) {
        if (k * NT >= n)
            break;
        const int i = min(k * NT + (int)threadIdx.x, n - 1);
        const int t = quotient(i, half), p = i - t * half; // p = 8 l + e
        const int l = p >> 3, e = p & 7;
        const int pair = !INTER ? p : e < 4 ? 4 * l + e : A.R / 4 + 4 * l + e - 4;
        const int64_t pos = A.pos ? A.pos[t0 + t] : t0 + t;
        const double turns = (double)pos * (double)A.inv_freq[pair] * 0.15915494309189535;
        turn[k] = 2.0f * (float)(turns - rint(turns));
    }
#pragma unroll
    for (int k = 0; k < UP; ++k)
        if (k * NT < n)
            cs[k * NT + threadIdx.x] = turn[k];
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += NT) {
        float s, c;
        sincospif(cs[i], &s, &c);
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

template <int G> __device__ __forceinline__ float head_sum(float s)
{
    auto step = [](float v, auto c) {
        return v + __uint_as_float(dpp_mov<decltype(c)::value>(__float_as_uint(v)));
    };
    s = step(s, std::integral_constant<int, 0xB1>{});
    s = step(s, std::integral_constant<int, 0x4E>{});
    if constexpr (G >= 8)
        s = step(s, std::integral_constant<int, 0x141>{});
    if constexpr (G >= 16)
        s = step(s, std::integral_constant<int, 0x140>{});
    if constexpr (G >= 32)
        s += __shfl_xor(s, 16);
    return s;
}

// Two adjacent elements of each of the lane's chunks.
struct Quad {
    float a0, a1, b0, b1;
};

__device__ __forceinline__ Quad widen(const uint4 &a, const uint4 &b, int i)
{
    const uint32_t x = i == 0 ? a.x : i == 1 ? a.y : i == 2 ? a.z : a.w;
    const uint32_t y = i == 0 ? b.x : i == 1 ? b.y : i == 2 ? b.z : b.w;
    return {bf16_lo(x), bf16_hi(x), bf16_lo(y), bf16_hi(y)};
}

// The compiler takes v as new: nothing computed from it before is kept.
__device__ __forceinline__ void opaque(uint4 (&v)[2])
{
#pragma unroll
    for (int i = 0; i < 2; ++i)
        asm volatile("" : "+v"(v[i].x), "+v"(v[i].y), "+v"(v[i].z), "+v"(v[i].w));
}

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const __bf16 x = (__bf16)a, y = (__bf16)b;
    return (uint32_t)__builtin_bit_cast(uint16_t, x) | ((uint32_t)__builtin_bit_cast(uint16_t, y) << 16);
}

// Turn elements 2 i, 2 i + 1 of the chunks by the lane's angles, or (BACK) by
// their negatives.
template <bool INTER, bool BACK>
__device__ __forceinline__ void turn(Quad &q, const float *cs, const float *sn, int i)
{
    auto one = [](float &x, float &y, float c, float s) {
        if (BACK)
            s = -s;
        const float t = __builtin_fmaf(x, c, -(y * s));
        y = __builtin_fmaf(y, c, x * s);
        x = t;
    };
    if constexpr (INTER) {
        one(q.a0, q.a1, cs[i], sn[i]);
        one(q.b0, q.b1, cs[4 + i], sn[4 + i]);
    } else {
        const float2 c = reinterpret_cast<const float2 *>(cs)[i], s = reinterpret_cast<const float2 *>(sn)[i];
        one(q.a0, q.b0, c.x, s.x);
        one(q.a1, q.b1, c.y, s.y);
    }
}

// 16 bytes at p, or zeros: without a branch, which would end with a wait for
// its own load.  `some` is an address that can be read.
__device__ __forceinline__ uint4 load16(const uint16_t *p, bool in, const uint16_t *some)
{
    const uint4 v = load_stream(reinterpret_cast<const uint4 *>(in ? p : some));
    return make_uint4(in ? v.x : 0, in ? v.y : 0, in ? v.z : 0, in ? v.w : 0);
}

// The lane's two chunks at p and p + step.
template <bool FULL>
__device__ __forceinline__ void load_chunks(uint4 (&v)[2], const uint16_t *p, int step, bool in_a,
                                            bool in_b, const uint16_t *some)
{
    if constexpr (FULL) {
        v[0] = load_stream(reinterpret_cast<const uint4 *>(p));
        v[1] = load_stream(reinterpret_cast<const uint4 *>(p + step));
    } else {
        v[0] = load16(p, in_a, some);
        v[1] = load16(p + step, in_b, some);
    }
}

__device__ __forceinline__ void store16(uint16_t *p, const uint32_t (&v)[4])
{
    __builtin_nontemporal_store(u32x4_t{v[0], v[1], v[2], v[3]}, reinterpret_cast<u32x4_t *>(p));
}

// A lane's place in its head, its item's head and token, and the gains of its
// chunks.  FULL: every lane of
// a wave holds two chunks that turn (R = D = 16 G, and the numbers of heads are
// multiples of 64 / G).
template <int G, bool FULL> struct Lane {
    int l, sub, ca, cb;
    bool in_a, in_b, rot;
    int hs, ts; // the lane's head and token within an item
    bool used;
    __device__ __forceinline__ Lane(const Args &A, const Heads &H)
    {
        const int lane = threadIdx.x & 63;
        l = lane % G;
        sub = lane / G;
        hs = sub;
        ts = 0;
        used = true;
        if constexpr (FULL) {
            ca = l;
            cb = l + G;
            in_a = in_b = rot = true;
        } else {
            if (H.tpi > 1) {
                ts = quotient(sub, H.heads);
                hs = sub - ts * H.heads;
                used = ts < H.tpi;
            }
            chunks_of(A.D, A.R, l, ca, cb);
            in_a = l < lanes_of(A.D, A.R);
            in_b = in_a && 8 * cb < A.D;
            rot = l < A.R / 16;
        }
    }
    __device__ __forceinline__ void gains(const uint16_t *gamma, uint4 (&g)[2]) const
    {
        const uint32_t one = 0x3F803F80u;
        g[0] = g[1] = make_uint4(one, one, one, one);
        if (gamma && in_a)
            g[0] = *reinterpret_cast<const uint4 *>(gamma + 8 * ca);
        if (gamma && in_b)
            g[1] = *reinterpret_cast<const uint4 *>(gamma + 8 * cb);
    }
};

// What a lane has loaded of one head: its chunks of x and, backward, of the
// gradient.
template <bool BWD> struct Loaded {
    uint4 x[2], gy[BWD ? 2 : 1];
};

// The lane's 16 elements, widened: four at a time.
struct Item {
    Quad q[4];
};

__device__ __forceinline__ Item widen(const uint4 (&v)[2])
{
    return {{widen(v[0], v[1], 0), widen(v[0], v[1], 1), widen(v[0], v[1], 2), widen(v[0], v[1], 3)}};
}

// r = (sum x^2 / D + eps)^(-1/2) of the lane's head: the sum in float where its
// squares cannot leave float's range (between 2^-100 and 2^100), else in double;
// 0 for a radicand that is zero or infinite.  A wave computes the double sums if
// one of its heads needs them, but each head takes its own, so that its bits do
// not depend on the others.  Lanes without a head (`on` false), whose elements
// are zeros, ask for none, and get an r that is finite for any eps.
// Without eps a head of subnormals has an r of up to 2^138, beyond float: r is
// then 2^-64 of it and v becomes 2^64 v, exactly, so that x r is what it should
// be.  (v and not its widened elements, which need not be kept for it: twice the
// registers made the forward up to 11% slower.)  Returns 2^64 there, else 1.
template <int G>
__device__ __forceinline__ float inverse_rms(const Args &A, uint4 (&v)[2], bool on, float &r)
{
    const Item x = widen(v);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s = __builtin_fmaf(x.q[i].a0, x.q[i].a0, s);
        s = __builtin_fmaf(x.q[i].a1, x.q[i].a1, s);
        s = __builtin_fmaf(x.q[i].b0, x.q[i].b0, s);
        s = __builtin_fmaf(x.q[i].b1, x.q[i].b1, s);
    }
    s = head_sum<G>(s);
    s = on ? s : 1.0f;
    const bool far = !(s > 0x1p-100f && s < 0x1p100f);
    float up = 1.0f;
    r = __builtin_amdgcn_rsqf(__builtin_fmaf(s, (float)A.inv_d, A.eps));
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(far) != 0, 0)) {
        double S = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double a = x.q[i].a0, b = x.q[i].a1, c = x.q[i].b0, d = x.q[i].b1;
            S += a * a + b * b + c * c + d * d;
        }
        const double u = head_sum<G>(S) * A.inv_d + (double)A.eps;
        const double w = u == 0.0 || u == INFINITY ? 0.0 : 1.0 / sqrt(u);
        up = far && w > 0x1p126 ? 0x1p64f : 1.0f;
        if (far)
            r = (float)(up > 1.0f ? w * 0x1p-64 : w);
        if (up > 1.0f) {
            auto raise = [&](uint32_t &w) { w = pack2(bf16_lo(w) * up, bf16_hi(w) * up); };
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                raise(v[i].x);
                raise(v[i].y);
                raise(v[i].z);
                raise(v[i].w);
            }
        }
    }
    return up;
}

template <int G, bool INTER, bool FULL>
__device__ __forceinline__ void forward_item(const Args &A, const Lane<G, FULL> &L, bool on, Loaded<false> &v,
                                             const uint4 (&gain)[2], const float *cs, const float *sn,
                                             uint32_t (&a)[4], uint32_t (&b)[4])
{
    float r;
    inverse_rms<G>(A, v.x, on, r);
    const Item x = widen(v.x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Quad g = widen(gain[0], gain[1], i), q = x.q[i];
        Quad y = {q.a0 * r * g.a0, q.a1 * r * g.a1, q.b0 * r * g.b0, q.b1 * r * g.b1};
        if (L.rot)
            turn<INTER, false>(y, cs, sn, i);
        a[i] = pack2(y.a0, y.a1);
        b[i] = pack2(y.b0, y.b1);
    }
}

// The gradient of x is r (v - k n) with n = x r and k = (1/D) sum v n: no term
// overflows or underflows where x is huge or tiny, unless the gradient does.
template <int G, bool INTER, bool FULL>
__device__ __forceinline__ void backward_item(const Args &A, const Lane<G, FULL> &L, bool on, Loaded<true> &v,
                                              const uint4 (&gain)[2], const float *cs, const float *sn,
                                              uint32_t (&a)[4], uint32_t (&b)[4], float (&sum)[16])
{
    float r;
    const float up = inverse_rms<G>(A, v.x, on, r);
    Item n = widen(v.x), w;
    float u = 0.0f;
    auto one = [&](float &x, float m, float g, float &to) {
        x = x * r;
        to = __builtin_fmaf(x, m, to);
        const float t = m * g;
        u = __builtin_fmaf(x, t, u);
        return t;
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Quad g = widen(gain[0], gain[1], i);
        Quad m = widen(v.gy[0], v.gy[1], i);
        if (L.rot)
            turn<INTER, true>(m, cs, sn, i);
        w.q[i] = {one(n.q[i].a0, m.a0, g.a0, sum[2 * i]), one(n.q[i].a1, m.a1, g.a1, sum[2 * i + 1]),
                  one(n.q[i].b0, m.b0, g.b0, sum[8 + 2 * i]), one(n.q[i].b1, m.b1, g.b1, sum[9 + 2 * i])};
    }
    const float k = head_sum<G>(u) * (float)A.inv_d;
    auto store = [&](auto grad) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = pack2(grad(n.q[i].a0, w.q[i].a0), grad(n.q[i].a1, w.q[i].a1));
            b[i] = pack2(grad(n.q[i].b0, w.q[i].b0), grad(n.q[i].b1, w.q[i].b1));
        }
    };
    // (the common case apart: no multiplication, and no copies of w kept for one)
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(up > 1.0f) != 0, 0))
        store([&](float x, float t) { return r * (up * __builtin_fmaf(-k, x, t)); });
    else
        store([&](float x, float t) { return r * __builtin_fmaf(-k, x, t); });
}

// Steps s, s + nwg, ... below H.steps of one kind of heads, a step being H.tb
// tokens: wave w takes items w, w + NW, ... of their blocks of heads, an item's
// loads issued before the item ahead of it is computed, the first before the
// tokens' angles.  Backward, fold() takes the sums after every CHAIN items.
// Returns the first step past them.
constexpr int CHAIN = 64;
template <int G, bool INTER, bool FULL, bool BWD, class Fold>
__device__ __forceinline__ int64_t heads_of_kind(const Args &A, const Heads &H, int64_t s, int64_t nwg,
                                                 float *cs, float *sn, float (&sum)[16], Fold fold)
{
    int chain = 0;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = A.R / 2;
    const Lane<G, FULL> L(A, H);
    uint4 gain[2];
    L.gains(H.gamma, gain);
    // an item is the wave's, so its first head's address is scalar; a lane adds
    // its own head and chunk
    const int64_t xl = L.hs * H.in_h + L.ts * H.in_t + 8 * L.ca,
                  gl = BWD ? L.hs * H.gy_h + L.ts * H.gy_t + 8 * L.ca : 0,
                  yl = L.hs * H.out_h + L.ts * H.out_t + 8 * L.ca;
    const int step = 8 * (L.cb - L.ca);
#pragma unroll 1
    for (; s < H.steps; s += nwg) {
        const int64_t t0 = s * H.tb;
        const int nt = (int)min((int64_t)H.tb, A.T - t0), n = (nt + H.tpi - 1) / H.tpi * H.blocks;
        auto place = [&](int i, int &t, int &h) {
            t = i / H.blocks;
            h = (i - t * H.blocks) * (64 / G);
            if constexpr (!FULL)
                t *= H.tpi;
        };
        auto load = [&](int i, Loaded<BWD> &v) {
            int t, h;
            place(i, t, h);
            // past the last item every lane reads the tensor's first bytes: a
            // branch around the loads would end with a wait for them
            const bool more = i < n;
            const bool on = FULL || (more && L.used && h + L.hs < H.heads && t + L.ts < nt);
            const int sp = more ? step : 0;
            const uint16_t *x = more ? H.in + (t0 + t) * H.in_t + h * H.in_h : H.in;
            load_chunks<FULL>(v.x, x + (more ? xl : 0), sp, on && L.in_a, on && L.in_b, H.in);
            if constexpr (BWD) {
                const uint16_t *gy = more ? H.gy + (t0 + t) * H.gy_t + h * H.gy_h : H.gy;
                load_chunks<FULL>(v.gy, gy + (more ? gl : 0), sp, on && L.in_a, on && L.in_b, H.gy);
            }
        };
        Loaded<BWD> next;
        load(w, next);
        __syncthreads(); // the angles of the tokens before are read
        fill_angles<INTER>(A, t0, nt, cs, sn);
        __syncthreads();
#pragma unroll 1
        for (int i = w; i < n; i += NW) {
            Loaded<BWD> v = next;
            load(i + NW, next);
            int t, h;
            place(i, t, h);
            const bool on = FULL || (L.used && h + L.hs < H.heads && t + L.ts < nt);
            // (a lane without a token turns zeros, by any angles)
            const int at = (on ? t + L.ts : 0) * half + 8 * L.l;
            const float *c = cs + at, *d = sn + at;
            uint16_t *y = H.out + (t0 + t) * H.out_t + h * H.out_h + yl;
            opaque(gain); // or they are all kept widened, 16 registers more
            uint32_t a[4], b[4];
            if constexpr (BWD)
                backward_item<G, INTER, FULL>(A, L, on, v, gain, c, d, a, b, sum);
            else
                forward_item<G, INTER, FULL>(A, L, on, v, gain, c, d, a, b);
            if (on && L.in_a)
                store16(y, a);
            if (on && L.in_b)
                store16(y + step, b);
            if constexpr (BWD) {
                if (__builtin_expect(++chain == CHAIN, 0)) {
                    fold();
                    chain = 0;
                }
            }
        }
    }
    return s;
}

// The steps of queries and then those of keys, dealt to the workgroups in one
// sequence.
template <int G, bool INTER, bool FULL> __global__ void __launch_bounds__(NT) fwd_kernel(Args A)
{
    __shared__ __attribute__((aligned(16))) float cs[ANGLES], sn[ANGLES];
    float none[16];
    const int64_t s =
        heads_of_kind<G, INTER, FULL, false>(A, A.q, blockIdx.x, gridDim.x, cs, sn, none, [] {});
    heads_of_kind<G, INTER, FULL, false>(A, A.k, s - A.q.steps, gridDim.x, cs, sn, none, [] {});
}

// As the forward; each lane also keeps the gain gradients of its chunks, in
// float over CHAIN heads and from then on in double in LDS, so that their error
// does not grow with the tokens.  After each kind the workgroup's lanes are added
// in a fixed order into its row of the partial sums: in float where no wave had
// more than CHAIN items (in double always: up to 2 us more), else in double.
template <int G, bool INTER, bool FULL>
__global__ void __launch_bounds__(NT) bwd_kernel(Args A)
{
    constexpr int GW = 64 / G; // groups of a wave
    __shared__ __attribute__((aligned(16))) float cs[ANGLES], sn[ANGLES];
    __shared__ float red[NW * GW][16 * G]; // D <= 16 G
    __shared__ double kept[NW * GW][16 * G];
    __shared__ bool folded[NW];
    const Lane<G, FULL> L(A, A.q);
    const int w = threadIdx.x >> 6, row = w * GW + L.sub;
    float sum[16] = {};
    bool some = false; // this wave has folded its sums
    auto fold = [&] {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (L.in_a) {
                double &to = kept[row][8 * L.ca + e];
                to = (some ? to : 0.0) + (double)sum[e];
            }
            if (L.in_b) {
                double &to = kept[row][8 * L.cb + e];
                to = (some ? to : 0.0) + (double)sum[8 + e];
            }
            sum[e] = sum[8 + e] = 0.0f;
        }
        some = true;
    };
    auto finish = [&](int which, bool any) {
        if (!A.part)
            return;
        float *to = A.part + ((int64_t)which * gridDim.x + blockIdx.x) * A.D;
        if (!any) {
            for (int e = threadIdx.x; e < A.D; e += NT)
                to[e] = 0.0f;
            return;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (L.in_a)
                red[row][8 * L.ca + e] = sum[e];
            if (L.in_b)
                red[row][8 * L.cb + e] = sum[8 + e];
            sum[e] = sum[8 + e] = 0.0f;
        }
        if ((threadIdx.x & 63) == 0)
            folded[w] = some;
        __syncthreads();
        const bool f[NW] = {folded[0], folded[1], folded[2], folded[3]};
        const bool in_double = f[0] || f[1] || f[2] || f[3];
        for (int e = threadIdx.x; e < A.D; e += NT) {
            if (in_double) {
                double t = 0.0;
#pragma unroll
                for (int v = 0; v < NW; ++v)
#pragma unroll 2
                    for (int g = v * GW; g < (v + 1) * GW; ++g)
                        t += (f[v] ? kept[g][e] : 0.0) + (double)red[g][e];
                to[e] = (float)t;
            } else {
                float t = 0.0f;
#pragma unroll 16
                for (int g = 0; g < NW * GW; ++g)
                    t += red[g][e];
                to[e] = t;
            }
        }
        __syncthreads();
        some = false;
    };
    const int64_t s = heads_of_kind<G, INTER, FULL, true>(A, A.q, blockIdx.x, gridDim.x, cs, sn, sum, fold);
    finish(0, blockIdx.x < A.q.steps);
    heads_of_kind<G, INTER, FULL, true>(A, A.k, s - A.q.steps, gridDim.x, cs, sn, sum, fold);
    finish(1, s - A.q.steps < A.k.steps);
}

// Gain gradients: the workgroups' partial rows [2][P][D] added in double in a
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
    part += (int64_t)which * P * D;
    for (int p = g; p < P; p += GAIN_GROUPS) {
        const float4 v = *reinterpret_cast<const float4 *>(part + (int64_t)p * D + j);
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

template <bool BWD, int G, bool INTER> void launch_group(const Args &A, unsigned grid, hipStream_t st)
{
    if (A.D == 16 * G && A.R == A.D && A.q.heads % (64 / G) == 0 && A.k.heads % (64 / G) == 0) {
        if constexpr (BWD)
            hipLaunchKernelGGL((bwd_kernel<G, INTER, true>), dim3(grid), dim3(NT), 0, st, A);
        else
            hipLaunchKernelGGL((fwd_kernel<G, INTER, true>), dim3(grid), dim3(NT), 0, st, A);
    } else {
        if constexpr (BWD)
            hipLaunchKernelGGL((bwd_kernel<G, INTER, false>), dim3(grid), dim3(NT), 0, st, A);
        else
            hipLaunchKernelGGL((fwd_kernel<G, INTER, false>), dim3(grid), dim3(NT), 0, st, A);
    }
}

template <bool BWD> void launch(const Args &A, bool inter, unsigned grid, hipStream_t st)
{
    switch (group_of(A.D, A.R)) {
    case 4: return inter ? launch_group<BWD, 4, true>(A, grid, st)
                         : launch_group<BWD, 4, false>(A, grid, st);
    case 8: return inter ? launch_group<BWD, 8, true>(A, grid, st)
                         : launch_group<BWD, 8, false>(A, grid, st);
    case 16: return inter ? launch_group<BWD, 16, true>(A, grid, st)
                         : launch_group<BWD, 16, false>(A, grid, st);
    default: return inter ? launch_group<BWD, 32, true>(A, grid, st)
                         : launch_group<BWD, 32, false>(A, grid, st);
    }
}

// Tokens of a step: four items (one a wave) with an angle a lane, and up to 16
// as far as the angles fit and that leaves a step for each of `least` workgroups: the next item's
// loads then hide behind the one at hand, and backward a workgroup's sums are
// added once.  12 + 4 heads of 64, 2000 tokens backward: 12.4 us, 14.5 with
// four times as many steps; 8000 tokens 24.1 and 29.0, forward 12.9 and 15.5.
// Fewer workgroups than 224 backward or 360 forward leave compute units idle:
// 32 + 8 heads of 128, 500 tokens 10.6 us backward, 12.1 with 120 of them; 4096
// tokens 19.1 us forward, 19.8 with 256.
inline void steps_of(Heads &H, int64_t T, int R, int64_t least)
{
    H.tb = 1;
    H.steps = 0;
    if (H.heads == 0) // no items, however many tokens: nothing below would bound tb
        return;
    auto items = [&](int tb) { return (tb + H.tpi - 1) / H.tpi * H.blocks; };
    auto angles = [&](int tb) { return tb * (R / 2); };
    while (angles(2 * H.tb) <= ANGLES &&
           ((items(2 * H.tb) <= NW && angles(2 * H.tb) <= NT) ||
            (items(2 * H.tb) <= 4 * NW && T / (2 * H.tb) >= least)))
        H.tb *= 2;
    H.steps = (T + H.tb - 1) / H.tb;
}

// Workgroups: forward one for each step, backward at most two a compute unit,
// each with a row of partial sums for either gain (32768 tokens of 40 heads of
// 128: 188 us with 512, 210 with 768, 187 with 1024, 226 with 256).
constexpr int MAX_ROWS = 512;
inline unsigned workgroups(const Args &A, bool bwd)
{
    return (unsigned)std::min<int64_t>(A.q.steps + A.k.steps, bwd ? MAX_ROWS : 1 << 20);
}

} // namespace mxq

namespace {

using mxk::aligned;
using mxk::check_heads;
using mxk::launched;

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
    H.tpi = H.heads ? std::max(64 / G / H.heads, 1) : 1;
    return H;
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
    A.eps = eps;
    A.inv_d = 1.0 / (double)D;
    mxq::steps_of(A.q, T, A.R, 360);
    mxq::steps_of(A.k, T, A.R, 360);
    mxq::launch<false>(A, interleaved != 0, mxq::workgroups(A, false), stream);
    return launched();
}

size_t qk_norm_rope_bwd_workspace_bytes(int64_t T, int64_t D)
{
    if (T <= 0 || D <= 0 || T > ((int64_t)1 << 40) || D > mxq::MAX_D)
        return 0;
    // no more steps than tokens of each kind
    return 2 * (size_t)std::min<int64_t>(mxq::MAX_ROWS, 2 * T) * (size_t)D * sizeof(float);
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
    A.eps = eps;
    A.inv_d = 1.0 / (double)D;
    mxq::steps_of(A.q, T, A.R, 224);
    mxq::steps_of(A.k, T, A.R, 224);
    const unsigned grid = mxq::workgroups(A, true);
    if (grid == 0 && !gains)
        return MX_OK;
    if (grid > 0)
        mxq::launch<true>(A, interleaved != 0, grid, stream);
    if (gains)
        hipLaunchKernelGGL(mxq::gain_kernel, dim3((unsigned)(D / 8), 2), dim3(1024), 0, stream,
                           A.part, (int)grid, (int)D, grad_q_gamma, grad_k_gamma);
    return launched();
}

} // extern "C"

// window_attn.hip -- causal attention of packed sequences with a sliding window
// and sinks, forward and backward.
//
// Query i of a sequence of lq queries and lk keys stands at p = i + lk - lq and
// sees key j where j <= p and (p - j < window or j < sinks).  With s = scale q.k,
//   forward:  o = sum_j exp(s_j - m) v_j / l,  l = sum_j exp(s_j - m),  lse = m + log l;
//   backward: P = exp(s - lse),  delta = grad_o . o,  dS = P (grad_o . v - delta),
//     grad_q = scale sum_j dS k_j,  grad_k = scale sum_i dS q_i,  grad_v = sum_i P grad_o_i.
//
// One pass over the keys with a running maximum; scores and P stay in registers, tiles
// of 64 rows come by LDS DMA.  The backward forms S and dP twice, once by queries for
// grad_q and once by keys for grad_k and grad_v: 7 products for the formulas' 5, but no
// atomics, so the same call gives the same bits.  A block of the sinks' keys has every
// query of the sequence: those behind its window are summed apart, in chunks.
//
// What bounds it (8192 tokens, 32 + 8 heads of 128): forward without a window 528 to
// 585 us, 0.94 to 1.04 PFLOP/s (the clock falls to 1.84 GHz under it).  Its matrix
// instructions alone take 317, with the exponentials 400, with the LDS reads instead
// 479: the three overlap in part, two waves a SIMD.  A transposing LDS read brings 64
// bytes a cycle, half of a plain one, and a tile is read by all of a workgroup's waves;
// more rows a wave, which would halve that, need more than the 256 registers of two
// waves a SIMD.  Two halves of a workgroup in opposite phases, products beside
// exponentials by two barriers a tile, took 595.  Backward with a window of 4096 1600
// to 1680: grad_q 590 to 610 (1.05 PFLOP/s of its three products), grad_k and grad_v 970
// to 1045 (0.83 of its four; matrix instructions alone 511, without LDS reads 767, without
// the exponentials and the hand-over of P 800), the sinks' far queries 45.
#include <type_traits>

#include "attn.h"
#include "testing.h"

namespace mxa {

constexpr int BK = 64;        // keys of a tile, queries of a backward tile
constexpr int FAR_CHUNK = 256; // queries that a pair of waves sums for the sinks, at least

struct Args {
    In q, k, v, go, o;
    Out out, gk, gv;      // out: the output, or grad_q
    const float *lse;     // backward: [Hq, Tq]
    float *lse_out;       // forward: or NULL
    float *lse_s, *delta; // backward: -lse / scale and -delta, where scores and grad_o . v start, [Hq, Tq]
    float *far;           // backward: the sinks' sums over queries far behind them, by chunk and share
    float *near;          // with shares of near queries: their sums
    const int *qs, *ks;   // [B + 1], or NULL: one sequence
    int Tq, Tk, B, Hk, G, D;
    int tiles, window, sinks, chunk, far_blocks, far_shares, shares;
    float c, scale;       // scale log2(e), scale
};

struct Span {
    int q0, lq, k0, lk, off; // off = lk - lq
};

__device__ __forceinline__ int start_of(const int *s, int b, int T) { return min(max(s[b], 0), T); }

// The sequence that tile `tile` belongs to and the tile's first row in it.  The
// sequences' tiles of R rows are numbered from floor(start / R) + b on: that
// leaves room for each, and starts that are not in order stay within bounds.
__device__ __forceinline__ bool span_of(const Args &A, const int *s, int T, int tile, int R, bool keys, Span &S, int &b, int &r0)
{
    b = 0;
    if (!s) {
        S = {0, A.Tq, 0, A.Tk, A.Tk - A.Tq};
        r0 = tile * R;
        return r0 < T;
    }
    int hi = A.B - 1;
    while (b < hi) {
        const int mid = (b + hi + 1) >> 1;
        if (start_of(s, mid, T) / R + mid <= tile)
            b = mid;
        else
            hi = mid - 1;
    }
    S.q0 = start_of(A.qs, b, A.Tq);
    S.lq = max(start_of(A.qs, b + 1, A.Tq) - S.q0, 0);
    S.k0 = start_of(A.ks, b, A.Tk);
    S.lk = max(start_of(A.ks, b + 1, A.Tk) - S.k0, 0);
    S.off = S.lk - S.lq;
    r0 = (tile - ((keys ? S.k0 : S.q0) / R + b)) * R;
    return r0 >= 0 && r0 < (keys ? S.lk : S.lq);
}

// Workgroup id of a launch over tiles, key heads and their G query heads, so that
// an XCD has whole key heads, or every (8 / Hk)-th tile of one: its L2 then holds
// what its workgroups share, and each XCD has long and short tiles alike.
__device__ __forceinline__ bool item_of(int id, int tiles, int Hk, int G, int &rank, int &hk, int &g)
{
    const int per = tiles * G, x = id % NXCD;
    int r;
    if (Hk % NXCD == 0) {
        r = id / NXCD;
        hk = x + NXCD * (r / per);
        r %= per;
    } else if (NXCD % Hk == 0) {
        hk = x % Hk;
        r = id / NXCD * (NXCD / Hk) + x / Hk;
    } else {
        hk = id % Hk;
        r = id / Hk;
    }
    rank = r / G;
    g = r % G;
    return r < per;
}

inline int64_t items(int64_t tiles, int64_t Hk, int64_t G)
{
    if (NXCD % Hk == 0)
        return NXCD * ((tiles * G * Hk + NXCD - 1) / NXCD);
    return tiles * G * Hk;
}

// The key tiles that queries at p0 .. p1 see: those of the sinks, then the window's.
struct Tiles {
    int sinks, first, n;
    __device__ __forceinline__ Tiles(const Args &A, int p0, int p1)
    {
        first = max(p0 - A.window + 1, 0) / BK;
        sinks = min((A.sinks + BK - 1) / BK, first);
        n = p1 < 0 ? 0 : sinks + p1 / BK - first + 1;
    }
    __device__ __forceinline__ int operator[](int i) const { return (i < sinks ? i : first + i - sinks) * BK; }
};

__device__ __forceinline__ bool sees(const Args &A, int p, int j)
{
    return j <= p && (p - j < A.window || j < A.sinks);
}

// The same of the keys j0 + c, for constants c.  The sums are hidden from the
// compiler, which would keep one for every c in a register.
struct Mask {
    int most, least, sinks;
    __device__ __forceinline__ Mask(const Args &A, int p, int j0) : most(p - j0), least(p - j0 - A.window), sinks(A.sinks - j0)
    {
        asm volatile("" : "+v"(most), "+v"(least), "+v"(sinks));
    }
    __device__ __forceinline__ bool operator()(int c) const { return c <= most && (c > least || c < sinks); }
};

// floor(x / BK) for any x
__device__ __forceinline__ int tile_floor(int x) { return x >> 6; }
static_assert(BK == 64, "tile_floor");

// What queries at p0 .. p1 (p1 < p0: none) see of the tiles, by their number in the list.
__device__ __forceinline__ Seen seen_of(const Args &A, const Tiles &T, int p0, int p1)
{
    const int shift = T.first - T.sinks;
    Seen S;
    S.some = max(tile_floor(p0 - A.window + 1) - shift, T.sinks);
    S.none = p1 < p0 ? 0 : tile_floor(p1) + 1 - shift;
    S.sinks = min(max(tile_floor(A.sinks + BK - 1) - shift, T.sinks), S.none);
    S.all = max(tile_floor(p1 - A.window) + 1 - shift, T.sinks);
    S.less = p1 < p0 ? 0 : tile_floor(p0 + 1) - shift;
    return S;
}

// Waves of a workgroup, 32 queries each.  Two workgroups of four have room on a compute
// unit, and what one waits for at its barrier the other fills (eight in one, with
// three stages: 8192 tokens of 32 + 8 heads of 128 567 us, so 552; 5003 of 12 + 4 of
// 80, window 1000, 41 and 34).
constexpr int QW = 4;
// Stages of keys and values: three, or two where that makes the room.
template <int DB> constexpr int kStages = DB > 2 ? 2 : 3;
template <int DB> constexpr int kTiles = kStages<DB> * 2 * BK * kRow<DB>;

// Where few workgroups leave compute units idle, two groups of waves (KW = 2) take the
// tiles in turn, and the second hands its sums over at the end (in LDS: the sums, the
// rows' maxima and sums, the rows on their way out).
template <int DB> constexpr int kSums = QW * DB * 4096;
template <int DB, int KW> constexpr int kRows = KW == 1 ? 0 : kSums<DB> + QW * 256;

// False in the second group, whose sums are then in LDS.
template <int DB> __device__ __forceinline__ bool hand_over(const f16v (&o)[DB], LDS_AS uint8_t *lds, int w, int kw, int l)
{
    static_assert(kRows<DB, 2> + QW * 32 * kRow<DB> <= 2 * kTiles<DB>, "room for all");
    LDS_AS float *const to = reinterpret_cast<LDS_AS float *>(lds) + w * DB * 1024 + l;
    if (kw == 1)
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                to[(d * 16 + e) * 64] = o[d][e];
    __syncthreads();
    return kw == 0;
}

// o = a o + b (the second group's)
template <int DB> __device__ __forceinline__ void take_over(f16v (&o)[DB], float a, float b, const LDS_AS uint8_t *lds, int w, int l)
{
    const LDS_AS float *const from = reinterpret_cast<const LDS_AS float *>(lds) + w * DB * 1024 + l;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            o[d][e] = o[d][e] * a + from[(d * 16 + e) * 64] * b;
}

// ---------------------------------------------------------------- forward --

template <int DB, bool FULL, int KW, bool CAREFUL>
__device__ __forceinline__ bool forward(const Args &A, LDS_AS uint8_t *lds, const Span &S, int i0, int hk, int hq)
{
    constexpr int TILE = BK * kRow<DB>;
    const int thread = thread_number<CAREFUL>();
    const int wave = __builtin_amdgcn_readfirstlane(thread >> 6), l = thread & 63, n = l & 31, h = l >> 5;
    const int w = wave % QW, kw = wave / QW;
    LDS_AS uint8_t *const mine = lds + kw * kTiles<DB>;
    const uint32_t base = lds_address(mine);
    const Lane<DB> L(l);
    const uint16_t *kh = A.k.p + S.k0 * A.k.ts + hk * A.k.hs, *vh = A.v.p + S.k0 * A.v.ts + hk * A.v.hs;
    const Tiles tiles(A, i0 + S.off, min(i0 + 32 * QW, S.lq) - 1 + S.off);
    using Load = Loader<DB, BK, QW, FULL>;
    const Load kl(A.k.ts, A.D, w, l), vl(A.v.ts, A.D, w, l);
    auto load = [&](int it, int stage) {
        const uint32_t to = base + stage * 2 * TILE;
        const int j0 = tiles[min(it * KW + kw, tiles.n - 1)]; // a group without a last tile loads for the count's sake
        kl.load(kh, j0, S.lk - 1, to, l);
        vl.load(vh, j0, S.lk - 1, to + TILE, l);
    };
    const int iw = i0 + 32 * w;                             // the wave's first query
    const int p0 = iw + S.off, p1 = min(iw + 31, S.lq - 1) + S.off;
    const int p = min(iw + n, S.lq - 1) + S.off;
    const Seen what = seen_of(A, tiles, p0, p1);
    b8 q[2 * DB];
    load_rows<DB>(q, A.q.p + S.q0 * A.q.ts + hq * A.q.hs, A.q.ts, iw, S.lq - 1, A.D, l);
    settle(q);
    f16v o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
        o[d] = zero16();
    float m = -FLT_MAX, sum = 0.0f; // m: of scores in powers of two; sum: the lane's half of the keys
    auto work = [&](int it, int stage) {
        const int t = it * KW + kw;
        const int see = t < tiles.n ? what(t) : 0, j0 = tiles[t];
        if (see == 0)
            return;
        const LDS_AS uint8_t *kt = mine + stage * 2 * TILE, *vt = kt + TILE;
        f16v x[2]; // scores, then P
        scores<DB>(x, kt, L, q);
        if (see == 1) {
            const Mask mask(A, p, j0 + 4 * h);
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    x[b][e] = mask(32 * b + c_row(e, 0)) ? x[b][e] : -INFINITY;
        }
        float mt = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                mt = fmaxf(mt, x[b][e]);
        mt = halves_max(mt) * A.c;
        // The maximum is followed only where it grows by more than 2^8: what
        // exponentials and sums gain from that stays far inside float and bf16.
        if (__builtin_amdgcn_ballot_w64(mt > m + 8.0f)) {
            const float mn = fmaxf(m, mt), by = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            sum *= by;
#pragma unroll
            for (int d = 0; d < DB; ++d)
                o[d] *= by;
        }
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                x[b][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][e], A.c, -m));
                sum += x[b][e];
            }
        if (CAREFUL && see == 1)
            careful_products<DB, 2>(o, vt, L, x, h, [&](int r) { return sees(A, p, j0 + r); });
        else
            products<DB, 2>(o, vt, L, x);
    };
    tile_loop<kStages<DB>, 2 * Load::N>((tiles.n + KW - 1) / KW, load, work);
    if (!CAREFUL && __syncthreads_or(iw + n < S.lq && not_finite<DB>(o)))
        return false;
    if (CAREFUL)
        __syncthreads();
    sum = halves_sum(sum);
    if constexpr (KW == 2) {
        LDS_AS float *const stat = reinterpret_cast<LDS_AS float *>(lds + kSums<DB>) + w * 64 + n;
        if (kw == 1 && h == 0) {
            stat[0] = m;
            stat[32] = sum;
        }
        if (!hand_over<DB>(o, lds, w, kw, l))
            return true;
        const float m1 = stat[0], mn = fmaxf(m, m1);
        const float a = __builtin_amdgcn_exp2f(m - mn), a1 = __builtin_amdgcn_exp2f(m1 - mn);
        sum = sum * a + stat[32] * a1;
        m = mn;
        take_over<DB>(o, a, a1, lds, w, l);
    }
    // a row that sees no key gives 0; one that sees only scores of -inf NaN
    const float by = p < 0 ? 0.0f : 1.0f / sum;
    if (A.lse_out && h == 0 && iw + n < S.lq)
        A.lse_out[(int64_t)hq * A.Tq + S.q0 + iw + n] =
            p < 0 ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * LN2;
    store_rows<DB>(o, by, lds + kRows<DB, KW> + w * 32 * kRow<DB>, A.out.p + (int64_t)(S.q0 + iw) * A.out.ts + hq * A.out.hs, A.out.ts,
                   S.lq - iw, A.D, l);
    return true;
}

template <int DB, bool FULL, int KW>
__global__ void __launch_bounds__(64 * QW * KW, 2) fwd_kernel(Args A)
{
    __shared__ __attribute__((aligned(1024))) uint8_t smem[KW * kTiles<DB>];
    LDS_AS uint8_t *lds = (LDS_AS uint8_t *)smem;
    int rank, hk, g, b, i0;
    Span S;
    if (!item_of(blockIdx.x, A.tiles, A.Hk, A.G, rank, hk, g) ||
        !span_of(A, A.qs, A.Tq, A.tiles - 1 - rank, 32 * QW, false, S, b, i0))
        return;
    if (!FULL)
        zero_lds<KW * kTiles<DB>>(lds, 64 * QW * KW);
    if (!forward<DB, FULL, KW, false>(A, lds, S, i0, hk, hk * A.G + g))
        forward<DB, FULL, KW, true>(A, lds, S, i0, hk, hk * A.G + g);
}

// --------------------------------------------------------------- backward --

// grad_q, and for the other kernels where a query's scores and grad_out . v start.
template <int DB, bool FULL, int KW, bool CAREFUL>
__device__ __forceinline__ bool backward_q(const Args &A, LDS_AS uint8_t *lds, const Span &S, int i0, int hk, int hq)
{
    constexpr int TILE = BK * kRow<DB>;
    const int thread = thread_number<CAREFUL>();
    const int wave = __builtin_amdgcn_readfirstlane(thread >> 6), l = thread & 63, n = l & 31, h = l >> 5;
    const int w = wave % QW, kw = wave / QW;
    LDS_AS uint8_t *const mine = lds + kw * kTiles<DB>;
    const uint32_t base = lds_address(mine);
    const Lane<DB> L(l);
    const uint16_t *kh = A.k.p + S.k0 * A.k.ts + hk * A.k.hs, *vh = A.v.p + S.k0 * A.v.ts + hk * A.v.hs;
    const Tiles tiles(A, i0 + S.off, min(i0 + 32 * QW, S.lq) - 1 + S.off);
    using Load = Loader<DB, BK, QW, FULL>;
    const Load kl(A.k.ts, A.D, w, l), vl(A.v.ts, A.D, w, l);
    auto load = [&](int it, int stage) {
        const uint32_t to = base + stage * 2 * TILE;
        const int j0 = tiles[min(it * KW + kw, tiles.n - 1)]; // a group without a last tile loads for the count's sake
        kl.load(kh, j0, S.lk - 1, to, l);
        vl.load(vh, j0, S.lk - 1, to + TILE, l);
    };
    const int iw = i0 + 32 * w;
    const int p0 = iw + S.off, p1 = min(iw + 31, S.lq - 1) + S.off;
    const int p = min(iw + n, S.lq - 1) + S.off;
    b8 q[2 * DB], go[2 * DB];
    load_rows<DB>(go, A.o.p + S.q0 * A.o.ts + hq * A.o.hs, A.o.ts, iw, S.lq - 1, A.D, l);
    load_rows<DB>(q, A.go.p + S.q0 * A.go.ts + hq * A.go.hs, A.go.ts, iw, S.lq - 1, A.D, l);
    float delta = 0.0f;
#pragma unroll
    for (int ks = 0; ks < 2 * DB; ++ks)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            delta = __builtin_fmaf((float)q[ks][e], (float)go[ks][e], delta);
    delta = halves_sum(delta);
#pragma unroll
    for (int ks = 0; ks < 2 * DB; ++ks)
        go[ks] = q[ks];
    load_rows<DB>(q, A.q.p + S.q0 * A.q.ts + hq * A.q.hs, A.q.ts, iw, S.lq - 1, A.D, l);
    const int64_t row = (int64_t)hq * A.Tq + S.q0 + min(iw + n, S.lq - 1);
    float lse2 = A.lse[row] * LOG2E;
    settle(q);
    settle(lse2);
    if (h == 0 && iw + n < S.lq) {
        A.lse_s[row] = -A.lse[row] / A.scale;
        A.delta[row] = -delta;
    }
    const Seen what = seen_of(A, tiles, p0, p1);
    f16v o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
        o[d] = zero16();
    auto work = [&](int it, int stage) {
        const int t = it * KW + kw;
        const int see = t < tiles.n ? what(t) : 0, j0 = tiles[t];
        if (see == 0)
            return;
        const LDS_AS uint8_t *kt = mine + stage * 2 * TILE, *vt = kt + TILE;
        f16v x[2], y[2]; // x: scores, then dS
        scores<DB>(x, kt, L, q);
        scores<DB>(y, vt, L, go);
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float pr = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][e], A.c, -lse2));
                x[b][e] = pr * (y[b][e] - delta);
            }
        if (see == 1) {
            const Mask mask(A, p, j0 + 4 * h);
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    x[b][e] = mask(32 * b + c_row(e, 0)) ? x[b][e] : 0.0f;
        }
        if (CAREFUL && see == 1)
            careful_products<DB, 2>(o, kt, L, x, h, [&](int r) { return sees(A, p, j0 + r); });
        else
            products<DB, 2>(o, kt, L, x);
    };
    tile_loop<kStages<DB>, 2 * Load::N>((tiles.n + KW - 1) / KW, load, work);
    if (!CAREFUL && __syncthreads_or(iw + n < S.lq && not_finite<DB>(o)))
        return false;
    if (CAREFUL)
        __syncthreads();
    if constexpr (KW == 2) {
        if (!hand_over<DB>(o, lds, w, kw, l))
            return true;
        take_over<DB>(o, 1.0f, 1.0f, lds, w, l);
    }
    store_rows<DB>(o, A.scale, lds + kRows<DB, KW> + w * 32 * kRow<DB>, A.out.p + (int64_t)(S.q0 + iw) * A.out.ts + hq * A.out.hs, A.out.ts,
                   S.lq - iw, A.D, l);
    return true;
}

template <int DB, bool FULL, int KW>
__global__ void __launch_bounds__(64 * QW * KW, 2) bwd_q_kernel(Args A)
{
    __shared__ __attribute__((aligned(1024))) uint8_t smem[KW * kTiles<DB>];
    LDS_AS uint8_t *lds = (LDS_AS uint8_t *)smem;
    int rank, hk, g, b, i0;
    Span S;
    if (!item_of(blockIdx.x, A.tiles, A.Hk, A.G, rank, hk, g) ||
        !span_of(A, A.qs, A.Tq, A.tiles - 1 - rank, 32 * QW, false, S, b, i0))
        return;
    if (!FULL)
        zero_lds<KW * kTiles<DB>>(lds, 64 * QW * KW);
    if (!backward_q<DB, FULL, KW, false>(A, lds, S, i0, hk, hk * A.G + g))
        backward_q<DB, FULL, KW, true>(A, lds, S, i0, hk, hk * A.G + g);
}

// Sums of 32 keys as the waves hold them: a plane each for grad_k and grad_v.
template <int DB> constexpr int kPlane = DB * 16 * 64;

// Of block kb of the sinks, over share s of the queries of chunk `at` (see Chunks) that
// lie the window or more behind.
template <int DB> __device__ __forceinline__ float *far_part(const Args &A, int at, int hk, int kb, int s)
{
    return A.far + ((((int64_t)at * A.Hk + hk) * A.far_blocks + kb) * A.far_shares + s) * (2 * kPlane<DB>);
}

// Of key block `at` (numbered as tiles of 32), over share s of its near queries.
template <int DB> __device__ __forceinline__ float *near_part(const Args &A, int at, int hk, int s)
{
    return A.near + (((int64_t)at * A.Hk + hk) * A.shares + s) * (2 * kPlane<DB>);
}

// The chunks with far queries of sink block jw: first and last, and the number of chunk 0.
// Chunks are numbered as tiles are, but only sequences with far queries need room of
// their own: those have more keys than the window, so floor(k_start / (window + 1)) tells
// them apart, and the sums' room does not grow with the short sequences of a batch.
struct Chunks {
    int first, last, at;
    __device__ __forceinline__ Chunks(const Args &A, const Span &S, int b, int jw)
    {
        const int i = max(jw + A.window - S.off, 0);
        const bool any = jw < A.sinks && i < S.lq;
        first = any ? i / A.chunk : 0;
        last = any ? (S.lq - 1) / A.chunk : -1;
        at = number(A, S, b);
    }
    __device__ __forceinline__ static int number(const Args &A, const Span &S, int b)
    {
        return S.q0 / A.chunk + min(b, S.k0 / (A.window + 1));
    }
};

// grad_k and grad_v of 32 keys for each of NP pairs of waves, from share `share` of
// `shares` of the tiles of queries i0 .. i1 of the group's heads, one head behind the
// other.  FAR: those that see them as sinks, not through the window.
//
// A wave has registers for one of the two sums at two waves a SIMD.  So of a pair
// the first wave forms the scores, P and grad_v += grad_out^T P, and the second, a
// tile of queries later, grad_out . v, dS from the P that the first left in LDS,
// and grad_k += Q^T dS: two products each, one barrier a tile.  P goes over as the upper 24 bits of its
// float, within 2^-15, so dS is rounded to bf16 from what is nearly float (P in bf16
// would double that rounding, whole floats do not fit).
template <int DB> constexpr int kStageKV = 2 * BK * kRow<DB> + 8 * BK;
template <int DB, int NP> constexpr int kBytesKV = 3 * kStageKV<DB> + NP * 2 * BK * 96;
template <int DB, int NP, bool FULL, bool FAR, bool CAREFUL>
__device__ __forceinline__ bool backward_kv(const Args &A, LDS_AS uint8_t *lds, const Span &S, int j0, int i0, int i1, int hk,
                                            int b, int chunk, int share, int shares)
{
    constexpr int TILE = BK * kRow<DB>, STAGE = kStageKV<DB>, NW = 2 * NP;
    const int thread = thread_number<CAREFUL>();
    const int w = __builtin_amdgcn_readfirstlane(thread >> 6), l = thread & 63, n = l & 31, h = l >> 5;
    const int pair = w % NP, second = w / NP;
    const uint32_t base = lds_address(lds);
    const Lane<DB> L(l);
    const int steps = i1 < i0 ? 0 : (i1 - i0) / BK + 1;
    const int from = (int)((int64_t)steps * A.G * share / shares), total = (int)((int64_t)steps * A.G * (share + 1) / shares) - from;
    const int u0 = steps ? from % steps : 0;
    using Load = Loader<DB, BK, NW, FULL>;
    const Load ql(A.q.ts, A.D, w, l), gl(A.go.ts, A.D, w, l);
    int lr = i0 + u0 * BK, lq = hk * A.G + (steps ? from / steps : 0); // of the tile to load next: first query, head
    auto load = [&](int stage) { // the next one
        const uint32_t to = base + stage * STAGE;
        ql.load(A.q.p + S.q0 * A.q.ts + lq * A.q.hs, lr, i1, to, l);
        gl.load(A.go.p + S.q0 * A.go.ts + lq * A.go.hs, lr, i1, to + TILE, l);
        // where the rows start
        const int64_t row = (int64_t)lq * A.Tq + S.q0 + min(lr + l, i1);
        if (w < 2)
            mxg::lds_load4((w ? A.delta : A.lse_s) + row, to + 2 * TILE + w * 4 * BK);
        lr += BK;
        if (lr > i1) {
            lr = i0;
            ++lq;
        }
    };
    const int jw = j0 + 32 * pair, j = jw + n;
    b8 x[2 * DB];
    const In &kv = second ? A.v : A.k;
    load_rows<DB>(x, kv.p + S.k0 * kv.ts + hk * kv.hs, kv.ts, jw, S.lk - 1, A.D, l);
    settle(x);
    f16v acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
        acc[d] = zero16();
    auto sees_key = [&](int i) {
        const int back = i + S.off - j;
        return i <= i1 && (FAR ? back >= A.window && j < A.sinks : back >= 0 && back < A.window);
    };
    LDS_AS uint8_t *ps = lds + 3 * STAGE + pair * 2 * BK * 96 + l * 16;
    // What of the wave's keys the tiles of a head's queries see.
    auto tiles_to = [&](int i) { return tile_floor(i - i0 + BK - 1); }; // tiles that start before query i
    Seen what{0, 0, 0, 0, jw < S.lk ? steps : 0};
    if (!FAR && jw < S.lk) {
        what.some = tiles_to(jw - S.off - BK + 1);
        what.none = tiles_to(jw + 31 - S.off + A.window);
        what.all = tiles_to(jw + 31 - S.off);
        what.less = tile_floor(min(i1, jw + A.window - 1 - S.off) - BK + 1 - i0) + 1;
    }
    auto work = [&](int u, int stage, int odd) { // tile u of a head; odd: that of all heads' tiles
        const int see = what(u), r0 = i0 + u * BK;
        if (see == 0)
            return;
        const LDS_AS uint8_t *qt = lds + stage * STAGE, *gt = qt + TILE;
        LDS_AS uint8_t *pt = ps + odd * BK * 96;
        // scores less lse / scale, or grad_out . v less delta; then P or dS
        const LDS_AS float *st = reinterpret_cast<const LDS_AS float *>(qt + 2 * TILE) + second * BK + 4 * h;
        f16v s[2];
#pragma unroll
        for (int qb = 0; qb < 2; ++qb)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                s[qb][e] = st[32 * qb + 8 * (e >> 2) + (e & 3)];
        add_scores<DB>(s, second ? gt : qt, L, x);
        if (second) { // dS: cells 0 .. 3 hold P's upper halves, 4 and 5 the bytes below
            u32x4 low[2];
#pragma unroll
            for (int c = 0; c < 2; ++c)
                low[c] = *reinterpret_cast<const LDS_AS u32x4 *>(pt + (4 + c) * 1024);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const u32x4 up = *reinterpret_cast<const LDS_AS u32x4 *>(pt + c * 1024);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    constexpr uint32_t BYTES[4] = {0x0504000Cu, 0x0706010Cu, 0x0504020Cu, 0x0706030Cu};
                    const int e = 8 * (c & 1) + i;
                    const float pr =
                        __uint_as_float(__builtin_amdgcn_perm(up[i / 2], low[c >> 1][2 * (c & 1) + i / 4], BYTES[i & 3]));
                    s[c >> 1][e] *= pr;
                }
            }
        } else { // P
#pragma unroll
            for (int qb = 0; qb < 2; ++qb)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    s[qb][e] = __builtin_amdgcn_exp2f(s[qb][e] * A.c);
        }
        if (see == 1) { // queries first + c, for constants c (hidden sums as in Mask)
            const int first = r0 + 4 * h;
            int least = FAR ? (j < A.sinks ? j + A.window - S.off - first : 64) : j - S.off - first;
            int most = FAR ? i1 - first : min(i1 - first, least + A.window - 1);
            asm volatile("" : "+v"(least), "+v"(most));
#pragma unroll
            for (int qb = 0; qb < 2; ++qb)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int c = 32 * qb + c_row(e, 0);
                    s[qb][e] = c >= least && c <= most ? s[qb][e] : 0.0f;
                }
        }
        if (!second) {
            u32x4 low[2];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                u32x4 up;
                uint32_t y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    y[i] = __float_as_uint(s[c >> 1][8 * (c & 1) + i]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    up[i] = __builtin_amdgcn_perm(y[2 * i + 1], y[2 * i], 0x07060302u);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    low[c >> 1][2 * (c & 1) + i] = __builtin_amdgcn_perm(y[4 * i + 1], y[4 * i], 0x0C0C0501u) |
                                                   __builtin_amdgcn_perm(y[4 * i + 3], y[4 * i + 2], 0x05010C0Cu);
                *reinterpret_cast<LDS_AS u32x4 *>(pt + c * 1024) = up;
            }
#pragma unroll
            for (int c = 0; c < 2; ++c)
                *reinterpret_cast<LDS_AS u32x4 *>(pt + (4 + c) * 1024) = low[c];
        }
        const LDS_AS uint8_t *down = second ? qt : gt;
        if (CAREFUL && see == 1)
            careful_products<DB, 2>(acc, down, L, s, h, [&](int i) { return sees_key(r0 + i); });
        else
            products<DB, 2>(acc, down, L, s);
    };
    if (total > 0)
        load(0);
    int stage = second ? 2 : 0, next = 1, u = u0 - second; // the wave's stage and tile; the stage to load next
    for (int it = 0; it <= total; ++it) {
        wait_vmcnt<0>();
        barrier();
        if (it + 1 < total)
            load(next);
        if (it - second >= 0 && it - second < total)
            work(u, stage, (it - second) & 1);
        u = u + 1 == steps ? 0 : u + 1;
        stage = stage == 2 ? 0 : stage + 1;
        next = next == 2 ? 0 : next + 1;
    }
    if (!CAREFUL && __syncthreads_or(j < S.lk && not_finite<DB>(acc)))
        return false;
    if (CAREFUL)
        __syncthreads();
    const int plane = second ? 0 : kPlane<DB>;
    if (FAR || shares > 1) {
        if (jw >= S.lk)
            return true;
        float *to = (FAR ? far_part<DB>(A, chunk, hk, j0 / 32, share)
                         : near_part<DB>(A, (A.ks ? S.k0 / 32 + b : 0) + jw / 32, hk, share)) + plane + l;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                to[(d * 16 + e) * 64] = acc[d][e];
        return true;
    }
    if (jw < S.lk) { // add the sums that sinks have from far queries
        const Chunks C(A, S, b, jw);
        for (int c = C.first; c <= C.last; ++c)
            for (int f = 0; f < A.far_shares; ++f) {
                const float *from = far_part<DB>(A, C.at + c, hk, jw / 32, f) + plane + l;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        acc[d][e] += from[(d * 16 + e) * 64];
            }
    }
    const Out &to = second ? A.gk : A.gv;
    store_rows<DB>(acc, second ? A.scale : 1.0f, lds + w * 32 * kRow<DB>,
                   to.p + (int64_t)(S.k0 + jw) * to.ts + hk * to.hs, to.ts, S.lk - jw, A.D, l);
    return true;
}

template <int DB, int NP, bool FULL>
__global__ void __launch_bounds__(128 * NP, 2) bwd_kv_kernel(Args A)
{
    __shared__ __attribute__((aligned(1024))) uint8_t smem[kBytesKV<DB, NP>];
    LDS_AS uint8_t *lds = (LDS_AS uint8_t *)smem;
    int rank, hk, share, b, j0;
    Span S;
    if (!item_of(blockIdx.x, A.tiles, A.Hk, A.shares, rank, hk, share) ||
        !span_of(A, A.ks, A.Tk, rank, 32 * NP, true, S, b, j0))
        return;
    if (!FULL)
        zero_lds<3 * kStageKV<DB>>(lds, 128 * NP);
    const int i0 = max(j0 - S.off, 0);
    const int i1 = min(min(j0 + 32 * NP, S.lk) - 2 + A.window - S.off, S.lq - 1);
    if (!backward_kv<DB, NP, FULL, false, false>(A, lds, S, j0, i0, i1, hk, b, 0, share, A.shares))
        backward_kv<DB, NP, FULL, false, true>(A, lds, S, j0, i0, i1, hk, b, 0, share, A.shares);
}

// The shares of 32 keys' sums added in order, near queries' and then far ones', and
// rounded: wave d of a plane's DB takes its elements 32 d ..
template <int DB> __global__ void __launch_bounds__(128 * DB) bwd_sum_kernel(Args A)
{
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63, n = l & 31, h = l >> 5, d = w % DB;
    const bool key = w < DB; // grad_k
    const int hk = blockIdx.y;
    int b, jw;
    Span S;
    if (!span_of(A, A.ks, A.Tk, blockIdx.x, 32, true, S, b, jw))
        return;
    const int at = (key ? 0 : kPlane<DB>) + d * 1024 + l;
    float acc[16];
#pragma unroll
    for (int e = 0; e < 16; ++e)
        acc[e] = 0.0f;
#pragma unroll 4
    for (int s = 0; s < A.shares; ++s)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            acc[e] += near_part<DB>(A, blockIdx.x, hk, s)[at + e * 64];
    const Chunks C(A, S, b, jw);
    for (int c = C.first; c <= C.last; ++c)
        for (int f = 0; f < A.far_shares; ++f)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                acc[e] += far_part<DB>(A, C.at + c, hk, jw / 32, f)[at + e * 64];
    if (jw + n >= S.lk)
        return;
    const Out &to = key ? A.gk : A.gv;
    const float by = key ? A.scale : 1.0f;
    uint16_t *row = to.p + (int64_t)(S.k0 + jw + n) * to.ts + hk * to.hs + 32 * d + 4 * h;
#pragma unroll
    for (int g = 0; g < 4; ++g)
        if (32 * d + 8 * g + 4 * h < A.D)
            *reinterpret_cast<u32x2 *>(row + 8 * g) = u32x2{pack_bf16(acc[4 * g] * by, acc[4 * g + 1] * by),
                                                            pack_bf16(acc[4 * g + 2] * by, acc[4 * g + 3] * by)};
}

template <int DB, bool FULL>
__global__ void __launch_bounds__(128) bwd_far_kernel(Args A)
{
    __shared__ __attribute__((aligned(1024))) uint8_t smem[kBytesKV<DB, 1>];
    LDS_AS uint8_t *lds = (LDS_AS uint8_t *)smem;
    int b, i0;
    Span S;
    const int hk = blockIdx.y / A.far_shares, share = blockIdx.y % A.far_shares, j0 = 32 * blockIdx.z;
    if (!span_of(A, A.qs, A.Tq, blockIdx.x, A.chunk, false, S, b, i0))
        return;
    const int i1 = min(i0 + A.chunk, S.lq) - 1, at = Chunks::number(A, S, b) + i0 / A.chunk;
    i0 = max(i0, j0 + A.window - S.off);
    if (j0 >= S.lk || i0 > i1)
        return;
    if (!FULL)
        zero_lds<3 * kStageKV<DB>>(lds, 128);
    if (!backward_kv<DB, 1, FULL, true, false>(A, lds, S, j0, i0, i1, hk, b, at, share, A.far_shares))
        backward_kv<DB, 1, FULL, true, true>(A, lds, S, j0, i0, i1, hk, b, at, share, A.far_shares);
}

// ------------------------------------------------------------------- host --

enum Kind { FWD, FWD_FEW, BWD_Q, BWD_Q_FEW, BWD_KV, BWD_FAR, BWD_SUM };

template <Kind K, int DB, bool FULL> void launch_full(const Args &A, dim3 grid, hipStream_t st)
{
    if constexpr (K == FWD)
        hipLaunchKernelGGL((fwd_kernel<DB, FULL, 1>), grid, dim3(64 * QW), 0, st, A);
    else if constexpr (K == FWD_FEW)
        hipLaunchKernelGGL((fwd_kernel<DB, FULL, 2>), grid, dim3(128 * QW), 0, st, A);
    else if constexpr (K == BWD_Q)
        hipLaunchKernelGGL((bwd_q_kernel<DB, FULL, 1>), grid, dim3(64 * QW), 0, st, A);
    else if constexpr (K == BWD_Q_FEW)
        hipLaunchKernelGGL((bwd_q_kernel<DB, FULL, 2>), grid, dim3(128 * QW), 0, st, A);
    else if constexpr (K == BWD_KV)
        hipLaunchKernelGGL((bwd_kv_kernel<DB, 4, FULL>), grid, dim3(512), 0, st, A);
    else if constexpr (K == BWD_FAR)
        hipLaunchKernelGGL((bwd_far_kernel<DB, FULL>), grid, dim3(128), 0, st, A);
    else
        hipLaunchKernelGGL((bwd_sum_kernel<DB>), grid, dim3(128 * DB), 0, st, A);
}

// f(DB, FULL) for heads of D elements
template <typename F> auto by_head_size(int D, F f)
{
    using std::integral_constant;
    switch (D) {
    case 64: return f(integral_constant<int, 2>(), std::true_type());
    case 96: return f(integral_constant<int, 3>(), std::true_type());
    case 128: return f(integral_constant<int, 4>(), std::true_type());
    default:
        return D < 64   ? f(integral_constant<int, 2>(), std::false_type())
               : D < 96 ? f(integral_constant<int, 3>(), std::false_type())
                        : f(integral_constant<int, 4>(), std::false_type());
    }
}

template <Kind K> void launch(const Args &A, dim3 grid, hipStream_t st)
{
    by_head_size(A.D, [&](auto db, auto full) { launch_full<K, db(), full()>(A, grid, st); });
}

// How often the loads of a tile by NW waves bring each 16-byte piece of its rows.
template <int DB, int NW, bool FULL> void count_loads(int D, uint8_t (*count)[16])
{
    using Load = Loader<DB, BK, NW, FULL>;
    for (int w = 0; w < NW; ++w)
        for (int l = 0; l < 64; ++l) {
            const Load load(0, D, w, l);
            for (int i = 0; i < Load::N; ++i)
                if (load.has(i, l))
                    ++count[load.row(i, l)][load.chunk(i, l)];
        }
}

// tiles of R rows that T rows of B sequences may have, numbered as span_of does
inline int64_t tiles_of(int64_t T, int64_t R, int64_t B, bool packed)
{
    return packed ? T / R + B : (T + R - 1) / R;
}

// queries of a chunk of the sinks' far sums: at most about 64 chunks
inline int64_t chunk_of(int64_t Tq)
{
    int64_t c = FAR_CHUNK;
    while (c * 64 < Tq)
        c *= 2;
    return c;
}

inline int64_t blocks_of(int64_t D) { return D <= 64 ? 2 : D <= 96 ? 3 : 4; }

// Blocks of 32 sinks that can have queries the window or more behind them, and chunks of
// such queries.
inline int64_t far_blocks(int64_t Tk, int64_t window, int64_t sinks)
{
    return window == 0 ? 0 : (std::min(sinks, std::max<int64_t>(Tk - window, 0)) + 31) / 32;
}
inline int64_t far_chunks(int64_t Tq, int64_t Tk, int64_t B, int64_t window)
{
    return Tq / chunk_of(Tq) + std::min(B - 1, Tk / (std::min<int64_t>(window, MX_ATTN_MAX_TOKENS) + 1)) + 1;
}

// floats of the sinks' far sums
inline int64_t far_floats(int64_t Tq, int64_t Tk, int64_t Hk, int64_t D, int64_t B, int64_t window, int64_t sinks, int64_t shares)
{
    return far_chunks(Tq, Tk, B, window) * Hk * far_blocks(Tk, window, sinks) * shares * blocks_of(D) * (2 * 16 * 64);
}

inline int64_t round256(int64_t n) { return (n + 255) / 256 * 256; }
inline int64_t row_bytes(int64_t Tq, int64_t Hq) { return round256(4 * Tq * Hq); }

// A launch of tiles of queries, with two groups of waves where there are fewer
// workgroups than compute units, or not many more and the last queries of a sequence
// without a window see twice the average (3000 tokens of 16 heads of 128: 70 us, so 57;
// 2000 of 32 of 64 with a window of 500: 26, so 30).
template <Kind MANY, Kind FEW> void launch_queries(Args &A, hipStream_t st)
{
    A.tiles = (int)tiles_of(A.Tq, 32 * QW, A.B, A.qs != nullptr);
    const dim3 grid((unsigned)items(A.tiles, A.Hk, A.G));
    const int64_t n = (int64_t)A.tiles * A.Hk * A.G;
    n <= 256 || (n <= 600 && A.window == MX_ATTN_MAX_TOKENS) ? launch<FEW>(A, grid, st) : launch<MANY>(A, grid, st);
}

// Shares of the queries that a block of 128 keys, and the sinks' far sums of a chunk,
// are summed over.  A tile of 64 queries takes a workgroup about 1.8 us, and few
// workgroups leave compute units idle; but shares are written, read and added (about
// 4 us and 0.5 us a MB).
struct BwdPlan {
    int shares, far_shares;
};

inline BwdPlan bwd_plan(int64_t Tq, int64_t Tk, int64_t Hq, int64_t Hk, int64_t D, int64_t B, int64_t window, int64_t sinks)
{
    BwdPlan P{1, 1};
    const int64_t G = Hq / Hk, tiles = tiles_of(Tk, 128, B, true) * Hk;
    const int64_t length = std::max<int64_t>(Tq / B, 1), seen = window > 0 ? std::min(std::min(window, length) + 128, length) : length;
    const double steps = (double)(G * (seen / BK + 1)), mb = (double)tiles * 4 * blocks_of(D) * 8e-3;
    double best = 1e30;
    for (int s = 1; s <= 8 && (s == 1 || tiles < 192); ++s) {
        const double rounds = (double)((tiles * s + 255) / 256);
        const double us = rounds * (steps / s * 1.8 + 4) + (s > 1 ? 4 + 0.5 * s * mb : 0);
        if (us < 0.95 * best) {
            best = us;
            P.shares = s;
        }
    }
    const int64_t far = tiles_of(Tq, chunk_of(Tq), B, true) * Hk * std::max<int64_t>((sinks + 31) / 32, 1);
    P.far_shares = (int)std::max<int64_t>(std::min<int64_t>(256 / far, 8), 1);
    return P;
}

} // namespace mxa

namespace {

using mxk::aligned;
using mxk::check_heads;
using mxk::fail;
using mxk::launched;

mx_status check_common(const mx_heads *q, const mx_heads *k, const mx_heads *v, int64_t Tq, int64_t Tk, int64_t D,
                       const int32_t *q_start, const int32_t *k_start, int64_t sequences, int64_t window, int64_t sinks,
                       float scale, bool backward)
{
    if (Tq < 0 || Tk < 0)
        return fail(MX_EINVAL, "Tq and Tk must be >= 0");
    if (D <= 0 || D % 8 != 0)
        return fail(MX_EINVAL, "D must be a positive multiple of 8");
    if (!q || !k || !v || q->heads < 1 || k->heads < 1 || q->heads % k->heads != 0)
        return fail(MX_EINVAL, "q, k and v must be given, q's heads a multiple of k's");
    if (window < 0 || sinks < 0)
        return fail(MX_EINVAL, "window and sinks must be >= 0");
    if (!(scale >= 0x1p-100f && scale <= 0x1p100f))
        return fail(MX_EINVAL, "scale must be from 2^-100 to 2^100");
    if (q_start ? sequences < 1 || !aligned(q_start, 4) || !aligned(k_start, 4) : sequences != 1 || k_start != nullptr)
        return fail(MX_EINVAL, "q_start must hold sequences + 1 starts; without it there is one sequence, and no k_start");
    if (q_start && !k_start && Tq != Tk)
        return fail(MX_EINVAL, "without k_start, k must have the tokens of q");
    if (D > MX_ATTN_MAX_D || sinks > MX_ATTN_MAX_SINKS)
        return fail(MX_EUNSUPPORTED, "heads of more than %d elements, or more than %d sinks", MX_ATTN_MAX_D, MX_ATTN_MAX_SINKS);
    if (Tq > MX_ATTN_MAX_TOKENS || Tk > MX_ATTN_MAX_TOKENS || q->heads > 4096 || sequences > 1 << 20)
        return fail(MX_EUNSUPPORTED, "at most %d tokens, 4096 heads and 2^20 sequences", MX_ATTN_MAX_TOKENS);
    // workgroups as they are launched (a key block has shares only where its blocks are few)
    const int64_t G = q->heads / k->heads;
    if ((mxa::tiles_of(std::max(Tq, Tk), 128, sequences, true) + 1) * q->heads > 1 << 30 ||
        !mxk::launchable(mxa::items(mxa::tiles_of(Tq, 128, sequences, q_start != nullptr), k->heads, G), 256) ||
        (backward && !mxk::launchable(mxa::items(mxa::tiles_of(Tk, 128, sequences, q_start != nullptr), k->heads, 1), 512)))
        return fail(MX_EUNSUPPORTED, "too many tokens times heads");
    return MX_OK;
}

mxa::In in_of(const mx_heads *h)
{
    return {static_cast<const uint16_t *>(h->data), h->token_stride, h->head_stride};
}
mxa::Out out_of(const mx_heads *h)
{
    return {static_cast<uint16_t *>(h->data), h->token_stride, h->head_stride};
}

mxa::Args arguments(const mx_heads *q, const mx_heads *k, const mx_heads *v, int64_t Tq, int64_t Tk, int64_t D,
                    const int32_t *q_start, const int32_t *k_start, int64_t sequences, int64_t window, int64_t sinks,
                    float scale)
{
    mxa::Args A{};
    A.q = in_of(q);
    A.k = in_of(k);
    A.v = in_of(v);
    A.qs = q_start;
    A.ks = k_start ? k_start : q_start;
    A.Tq = (int)Tq;
    A.Tk = (int)Tk;
    A.B = (int)sequences;
    A.Hk = (int)k->heads;
    A.G = (int)(q->heads / k->heads);
    A.D = (int)D;
    // no two positions are further apart than 2^30
    A.window = window == 0 || window > MX_ATTN_MAX_TOKENS ? MX_ATTN_MAX_TOKENS : (int)window;
    A.sinks = A.window == MX_ATTN_MAX_TOKENS ? 0 : (int)sinks;
    A.scale = scale;
    A.c = scale * mxa::LOG2E;
    return A;
}

} // namespace

extern "C" {

mx_status window_attn_fwd(const mx_heads *q, const mx_heads *k, const mx_heads *v, int64_t Tq, int64_t Tk, int64_t D,
                          const int32_t *q_start, const int32_t *k_start, int64_t sequences, int64_t window, int64_t sinks,
                          float scale, const mx_heads *out, float *lse, hipStream_t stream)
{
    mxk::clear_error();
    mx_status st = check_common(q, k, v, Tq, Tk, D, q_start, k_start, sequences, window, sinks, scale, false);
    if (st != MX_OK || (st = check_heads(q, "q", Tq, D, q->heads, false)) != MX_OK ||
        (st = check_heads(k, "k", Tk, D, k->heads, false)) != MX_OK ||
        (st = check_heads(v, "v", Tk, D, k->heads, false)) != MX_OK ||
        (st = check_heads(out, "out", Tq, D, q->heads, true)) != MX_OK)
        return st;
    if (!aligned(lse, 4))
        return fail(MX_EINVAL, "lse must be 4-byte aligned");
    if (Tq == 0)
        return MX_OK;
    mxa::Args A = arguments(q, k, v, Tq, Tk, D, q_start, k_start, sequences, window, sinks, scale);
    A.out = out_of(out);
    A.lse_out = lse;
    mxa::launch_queries<mxa::FWD, mxa::FWD_FEW>(A, stream);
    return launched();
}

size_t window_attn_bwd_workspace_bytes(int64_t Tq, int64_t Tk, int64_t q_heads, int64_t k_heads, int64_t D, int64_t sequences,
                                       int64_t window, int64_t sinks)
{
    if (Tq <= 0 || Tq > MX_ATTN_MAX_TOKENS || Tk < 0 || Tk > MX_ATTN_MAX_TOKENS || q_heads < 1 || q_heads > 4096 || k_heads < 1 ||
        k_heads > q_heads || D < 1 || D > MX_ATTN_MAX_D || sequences < 1 || sequences > 1 << 20 || window < 0 || sinks < 0 ||
        sinks > MX_ATTN_MAX_SINKS)
        return 0;
    const mxa::BwdPlan P = mxa::bwd_plan(Tq, Tk, q_heads, k_heads, D, sequences, window, sinks);
    const int64_t block = mxa::blocks_of(D) * (2 * 16 * 64 * 4);
    const int64_t near = P.shares > 1 ? mxa::tiles_of(Tk, 32, sequences, true) + 1 : 0;
    return 2 * mxa::row_bytes(Tq, q_heads) + k_heads * block * near * P.shares +
           sizeof(float) * mxa::far_floats(Tq, Tk, k_heads, D, sequences, window, sinks, P.far_shares);
}

mx_status window_attn_bwd(const mx_heads *grad_out, const mx_heads *q, const mx_heads *k, const mx_heads *v,
                          const mx_heads *out, const float *lse, int64_t Tq, int64_t Tk, int64_t D, const int32_t *q_start,
                          const int32_t *k_start, int64_t sequences, int64_t window, int64_t sinks, float scale,
                          const mx_heads *grad_q, const mx_heads *grad_k, const mx_heads *grad_v, void *workspace,
                          size_t workspace_bytes, hipStream_t stream)
{
    mxk::clear_error();
    mx_status st = check_common(q, k, v, Tq, Tk, D, q_start, k_start, sequences, window, sinks, scale, true);
    if (st != MX_OK || (st = check_heads(grad_out, "grad_out", Tq, D, q->heads, false)) != MX_OK ||
        (st = check_heads(q, "q", Tq, D, q->heads, false)) != MX_OK ||
        (st = check_heads(k, "k", Tk, D, k->heads, false)) != MX_OK ||
        (st = check_heads(v, "v", Tk, D, k->heads, false)) != MX_OK ||
        (st = check_heads(out, "out", Tq, D, q->heads, false)) != MX_OK ||
        (st = check_heads(grad_q, "grad_q", Tq, D, q->heads, true)) != MX_OK ||
        (st = check_heads(grad_k, "grad_k", Tk, D, k->heads, true)) != MX_OK ||
        (st = check_heads(grad_v, "grad_v", Tk, D, k->heads, true)) != MX_OK)
        return st;
    const size_t need = window_attn_bwd_workspace_bytes(Tq, Tk, q->heads, k->heads, D, sequences, window, sinks);
    if (Tq > 0 && (!lse || !aligned(lse, 4) || !workspace || !aligned(workspace, 256) || workspace_bytes < need))
        return fail(MX_EINVAL, "lse must be given, 4-byte aligned, and a 256-byte aligned workspace of %zu bytes", need);
    if (Tq == 0 && Tk == 0)
        return MX_OK;
    mxa::Args A = arguments(q, k, v, Tq, Tk, D, q_start, k_start, sequences, window, sinks, scale);
    const bool packed = q_start != nullptr;
    if (Tq > 0) {
        A.go = in_of(grad_out);
        A.o = in_of(out);
        A.lse = lse;
        A.lse_s = static_cast<float *>(workspace);
        A.delta = A.lse_s + mxa::row_bytes(Tq, q->heads) / 4;
        A.chunk = (int)mxa::chunk_of(Tq);
        const mxa::BwdPlan P = mxa::bwd_plan(Tq, Tk, q->heads, k->heads, D, sequences, window, sinks);
        A.shares = P.shares;
        A.far_shares = P.far_shares;
        A.far = A.delta + mxa::row_bytes(Tq, q->heads) / 4;
        A.far_blocks = (int)mxa::far_blocks(Tk, window, sinks);
        A.near = A.far + mxa::far_floats(Tq, Tk, k->heads, D, sequences, window, sinks, P.far_shares);
        A.out = out_of(grad_q);
        mxa::launch_queries<mxa::BWD_Q, mxa::BWD_Q_FEW>(A, stream);
    } else {
        A.chunk = A.shares = A.far_shares = 1;
    }
    if (Tk > 0) {
        A.gk = out_of(grad_k);
        A.gv = out_of(grad_v);
        if (A.far_blocks > 0)
            mxa::launch<mxa::BWD_FAR>(A, dim3((unsigned)mxa::tiles_of(Tq, A.chunk, sequences, packed), (unsigned)(A.Hk * A.far_shares),
                                              (unsigned)A.far_blocks), stream);
        A.tiles = (int)mxa::tiles_of(Tk, 128, sequences, packed);
        mxa::launch<mxa::BWD_KV>(A, dim3((unsigned)mxa::items(A.tiles, A.Hk, A.shares)), stream);
        if (A.shares > 1)
            mxa::launch<mxa::BWD_SUM>(A, dim3((unsigned)mxa::tiles_of(Tk, 32, sequences, packed), (unsigned)A.Hk), stream);
    }
    return launched();
}

int mxt_attn_tile_loads(int64_t D, int waves, uint8_t *count)
{
    if (D <= 0 || D % 8 != 0 || D > MX_ATTN_MAX_D || (waves != 2 && waves != 4 && waves != 8))
        return -1;
    uint8_t(*rows)[16] = reinterpret_cast<uint8_t(*)[16]>(count);
    mxa::by_head_size((int)D, [&](auto db, auto full) {
        waves == 2   ? mxa::count_loads<db(), 2, full()>((int)D, rows)
        : waves == 4 ? mxa::count_loads<db(), 4, full()>((int)D, rows)
                     : mxa::count_loads<db(), 8, full()>((int)D, rows);
    });
    return mxa::BK;
}

} // extern "C"

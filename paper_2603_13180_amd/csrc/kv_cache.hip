// kv_cache.hip -- a paged cache of keys and values: new tokens' heads into it, and
// attention of new tokens (one a sequence, or a tree of drafted ones) over it.
//
// Sequence b has length[b] cached tokens; its new ones stand behind them, drafted
// token i at key length + i.  Token i sees cached key j where place - j < window or
// j < sinks, and drafted key u where bit u of its mask is set and the same holds of
// u's place; a token's place is length + popcount(mask) - 1.
//
// The group's query heads and the sequence's new tokens are rows of one product, so
// the cache is read once for all of them.  A workgroup takes one key head of one
// sequence, RB blocks of 32 rows and a share of the keys; KW groups of RB waves take
// tiles of keys in turn, each with its own maximum and sums, joined at the end, and
// across workgroups by a second kernel.
//
// What bounds it: for single tokens the cache's bytes.  One token behind 131072 (8 key
// heads of 128, 537 MB) 81 to 84 us and 6 for the join, 6.4 TB/s (16 loads of 1 KB in
// flight a wave; with twice the workgroups 86, of those reads through the caches 109, and
// pages looked up in the tile itself instead of one ahead 139); 61 tokens behind 4916 to
// 16384 in E4M3 (1.37 GB) 264 to 300, 4.6 to 5.2 TB/s, of which the sequences' lengths
// cost a tenth.  For trees the products: 63 tokens behind 16 sequences of up to 8192 145
// to 170 us, 0.5 to 0.6 PFLOP/s (the whole call over codes 166, over bf16 152).  The append
// moves 134 MB in 21.2 to 22.3 us, 6.0 TB/s; 102 MB into codes, the whole call, in 20.7.
#include "attn.h"
#include "norm_cast.h"

namespace mxa {

struct Cache {
    uint8_t *k, *v;          // pages [heads, slots, D] of bf16 elements or E4M3 codes
    uint8_t *ks, *vs;        // E8M0 scales [heads, slots, D / 32] of codes
    int64_t page_bytes, page_scales; // from page to page
    int pages, shift;        // 2^shift slots
    const int *table;        // [B, width] pages of every sequence
    const int *length;       // [B]
    int width, B, Hk, D;
};

// New tokens: sequence b's are start[b] .. start[b + 1] - 1, or without starts
// token b.
__device__ __forceinline__ int first_of(const int *start, int b, int T)
{
    return start ? min(max(start[b], 0), T) : min(b, T);
}

// ----------------------------------------------------------------- append --

struct AppendArgs {
    Cache C;
    In k, v;
    const int *start, *rows;
    int T, S; // new tokens, rows of k and v
    int tpw;  // tokens of a workgroup
};

constexpr int APPEND_THREADS = 256, APPEND_TOKENS = 64, APPEND_STARTS = 1024;

template <bool MX> __global__ void __launch_bounds__(APPEND_THREADS) append_kernel(AppendArgs A)
{
    __shared__ int starts[APPEND_STARTS];
    __shared__ int64_t to[APPEND_TOKENS]; // page's first row of the head 0 and slot, or -1
    __shared__ int from[APPEND_TOKENS];
    __shared__ int slots[APPEND_TOKENS];
    const Cache &C = A.C;
    const int t0 = blockIdx.x * A.tpw, nt = min(A.tpw, A.T - t0);
    const bool near = A.start && C.B < APPEND_STARTS;
    if (near)
        for (int i = threadIdx.x; i <= C.B; i += APPEND_THREADS)
            starts[i] = first_of(A.start, i, A.T);
    __syncthreads();
    if ((int)threadIdx.x < nt) {
        const int t = t0 + threadIdx.x;
        auto first = [&](int b) { return near ? starts[b] : first_of(A.start, b, A.T); };
        int b = A.start ? 0 : t, hi = A.start ? C.B - 1 : t;
        while (b < hi) {
            const int mid = (b + hi + 1) >> 1;
            if (first(mid) <= t)
                b = mid;
            else
                hi = mid - 1;
        }
        const int i = t - first(b), src = A.rows ? A.rows[t] : t;
        int page = -1, slot = 0;
        if (b < C.B && i >= 0 && t < first(b + 1) && (unsigned)src < (unsigned)A.S) {
            const int64_t at = (int64_t)max(C.length[b], 0) + i;
            slot = (int)(at & ((1 << C.shift) - 1));
            if (at >> C.shift < C.width)
                page = C.table[(int64_t)b * C.width + (at >> C.shift)];
        }
        to[threadIdx.x] = (unsigned)page < (unsigned)C.pages ? page : -1;
        slots[threadIdx.x] = slot;
        from[threadIdx.x] = src;
    }
    __syncthreads();
    const int row = C.D / 8, per = C.Hk * row; // 16-byte chunks
    for (int i = threadIdx.x; i < nt * per; i += APPEND_THREADS) {
        const int t = i / per, h = (i - t * per) / row, c = i - t * per - h * row;
        const int64_t page = to[t], src = from[t];
        if (page < 0)
            continue;
        const int64_t slot = ((int64_t)h << C.shift) + slots[t];
        const u32x4 k = *reinterpret_cast<const u32x4 *>(A.k.p + src * A.k.ts + h * A.k.hs + c * 8);
        const u32x4 v = *reinterpret_cast<const u32x4 *>(A.v.p + src * A.v.ts + h * A.v.hs + c * 8);
        if constexpr (!MX) {
            *reinterpret_cast<u32x4 *>(C.k + page * C.page_bytes + (slot * C.D + c * 8) * 2) = k;
            *reinterpret_cast<u32x4 *>(C.v + page * C.page_bytes + (slot * C.D + c * 8) * 2) = v;
        } else {
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                const u32x4 x = which ? v : k;
                // the block's largest magnitude: four lanes hold its 32 elements
                uint32_t m = 0;
                float t8[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    m = max(m, max(x[e] & 0x7FFFu, (x[e] >> 16) & 0x7FFFu));
                    t8[2 * e] = __uint_as_float(x[e] << 16);
                    t8[2 * e + 1] = __uint_as_float(x[e] & 0xFFFF0000u);
                }
                m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));
                m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));
                const uint32_t byte = mxk::e8m0_byte<false>(__uint_as_float(m << 16), MX_SCALE_RCEIL);
                const float scale = __uint_as_float(byte << 23);
                u32x2 codes = {mxk::e4m3x4_hw(t8[0], t8[1], t8[2], t8[3], scale),
                               mxk::e4m3x4_hw(t8[4], t8[5], t8[6], t8[7], scale)};
                if (byte == 0xFFu)
                    codes = u32x2{mxk::nan_codes_e4m3(x[0], x[1]), mxk::nan_codes_e4m3(x[2], x[3])};
                *reinterpret_cast<u32x2 *>((which ? C.v : C.k) + page * C.page_bytes + slot * C.D + c * 8) = codes;
                if (c % 4 == 0)
                    (which ? C.vs : C.ks)[page * C.page_scales + slot * (C.D / 32) + c / 4] = (uint8_t)byte;
            }
        }
    }
}

// -------------------------------------------------------------- attention --

constexpr int MAX_NEW = MX_ATTN_MAX_NEW;
// Sequences that a launch takes by length: workgroups are started in order, and a long
// one that comes last is waited for (61 of 5000 to 16384 keys of codes: 295 us, in their own order 321).
constexpr int MAX_SORTED = 256;

struct CachedArgs {
    Cache C;
    In q;
    Out out;
    const int *start;
    const int64_t *bits; // [T] or NULL: every token sees the ones before it and itself
    float *part;         // [T, Hq, splits, D] sums and
    float2 *stat;        // [T, Hq, splits] maxima (powers of two) and sums of exponentials
    int T, G, max_new, blocks; // blocks of 32 RB rows
    int splits, window, sinks;
    int by_length; // sequences in the order of their lengths, the longest first
    float c;
};

// A sequence of a workgroup.
struct Rows {
    int t0, n, len, R; // first token, tokens, cached tokens, rows
    int end;           // keys that the table has pages for
    const int *pages;
    // the page of key j, or one that the cache does not have
    __device__ __forceinline__ int page_of(int j, int shift) const { return j < end ? pages[j >> shift] : -1; }
};

template <int RB> struct Shape {
    static constexpr int KW = RB >= 4 ? 1 : 4 / RB, NW = RB * KW;
    static constexpr int NB = RB >= 4 ? 2 : 1, KEYS = 32 * NB; // of a tile
    static constexpr int STAGES = RB == 1 ? 1 : 2;
};

// The pages of a tile's runs of 16 keys: the same for every thread of its group.
template <int RB> struct Pages {
    static constexpr int RUNS = Shape<RB>::KEYS / 16;
    int id[RUNS];
    __device__ __forceinline__ Pages(const Rows &S, int shift, int j0)
    {
#pragma unroll
        for (int y = 0; y < RUNS; ++y)
            id[y] = __builtin_amdgcn_readfirstlane(S.page_of(j0 + 16 * y, shift));
    }
};

// A thread's part of a tile of keys and values on its way to LDS.
template <int DB, int RB, bool MX> struct Staged {
    using O = Shape<RB>;
    static constexpr int PER = kChunks<DB> / (MX ? 2 : 1);      // 16-byte pieces of a row
    static constexpr int PIECES = O::KEYS * PER, N = (PIECES + 64 * RB - 1) / (64 * RB);
    static constexpr int RUNS = O::KEYS / 16;
    u32x4 k[N], v[N];
    u32x4 scales;   // the wave's copy of the tile's scale bytes, 16 a lane: K's rows, V's rows
    uint32_t there; // bit y: run y's page is there
    int rows;       // that the tile has

    // Keys j0 .. of the tile, those past the end and those of pages that are not
    // there as zeros.  i: the thread's number among those of its group.
    __device__ __forceinline__ void load(const Cache &C, const Rows &S, const Pages<RB> &P, int hk, int j0, int i)
    {
        const uint8_t *kb[RUNS], *vb[RUNS];
        there = 0;
        rows = S.end - j0;
        if constexpr (MX) // a run's scales lie one behind the other
            scales = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int y = 0; y < RUNS; ++y) {
            const bool is = (unsigned)P.id[y] < (unsigned)C.pages;
            there |= (uint32_t)is << y;
            const int64_t slot = ((int64_t)hk << C.shift) + ((j0 + 16 * y) & ((1 << C.shift) - 1));
            const int64_t at = (is ? P.id[y] : 0) * C.page_bytes + slot * C.D * (MX ? 1 : 2);
            kb[y] = C.k + at;
            vb[y] = C.v + at;
            if constexpr (MX) {
                const int64_t sc = (is ? P.id[y] : 0) * C.page_scales + slot * (C.D / 32);
                const int n = C.D / 32, l = i & 63, of = l - y * n; // K's run y, then V's behind all of K's
                if (is && of >= 0 && of < n)
                    scales = *reinterpret_cast<const u32x4 *>(C.ks + sc + of * 16);
                if (is && of - RUNS * n >= 0 && of - RUNS * n < n)
                    scales = *reinterpret_cast<const u32x4 *>(C.vs + sc + (of - RUNS * n) * 16);
            }
        }
#pragma unroll
        for (int x = 0; x < N; ++x) {
            constexpr int STEP = 64 * RB / PER; // rows that the group's threads take at once
            const int p = x * 64 * RB + i, r = p / PER, c = p % PER;
            k[x] = v[x] = u32x4{0, 0, 0, 0};
            int y = x * STEP / 16;
            const uint8_t *kp = kb[y < RUNS ? y : 0], *vp = vb[y < RUNS ? y : 0];
            if constexpr (STEP > 16) { // several runs: the thread's own
                y = r / 16;
#pragma unroll
                for (int z = 0; z < RUNS; ++z) {
                    kp = y == z ? kb[z] : kp;
                    vp = y == z ? vb[z] : vp;
                }
            }
            if ((PIECES % (64 * RB) == 0 || p < PIECES) && j0 + r < S.end && (there >> y & 1) && c * (MX ? 16 : 8) < C.D) {
                const uint32_t off = (uint32_t)((r & 15) * C.D * (MX ? 1 : 2) + c * 16);
                k[x] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(kp + off));
                v[x] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(vp + off));
            }
        }
    }

    // 16 codes times 2^(s - 127) as bf16 (exact but for bf16's subnormals)
    __device__ __forceinline__ static void decode(u32x4 codes, uint32_t s, u32x4 &lo, u32x4 &hi)
    {
        const float by = __uint_as_float(s << 23);
        u32x4 o[2];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            o[e / 2][e % 2 * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[e], by, false));
            o[e / 2][e % 2 * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[e], by, true));
        }
        if (s == 255) // a scale that is not a number
            o[0] = o[1] = u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
        lo = o[0];
        hi = o[1];
    }

    // `area`: the wave's, for scales.
    __device__ __forceinline__ void store(const Cache &C, LDS_AS uint8_t *tile, LDS_AS uint8_t *area, int i) const
    {
        constexpr int TILE = O::KEYS * kRow<DB>;
        const int n = C.D / 32;
        if constexpr (MX) {
            if ((i & 63) < 2 * RUNS * n)
                *reinterpret_cast<LDS_AS u32x4 *>(area + (i & 63) * 16) = scales;
        }
#pragma unroll
        for (int x = 0; x < N; ++x) {
            const int p = x * 64 * RB + i, r = p / PER, c = p % PER;
            if (PIECES % (64 * RB) != 0 && p >= PIECES)
                continue;
            LDS_AS uint8_t *row = tile + r * kRow<DB>;
            if constexpr (MX) {
                u32x4 lo, hi;
                const int a = ((2 * c) ^ swz<DB>(r)) * 16, b = ((2 * c + 1) ^ swz<DB>(r)) * 16;
                // what slots past the end have for scales does not count
                const bool is = r < rows && c * 16 < C.D;
                const uint32_t sk = is ? area[r * n + c / 2] : 127, sv = is ? area[(O::KEYS + r) * n + c / 2] : 127;
                decode(k[x], sk, lo, hi);
                *reinterpret_cast<LDS_AS u32x4 *>(row + a) = lo;
                *reinterpret_cast<LDS_AS u32x4 *>(row + b) = hi;
                decode(v[x], sv, lo, hi);
                *reinterpret_cast<LDS_AS u32x4 *>(row + TILE + a) = lo;
                *reinterpret_cast<LDS_AS u32x4 *>(row + TILE + b) = hi;
            } else {
                const int a = (c ^ swz<DB>(r)) * 16;
                *reinterpret_cast<LDS_AS u32x4 *>(row + a) = k[x];
                *reinterpret_cast<LDS_AS u32x4 *>(row + TILE + a) = v[x];
            }
        }
    }
};

// A workgroup's LDS: the groups' tiles, or their sums when they are joined; the queries.
template <int DB, int RB>
constexpr int kQueriesAt = std::max(Shape<RB>::KW * Shape<RB>::STAGES * 2 * Shape<RB>::KEYS * kRow<DB>,
                                    Shape<RB>::KW > 1 ? Shape<RB>::KW *RB *(DB * 1024 + 96) * 4 : 0);

template <int DB, int RB, bool MX, bool CAREFUL>
__device__ __forceinline__ bool cached(const CachedArgs &A, LDS_AS uint8_t *lds, const LDS_AS int *places, const Rows &S,
                                       int hk, int split, int r0)
{
    using O = Shape<RB>;
    constexpr int TILE = O::KEYS * kRow<DB>, GROUP = O::STAGES * 2 * TILE;
    const Cache &C = A.C;
    const int thread = thread_number<CAREFUL>();
    const int w = __builtin_amdgcn_readfirstlane(thread >> 6), l = thread & 63, n = l & 31, h = l >> 5;
    const int kw = w / RB, in_group = thread - kw * RB * 64;
    const Lane<DB> L(l);
    const int rw = r0 + 32 * (w % RB), r = min(rw + n, S.R - 1), i = r / A.G, hq = hk * A.G + r % A.G;
    const bool mine = rw + n < S.R;
    // The rows' queries: in registers, or in LDS for the KW groups that share them (the
    // tiles in flight take the registers).
    constexpr bool SHARED = RB == 1;
    LDS_AS uint8_t *const qt = lds + kQueriesAt<DB, RB>;
    u32x4 x[2 * DB]; // all on their way before the first is waited for
    if (!SHARED || kw == 0) {
        const uint16_t *row = A.q.p + (int64_t)(S.t0 + i) * A.q.ts + hq * A.q.hs;
#pragma unroll
        for (int ks = 0; ks < 2 * DB; ++ks)
            x[ks] = *reinterpret_cast<const u32x4 *>(row + min(16 * ks + 8 * h, C.D - 8));
    }
    LDS_AS uint8_t *const area = qt + (SHARED ? 32 * kRow<DB> : 0) + w * (O::KEYS * 8);
    const uint64_t all = S.n >= 64 ? ~0ull : (1ull << S.n) - 1;
    uint64_t bits = (A.bits ? (uint64_t)A.bits[S.t0 + i] : (2ull << i) - 1) & all;
    const int place = S.len + __popcll(bits) - 1;
    if (A.window <= MAX_NEW) // drafted tokens that lie the window before (places differ by 64 at most)
        for (int u = 0; u < S.n; ++u)
            if (place - places[u] >= A.window && places[u] >= A.sinks)
                bits &= ~(1ull << u);
    // Tiles: the sinks', then from the first key that the window of a token at
    // length - 1 holds.  Row blocks differ in their places, not in their tiles.
    const int first = max(S.len - A.window, 0) / O::KEYS;
    const int sinks = min((min(A.sinks, S.end) + O::KEYS - 1) / O::KEYS, first);
    const int tiles = sinks + max((S.end + O::KEYS - 1) / O::KEYS - first, 0);
    const int from = (int)((int64_t)tiles * split / A.splits), to = (int)((int64_t)tiles * (split + 1) / A.splits);
    auto key_of = [&](int t) { return (t < sinks ? t : first + t - sinks) * O::KEYS; };
    // The keys of a tile that the row sees, a bit each: of the cached ones those of the
    // window and the sinks, of the drafted ones its bits.
    auto below = [&](int x) { return x <= 0 ? 0ull : x >= 64 ? ~0ull : (1ull << x) - 1; };
    auto seen_of = [&](int j0, uint32_t there) {
        const int to_draft = S.len - j0;
        uint64_t m = (below(to_draft) & ~below(place - A.window + 1 - j0)) | below(min(A.sinks, S.len) - j0);
        if (to_draft < 64 && to_draft > -64)
            m |= to_draft >= 0 ? bits << to_draft : bits >> -to_draft;
#pragma unroll
        for (int y = 0; y < O::KEYS / 16; ++y)
            m &= there >> y & 1 ? ~0ull : ~(0xFFFFull << 16 * y);
        return m;
    };
    f16v o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
        o[d] = zero16();
    float m = -FLT_MAX, sum = 0.0f;
    bool any = false;
    const int rounds = (to - from + O::KW - 1) / O::KW;
    auto tile_of = [&](int it) { return from + it * O::KW + kw; };
    // A tile goes through registers to LDS; DEPTH tiles are in flight, and the pages
    // of the one after them are on their way as well.  (Codes are half the bytes: with
    // one tile of them a wave, too little is in flight for the memory's latency.)
    constexpr int DEPTH = MX && RB == 1 ? 2 : 1;
    Staged<DB, RB, MX> staged[DEPTH];
    const int last = max(to - 1, from);
    Pages<RB> pages(S, C.shift, key_of(min(tile_of(0), last)));
    auto load = [&](Staged<DB, RB, MX> &next, int it) {
        if (tile_of(it) < to)
            next.load(C, S, pages, hk, key_of(tile_of(it)), in_group);
        pages = Pages<RB>(S, C.shift, key_of(min(tile_of(it + 1), last)));
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        load(staged[d], d);
    b8 q[SHARED ? 1 : 2 * DB];
#pragma unroll
    for (int ks = 0; ks < 2 * DB; ++ks) {
        const u32x4 own = 16 * ks + 8 * h < C.D ? x[ks] : u32x4{0, 0, 0, 0};
        if constexpr (!SHARED)
            q[ks] = __builtin_bit_cast(b8, own);
        else if (kw == 0)
            *reinterpret_cast<LDS_AS u32x4 *>(qt + n * kRow<DB> + ((2 * ks + h) ^ swz<DB>(n)) * 16) = own;
    }
    auto query = [&](int ks) { return SHARED ? row_frag<DB>(qt, L, ks, 0) : q[SHARED ? 0 : ks]; };
    if (SHARED)
        __syncthreads();
    auto step = [&](Staged<DB, RB, MX> &next, int it) __attribute__((always_inline)) {
        const int t = tile_of(it);
        LDS_AS uint8_t *kt = lds + kw * GROUP + (O::STAGES == 2 ? (it & 1) * 2 * TILE : 0), *vt = kt + TILE;
        const uint32_t there = next.there;
        if (t < to)
            next.store(C, kt, area, in_group);
        if (RB > 1)
            __syncthreads();
        load(next, it + DEPTH);
        if (t >= to || rw >= S.R)
            return;
        const int j0 = key_of(t);
        const bool full = j0 + O::KEYS <= S.len && there == (1u << O::KEYS / 16) - 1 &&
                          S.len + S.n - 1 - j0 < A.window;
        const uint64_t keys = full ? ~0ull : seen_of(j0, there);
        auto seen = [&](int x) { return (keys >> x & 1) != 0; };
        f16v s[O::NB];
#pragma unroll
        for (int x = 0; x < O::NB; ++x)
            s[x] = zero16();
#pragma unroll
        for (int ks = 0; ks < 2 * DB; ++ks)
#pragma unroll
            for (int x = 0; x < O::NB; ++x)
                s[x] = mfma(row_frag<DB>(kt, L, ks, x), query(ks), s[x]);
        if (!full) {
            const uint64_t half = keys >> (4 * h);
#pragma unroll
            for (int x = 0; x < O::NB; ++x)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    s[x][e] = (uint32_t)(half >> 32 * x) & 1u << c_row(e, 0) ? s[x][e] : -INFINITY;
        }
        any |= O::KEYS == 64 ? keys != 0 : (uint32_t)keys != 0;
        float mt = -INFINITY;
#pragma unroll
        for (int x = 0; x < O::NB; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                mt = fmaxf(mt, s[x][e]);
        mt = halves_max(mt) * A.c;
        if (__builtin_amdgcn_ballot_w64(mt > m + 8.0f)) { // as in the packed sequences' kernel
            const float mn = fmaxf(m, mt), by = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            sum *= by;
#pragma unroll
            for (int d = 0; d < DB; ++d)
                o[d] *= by;
        }
#pragma unroll
        for (int x = 0; x < O::NB; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[x][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][e], A.c, -m));
                sum += s[x][e];
            }
        if (CAREFUL && !full)
            careful_products<DB, O::NB>(o, vt, L, s, h, seen);
        else
            products<DB, O::NB>(o, vt, L, s);
    };
    for (int it = 0; it < rounds; it += DEPTH)
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (d == 0 || it + d < rounds)
                step(staged[d], it + d);
    if (!CAREFUL && __syncthreads_or(mine && not_finite<DB>(o)))
        return false;
    if (CAREFUL)
        __syncthreads();
    sum = halves_sum(sum);
    any = halves_max(any ? 1.0f : 0.0f) > 0.0f;
    // join the key groups: group kw takes over blocks of 32 elements
    if constexpr (O::KW > 1) {
        LDS_AS float *stat = reinterpret_cast<LDS_AS float *>(lds) + RB * DB * O::KW * 1024;
        auto cell = [&](int g, int what) { return stat + ((g * RB + w % RB) * 3 + what) * 32 + n; };
        if (h == 0) {
            *cell(kw, 0) = m;
            *cell(kw, 1) = sum;
            *cell(kw, 2) = any ? 1.0f : 0.0f;
        }
        __syncthreads();
        float mn = m;
        for (int g = 0; g < O::KW; ++g)
            mn = fmaxf(mn, *cell(g, 0));
        sum = 0.0f;
        for (int g = 0; g < O::KW; ++g) {
            sum += *cell(g, 1) * __builtin_amdgcn_exp2f(*cell(g, 0) - mn);
            any |= *cell(g, 2) != 0.0f;
        }
        const float by = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        LDS_AS float *sums = reinterpret_cast<LDS_AS float *>(lds);
        auto at = [&](int g, int d, int e) { return sums + (((g * RB + w % RB) * DB + d) * 16 + e) * 64 + l; };
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                *at(kw, d, e) = o[d][e] * by;
        __syncthreads();
        if (kw != 0)
            return true;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                float t = 0.0f;
#pragma unroll
                for (int g = 0; g < O::KW; ++g)
                    t += *at(g, d, e);
                o[d][e] = t;
            }
    }
    if (rw >= S.R)
        return true;
    if (A.splits > 1) {
        // a share that sees nothing is marked by a sum of 0, one that sees only
        // scores of -inf by -1
        const int64_t row = ((int64_t)(S.t0 + i) * A.G * C.Hk + hq) * A.splits + split;
        if (mine && h == 0)
            A.stat[row] = float2{m, sum > 0.0f || sum != sum ? sum : any ? -1.0f : 0.0f};
        if (mine)
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    if (32 * d + 8 * g + 4 * h < C.D)
                        *reinterpret_cast<float4 *>(A.part + row * C.D + 32 * d + 8 * g + 4 * h) =
                            float4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
        return true;
    }
    const float by = any ? 1.0f / sum : 0.0f;
    if (mine)
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (32 * d + 8 * g + 4 * h < C.D)
                    *reinterpret_cast<u32x2 *>(A.out.p + (int64_t)(S.t0 + i) * A.out.ts + hq * A.out.hs + 32 * d + 8 * g + 4 * h) =
                        u32x2{pack_bf16(o[d][4 * g] * by, o[d][4 * g + 1] * by),
                              pack_bf16(o[d][4 * g + 2] * by, o[d][4 * g + 3] * by)};
    return true;
}

template <int DB, int RB, bool MX> __global__ void __launch_bounds__(64 * Shape<RB>::NW, 2) cached_kernel(CachedArgs A)
{
    __shared__ __attribute__((aligned(1024))) uint8_t smem[kQueriesAt<DB, RB> + (RB == 1 ? 32 * kRow<DB> : 0) +
                                                            (MX ? Shape<RB>::NW * Shape<RB>::KEYS * 8 : 0)];
    __shared__ int places[MAX_NEW];
    __shared__ int lengths[MAX_SORTED], sequence;
    LDS_AS uint8_t *lds = (LDS_AS uint8_t *)smem;
    const Cache &C = A.C;
    int id = blockIdx.x;
    const int split = id % A.splits;
    id /= A.splits;
    const int hk = id % C.Hk;
    id /= C.Hk;
    const int block = id % A.blocks;
    int b = id / A.blocks;
    if (A.by_length) { // the sequence with b longer ones
        for (int i = threadIdx.x; i < C.B; i += 64 * Shape<RB>::NW)
            lengths[i] = C.length[i];
        __syncthreads();
        if ((int)threadIdx.x < C.B) {
            const int mine = lengths[threadIdx.x];
            int longer = 0;
            for (int i = 0; i < C.B; ++i)
                longer += lengths[i] > mine || (lengths[i] == mine && i < (int)threadIdx.x);
            if (longer == b)
                sequence = threadIdx.x;
        }
        __syncthreads();
        b = sequence;
    }
    Rows S;
    S.t0 = first_of(A.start, b, A.T);
    S.n = min(min(first_of(A.start, b + 1, A.T) - S.t0, A.max_new), MAX_NEW);
    S.R = S.n * A.G;
    const int r0 = block * 32 * RB;
    if (S.n <= 0 || r0 >= S.R)
        return;
    S.len = min(max(C.length[b], 0), MX_ATTN_MAX_TOKENS);
    S.end = min(S.len + S.n, C.width << C.shift);
    S.pages = C.table + (int64_t)b * C.width;
    if ((int)threadIdx.x < S.n) {
        const uint64_t all = S.n >= 64 ? ~0ull : (1ull << S.n) - 1;
        places[threadIdx.x] = S.len - 1 + (A.bits ? __popcll((uint64_t)A.bits[S.t0 + threadIdx.x] & all) : (int)threadIdx.x + 1);
    }
    __syncthreads();
    if (!cached<DB, RB, MX, false>(A, lds, (const LDS_AS int *)places, S, hk, split, r0))
        cached<DB, RB, MX, true>(A, lds, (const LDS_AS int *)places, S, hk, split, r0);
}

// A row's shares joined, in order: a workgroup takes one row, groups of 32 lanes
// every eighth share, four elements a lane.
constexpr int MAX_SPLITS = 128;
__global__ void __launch_bounds__(256) join_kernel(CachedArgs A)
{
    __shared__ float weight[MAX_SPLITS];
    __shared__ float4 sums[8][32];
    __shared__ float part[8];
    const Cache &C = A.C;
    const int64_t row = blockIdx.x;
    const int Hq = A.G * C.Hk, l = threadIdx.x & 63, sub = threadIdx.x >> 5;
    const int64_t t = row / Hq;
    if (t < first_of(A.start, 0, A.T) || t >= first_of(A.start, C.B, A.T))
        return;
    // every wave finds the maximum by itself
    const float2 none = {-FLT_MAX, 0.0f};
    const float2 x0 = l < A.splits ? A.stat[row * A.splits + l] : none;
    const float2 x1 = l + 64 < A.splits ? A.stat[row * A.splits + l + 64] : none;
    float m = fmaxf(x0.x, x1.x);
    for (int x = 32; x; x >>= 1)
        m = fmaxf(m, __shfl_xor(m, x));
    const bool any = __builtin_amdgcn_ballot_w64(x0.y != 0.0f || x1.y != 0.0f) != 0;
    if (threadIdx.x < 64) { // shares without a sum have no weight, and their sums are not there
        auto w = [&](float2 x) { return x.y == 0.0f || x.y == -1.0f ? -1.0f : __builtin_amdgcn_exp2f(x.x - m); };
        weight[l] = w(x0);
        weight[l + 64] = w(x1);
    }
    __syncthreads();
    const int e = 4 * (threadIdx.x & 31);
    float sum = 0.0f;
    float4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int s = sub; s < A.splits; s += 8) {
        const float by = weight[s];
        if (by == -1.0f)
            continue;
        sum = __builtin_fmaf(A.stat[row * A.splits + s].y, by, sum);
        if (e < C.D) {
            const float4 v = *reinterpret_cast<const float4 *>(A.part + (row * A.splits + s) * C.D + e);
            o.x = __builtin_fmaf(v.x, by, o.x);
            o.y = __builtin_fmaf(v.y, by, o.y);
            o.z = __builtin_fmaf(v.z, by, o.z);
            o.w = __builtin_fmaf(v.w, by, o.w);
        }
    }
    sums[sub][threadIdx.x & 31] = o;
    if ((threadIdx.x & 31) == 0)
        part[sub] = sum;
    __syncthreads();
    if (threadIdx.x >= 32 || e >= C.D)
        return;
    for (int g = 1; g < 8; ++g) {
        const float4 v = sums[g][threadIdx.x];
        o.x += v.x;
        o.y += v.y;
        o.z += v.z;
        o.w += v.w;
        sum += part[g];
    }
    const float by = any ? 1.0f / sum : 0.0f;
    *reinterpret_cast<u32x2 *>(A.out.p + t * A.out.ts + (row - t * Hq) * A.out.hs + e) =
        u32x2{pack_bf16(o.x * by, o.y * by), pack_bf16(o.z * by, o.w * by)};
}

// The same for few shares: 32 lanes a row, eight rows a workgroup.
constexpr int FEW_SPLITS = 16;
__global__ void __launch_bounds__(256) join_few_kernel(CachedArgs A)
{
    const Cache &C = A.C;
    const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int Hq = A.G * C.Hk, l = threadIdx.x & 31, e = 4 * l;
    const int64_t t = row / Hq;
    if (t < first_of(A.start, 0, A.T) || t >= first_of(A.start, C.B, A.T))
        return;
    const float2 mine = l < A.splits ? A.stat[row * A.splits + l] : float2{-FLT_MAX, 0.0f};
    float m = mine.x;
    for (int x = 8; x; x >>= 1)
        m = fmaxf(m, __shfl_xor(m, x, 16));
    m = __shfl(m, 0, 32);
    // shares without a sum have no weight, and their sums are not there
    const float w = mine.y == 0.0f || mine.y == -1.0f ? -1.0f : __builtin_amdgcn_exp2f(mine.x - m);
    float sum = 0.0f;
    bool any = false;
    float4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < A.splits; ++s) {
        const float by = __shfl(w, s, 32), y = __shfl(mine.y, s, 32);
        any |= y != 0.0f;
        if (by == -1.0f)
            continue;
        sum = __builtin_fmaf(y, by, sum);
        if (e < C.D) {
            const float4 v = *reinterpret_cast<const float4 *>(A.part + (row * A.splits + s) * C.D + e);
            o.x = __builtin_fmaf(v.x, by, o.x);
            o.y = __builtin_fmaf(v.y, by, o.y);
            o.z = __builtin_fmaf(v.z, by, o.z);
            o.w = __builtin_fmaf(v.w, by, o.w);
        }
    }
    const float by = any ? 1.0f / sum : 0.0f;
    if (e < C.D)
        *reinterpret_cast<u32x2 *>(A.out.p + t * A.out.ts + (row - t * Hq) * A.out.hs + e) =
            u32x2{pack_bf16(o.x * by, o.y * by), pack_bf16(o.z * by, o.w * by)};
}

// ------------------------------------------------------------------- host --

// Blocks of 32 rows of a workgroup, workgroups a sequence and head takes for its
// rows, shares of its keys.
struct CachedPlan {
    int RB, blocks, splits;
};

inline CachedPlan cached_plan(int64_t B, int64_t Hk, int64_t G, int64_t max_new, int64_t keys)
{
    CachedPlan P;
    const int64_t rows = max_new * G;
    P.RB = rows <= 32 ? 1 : rows <= 64 ? 2 : rows <= 128 ? 4 : 8;
    P.blocks = (int)((rows + 32 * P.RB - 1) / (32 * P.RB));
    // As many workgroups as run at once, two a compute unit; twice that where sequences of
    // different lengths have few rows and shares would be long, so that short ones make
    // room (32 + 8 heads of 128, new tokens behind uneven lengths, us with 512 and with 1024
    // workgroups: 61 behind up to 2048 60 and 67, 8 behind 8192 39 and 46, 16 behind 16384
    // 121 and 120, 61 behind 16384 of codes 303 and 261; one behind 131072 89 and 94).
    const int64_t groups = std::max<int64_t>(B * Hk * P.blocks, 1);
    const int64_t want = P.RB < 8 && B > 1 && groups * keys >= 512 * 4096 ? 1024 : 512;
    // at least 256 keys a share
    const int64_t most = std::max<int64_t>(keys / 256, 1);
    P.splits = (int)std::max<int64_t>(std::min<int64_t>(std::min<int64_t>(want / groups, most), MAX_SPLITS), 1);
    return P;
}

template <int DB, bool MX> void launch_cached(const CachedArgs &A, int RB, unsigned grid, hipStream_t st)
{
    switch (RB) {
    case 1: hipLaunchKernelGGL((cached_kernel<DB, 1, MX>), dim3(grid), dim3(256), 0, st, A); break;
    case 2: hipLaunchKernelGGL((cached_kernel<DB, 2, MX>), dim3(grid), dim3(256), 0, st, A); break;
    case 4: hipLaunchKernelGGL((cached_kernel<DB, 4, MX>), dim3(grid), dim3(256), 0, st, A); break;
    default: hipLaunchKernelGGL((cached_kernel<DB, 8, MX>), dim3(grid), dim3(512), 0, st, A); break;
    }
}

} // namespace mxa

namespace {

using mxk::aligned;
using mxk::check_heads;
using mxk::fail;
using mxk::launched;

mx_status check_cache(const mx_kv_cache *c, int64_t D, const int32_t *table, int64_t width, const int32_t *length,
                      const int32_t *start, int64_t T, int64_t sequences)
{
    if (!c || c->heads < 1 || c->pages < 0 || width < 0 || T < 0 || sequences < 0)
        return fail(MX_EINVAL, "the cache must be given, with a head at least; sizes must be >= 0");
    if (c->type != MX_CACHE_BF16 && c->type != MX_CACHE_E4M3)
        return fail(MX_EINVAL, "the cache's type must be MX_CACHE_BF16 or MX_CACHE_E4M3");
    const bool mx = c->type == MX_CACHE_E4M3;
    const int64_t step = mx ? 32 : 8;
    if (D <= 0 || D % step != 0)
        return fail(MX_EINVAL, "D must be a positive multiple of %d", (int)step);
    if (D > MX_ATTN_MAX_D || c->heads > 4096 || sequences > 1 << 20 || T > MX_ATTN_MAX_TOKENS || c->pages > 0x7FFFFFFF)
        return fail(MX_EUNSUPPORTED, "at most %d elements a head, 4096 heads, 2^20 sequences, %d tokens, 2^31 pages",
                    MX_ATTN_MAX_D, MX_ATTN_MAX_TOKENS);
    if (c->page_size < 16 || (c->page_size & (c->page_size - 1)) != 0)
        return fail(MX_EINVAL, "page_size must be a power of two from 16 on");
    if (c->page_size > MX_ATTN_MAX_TOKENS || width > MX_ATTN_MAX_TOKENS / c->page_size)
        return fail(MX_EUNSUPPORTED, "a sequence's pages hold more than %d tokens", MX_ATTN_MAX_TOKENS);
    const int64_t page = c->heads * c->page_size * D;
    if (c->pages > 1 && (c->page_stride < page || c->page_stride % (mx ? 16 : 8) != 0 || c->page_stride > INT64_MAX / 8 / c->pages))
        return fail(MX_EINVAL, "page_stride must be at least heads page_size D elements, whole 16-byte pieces");
    if (mx && c->pages > 1 && (c->scale_page_stride < page / 32 || c->scale_page_stride % 16 != 0 || c->scale_page_stride > INT64_MAX / 8 / c->pages))
        return fail(MX_EINVAL, "scale_page_stride must be at least heads page_size D / 32, whole 16-byte pieces");
    if (T == 0 || sequences == 0)
        return MX_OK;
    if (c->pages > 0 && (!c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16) || (mx && (!c->k_scales || !c->v_scales || !aligned(c->k_scales, 16) || !aligned(c->v_scales, 16)))))
        return fail(MX_EINVAL, "the cache's k and v, and the scales of codes, must be non-NULL and 16-byte aligned");
    if ((width > 0 && !table) || !aligned(table, 4) || !length || !aligned(length, 4) || !aligned(start, 4))
        return fail(MX_EINVAL, "table and length must be non-NULL; table, length and start 4-byte aligned");
    if (!start && T != sequences)
        return fail(MX_EINVAL, "without start every sequence has one new token");
    return MX_OK;
}

mxa::Cache cache_of(const mx_kv_cache *c, int64_t D, const int32_t *table, int64_t width, const int32_t *length,
                    int64_t sequences)
{
    mxa::Cache C{};
    C.k = static_cast<uint8_t *>(c->k);
    C.v = static_cast<uint8_t *>(c->v);
    C.ks = c->k_scales;
    C.vs = c->v_scales;
    C.page_bytes = c->pages > 1 ? c->page_stride * (c->type == MX_CACHE_E4M3 ? 1 : 2) : 0;
    C.page_scales = c->pages > 1 ? c->scale_page_stride : 0;
    C.pages = (int)c->pages;
    C.shift = __builtin_ctzll((uint64_t)c->page_size);
    C.table = table;
    C.length = length;
    C.width = (int)width;
    C.B = (int)sequences;
    C.Hk = (int)c->heads;
    C.D = (int)D;
    return C;
}

// Keys that a token can see at most.
int64_t keys_of(int64_t width, int64_t page_size, int64_t max_new, int64_t max_length, int64_t window, int64_t sinks)
{
    int64_t n = width * page_size;
    if (max_length > 0)
        n = std::min(n, max_length + max_new);
    if (window > 0) // either may be as large as an int64
        n = std::min(n, std::min(window, n) + max_new + std::min(sinks, n));
    return n;
}

} // namespace

extern "C" {

mx_status kv_cache_append(const mx_kv_cache *cache, const mx_heads *k, const mx_heads *v, int64_t T, int64_t S, int64_t D,
                          const int32_t *table, int64_t table_width, const int32_t *length, const int32_t *start,
                          int64_t sequences, const int32_t *rows, hipStream_t stream)
{
    mxk::clear_error();
    mx_status st = check_cache(cache, D, table, table_width, length, start, T, sequences);
    if (st != MX_OK)
        return st;
    if (S < 0 || S > MX_ATTN_MAX_TOKENS || (!rows && S < T) || !aligned(rows, 4))
        return fail(MX_EINVAL, "k and v must have a row for every new token, or rows (4-byte aligned) name theirs");
    if ((st = check_heads(k, "k", S, D, cache->heads, false)) != MX_OK ||
        (st = check_heads(v, "v", S, D, cache->heads, false)) != MX_OK)
        return st;
    if (T == 0 || S == 0 || sequences == 0 || cache->pages == 0)
        return MX_OK;
    mxa::AppendArgs A{};
    A.C = cache_of(cache, D, table, table_width, length, sequences);
    A.k = {static_cast<const uint16_t *>(k->data), k->token_stride, k->head_stride};
    A.v = {static_cast<const uint16_t *>(v->data), v->token_stride, v->head_stride};
    A.start = start;
    A.rows = rows;
    A.T = (int)T;
    A.S = (int)S;
    const int64_t per = cache->heads * D / 8;
    A.tpw = (int)std::min<int64_t>(std::max<int64_t>(mxa::APPEND_THREADS / per, 1), mxa::APPEND_TOKENS);
    const dim3 grid((unsigned)((T + A.tpw - 1) / A.tpw));
    if (!mxk::launchable(grid.x, mxa::APPEND_THREADS))
        return fail(MX_EUNSUPPORTED, "too many tokens");
    if (cache->type == MX_CACHE_E4M3)
        hipLaunchKernelGGL((mxa::append_kernel<true>), grid, dim3(mxa::APPEND_THREADS), 0, stream, A);
    else
        hipLaunchKernelGGL((mxa::append_kernel<false>), grid, dim3(mxa::APPEND_THREADS), 0, stream, A);
    return launched();
}

size_t kv_cache_attn_fwd_workspace_bytes(int64_t T, int64_t q_heads, int64_t k_heads, int64_t D, int64_t sequences,
                                         int64_t page_size, int64_t table_width, int64_t max_new, int64_t max_length,
                                         int64_t window, int64_t sinks)
{
    if (T <= 0 || T > MX_ATTN_MAX_TOKENS || k_heads < 1 || q_heads < k_heads || q_heads > 4096 || D < 1 || D > MX_ATTN_MAX_D ||
        sequences < 1 || sequences > 1 << 20 || page_size < 1 || table_width < 0 ||
        table_width > MX_ATTN_MAX_TOKENS / page_size || max_new < 1 || max_new > MX_ATTN_MAX_NEW || max_length < 0 ||
        max_length > MX_ATTN_MAX_TOKENS || window < 0 || sinks < 0)
        return 0;
    const mxa::CachedPlan P = mxa::cached_plan(sequences, k_heads, q_heads / k_heads, max_new,
                                               keys_of(table_width, page_size, max_new, max_length, window, sinks));
    return P.splits == 1 ? 0 : (size_t)T * q_heads * P.splits * (D + 2) * sizeof(float);
}

mx_status kv_cache_attn_fwd(const mx_kv_cache *cache, const mx_heads *q, int64_t T, int64_t D, const int32_t *table,
                            int64_t table_width, const int32_t *length, const int32_t *start, int64_t sequences,
                            int64_t max_new, int64_t max_length, const int64_t *ancestors, int64_t window, int64_t sinks,
                            float scale, const mx_heads *out, void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    mxk::clear_error();
    mx_status st = check_cache(cache, D, table, table_width, length, start, T, sequences);
    if (st != MX_OK)
        return st;
    if (!q || q->heads < 1 || q->heads % cache->heads != 0)
        return fail(MX_EINVAL, "q must be given, its heads a multiple of the cache's");
    if (q->heads > 4096)
        return fail(MX_EUNSUPPORTED, "at most 4096 heads");
    if ((st = check_heads(q, "q", T, D, q->heads, false)) != MX_OK ||
        (st = check_heads(out, "out", T, D, q->heads, true)) != MX_OK)
        return st;
    if (max_new < 1 || max_length < 0 || window < 0 || sinks < 0)
        return fail(MX_EINVAL, "max_new must be >= 1; max_length, window and sinks >= 0");
    if (max_new > MX_ATTN_MAX_NEW || max_length > MX_ATTN_MAX_TOKENS)
        return fail(MX_EUNSUPPORTED, "at most %d new tokens a sequence, and %d cached", MX_ATTN_MAX_NEW, MX_ATTN_MAX_TOKENS);
    if (!(scale >= 0x1p-100f && scale <= 0x1p100f))
        return fail(MX_EINVAL, "scale must be from 2^-100 to 2^100");
    if (!aligned(ancestors, 8))
        return fail(MX_EINVAL, "ancestors must be 8-byte aligned");
    if (T == 0 || sequences == 0)
        return MX_OK;
    const int64_t Hk = cache->heads, G = q->heads / Hk;
    const mxa::CachedPlan P = mxa::cached_plan(
        sequences, Hk, G, max_new, keys_of(table_width, cache->page_size, max_new, max_length, window, sinks));
    const int64_t grid = (int64_t)P.splits * Hk * P.blocks * sequences, rows = T * q->heads;
    const int64_t joins = P.splits == 1 ? 0 : P.splits <= mxa::FEW_SPLITS ? (rows + 7) / 8 : rows;
    if (!mxk::launchable(grid, P.RB == 8 ? 512 : 256) || !mxk::launchable(joins, 256))
        return fail(MX_EUNSUPPORTED, "too many sequences, or tokens, times heads");
    const size_t need = P.splits == 1 ? 0 : (size_t)rows * P.splits * (D + 2) * sizeof(float);
    if (need && (!workspace || !aligned(workspace, 256) || workspace_bytes < need))
        return fail(MX_EINVAL, "a 256-byte aligned workspace of %zu bytes is needed", need);
    mxa::CachedArgs A{};
    A.C = cache_of(cache, D, table, table_width, length, sequences);
    A.q = {static_cast<const uint16_t *>(q->data), q->token_stride, q->head_stride};
    A.out = {static_cast<uint16_t *>(out->data), out->token_stride, out->head_stride};
    A.start = start;
    A.bits = ancestors;
    A.part = static_cast<float *>(workspace);
    A.stat = reinterpret_cast<float2 *>(A.part + rows * P.splits * D);
    A.T = (int)T;
    A.G = (int)G;
    A.max_new = (int)max_new;
    A.blocks = P.blocks;
    A.splits = P.splits;
    A.window = window == 0 || window > MX_ATTN_MAX_TOKENS ? MX_ATTN_MAX_TOKENS * 2 : (int)window;
    A.sinks = (int)std::min<int64_t>(sinks, MX_ATTN_MAX_TOKENS);
    A.c = scale * mxa::LOG2E;
    A.by_length = sequences > 1 && sequences <= mxa::MAX_SORTED && grid > 256 &&
                  keys_of(table_width, cache->page_size, max_new, max_length, window, sinks) >= 2048;
    const int DB = D <= 64 ? 2 : D <= 96 ? 3 : 4;
    if (cache->type == MX_CACHE_E4M3) {
        switch (DB) {
        case 2: mxa::launch_cached<2, true>(A, P.RB, (unsigned)grid, stream); break;
        case 3: mxa::launch_cached<3, true>(A, P.RB, (unsigned)grid, stream); break;
        default: mxa::launch_cached<4, true>(A, P.RB, (unsigned)grid, stream); break;
        }
    } else {
        switch (DB) {
        case 2: mxa::launch_cached<2, false>(A, P.RB, (unsigned)grid, stream); break;
        case 3: mxa::launch_cached<3, false>(A, P.RB, (unsigned)grid, stream); break;
        default: mxa::launch_cached<4, false>(A, P.RB, (unsigned)grid, stream); break;
        }
    }
    if (P.splits > 1 && P.splits <= mxa::FEW_SPLITS)
        hipLaunchKernelGGL(mxa::join_few_kernel, dim3((unsigned)joins), dim3(256), 0, stream, A);
    else if (P.splits > 1)
        hipLaunchKernelGGL(mxa::join_kernel, dim3((unsigned)joins), dim3(256), 0, stream, A);
    return launched();
}

} // extern "C"

// attn.h -- what the attention kernels share: tiles of heads in LDS, their
// fragments for the matrix cores, the masked products.
//
// All products are v_mfma_f32_32x32x16_bf16: A [32, 16], B [16, 32], C [32, 32],
// lane l with n = l % 32 and half h = l / 32 holding row n of A and column n of
// B at k = 8 h .. 8 h + 7, and of C column n at rows 8 g + 4 h + e (g, e = 0 .. 3,
// element 4 g + e).  A kernel computes scores with the axis it sums over as C's
// rows: a lane then has 16 of one row's 32 scores, its sums need one exchange
// between the halves, and elements 8 s .. 8 s + 7, rounded to bf16, are the B
// operand of the next product at the k order 16 s + 8 u + 4 h + j (element 4 u +
// j).  That product's A is a tile read down its columns in the same order: two
// transposing 8-byte LDS reads.
#pragma once

#include <hip/hip_runtime.h>
#include <float.h>
#include <stdint.h>

#include <algorithm>
#include <utility>

#include "heads.h"
#include "mx_gemm.h"
#include "mxnorm.h"

#pragma clang fp contract(off)

namespace mxa {

using mxg::barrier;
using mxg::NXCD;
using mxg::u32x4;
using mxg::wait_vmcnt;

typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// two floats to bf16, to nearest even, the first in the low half
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{a, b}), b2));
}

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// Heads of up to 32 DB elements; a tile's rows in LDS hold 64 or 128, 16-byte
// chunk c of row r at chunk c ^ swz(r).
template <int DB> constexpr int kRow = DB <= 2 ? 128 : 256; // bytes
template <int DB> constexpr int kChunks = kRow<DB> / 16;

// The 16 rows of a group of lanes that read one chunk each, and the 4 rows by 64
// bytes of a transposing read, lie in different banks.
template <int DB> __host__ __device__ __forceinline__ int swz(int r)
{
    return DB <= 2 ? ((r >> 1) & 1) << 2 | ((r >> 2) & 3) : (r & 3) << 2 | ((r >> 2) & 3);
}

__device__ __forceinline__ void lds_load16(const void *p, uint32_t lds_base)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "{m0}"(lds_base) : "memory");
}

__device__ __forceinline__ uint32_t lds_address(const LDS_AS uint8_t *p) { return (uint32_t)(uintptr_t)p; }
__device__ __forceinline__ LDS_AS uint8_t *lds_pointer(uint32_t a) { return (LDS_AS uint8_t *)(uintptr_t)a; }

// The thread's number.  A kernel's second, careful pass asks apart: what the compiler
// could keep for it from the first would take registers from the first's loop.
template <bool APART> __device__ __forceinline__ int thread_number()
{
    int t = threadIdx.x;
    if (APART)
        asm volatile("" : "+v"(t));
    return t;
}

// One kind of heads: element (t, h, e) at p[t ts + h hs + e].
struct In {
    const uint16_t *p;
    int64_t ts, hs;
};
struct Out {
    uint16_t *p;
    int64_t ts, hs;
};

// Loads tiles of ROWS rows of a head into LDS, by NW waves.  FULL: the heads have all
// of their 32 DB elements.  Chunks past D keep what the LDS held: behind the last head
// there may be no memory to read.
template <int DB, int ROWS, int NW, bool FULL> struct Loader {
    static constexpr int RPL = 64 / kChunks<DB>, N = ROWS / RPL / NW; // rows of a load, loads of a wave
    static_assert(ROWS % (RPL * NW) == 0, "whole loads for every wave");
    int64_t ts;
    uint32_t off[N]; // the lane's bytes from the tile's first row
    int first, D;    // the wave's first row

    __host__ __device__ __forceinline__ Loader(int64_t stride, int d, int w, int l) : ts(stride), first(w * N * RPL), D(d)
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
            off[i] = (uint32_t)row(i, l) * (uint32_t)ts * 2 + chunk(i, l) * 16;
    }
    __host__ __device__ __forceinline__ int row(int i, int l) const { return first + i * RPL + l / kChunks<DB>; }
    __host__ __device__ __forceinline__ uint32_t chunk(int i, int l) const { return (l % kChunks<DB>) ^ swz<DB>(row(i, l)); }
    // Whether the head has the chunk.  FULL: a lane's rows differ in the lower two bits of
    // swz alone, so its chunks are all before 4 DB or none is (all, but for DB = 3).
    __host__ __device__ __forceinline__ bool has(int i, int l) const
    {
        return FULL ? 4 * DB == kChunks<DB> || (int)chunk(0, l) < 4 * DB : (int)chunk(i, l) * 8 < D;
    }

    // rows r0 .. (those past `last` as `last`)
    __device__ __forceinline__ void load(const uint16_t *head, int r0, int last, uint32_t lds, int l) const
    {
        const uint16_t *base = head + (int64_t)r0 * ts;
        const uint32_t to = lds + w_bytes();
        if (__builtin_expect(ts >= 1 << 24, 0)) { // 32-bit offsets do not hold a tile
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (has(i, l))
                    lds_load16(head + (int64_t)min(r0 + row(i, l), last) * ts + chunk(i, l) * 8, to + i * 1024);
        } else if (r0 + ROWS - 1 > last) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (has(i, l))
                    mxg::lds_load16(base, (uint32_t)min(row(i, l), last - r0) * (uint32_t)ts * 2 + chunk(i, l) * 16, to + i * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (has(i, l))
                    mxg::lds_load16(base, off[i], to + i * 1024);
        }
    }
    __device__ __forceinline__ uint32_t w_bytes() const { return first / RPL * 1024; }
};

// A run of tiles by what a wave's rows see of them: 0 before `some` and from `none`
// on, 2 (all) from `all` to `less` - 1, 1 (some) else.
// `sinks` tiles in front of the run are seen in part.
struct Seen {
    int sinks, some, all, less, none;
    __device__ __forceinline__ int operator()(int t) const
    {
        return t >= all && t < less ? 2 : t < sinks || (t >= some && t < none) ? 1 : 0;
    }
};

// Tiles 0 .. n - 1 through STAGES LDS stages (2 or 3), loads STAGES - 1 tiles ahead,
// one barrier a tile.  LOADS: a wave's loads of a tile.
template <int STAGES, int LOADS, typename Load, typename Work>
__device__ __forceinline__ void tile_loop(int n, Load load, Work work)
{
    constexpr int AHEAD = STAGES - 1;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (i < n)
            load(i, i);
    int mine = 0, next = AHEAD; // the stage of tile it, and of tile it + AHEAD
    for (int it = 0; it < n; ++it) {
        if (AHEAD > 1 && it + 1 < n)
            wait_vmcnt<LOADS>();
        else
            wait_vmcnt<0>();
        barrier();
        if (it + AHEAD < n)
            load(it + AHEAD, next);
        work(it, mine);
        mine = mine == AHEAD ? 0 : mine + 1;
        next = next == AHEAD ? 0 : next + 1;
    }
}

// A lane's offsets into a tile.  Of an offset, the bits that say which 16 bytes (ks)
// or which 32 columns (d) of its row are its own: they are XORed in when it is used,
// behind a sum that differs from tile to tile, so that no register holds them.
template <int DB> struct Lane {
    uint32_t row;   // chunk h of row n
    uint32_t tr[2]; // the transposing read of rows 8 u + 4 h .. + 3, columns 0 .. 31

    __device__ __forceinline__ explicit Lane(int l)
    {
        const int n = l & 31, h = l >> 5, i = l & 15;
        row = n * kRow<DB> + (h ^ swz<DB>(n)) * 16;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = 8 * u + 4 * h + (i >> 2), c = 2 * ((l >> 4) & 1) + ((i & 3) >> 1);
            tr[u] = r * kRow<DB> + (c ^ swz<DB>(r)) * 16 + (i & 1) * 8;
        }
    }
};

// elements 16 ks + 8 h .. of rows 32 b + n
template <int DB>
__device__ __forceinline__ b8 row_frag(const LDS_AS uint8_t *tile, const Lane<DB> &L, int ks, int b)
{
    return *reinterpret_cast<const LDS_AS b8 *>(lds_pointer((lds_address(tile) + L.row) ^ (ks * 32)) + b * 32 * kRow<DB>);
}

// elements 32 d + n of rows 16 s + 8 u + 4 h + j
template <int DB>
__device__ __forceinline__ b8 col_frag(const LDS_AS uint8_t *tile, const Lane<DB> &L, int s, int d)
{
    typedef short s4 __attribute__((ext_vector_type(4)));
    s4 x[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
        x[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_AS s4 *>(
            lds_pointer((lds_address(tile) + L.tr[u]) ^ (d * 64)) + s * 16 * kRow<DB>));
    return __builtin_bit_cast(b8, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
}

__device__ __forceinline__ f16v mfma(b8 a, b8 b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ f16v zero16()
{
    return f16v{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
}

// elements 8 s .. 8 s + 7, rounded to nearest even
__device__ __forceinline__ b8 pack8(const f16v &x, int s)
{
    const u32x4 w = {pack_bf16(x[8 * s], x[8 * s + 1]), pack_bf16(x[8 * s + 2], x[8 * s + 3]),
                     pack_bf16(x[8 * s + 4], x[8 * s + 5]), pack_bf16(x[8 * s + 6], x[8 * s + 7])};
    return __builtin_bit_cast(b8, w);
}

// the row of element e of C, from the block's first
__device__ __forceinline__ int c_row(int e, int h) { return 8 * (e >> 2) + 4 * h + (e & 3); }

// max and sum over the two lanes that share a column
__device__ __forceinline__ float halves_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// acc += tile^T x, the tile of 32 NB rows, x in C's layout and rounded to bf16
template <int DB, int NB>
__device__ __forceinline__ void products(f16v (&acc)[DB], const LDS_AS uint8_t *tile, const Lane<DB> &L, const f16v (&x)[NB])
{
#pragma unroll
    for (int s = 0; s < 2 * NB; ++s) {
        const b8 y = pack8(x[s >> 1], s & 1);
#pragma unroll
        for (int d = 0; d < DB; ++d)
            acc[d] = mfma(col_frag<DB>(tile, L, s, d), y, acc[d]);
    }
}

// s += the tile's 64 rows times x
template <int DB>
__device__ __forceinline__ void add_scores(f16v (&s)[2], const LDS_AS uint8_t *tile, const Lane<DB> &L, const b8 (&x)[2 * DB])
{
#pragma unroll
    for (int ks = 0; ks < 2 * DB; ++ks)
#pragma unroll
        for (int b = 0; b < 2; ++b)
            s[b] = mfma(row_frag<DB>(tile, L, ks, b), x[ks], s[b]);
    // eight fragments are on their way ahead of the products
    __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
    for (int i = 0; i < 4 * DB - 8; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x8, 8, 0);
}

// s = the tile's 64 rows times x
template <int DB>
__device__ __forceinline__ void scores(f16v (&s)[2], const LDS_AS uint8_t *tile, const Lane<DB> &L, const b8 (&x)[2 * DB])
{
    s[0] = s[1] = zero16();
    add_scores<DB>(s, tile, L, x);
}

// acc += tile^T x of a tile some of whose rows are masked and may hold infinities or
// NaN: 0 times those is NaN, so every row is a product of its own, kept where
// seen(row) of the lane's column.  Only for tiles where the plain product gave
// something that is not finite.
template <int DB, int NB, typename Seen>
__device__ __forceinline__ void careful_products(f16v (&acc)[DB], const LDS_AS uint8_t *tile, const Lane<DB> &L,
                                                 const f16v (&x)[NB], int h, Seen seen)
{
    typedef short s8 __attribute__((ext_vector_type(8)));
#pragma unroll
    for (int s = 0; s < 2 * NB; ++s) {
        const s8 xi = __builtin_bit_cast(s8, pack8(x[s >> 1], s & 1));
#pragma unroll 1
        for (int r = 0; r < 16; ++r) {
            const bool mine = ((r >> 2) & 1) == h, see = seen(16 * s + r);
            const int e = 4 * (r >> 3) + (r & 3);
            s8 xr;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                xr[i] = mine && i == e ? xi[i] : (short)0;
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                s8 a = __builtin_bit_cast(s8, col_frag<DB>(tile, L, s, d));
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    a[i] = mine && i == e ? a[i] : (short)0;
                const f16v t = mfma(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, xr), acc[d]);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    acc[d][i] = see ? t[i] : acc[d][i];
            }
        }
    }
}

// whether any of the lane's sums is not finite
template <int DB> __device__ __forceinline__ bool not_finite(const f16v (&acc)[DB])
{
    float t = 0.0f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            t = __builtin_fmaf(acc[d][i], 0.0f, t);
    return !(t == 0.0f);
}

// 32 rows (columns n of acc) times `by` to global memory as bf16, transposed in
// the wave's own LDS; row r at out + r ts, rows from `rows` on are not written.
template <int DB>
__device__ __forceinline__ void store_rows(const f16v (&acc)[DB], float by, LDS_AS uint8_t *mine, uint16_t *out, int64_t ts,
                                           int rows, int D, int l)
{
    const int n = l & 31, h = l >> 5;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const u32x2 v = {pack_bf16(acc[d][4 * g] * by, acc[d][4 * g + 1] * by),
                             pack_bf16(acc[d][4 * g + 2] * by, acc[d][4 * g + 3] * by)};
            *reinterpret_cast<LDS_AS u32x2 *>(mine + n * kRow<DB> + ((4 * d + g) ^ swz<DB>(n)) * 16 + 8 * h) = v;
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    constexpr int RPL = 64 / kChunks<DB>;
#pragma unroll
    for (int i = 0; i < 32 / RPL; ++i) {
        const int r = i * RPL + l / kChunks<DB>, c = l % kChunks<DB> ^ swz<DB>(r);
        const u32x4 v = *reinterpret_cast<const LDS_AS u32x4 *>(mine + i * 1024 + l * 16);
        if (r < rows && c * 8 < D)
            *reinterpret_cast<u32x4 *>(out + r * ts + c * 8) = v;
    }
}

// 32 rows of a head straight to registers: row n (at most `last`), the B (or A)
// operands of the 2 DB steps along its elements.
template <int DB>
__device__ __forceinline__ void load_rows(b8 (&x)[2 * DB], const uint16_t *head, int64_t ts, int r0, int last, int D, int l)
{
    const uint16_t *row = head + (int64_t)min(r0 + (l & 31), last) * ts;
#pragma unroll
    for (int ks = 0; ks < 2 * DB; ++ks) {
        const int e = 16 * ks + 8 * (l >> 5);
        u32x4 v = {0, 0, 0, 0};
        if (e < D)
            v = *reinterpret_cast<const u32x4 *>(row + e);
        x[ks] = __builtin_bit_cast(b8, v);
    }
}

// Waits for loads to registers here.  Left to their first use, inside the loop over
// tiles, the wait would stand there in every turn, and for the tile in flight too:
// the compiler does not see the LDS DMA that comes after them.
template <int N> __device__ __forceinline__ void settle(b8 (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        asm volatile("" : "+v"(x[i]));
}
__device__ __forceinline__ void settle(float &x) { asm volatile("" : "+v"(x)); }

template <int BYTES> __device__ __forceinline__ void zero_lds(LDS_AS uint8_t *lds, int threads)
{
    for (int i = threadIdx.x * 16; i < BYTES; i += threads * 16)
        *reinterpret_cast<LDS_AS u32x4 *>(lds + i) = u32x4{0, 0, 0, 0};
    __syncthreads();
}

} // namespace mxa

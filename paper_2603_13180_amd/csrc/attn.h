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
template <int DB> __device__ __forceinline__ int swz(int r)
{
    return DB <= 2 ? ((r >> 1) & 1) << 2 | ((r >> 2) & 3) : (r & 3) << 2 | ((r >> 2) & 3);
}

__device__ __forceinline__ void lds_load16(const void *p, uint32_t lds_base)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "{m0}"(lds_base) : "memory");
}

__device__ __forceinline__ uint32_t lds_address(const LDS_AS uint8_t *p) { return (uint32_t)(uintptr_t)p; }

// One kind of heads: element (t, h, e) at p[t ts + h hs + e].
struct In {
    const uint16_t *p;
    int64_t ts, hs;
};
struct Out {
    uint16_t *p;
    int64_t ts, hs;
};

// Rows r0 .. r0 + ROWS - 1 (those past `last` as `last`) of a head into LDS, by
// wave w of NW.  Chunks past D keep what the LDS held.
template <int DB, int ROWS, int NW>
__device__ __forceinline__ void load_tile(const uint16_t *head, int64_t ts, int r0, int last, int D,
                                          uint32_t lds, int w, int l)
{
    constexpr int RPL = 64 / kChunks<DB>, LOADS = ROWS / RPL;
    static_assert(LOADS % NW == 0, "whole loads for every wave");
    const int c = l % kChunks<DB>;
#pragma unroll
    for (int i = 0; i < LOADS / NW; ++i) {
        const int n = w * (LOADS / NW) + i, r = n * RPL + l / kChunks<DB>;
        const int ch = c ^ swz<DB>(r);
        if (ch * 8 < D)
            lds_load16(head + (int64_t)min(r0 + r, last) * ts + ch * 8, lds + n * 1024);
    }
}

// A lane's offsets into a tile.
template <int DB> struct Lane {
    uint32_t row;        // chunk h of row n
    uint32_t tr[2][DB];  // the transposing read of rows 8 u + 4 h .. + 3, columns 32 d ..

    __device__ __forceinline__ explicit Lane(int l)
    {
        const int n = l & 31, h = l >> 5, i = l & 15;
        row = n * kRow<DB> + (h ^ swz<DB>(n)) * 16;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const int r = 8 * u + 4 * h + (i >> 2);
                const int c = 4 * d + 2 * ((l >> 4) & 1) + ((i & 3) >> 1);
                tr[u][d] = r * kRow<DB> + (c ^ swz<DB>(r)) * 16 + (i & 1) * 8;
            }
    }
};

// elements 16 ks + 8 h .. of rows 32 b + n
template <int DB>
__device__ __forceinline__ b8 row_frag(const LDS_AS uint8_t *tile, const Lane<DB> &L, int ks, int b)
{
    return *reinterpret_cast<const LDS_AS b8 *>(tile + b * 32 * kRow<DB> + (L.row ^ (ks * 32)));
}

// elements 32 d + n of rows 16 s + 8 u + 4 h + j
template <int DB>
__device__ __forceinline__ b8 col_frag(const LDS_AS uint8_t *tile, const Lane<DB> &L, int s, int d)
{
    typedef short s4 __attribute__((ext_vector_type(4)));
    const s4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s4 *)(tile + s * 16 * kRow<DB> + L.tr[0][d]));
    const s4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s4 *)(tile + s * 16 * kRow<DB> + L.tr[1][d]));
    return __builtin_bit_cast(b8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
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

// acc += (rows 16 s .. of the tile)^T x
template <int DB>
__device__ __forceinline__ void product(f16v (&acc)[DB], const LDS_AS uint8_t *tile, const Lane<DB> &L, int s, b8 x)
{
#pragma unroll
    for (int d = 0; d < DB; ++d)
        acc[d] = mfma(col_frag<DB>(tile, L, s, d), x, acc[d]);
}

// The same of a tile some of whose rows are masked and may hold infinities or
// NaN: 0 times those is NaN, so every row is a product of its own, kept where
// seen(row) of the lane's column.  Only for tiles where the plain product gave
// something that is not finite.
template <int DB, typename Seen>
__device__ __forceinline__ void careful_product(f16v (&acc)[DB], const LDS_AS uint8_t *tile, const Lane<DB> &L, int s, b8 x,
                                                int h, Seen seen)
{
    typedef short s8 __attribute__((ext_vector_type(8)));
    const s8 xi = __builtin_bit_cast(s8, x);
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

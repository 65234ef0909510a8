// Device-side helpers of the microscaled formats: blocks of 32 values that share a scale 2^E (the OCP microscaling formats).
//
//   4 bits: e2m1 values (0, 0.5, 1, 1.5, 2, 3, 4, 6, sign in bit 3), E = floor(log2 of the largest magnitude) - 2
//   8 bits: whole numbers -127 .. 127 in steps of 1/64,               E = floor(log2 of the largest magnitude)
//
// E is at least -127 and is held as E + 127 in a byte; 255 stands for "not a number" and marks a block in which a value is not finite.  Values
// are bf16, whose exponent field gives E at once, and a division by 2^E is exact, so the only rounding is the one to the
// format's values: to nearest, ties to the even code, the magnitude limited to 6 and 127/64.
#pragma once

#include <stdint.h>

#include "lords_ptx.cuh"
#include "lords_tc_common.cuh"

namespace lords {
namespace mx {

constexpr int kBlock = 32;                  // values that share a scale
constexpr int kTileRows = 128;              // rows of a tile of 4-bit scales ...
constexpr int kTileBlocks = 4;              // ... and blocks: what one copy into TMEM takes
constexpr int kTileBytes = kTileRows * kTileBlocks;

__host__ __device__ inline int blocks_of(int cols) { return (cols + kBlock - 1) / kBlock; }
__host__ __device__ inline int scale_tiles_of(int cols) { return (blocks_of(cols) + kTileBlocks - 1) / kTileBlocks; }
__host__ __device__ inline size_t codes_pitch(int cols) { return (size_t)blocks_of(cols) * 16; }

// Blocks of rows on the grid's y axis, which ends at 65535, and on z behind it.
inline dim3 grid_of(unsigned col_blocks, unsigned row_blocks)
{
    const unsigned z = (row_blocks + 65534u) / 65535u;
    return dim3(col_blocks, (row_blocks + z - 1) / z, z);
}
__device__ __forceinline__ int row_block() { return (int)(blockIdx.z * gridDim.y + blockIdx.y); }

// Where the scale of row i and block b of a tile lies inside it: four words a lane, a word the four blocks of row 32 j + lane.
__host__ __device__ inline int scale_at(int i, int b) { return (i & 31) * 16 + (i >> 5) * 4 + b; }

// Magnitudes of a pair of bf16 values, and the larger ones of two or three pairs of magnitudes: as whole numbers they are in order, infinities and NaNs
// above all others.
__device__ __forceinline__ uint32_t magnitudes(uint32_t w) { return w & 0x7FFF7FFFu; }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return __vmaxu2(a, b); }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b, uint32_t c) { return __vimax3_u16x2(a, b, c); }
__device__ __forceinline__ uint32_t larger_half(uint32_t top) { return max(top & 0xFFFFu, top >> 16); }
__device__ __forceinline__ uint32_t bf16x2_mul(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// 2 N values of a row of `cols` from column c (below cols) on, as pairs, zeros behind the last; rows may begin anywhere, the matrix at a 16-byte boundary,
// and `end` is behind it.  The 16-byte words around are read and moved into place (4-byte words, 14336 x 4095 to 4 bits: 43 us).  (Ordinary loads:
// a dependent launch reads what another grid has written while it was already there, which the read-only path does not allow for.)
template <int N> __device__ __forceinline__ void load_values(const uint16_t *row, int cols, int c, const uint16_t *end, uint32_t (&w)[N])
{
    const uint16_t *src = row + c;
    if ((cols & 7) == 0) {                                   // (moved all the same, 14336 x 4088 30.9 us, 23.6 so)
#pragma unroll
        for (int j = 0; j < N / 4; ++j) {
            uint4 u = make_uint4(0u, 0u, 0u, 0u);
            if (c + 8 * j < cols) u = *reinterpret_cast<const uint4 *>(src + 8 * j);
            w[4 * j] = u.x; w[4 * j + 1] = u.y; w[4 * j + 2] = u.z; w[4 * j + 3] = u.w;
        }
        return;
    }
    const int left = cols - c < 2 * N ? cols - c : 2 * N, off = (int)((reinterpret_cast<uintptr_t>(src) >> 1) & 7), need = off + left;
    const uint16_t *at = src - off;
    const bool whole = at + ((need + 7) & ~7) <= end;        // no word reaches past the end
    uint32_t v[N + 4];
#pragma unroll
    for (int j = 0; j < N / 4 + 1; ++j) {
        uint4 u = make_uint4(0u, 0u, 0u, 0u);
        if (whole && 8 * j < need) u = *reinterpret_cast<const uint4 *>(at + 8 * j);
        v[4 * j] = u.x; v[4 * j + 1] = u.y; v[4 * j + 2] = u.z; v[4 * j + 3] = u.w;
    }
    if (!whole) {
#pragma unroll
        for (int k = 0; k < N + 4; ++k) {
            if (at + 2 * k + 2 <= end) v[k] = *reinterpret_cast<const uint32_t *>(at + 2 * k);
            else if (at + 2 * k < end) v[k] = at[2 * k];
        }
    }
    if (off & 4)
#pragma unroll
        for (int k = 0; k < N + 2; ++k) v[k] = v[k + 2];
    if (off & 2)
#pragma unroll
        for (int k = 0; k < N + 1; ++k) v[k] = v[k + 1];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t u = off & 1 ? __funnelshift_r(v[k], v[k + 1], 16) : v[k];
        w[k] = left >= 2 * k + 2 ? u : left > 2 * k ? u & 0xFFFFu : 0u;
    }
}
// Sixteen values to a 32-byte boundary: whole sectors.
__device__ __forceinline__ void store16(uint16_t *dst, uint4 a, uint4 b)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
                 : "memory");
}
// ... and to a row: a warp's lanes side by side, lane l from column c = c(0) + 8 l on; all 32 take part, those from column `cols` on store nothing.
// Rows that begin between two words: every lane stores its neighbour's last value with its own first ones, as whole words (byte by byte
// at the ends, 14336 x 4095 out of 4 bits took 79 us).
__device__ __forceinline__ void store8(uint16_t *row, int cols, int c, uint4 v, int lane)
{
    uint16_t *dst = row + c;
    if ((cols & 7) == 0) {
        if (c < cols) *reinterpret_cast<uint4 *>(dst) = v;
        return;
    }
    const bool between = (reinterpret_cast<uintptr_t>(row) & 2) != 0;      // the same for the whole warp
    uint32_t before = 0u;
    if (between) before = __shfl_up_sync(0xffffffffu, v.w, 1) >> 16;
    if (c + 8 <= cols) {
        if (!between) {
            uint32_t *w = reinterpret_cast<uint32_t *>(dst);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
            uint32_t *w = reinterpret_cast<uint32_t *>(dst + 1);
            if (lane > 0) w[-1] = before | v.x << 16;
            else dst[0] = (uint16_t)v.x;
            w[0] = v.x >> 16 | v.y << 16; w[1] = v.y >> 16 | v.z << 16; w[2] = v.z >> 16 | v.w << 16;
            if (lane == 31 || c + 8 == cols) dst[7] = (uint16_t)(v.w >> 16);
        }
    } else if (c < cols) {
        if (between && lane > 0) dst[-1] = (uint16_t)before;
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 7; ++k)
            if (c + k < cols) dst[k] = (uint16_t)(u[k >> 1] >> (16 * (k & 1)));
    }
}

// Scale byte from the bf16 pattern of the block's largest magnitude; BELOW: 2 for the 4-bit, 0 for the 8-bit format.
template <int BELOW> __device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    const uint32_t ex = top >> 7;
    return ex == 255u ? 255u : ex > (uint32_t)BELOW ? ex - (uint32_t)BELOW : 0u;
}
// 2^-E as a pair of bf16 numbers (zero for a block that is not finite: every code is 0 there).  E = 127 (8 bits only): 2^-127, a subnormal number.
__device__ __forceinline__ uint32_t inverse_scale(uint32_t byte)
{
    const uint32_t s = byte == 255u ? 0u : byte == 254u ? 0x0040u : (254u - byte) << 7;
    return s | s << 16;
}

// Eight bf16 values, times 2^-E already, to eight 4-bit codes, low nibble first: the first of each pair `a`, the second of each pair `b`.  (The
// product with 2^-E is exact: what falls out of bf16's range below is far from the least code.)
__device__ __forceinline__ uint32_t codes_of(float a0, float b0, float a1, float b1, float a2, float b2, float a3, float b3)
{
    uint32_t c;
    asm("{\n"
        ".reg .b8 b0, b1, b2, b3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
        "mov.b32 %0, {b0, b1, b2, b3};\n"
        "}\n"
        : "=r"(c)
        : "f"(a0), "f"(b0), "f"(a1), "f"(b1), "f"(a2), "f"(b2), "f"(a3), "f"(b3));
    return c;
}
__device__ __forceinline__ float low_half(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float high_half(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }
// Eight bf16 values as pairs, low half first, with the block's scale byte.  (Infinities and NaNs times the zero that stands for 2^-E of a block that is
// not finite are NaN, which the conversion makes 6: zeroed at the end.)
__device__ __forceinline__ uint32_t to_codes4(const uint32_t *w, uint32_t byte)
{
    const uint32_t inv = inverse_scale(byte);
    const uint32_t u0 = bf16x2_mul(w[0], inv), u1 = bf16x2_mul(w[1], inv), u2 = bf16x2_mul(w[2], inv), u3 = bf16x2_mul(w[3], inv);
    const uint32_t c = codes_of(low_half(u0), high_half(u0), low_half(u1), high_half(u1), low_half(u2), high_half(u2), low_half(u3), high_half(u3));
    return byte == 255u ? 0u : c;
}

}  // namespace mx

namespace ptx {

// Whole 16-byte words from global into this CTA's shared memory, counted in bytes on `bar`.
__device__ __forceinline__ void load_words(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// A tile of scales (512 bytes, 32 rows of 16) into four TMEM columns, the 32 lanes repeated in all four quadrants; ordered before the MMAs that
// the same thread issues next, and after those it has issued.
__device__ __forceinline__ void scales_to_tmem(uint32_t taddr, uint64_t desc, uint32_t leader)
{
    asm volatile(
        "{\n"
        ".reg .pred q;\n"
        "setp.ne.b32 q, %2, 0;\n"
        "@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n"
        "}\n" ::"r"(taddr), "l"(desc), "r"(leader)
        : "memory");
}
// The same in both CTAs of a pair, each from its own shared memory at the same offset; one thread of the even CTA.
__device__ __forceinline__ void scales_to_tmem2(uint32_t taddr, uint64_t desc, uint32_t leader)
{
    asm volatile(
        "{\n"
        ".reg .pred q;\n"
        "setp.ne.b32 q, %2, 0;\n"
        "@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n"
        "}\n" ::"r"(taddr), "l"(desc), "r"(leader)
        : "memory");
}
// Descriptor of such a tile: no swizzle, groups of 8 rows 128 bytes apart.
__device__ __forceinline__ uint64_t scales_desc(uint32_t smem_addr)
{
    return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)8 << 32) | ((uint64_t)1 << 46);
}
// Instruction descriptor of kind::mxf4: e2m1 operands, both K-major, scales 2^E, 64 values of K, two blocks of each row.  The scales' place in their
// TMEM words (the low or the high two bytes) is `half` = 0 or 1.
__host__ __device__ constexpr uint32_t umma_idesc_mxf4(int M, int N, int half)
{
    return ((uint32_t)(2 * half) << 4)        // B's scales: byte 0 or 2
           | (1u << 7) | (1u << 10)           // e2m1
           | ((uint32_t)(N >> 3) << 17) | (1u << 23)      // scales are powers of two
           | ((uint32_t)(M >> 4) << 24) | ((uint32_t)(2 * half) << 29);
}
// D[tmem] (+)= (A[smem] with its scales) * (B[smem] with its scales)
__device__ __forceinline__ void umma_mxf4_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sa_tmem, uint32_t sb_tmem,
                                             uint32_t accumulate, uint32_t leader)
{
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.b32 p, %6, 0;\n"
        "setp.ne.b32 q, %7, 0;\n"
        "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n"
        "}\n" ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa_tmem), "r"(sb_tmem), "r"(accumulate), "r"(leader)
        : "memory");
}
// The same on a CTA pair: each CTA holds half of A's rows with their scales, half of B's rows, and the scales of all of B's rows.
__device__ __forceinline__ void umma2_mxf4_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sa_tmem, uint32_t sb_tmem,
                                              uint32_t accumulate, uint32_t leader)
{
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.b32 p, %6, 0;\n"
        "setp.ne.b32 q, %7, 0;\n"
        "@q tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n"
        "}\n" ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa_tmem), "r"(sb_tmem), "r"(accumulate), "r"(leader)
        : "memory");
}

}  // namespace ptx
}  // namespace lords

// Activations kept for the backward pass in 8 bits (the format of lords_mx.cuh: whole numbers -127 .. 127 in steps of 1/64, a scale 2^E per 32
// values of a token), and taken up again in bf16.  A value of the format is a bf16 number, so only the store rounds.
//
// A thread has sixteen values, half a block, or eight on the way out into rows that do not begin at 32-byte boundaries.  Bound: the bytes, 2 + 33/32 a value
// either way.
#include <cuda_bf16.h>

#include "lords_internal.h"
#include "lords_mx.cuh"

namespace lords {

namespace {

using namespace mx;

constexpr int kCThreads = 256;
constexpr int kStoreRows = 2;               // rows a warp of the store (four: 2048 x 4096 6.0 us, two 5.4)

// A CTA takes eight warps' rows x 512 columns: a warp PER rows, a thread sixteen values of each, so that two threads are a block.  Small calls take one
// row a warp and more CTAs.  (Eight values a thread: 2048 x 4096 6.6 us.)
template <int PER>
__global__ void __launch_bounds__(kCThreads) lords_checkpoint_store_kernel(const uint16_t *x, int M, int n, int qp, int ep, int wide, uint8_t *q, uint8_t *e)
{
    const int lane = threadIdx.x & 31, t0 = (row_block() * (kCThreads / 32) + (threadIdx.x >> 5)) * PER;
    const int c = (int)blockIdx.x * 512 + lane * 16;
    const uint16_t *end = x + (size_t)M * n;
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    uint32_t w[PER][8];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
#pragma unroll
        for (int h = 0; h < 8; ++h) w[k][h] = 0u;
        if (t0 + k >= M || c >= n) continue;
        const uint16_t *row = x + (size_t)(t0 + k) * n;
        if (wide) {
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(w[k][0]), "=r"(w[k][1]), "=r"(w[k][2]), "=r"(w[k][3]), "=r"(w[k][4]), "=r"(w[k][5]), "=r"(w[k][6]), "=r"(w[k][7])
                         : "l"(row + c));
        } else {
            load_values<8>(row, n, c, end, w[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        uint32_t top = larger(magnitudes(w[k][0]), magnitudes(w[k][1]), magnitudes(w[k][2]));
        top = larger(top, magnitudes(w[k][3]), magnitudes(w[k][4]));
        top = larger(top, magnitudes(w[k][5]), magnitudes(w[k][6]));
        top = larger(top, magnitudes(w[k][7]));
        top = larger(top, __shfl_xor_sync(0xffffffffu, top, 1));
        const uint32_t byte = scale_byte<0>(larger_half(top));
        if (t0 + k >= M) continue;
        // value * 2^-E is exact in bf16; limited to 127/64 (which takes no more than half a step: the largest bf16 number below 2 is 127.5/64), then
        // times 64 onto 1.5 * 2^23, whose low bits are then the whole number: one rounding, ties to even
        const uint32_t inv = inverse_scale(byte);
        uint32_t out[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            uint32_t u[2];
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                u[g] = bf16x2_mul(w[k][2 * h + g], inv);
                asm("min.bf16x2 %0, %0, %1;\nmax.bf16x2 %0, %0, %2;" : "+r"(u[g]) : "r"(0x3FFE3FFEu), "r"(0xBFFEBFFEu));
            }
            auto whole = [](float v) { return __float_as_uint(fmaf(v, 64.0f, 12582912.0f)); };
            out[h] = __byte_perm(__byte_perm(whole(low_half(u[0])), whole(high_half(u[0])), 0x0040), __byte_perm(whole(low_half(u[1])), whole(high_half(u[1])), 0x0040), 0x5410);
            if (byte == 255u) out[h] = 0u;
        }
        if (c < qp) *reinterpret_cast<uint4 *>(q + (size_t)(t0 + k) * qp + c) = make_uint4(out[0], out[1], out[2], out[3]);
        if ((lane & 1) == 0 && c / kBlock < ep) e[(size_t)(t0 + k) * ep + c / kBlock] = (uint8_t)byte;
    }
}

// The eight values as bf16 pairs.  |q| <= 127 has seven bits and 2^(E - 6) is a bf16 number (2^-133, the least, included): the products are exact.
__device__ __forceinline__ uint4 values8(uint2 q, uint32_t byte)
{
    // a number's low seven bits as the mantissa of 128 + them, from which 128 is taken, or 256 where the sign bit is set
    const uint32_t s = byte == 255u ? 0x7FC0u : byte > 6u ? (byte - 6u) << 7 : 0x0080u >> (7u - byte), ss = s | s << 16;
    uint32_t v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t two = __byte_perm(k < 2 ? q.x : q.y, 0u, k & 1 ? 0x4342 : 0x4140);
        uint32_t d;
        asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"((two & 0x007F007Fu) | 0x43004300u), "r"((two & 0x00800080u) | 0xC300C300u));
        v[k] = bf16x2_mul(d, ss);
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// A warp takes PER rows x 256 columns, a thread eight values of each; WIDE, rows that begin at 32-byte boundaries: 512 columns, sixteen values.
template <int PER, bool WIDE>
__global__ void __launch_bounds__(kCThreads) lords_checkpoint_load_kernel(const uint8_t *q, const uint8_t *e, int M, int n, int qp, int ep, uint16_t *x)
{
    constexpr int VALUES = WIDE ? 16 : 8;
    const int lane = threadIdx.x & 31, t0 = (row_block() * (kCThreads / 32) + (threadIdx.x >> 5)) * PER;
    const int c = ((int)blockIdx.x * 32 + lane) * VALUES;
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    uint2 w[PER][VALUES / 8];
    uint32_t byte[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        byte[k] = 0u;
#pragma unroll
        for (int h = 0; h < VALUES / 8; ++h) w[k][h] = make_uint2(0u, 0u);
        if (t0 + k >= M || c >= n) continue;
        const uint8_t *src = q + (size_t)(t0 + k) * qp + c;
        if constexpr (WIDE) {
            const uint4 u = *reinterpret_cast<const uint4 *>(src);
            w[k][0] = make_uint2(u.x, u.y);
            w[k][1] = make_uint2(u.z, u.w);
        } else {
            w[k][0] = *reinterpret_cast<const uint2 *>(src);
        }
        byte[k] = e[(size_t)(t0 + k) * ep + c / kBlock];
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        if (t0 + k >= M) break;
        uint16_t *row = x + (size_t)(t0 + k) * n;
        if constexpr (WIDE) {
            if (c < n) store16(row + c, values8(w[k][0], byte[k]), values8(w[k][1], byte[k]));
        } else {
            store8(row, n, c, values8(w[k][0], byte[k]), lane);
        }
    }
}

// One row a warp where more would leave fewer than two CTAs an SM.
bool small(int M, int n, int cols, int per) { return (long long)((M + 8 * per - 1) / (8 * per)) * ((n + cols - 1) / cols) < 296; }
dim3 grid_of(int M, int n, int cols, int per) { return mx::grid_of((unsigned)((n + cols - 1) / cols), (unsigned)((M + 8 * per - 1) / (8 * per))); }

}  // namespace

int launch_checkpoint_store(const uint16_t *x, int M, int n, uint8_t *q, uint8_t *e, cudaStream_t stream)
{
    const int qp = blocks_of(n) * kBlock, ep = scale_tiles_of(n) * kTileBlocks;       // (whole words of scales are written)
    const int wide = n % 16 == 0 && reinterpret_cast<uintptr_t>(x) % 32 == 0;
    if (small(M, n, 512, kStoreRows)) return launch_dependent(lords_checkpoint_store_kernel<1>, grid_of(M, ep * kBlock, 512, 1), kCThreads, stream, x, M, n, qp, ep, wide, q, e);
    return launch_dependent(lords_checkpoint_store_kernel<kStoreRows>, grid_of(M, ep * kBlock, 512, kStoreRows), kCThreads, stream, x, M, n, qp, ep, wide, q, e);
}

int launch_checkpoint_load(const uint8_t *q, const uint8_t *e, int M, int n, uint16_t *x, cudaStream_t stream)
{
    const int qp = blocks_of(n) * kBlock, ep = scale_tiles_of(n) * kTileBlocks;
    auto launch = [&](auto kernel, int cols, int per) { return launch_dependent(kernel, grid_of(M, n, cols, per), kCThreads, stream, q, e, M, n, qp, ep, x); };
    if (n % 16 == 0 && reinterpret_cast<uintptr_t>(x) % 32 == 0)
        return small(M, n, 512, 2) ? launch(lords_checkpoint_load_kernel<1, true>, 512, 1) : launch(lords_checkpoint_load_kernel<2, true>, 512, 2);
    return small(M, n, 256, 4) ? launch(lords_checkpoint_load_kernel<1, false>, 256, 1) : launch(lords_checkpoint_load_kernel<4, false>, 256, 4);
}

}  // namespace lords

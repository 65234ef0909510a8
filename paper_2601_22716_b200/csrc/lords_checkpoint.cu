// Activations kept for the backward pass in 8 bits (the format of lords_mx.cuh: whole numbers -127 .. 127 in steps of 1/64, a scale 2^E per 32
// values of a token), and taken up again in bf16.  A value of the format is a bf16 number, so only the store rounds.
//
// A block is four neighbouring threads of eight values each.  Bound: the bytes, 2 + 33/32 a value either way.
#include <cuda_bf16.h>

#include "lords_internal.h"
#include "lords_mx.cuh"

namespace lords {

namespace {

using namespace mx;

constexpr int kCThreads = 256;

// rows of whole blocks and scales of four blocks: what a row of n values takes
__device__ __forceinline__ int q_pitch(int n) { return blocks_of(n) * kBlock; }
__device__ __forceinline__ int e_pitch(int n) { return scale_tiles_of(n) * kTileBlocks; }

// A CTA takes kCRows rows x 256 columns, a warp four rows, a thread eight values of each.
constexpr int kCPer = 4, kCRows = kCThreads / 32 * kCPer;

__global__ void __launch_bounds__(kCThreads) lords_checkpoint_store_kernel(const uint16_t *__restrict__ x, int M, int n, uint8_t *__restrict__ q,
                                                                           uint8_t *__restrict__ e)
{
    const int lane = threadIdx.x & 31, t0 = (int)blockIdx.y * kCRows + (threadIdx.x >> 5) * kCPer;
    const int c = (int)blockIdx.x * 256 + lane * 8, qp = q_pitch(n), ep = e_pitch(n);
    const uint16_t *end = x + (size_t)M * n;
    uint32_t w[kCPer][4];
#pragma unroll
    for (int k = 0; k < kCPer; ++k) {
        w[k][0] = w[k][1] = w[k][2] = w[k][3] = 0u;
        if (t0 + k < M && c < n) load8(x + (size_t)(t0 + k) * n, n, c, end, w[k]);
    }
#pragma unroll
    for (int k = 0; k < kCPer; ++k) {
        uint32_t top = max_magnitudes(max_magnitudes(w[k][0], w[k][1]), max_magnitudes(w[k][2], w[k][3]));
        top = max_magnitudes(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max_magnitudes(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const uint32_t byte = scale_byte<0>(max(top & 0xFFFFu, top >> 16));
        if (t0 + k >= M) continue;
        // whole numbers, value * 2^-E * 64: a bf16 product and a power of two, both exact, so only the conversion rounds
        const uint32_t inv = inverse_scale(byte);
        uint32_t out[2] = {0u, 0u};
#pragma unroll
        for (int h = 0; h < 8; ++h) {
            const uint32_t u = bf16x2_mul(w[k][h >> 1], inv);
            int i = __float2int_rn(__uint_as_float(h & 1 ? u & 0xFFFF0000u : u << 16) * 64.0f);
            i = i > 127 ? 127 : i < -127 ? -127 : i;
            out[h >> 2] |= (uint32_t)(i & 255) << (8 * (h & 3));
        }
        if (byte == 255u) out[0] = out[1] = 0u;
        if (c < qp) *reinterpret_cast<uint2 *>(q + (size_t)(t0 + k) * qp + c) = make_uint2(out[0], out[1]);
        if ((lane & 3) == 0 && c / kBlock < ep) e[(size_t)(t0 + k) * ep + c / kBlock] = (uint8_t)byte;
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

__global__ void __launch_bounds__(kCThreads) lords_checkpoint_load_kernel(const uint8_t *__restrict__ q, const uint8_t *__restrict__ e, int M, int n,
                                                                          uint16_t *__restrict__ x)
{
    const int lane = threadIdx.x & 31, t0 = (int)blockIdx.y * kCRows + (threadIdx.x >> 5) * kCPer;
    const int c = (int)blockIdx.x * 256 + lane * 8, qp = q_pitch(n), ep = e_pitch(n);
    if (c >= n) return;
    uint2 w[kCPer];
    uint32_t byte[kCPer];
#pragma unroll
    for (int k = 0; k < kCPer; ++k) {
        const int t = t0 + k < M ? t0 + k : M - 1;
        w[k] = __ldg(reinterpret_cast<const uint2 *>(q + (size_t)t * qp + c));
        byte[k] = __ldg(e + (size_t)t * ep + c / kBlock);
    }
#pragma unroll
    for (int k = 0; k < kCPer; ++k)
        if (t0 + k < M) store8(x + (size_t)(t0 + k) * n, n, c, values8(w[k], byte[k]));
}

}  // namespace

int launch_checkpoint_store(const uint16_t *x, int M, int n, uint8_t *q, uint8_t *e, cudaStream_t stream)
{
    // (whole words of scales are written)
    const dim3 grid((unsigned)((scale_tiles_of(n) * kTileBlocks * kBlock + 255) / 256), (unsigned)((M + kCRows - 1) / kCRows));
    lords_checkpoint_store_kernel<<<grid, kCThreads, 0, stream>>>(x, M, n, q, e);
    LORDS_CUDA_TRY(cudaGetLastError());
    return LORDS_OK;
}

int launch_checkpoint_load(const uint8_t *q, const uint8_t *e, int M, int n, uint16_t *x, cudaStream_t stream)
{
    const dim3 grid((unsigned)((n + 255) / 256), (unsigned)((M + kCRows - 1) / kCRows));
    lords_checkpoint_load_kernel<<<grid, kCThreads, 0, stream>>>(q, e, M, n, x);
    LORDS_CUDA_TRY(cudaGetLastError());
    return LORDS_OK;
}

}  // namespace lords

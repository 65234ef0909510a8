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

__global__ void __launch_bounds__(kCThreads) lords_checkpoint_store_kernel(const uint16_t *__restrict__ x, int M, int n, uint8_t *__restrict__ q,
                                                                           uint8_t *__restrict__ e)
{
    const int chunks = e_pitch(n) * 4;                       // of eight values, whole scale words
    const long long at = (long long)blockIdx.x * kCThreads + threadIdx.x;
    const int t = (int)(at / chunks), c = (int)(at % chunks) * 8;
    const bool in = t < M;
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if (in && c < n) {
        const uint16_t *src = x + (size_t)t * n + c;
        if ((n & 7) == 0) {
            const uint4 v = __ldg(reinterpret_cast<const uint4 *>(src));
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t lo = c + 2 * k < n ? __ldg(src + 2 * k) : 0u, hi = c + 2 * k + 1 < n ? __ldg(src + 2 * k + 1) : 0u;
                w[k] = lo | hi << 16;
            }
        }
    }
    uint32_t top = max_magnitudes(max_magnitudes(max_magnitudes(max_magnitudes(0u, w[0]), w[1]), w[2]), w[3]);
    top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t byte = scale_byte<0>(max(top & 0xFFFFu, top >> 16));
    if (!in) return;
    // whole numbers: value * 2^-E * 64, in two steps that are exact (2^-E alone may be 2^127)
    const float inv = inverse_scale(byte);
    uint32_t out[2] = {0u, 0u};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float v = __uint_as_float(k & 1 ? w[k >> 1] & 0xFFFF0000u : w[k >> 1] << 16) * inv * 64.0f;
        int i = __float2int_rn(v);
        i = i > 127 ? 127 : i < -127 ? -127 : i;
        out[k >> 2] |= (uint32_t)(i & 255) << (8 * (k & 3));
    }
    if (byte == 255u) out[0] = out[1] = 0u;
    if (c < q_pitch(n)) *reinterpret_cast<uint2 *>(q + (size_t)t * q_pitch(n) + c) = make_uint2(out[0], out[1]);
    if ((c & 31) == 0) e[(size_t)t * e_pitch(n) + c / 32] = (uint8_t)byte;
}

// The eight values as bf16 pairs.  |q| <= 127 has seven bits and 2^(E - 6) is a bf16 number (2^-133, the least, included): the products are exact.
__device__ __forceinline__ void values8(uint2 q, uint32_t byte, uint32_t (&w)[4])
{
    const float s = byte == 255u ? __uint_as_float(0x7FC00000u) : byte > 6u ? __uint_as_float((byte - 6u) << 23) : __uint_as_float(0x00800000u >> (7u - byte));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t src = k < 2 ? q.x : q.y;
        const int lo = (int)(src << (24 - 16 * (k & 1))) >> 24, hi = (int)(src << (16 - 16 * (k & 1))) >> 24;
        w[k] = __byte_perm(__float_as_uint((float)lo * s), __float_as_uint((float)hi * s), 0x7632);
    }
}

// Rows of `pitch` values (n, or a multiple of 8 behind which zeros are written).
__global__ void __launch_bounds__(kCThreads) lords_checkpoint_load_kernel(const uint8_t *__restrict__ q, const uint8_t *__restrict__ e, int M, int n, int pitch,
                                                                          uint16_t *__restrict__ x)
{
    const int chunks = (pitch + 7) / 8;
    const long long at = (long long)blockIdx.x * kCThreads + threadIdx.x;
    const int t = (int)(at / chunks), c = (int)(at % chunks) * 8;
    if (t >= M) return;
    uint32_t w[4];
    values8(__ldg(reinterpret_cast<const uint2 *>(q + (size_t)t * q_pitch(n) + c)), __ldg(e + (size_t)t * e_pitch(n) + c / 32), w);
    uint16_t *dst = x + (size_t)t * pitch + c;
    if ((pitch & 7) == 0) {
        *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (c + k < pitch) dst[k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
    }
}

}  // namespace

int launch_checkpoint_store(const uint16_t *x, int M, int n, uint8_t *q, uint8_t *e, cudaStream_t stream)
{
    const long long blocks = ((long long)M * scale_tiles_of(n) * 16 + kCThreads - 1) / kCThreads;
    if (blocks > 2147483647LL) return LORDS_ERR_SHAPE;
    lords_checkpoint_store_kernel<<<(unsigned)blocks, kCThreads, 0, stream>>>(x, M, n, q, e);
    LORDS_CUDA_TRY(cudaGetLastError());
    return LORDS_OK;
}

int launch_checkpoint_load(const uint8_t *q, const uint8_t *e, int M, int n, uint16_t *x, int pitch, cudaStream_t stream)
{
    const long long blocks = ((long long)M * ((pitch + 7) / 8) + kCThreads - 1) / kCThreads;
    if (blocks > 2147483647LL) return LORDS_ERR_SHAPE;
    lords_checkpoint_load_kernel<<<(unsigned)blocks, kCThreads, 0, stream>>>(q, e, M, n, pitch, x);
    LORDS_CUDA_TRY(cudaGetLastError());
    return LORDS_OK;
}

}  // namespace lords

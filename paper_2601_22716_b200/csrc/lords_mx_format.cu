// Tensors to and from the microscaled formats of lords_mx.cuh.
//
// Each kernel reads its input once and is bound by the bytes it moves.
#include <cuda_bf16.h>

#include "lords_internal.h"
#include "lords_mx.cuh"
#include "lords_tc_common.cuh"

namespace lords {

namespace {

using namespace mx;

// ------------------------------------------------------------------------------------------------ to 4 bits
// A CTA takes ROWS rows x 128 columns.  Along the rows, four neighbouring threads hold a block in registers.  Along the columns, a thread reads
// two columns x 32 rows back from shared memory.  Scales meet in shared memory as words of four blocks.
#ifndef QROWS
#define QROWS 64
#endif
constexpr int kQThreads = 256;
constexpr int kQPitch = 128 * 2 + 16;       // bytes per row of the tile in shared memory; 16-byte words stay aligned

struct QuantizeParams {
    const uint16_t *v;       // bf16 [rows][cols]
    uint8_t *codes, *scales;         // blocks along the rows (null: not asked for)
    uint8_t *codes_t, *scales_t;     // blocks along the columns: the same for the transposed matrix (null: not asked for)
    int rows, cols;
};

template <int ROWS, bool ALONG, bool ACROSS> __global__ void __launch_bounds__(kQThreads) lords_mxfp4_quantize_kernel(const QuantizeParams p)
{
    constexpr int PER = ROWS / 16;          // rows a thread loads eight values of
    __shared__ __align__(16) uint8_t tile[ACROSS ? ROWS * kQPitch : 16];
    __shared__ __align__(16) uint8_t sc[ROWS * 4], sct[kTileBytes];
    const int tid = threadIdx.x, r0 = (int)blockIdx.y * ROWS, c0 = (int)blockIdx.x * 128;
    const int seg = tid & 15, row_in = tid >> 4, c = c0 + seg * 8;
    const uint16_t *end = p.v + (size_t)p.rows * p.cols;
    uint32_t w[PER][4];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = r0 + k * 16 + row_in;
        w[k][0] = w[k][1] = w[k][2] = w[k][3] = 0u;
        if (i < p.rows && c < p.cols) load8(p.v + (size_t)i * p.cols, p.cols, c, end, w[k]);
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int rl = k * 16 + row_in;
        if constexpr (ACROSS) *reinterpret_cast<uint4 *>(tile + rl * kQPitch + seg * 16) = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
        if constexpr (ALONG) {
            uint32_t top = max_magnitudes(max_magnitudes(w[k][0], w[k][1]), max_magnitudes(w[k][2], w[k][3]));
            top = max_magnitudes(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max_magnitudes(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const uint32_t byte = scale_byte<2>(max(top & 0xFFFFu, top >> 16));
            if (r0 + rl < p.rows && c < (int)codes_pitch(p.cols) * 2)
                *reinterpret_cast<uint32_t *>(p.codes + (size_t)(r0 + rl) * codes_pitch(p.cols) + c / 2) = to_codes4(w[k], byte);
            if ((seg & 3) == 0) sc[rl * 4 + (seg >> 2)] = (uint8_t)byte;
        }
    }
    __syncthreads();
    // a row's four scales are a word of the tile of scales; the rows behind the last are part of it
    if (ALONG && tid < ROWS) {
        const int i = r0 + tid;
        *reinterpret_cast<uint32_t *>(p.scales + ((size_t)(i / kTileRows) * scale_tiles_of(p.cols) + blockIdx.x) * kTileBytes + scale_at(i % kTileRows, 0)) =
            *reinterpret_cast<const uint32_t *>(sc + tid * 4);
    }
    if constexpr (ACROSS) {
        for (int e = tid; e < 64 * (ROWS / 32); e += kQThreads) {
            const int pair = e & 63, b = e >> 6;        // two columns, a block of 32 rows
            uint32_t u[32];
            uint32_t top = 0u;
#pragma unroll
            for (int k = 0; k < 32; ++k) {
                u[k] = *reinterpret_cast<const uint32_t *>(tile + (b * 32 + k) * kQPitch + pair * 4);
                top = max_magnitudes(top, u[k]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t byte = scale_byte<2>(h ? top >> 16 : top & 0xFFFFu);
                uint32_t out[4];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    uint32_t x[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[k] = __byte_perm(u[8 * g + 2 * k], u[8 * g + 2 * k + 1], h ? 0x7632 : 0x5410);
                    out[g] = to_codes4(x, byte);
                }
                const int col = c0 + 2 * pair + h, r = r0 + b * 32;
                if (col < p.cols && r < p.rows)
                    *reinterpret_cast<uint4 *>(p.codes_t + (size_t)col * codes_pitch(p.rows) + r / 2) = make_uint4(out[0], out[1], out[2], out[3]);
                sct[(2 * pair + h) * (ROWS / 32) + b] = (uint8_t)byte;
            }
        }
        __syncthreads();
        // a column's scales of this CTA's rows are a part of a word (the whole of it with 128 rows)
        if (tid < 128) {
            uint8_t *dst = p.scales_t + ((size_t)blockIdx.x * scale_tiles_of(p.rows) + r0 / 128) * kTileBytes + scale_at(tid, r0 % 128 / 32);
            if constexpr (ROWS == 128) *reinterpret_cast<uint32_t *>(dst) = *reinterpret_cast<const uint32_t *>(sct + tid * 4);
            else *reinterpret_cast<uint16_t *>(dst) = *reinterpret_cast<const uint16_t *>(sct + tid * 2);
        }
    }
}

// ----------------------------------------------------------------------------------------------- from 4 bits
// A code's three low bits are a bf16 exponent's last two bits and the first of its mantissa, less 126 in the exponent: moved there and multiplied by 2^126,
// and by 2^E then, both exactly (zero and a half too, as a subnormal number times 2^126).  Two codes at a time; the word's nibbles k and
// k + 4 are taken together.
__device__ __forceinline__ uint4 values4(uint32_t w, uint32_t byte)
{
    // 2^E as a bf16 number: 2^-127 is subnormal, and the pattern of a NaN stands for 255
    const uint32_t s = byte == 255u ? 0x7FC0u : byte == 0u ? 0x0040u : byte << 7, ss = s | s << 16;
    uint32_t v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t sign = k < 3 ? w << (12 - 4 * k) : w, mag = k < 2 ? w << (6 - 4 * k) : w >> (4 * k - 6);
        v[k] = bf16x2_mul(bf16x2_mul((sign & 0x80008000u) | (mag & 0x01C001C0u), 0x7E807E80u), ss);
    }
    return make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410), __byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632));
}

// A CTA takes 128 rows x 256 columns, a warp four rows at a time, a thread eight values of each.
constexpr int kDThreads = 256, kDRows = 4;
__global__ void __launch_bounds__(kDThreads) lords_mxfp4_dequantize_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int rows,
                                                                           int cols, uint16_t *__restrict__ v)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = (int)blockIdx.x * 256 + lane * 8, r0 = (int)blockIdx.y * kTileRows, b = c / kBlock;
    if (c >= cols) return;
    const size_t pitch = codes_pitch(cols);
    const uint8_t *sc = scales + ((size_t)blockIdx.y * scale_tiles_of(cols) + b / kTileBlocks) * kTileBytes;
#pragma unroll 1
    for (int r = warp * kDRows; r < kTileRows && r0 + r < rows; r += kDThreads / 32 * kDRows) {
        uint32_t w[kDRows], e[kDRows];
#pragma unroll
        for (int k = 0; k < kDRows; ++k) {
            const bool in = r0 + r + k < rows;
            w[k] = in ? __ldg(reinterpret_cast<const uint32_t *>(codes + (size_t)(r0 + r + k) * pitch + c / 2)) : 0u;
            e[k] = __ldg(sc + scale_at(r + k, b % kTileBlocks));
        }
#pragma unroll
        for (int k = 0; k < kDRows; ++k) {
            if (r0 + r + k >= rows) break;
            store8(v + (size_t)(r0 + r + k) * cols, cols, c, values4(w[k], e[k]));
        }
    }
}

}  // namespace

template <int ROWS> static void launch_quantize_rows(const QuantizeParams &p, cudaStream_t stream)
{
    // (whole tiles of scales are written, the rows behind the last among them)
    const dim3 grid((unsigned)((p.cols + 127) / 128), (unsigned)((p.rows + 127) / 128 * (128 / ROWS)));
    if (p.codes && p.codes_t) lords_mxfp4_quantize_kernel<ROWS, true, true><<<grid, kQThreads, 0, stream>>>(p);
    else if (p.codes) lords_mxfp4_quantize_kernel<ROWS, true, false><<<grid, kQThreads, 0, stream>>>(p);
    else lords_mxfp4_quantize_kernel<ROWS, false, true><<<grid, kQThreads, 0, stream>>>(p);
}

int launch_mxfp4_quantize(const uint16_t *v, int rows, int cols, uint8_t *codes, uint8_t *scales, uint8_t *codes_t, uint8_t *scales_t, cudaStream_t stream)
{
    launch_quantize_rows<QROWS>({v, codes, scales, codes_t, scales_t, rows, cols}, stream);
    LORDS_CUDA_TRY(cudaGetLastError());
    return LORDS_OK;
}

int launch_mxfp4_dequantize(const uint8_t *codes, const uint8_t *scales, int rows, int cols, uint16_t *v, cudaStream_t stream)
{
    const dim3 grid((unsigned)((cols + 255) / 256), (unsigned)((rows + kTileRows - 1) / kTileRows));
    if (grid.y > 65535u) return LORDS_ERR_SHAPE;
    lords_mxfp4_dequantize_kernel<<<grid, kDThreads, 0, stream>>>(codes, scales, rows, cols, v);
    LORDS_CUDA_TRY(cudaGetLastError());
    return LORDS_OK;
}

}  // namespace lords

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
// A CTA takes 64 rows x 128 columns.  Along the rows, a thread holds a block in registers.  Along the columns, a thread reads two columns x 32 rows back
// from shared memory.  Scales meet in shared memory as words of four blocks.
//
// 14336 x 4096: rows 22.9 us (6.5 TB/s, the copy rate; with four threads to a block 30.7: 12.6 instructions a value kept the issue slots 81 % busy; with
// two 24.3), columns 29.8 and both 35.6 (46.5 with 16-byte stores along the columns; 5.0 TB/s: issue slots 67 % busy, load/store unit 61 %).
// Level or slower: 128 rows a CTA, 32 rows, 256 columns where all eight warps have columns (2048 x 4096 both ways 9.8 us in place of 7.2); rows off 16-byte
// pitches through shared memory, whole words of a row by neighbouring lanes (14336 x 4095 51 us, 32 so).
constexpr int kQRows = 64;                  // rows per CTA
constexpr int kQThreads = 256;
constexpr int kQPitch = 128 * 2 + 16;       // bytes per row of the tile in shared memory; 16-byte words stay aligned
constexpr int kQBlock = 32 * kQPitch + 64;  // ... and per 32 rows: the same columns of two neighbouring blocks lie in different banks

struct QuantizeParams {
    const uint16_t *v;       // bf16 [rows][cols]
    uint8_t *codes, *scales;         // blocks along the rows (null: not asked for)
    uint8_t *codes_t, *scales_t;     // blocks along the columns: the same for the transposed matrix (null: not asked for)
    int rows, cols;
    int pitch, pitch_t;              // bytes of a row of codes
    int ktiles, ktiles_t;            // tiles of scales in a row of them
    int wide, wide_t;                // rows of v, and of codes_t, begin at 32-byte boundaries
};

template <bool ALONG, bool ACROSS> __global__ void __launch_bounds__(kQThreads) lords_mxfp4_quantize_kernel(const QuantizeParams p)
{
    static_assert(kQRows * 4 == kQThreads, "a block of a row to a thread");
    __shared__ __align__(16) uint8_t tile[ACROSS ? kQRows / 32 * kQBlock : 16];
    __shared__ __align__(16) uint8_t sc[kQRows * 4], sct[128 * (kQRows / 32)];
    const int tid = threadIdx.x, r0 = (int)blockIdx.y * kQRows, c0 = (int)blockIdx.x * 128;
    const int seg = tid & 3, rl = tid >> 2, c = c0 + seg * kBlock, i = r0 + rl;
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    uint32_t w[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) w[e] = 0u;
    if (i < p.rows && c < p.cols) {
        const uint16_t *row = p.v + (size_t)i * p.cols;
        if (p.wide) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (h == 0 || c + 16 < p.cols)
                    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                                 : "=r"(w[8 * h]), "=r"(w[8 * h + 1]), "=r"(w[8 * h + 2]), "=r"(w[8 * h + 3]), "=r"(w[8 * h + 4]), "=r"(w[8 * h + 5]), "=r"(w[8 * h + 6]),
                                   "=r"(w[8 * h + 7])
                                 : "l"(row + c + 16 * h));
        } else {
            load_values<16>(row, p.cols, c, p.v + (size_t)p.rows * p.cols, w);
        }
    }
    if constexpr (ACROSS) {
        // (the second half of a row's threads begin with their second 32 bytes: no two of eight neighbours meet in a bank)
        const bool second = (seg & 2) != 0;
        uint4 *at = reinterpret_cast<uint4 *>(tile + (rl >> 5) * kQBlock + (rl & 31) * kQPitch + seg * 64);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int g = h ^ 2;
            at[second ? g : h] = second ? make_uint4(w[4 * g], w[4 * g + 1], w[4 * g + 2], w[4 * g + 3]) : make_uint4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]);
        }
    }
    if constexpr (ALONG) {
        uint32_t top = magnitudes(w[0]);
#pragma unroll
        for (int e = 1; e < 15; e += 2) top = larger(top, magnitudes(w[e]), magnitudes(w[e + 1]));
        top = larger(top, magnitudes(w[15]));
        const uint32_t byte = scale_byte<2>(larger_half(top));
        if (i < p.rows && c < p.cols)
            *reinterpret_cast<uint4 *>(p.codes + (size_t)i * p.pitch + c / 2) =
                make_uint4(to_codes4(w, byte), to_codes4(w + 4, byte), to_codes4(w + 8, byte), to_codes4(w + 12, byte));
        sc[rl * 4 + seg] = (uint8_t)byte;
    }
    __syncthreads();
    // a row's four scales are a word of the tile of scales; the rows behind the last are part of it
    if (ALONG && tid < kQRows) {
        const int i = r0 + tid;
        *reinterpret_cast<uint32_t *>(p.scales + ((size_t)(i / kTileRows) * p.ktiles + blockIdx.x) * kTileBytes + scale_at(i % kTileRows, 0)) =
            *reinterpret_cast<const uint32_t *>(sc + tid * 4);
    }
    if constexpr (ACROSS) {
        // two columns x 32 rows a thread; the lanes l and l + 16 of a warp have the same columns of neighbouring blocks and exchange halves, so that
        // each stores 32 bytes, a whole sector, of one column
        const int lane = tid & 31;
        for (int e = tid >> 5; e < 4 * (kQRows / 64); e += kQThreads / 32) {
            const int pair = (e & 3) * 16 + (lane & 15), half = lane >> 4, b = (e >> 2) * 2 + half;
            const uint8_t *at = tile + b * kQBlock + pair * 4;
            uint32_t u[32];
#pragma unroll
            for (int k = 0; k < 32; ++k) u[k] = *reinterpret_cast<const uint32_t *>(at + k * kQPitch);
            uint32_t top = magnitudes(u[0]);
#pragma unroll
            for (int k = 1; k < 31; k += 2) top = larger(top, magnitudes(u[k]), magnitudes(u[k + 1]));
            top = larger(top, magnitudes(u[31]));
            const uint32_t byte0 = scale_byte<2>(top & 0xFFFFu), byte1 = scale_byte<2>(top >> 16);
            const uint32_t inv = __byte_perm(inverse_scale(byte0), inverse_scale(byte1), 0x5410);       // each column its own
#pragma unroll
            for (int k = 0; k < 32; ++k) u[k] = bf16x2_mul(u[k], inv);
            uint32_t o0[4], o1[4], out[8];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint32_t *x = u + 8 * g;
                o0[g] = codes_of(low_half(x[0]), low_half(x[1]), low_half(x[2]), low_half(x[3]), low_half(x[4]), low_half(x[5]), low_half(x[6]), low_half(x[7]));
                o1[g] = codes_of(high_half(x[0]), high_half(x[1]), high_half(x[2]), high_half(x[3]), high_half(x[4]), high_half(x[5]), high_half(x[6]), high_half(x[7]));
                if (byte0 == 255u) o0[g] = 0u;
                if (byte1 == 255u) o1[g] = 0u;
            }
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint32_t theirs = __shfl_xor_sync(0xffffffffu, half ? o0[g] : o1[g], 16);
                out[g] = half ? theirs : o0[g];
                out[4 + g] = half ? o1[g] : theirs;
            }
            const int col = c0 + 2 * pair + half, r = r0 + (b & ~1) * 32;
            if (col < p.cols && r < p.rows) {
                uint8_t *dst = p.codes_t + (size_t)col * p.pitch_t + r / 2;
                if (p.wide_t) {
                    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(out[0]), "r"(out[1]), "r"(out[2]), "r"(out[3]), "r"(out[4]),
                                 "r"(out[5]), "r"(out[6]), "r"(out[7])
                                 : "memory");
                } else {
                    *reinterpret_cast<uint4 *>(dst) = make_uint4(out[0], out[1], out[2], out[3]);
                    if (r + 32 < p.rows) *reinterpret_cast<uint4 *>(dst + 16) = make_uint4(out[4], out[5], out[6], out[7]);
                }
            }
            sct[(2 * pair) * (kQRows / 32) + b] = (uint8_t)byte0;
            sct[(2 * pair + 1) * (kQRows / 32) + b] = (uint8_t)byte1;
        }
        __syncthreads();
        // a column's scales of this CTA's rows are half a word
        if (tid < 128) {
            uint8_t *dst = p.scales_t + ((size_t)blockIdx.x * p.ktiles_t + r0 / 128) * kTileBytes + scale_at(tid, r0 % 128 / 32);
            *reinterpret_cast<uint16_t *>(dst) = *reinterpret_cast<const uint16_t *>(sct + tid * 2);
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

// A warp takes four rows x 256 columns, a thread eight values of each (128 rows a CTA, four after four: 2048 x 4096 9.2 us, 14336 x 4096 28, so 4.5 and 24.9);
// WIDE, rows that begin at 32-byte boundaries: two rows x 512 columns, sixteen values of each.
constexpr int kDThreads = 256;
template <bool WIDE>
__global__ void __launch_bounds__(kDThreads) lords_mxfp4_dequantize_kernel(const uint8_t *codes, const uint8_t *scales, int rows, int cols, int pitch, int ktiles,
                                                                           uint16_t *v)
{
    constexpr int ROWS = WIDE ? 2 : 4, PER = WIDE ? 16 : 8;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = ((int)blockIdx.x * 32 + lane) * PER, r0 = (row_block() * (kDThreads / 32) + warp) * ROWS, b = c / kBlock;
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    // (the rows lie in one row of tiles)
    const uint8_t *sc = scales + ((size_t)(r0 / kTileRows) * ktiles + b / kTileBlocks) * kTileBytes;
    const uint8_t *src = codes + (size_t)r0 * pitch + c / 2;
    uint32_t w[ROWS][PER / 8], e[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k, src += pitch) {
        e[k] = 0u;
#pragma unroll
        for (int h = 0; h < PER / 8; ++h) w[k][h] = 0u;
        if (r0 + k >= rows || c >= cols) continue;
        if constexpr (WIDE) {
            const uint2 two = *reinterpret_cast<const uint2 *>(src);
            w[k][0] = two.x; w[k][1] = two.y;
        } else {
            w[k][0] = *reinterpret_cast<const uint32_t *>(src);
        }
        e[k] = sc[scale_at((r0 + k) % kTileRows, b % kTileBlocks)];
    }
    uint16_t *row = v + (size_t)r0 * cols;
#pragma unroll
    for (int k = 0; k < ROWS; ++k, row += cols) {
        if (r0 + k >= rows) break;
        if constexpr (WIDE) {
            if (c < cols) store16(row + c, values4(w[k][0], e[k]), values4(w[k][1], e[k]));
        } else {
            store8(row, cols, c, values4(w[k][0], e[k]), lane);
        }
    }
}

}  // namespace

template <bool ALONG, bool ACROSS> static int launch_quantize_variant(const QuantizeParams &p, cudaStream_t stream)
{
    // (whole tiles of scales are written, the rows behind the last among them)
    const dim3 grid((unsigned)((p.cols + 127) / 128), (unsigned)((p.rows + 127) / 128 * (128 / kQRows)));
    return launch_dependent(lords_mxfp4_quantize_kernel<ALONG, ACROSS>, grid, kQThreads, stream, p);
}

int launch_mxfp4_quantize(const uint16_t *v, int rows, int cols, uint8_t *codes, uint8_t *scales, uint8_t *codes_t, uint8_t *scales_t, cudaStream_t stream)
{
    const QuantizeParams p = {v, codes, scales, codes_t, scales_t, rows, cols, (int)codes_pitch(cols), (int)codes_pitch(rows), scale_tiles_of(cols),
                              scale_tiles_of(rows), cols % 16 == 0 && reinterpret_cast<uintptr_t>(v) % 32 == 0,
                              (rows + 31) / 32 % 2 == 0 && reinterpret_cast<uintptr_t>(codes_t) % 32 == 0};
    if (codes && codes_t) return launch_quantize_variant<true, true>(p, stream);
    return codes ? launch_quantize_variant<true, false>(p, stream) : launch_quantize_variant<false, true>(p, stream);
}

int launch_mxfp4_dequantize(const uint8_t *codes, const uint8_t *scales, int rows, int cols, uint16_t *v, cudaStream_t stream)
{
    const int pitch = (int)codes_pitch(cols), ktiles = scale_tiles_of(cols);
    auto launch = [&](auto kernel, int across, int down) {
        return launch_dependent(kernel, grid_of((unsigned)((cols + across - 1) / across), (unsigned)((rows + down - 1) / down)), kDThreads, stream, codes, scales, rows,
                                cols, pitch, ktiles, v);
    };
    if (cols % 16 == 0 && reinterpret_cast<uintptr_t>(v) % 32 == 0) return launch(lords_mxfp4_dequantize_kernel<true>, 512, 16);
    return launch(lords_mxfp4_dequantize_kernel<false>, 256, 32);
}

}  // namespace lords

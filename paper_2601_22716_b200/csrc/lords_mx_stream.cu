// y = x W^T on microscaled 4-bit operands, for few tokens.
//
// The tensor cores take e2m1 codes and their scales as they are stored (tcgen05.mma kind::mxf4, fp32 sums), so nothing is decoded: a
// CTA streams 128 rows of W through shared memory by TMA, 256 columns a step, as the MMA's 128-row operand; the tokens are its N = BN columns.
// The scales of a step follow their codes through shared memory and from there into TMEM (tcgen05.cp), where the MMA reads them.
//
//   QX:    x arrives in bf16; four warps bring each step's slice of it to 4 bits on the way (at most 16 tokens).  A token's slice
//          is worked on by every row tile, which costs less than a second launch.
//   else:  x arrives as codes and scales, by TMA like W.
//
// A cluster of CTAs divides a tile's steps where the row tiles alone leave SMs idle; token t is added up by CTA t mod cluster in distributed
// shared memory, in the order of the ranks, so results do not depend on timing.  No scratch memory: calls on different streams
// do not touch each other.
//
// Bound: the stream of codes and scales, 17/32 bytes a weight.  Everything is read in the stream's order.
//
// Every wait is bounded; on expiry the role records LORDS_ERR_TIMEOUT and leaves its loop.
#include <cuda.h>
#include <cuda_bf16.h>

#include "lords_internal.h"
#include "lords_mx.cuh"
#include "lords_ptx.cuh"
#include "lords_tc_common.cuh"

namespace lords {

namespace {

using namespace ptx;
using namespace mx;

constexpr int kRows = 128;                   // rows of W per CTA
constexpr int kStep = 256;                   // columns a step: 128 bytes of codes
constexpr int kConvWarp0 = 4;                // warps 4 .. 7: x to 4 bits, then the epilogue; 0: TMA, 1: MMA issuer, 2: TMEM
constexpr int kSThreads = 256;

template <int BN> struct SCfg {
    static constexpr int WTILE = kRows * 128;
    static constexpr int XTILE = BN * 128;
    static constexpr int SF = 2 * kTileBytes;                       // scales of a step: two tiles of four blocks
    static constexpr int STAGE = WTILE + XTILE + 2 * SF;            // a multiple of 1024 (BN is a multiple of 8)
    static constexpr int RECV = BN * kRows * 4;                     // partial sums from the cluster
    static constexpr int STAGES = (230 * 1024 - 2048 - RECV) / STAGE < 10 ? (230 * 1024 - 2048 - RECV) / STAGE : 10;
    static constexpr int SMEM = 1024 + STAGES * STAGE + RECV + 512;
    static constexpr uint32_t ACC = BN < 32 ? 32 : BN;              // accumulator columns; behind them two sets of scales
    static constexpr uint32_t TMEM = ACC + 32 <= 64 ? 64 : ACC + 32 <= 128 ? 128 : 256;
    static_assert(SMEM <= 232448 && STAGE % 1024 == 0, "shared memory");
};

struct alignas(64) StreamParams {
    CUtensorMap tm_w;        // bytes [m][pitch], box {128, 128}, 128-byte swizzle (zeros behind the last row and byte)
    CUtensorMap tm_x;        // bytes [M][pitch], box {128, BN}; not used with QX
    const uint8_t *ws;       // scale tiles of W
    const uint8_t *xs;       // scale tiles of x; not used with QX
    const uint16_t *x;       // bf16 [M][n]; QX only
    int M, m, n;
    int steps, blocks, ktiles;       // of a row: steps of 256 columns, blocks, scale tiles
    void *y;
    int y_f32;
    int *status;
};

template <int BN, bool QX>
__global__ void __launch_bounds__(kSThreads, 1) lords_mxfp4_stream_kernel(const __grid_constant__ StreamParams p)
{
    using C = SCfg<BN>;
    constexpr int STAGES = C::STAGES;
    extern __shared__ uint8_t s_smem[];
    const uint32_t base = (smem_u32(s_smem) + 1023u) & ~1023u;
    const uint32_t recv = base + STAGES * C::STAGE, bars = recv + C::RECV;
    const uint32_t bar_full = bars, bar_empty = bar_full + 8 * STAGES, bar_acc = bar_empty + 8 * STAGES, bar_recv = bar_acc + 8, tmem_slot = bar_recv + 8;
    static_assert(16 * STAGES + 24 <= 512, "barrier area");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster_ctarank(), split = (int)cluster_nctarank();
    const int rt = (int)(blockIdx.x / split), row0 = rt * kRows, tok0 = (int)blockIdx.y * BN;
    const int s_a = (int)((long long)p.steps * rank / split), s_b = (int)((long long)p.steps * (rank + 1) / split);
    const int tokens = p.M - tok0 < BN ? p.M - tok0 : BN;
    const int *status = p.status;
    bool failed = false;

    if (warp == 0) {
        if (lane == 0) {
            for (int s = 0; s < STAGES; ++s) { mbar_init(bar_full + 8 * s, QX ? 5 : 1); mbar_init(bar_empty + 8 * s, 1); }
            mbar_init(bar_acc, 1);
            mbar_init(bar_recv, 1);
            fence_mbar_init();
            const int own = tokens > rank ? (tokens - rank + split - 1) / split : 0;
            if (split > 1) mbar_expect_tx(bar_recv, (uint32_t)((split - 1) * own * kRows * 4));
            tma_prefetch_desc(&p.tm_w);
            if (!QX) tma_prefetch_desc(&p.tm_x);
        }
    } else if (warp == 2) {
        tmem_alloc(tmem_slot, C::TMEM);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (split > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // waited for before the first store to another CTA
    tc_fence_after_sync();
    uint32_t tmem_base;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem_base) : "r"(tmem_slot));
    griddep_launch_dependents();
    griddep_wait();

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA: codes and scales of W, and of x
        if (lane == 0) {
            int it = 0;
            for (int st = s_a; st < s_b; ++st, ++it) {
                const int s = it % STAGES;
                if (it >= STAGES && !mbar_wait(bar_empty + 8 * s, (uint32_t)((it / STAGES - 1) & 1), status, 61)) { failed = true; break; }
                const uint32_t dst = base + (uint32_t)(s * C::STAGE), bar = bar_full + 8 * s;
                const int kt = p.ktiles - 2 * st < 2 ? 1 : 2;
                mbar_expect_tx(bar, (uint32_t)(C::WTILE + kt * kTileBytes + (QX ? 0 : C::XTILE + kt * kTileBytes)));
                tma_load_2d(dst, &p.tm_w, st * 128, row0, bar);
                bulk_load(dst + C::WTILE + C::XTILE, p.ws + ((size_t)rt * p.ktiles + 2 * st) * kTileBytes, (uint32_t)(kt * kTileBytes), bar);
                if (!QX) {
                    tma_load_2d(dst + C::WTILE, &p.tm_x, st * 128, tok0, bar);
                    bulk_load(dst + C::WTILE + C::XTILE + C::SF, p.xs + ((size_t)(tok0 / kTileRows) * p.ktiles + 2 * st) * kTileBytes,
                              (uint32_t)(kt * kTileBytes), bar);
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        const uint32_t hi = (uint32_t)(umma_desc_sw128(0, 1024, 16) >> 32), lo0 = (uint32_t)umma_desc_sw128(0, 1024, 16);
        const uint32_t tmem_u = warp_uniform(tmem_base), leader = elect_one();
        const uint32_t xcol = QX ? 0u : (uint32_t)(tok0 % kTileRows / 32);      // x's tile of tokens inside its tile of scales
        int it = 0;
        for (int st = s_a; st < s_b; ++st, ++it) {
            const int s = it % STAGES;
            if (!mbar_wait_warp(bar_full + 8 * s, (uint32_t)((it / STAGES) & 1), status, 62)) { failed = true; break; }
            tc_fence_after_sync();
            const uint32_t at = base + (uint32_t)(s * C::STAGE), sw = at + C::WTILE + C::XTILE, sx = sw + C::SF;
            const uint32_t a_lo = lo0 | ((at & 0x3FFFFu) >> 4), b_lo = lo0 | (((at + C::WTILE) & 0x3FFFFu) >> 4);
            const int mmas = (p.blocks - 8 * st + 1) / 2 < 4 ? (p.blocks - 8 * st + 1) / 2 : 4;
            const uint32_t cw = tmem_u + C::ACC + (uint32_t)((it & 1) * 16), cx = cw + 8;
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if (2 * j < mmas) {
                    scales_to_tmem(cw + 4 * j, scales_desc(sw + (uint32_t)(j * kTileBytes)), leader);
                    scales_to_tmem(cx + 4 * j, scales_desc(sx + (uint32_t)(j * kTileBytes)), leader);
                }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < mmas)
                    umma_mxf4_ss(tmem_u, umma_desc_pack(a_lo + 2 * k, hi), umma_desc_pack(b_lo + 2 * k, hi), umma_idesc_mxf4(kRows, BN, k & 1), cw + 4 * (k >> 1),
                                 cx + 4 * (k >> 1) + xcol, (it > 0 || k > 0) ? 1u : 0u, leader);
            umma_commit(bar_empty + 8 * s, leader);
        }
        umma_commit(bar_acc, leader);
    } else if (warp >= kConvWarp0) {
        const int q = warp - kConvWarp0;
        if constexpr (QX) {
            // -------------------------------------------------------------- x to 4 bits: a block of a token per thread and step
            const int t = (tid - kConvWarp0 * 32) >> 3, b = tid & 7;
            const uint16_t *row = p.x + (size_t)(t < p.M ? t : 0) * p.n;
            auto load = [&](int st, uint32_t (&w)[16]) {
                const int c = st * kStep + b * kBlock;
#pragma unroll
                for (int k = 0; k < 16; ++k) w[k] = 0u;
                if (t >= p.M || c >= p.n) return;
                if ((p.n & 7) == 0) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (c + 8 * k < p.n) {
                            const uint4 v = __ldcg(reinterpret_cast<const uint4 *>(row + c) + k);
                            w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w;
                        }
                } else {
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const uint32_t lo = c + 2 * k < p.n ? __ldcg(row + c + 2 * k) : 0u, up = c + 2 * k + 1 < p.n ? __ldcg(row + c + 2 * k + 1) : 0u;
                        w[k] = lo | up << 16;
                    }
                }
            };
            uint32_t w[16], next[16];
            if (s_a < s_b) load(s_a, w);
            int it = 0;
            for (int st = s_a; st < s_b; ++st, ++it) {
                const int s = it % STAGES;
                if (st + 1 < s_b) load(st + 1, next);
                uint32_t top = 0u;
#pragma unroll
                for (int k = 0; k < 16; ++k) top = max_magnitudes(top, w[k]);
                const uint32_t byte = scale_byte<2>(max(top & 0xFFFFu, top >> 16));
                uint32_t out[4];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const uint32_t v[4] = {w[4 * g], w[4 * g + 1], w[4 * g + 2], w[4 * g + 3]};
                    out[g] = to_codes4(v, byte);
                }
                if (it >= STAGES && !mbar_wait_warp(bar_empty + 8 * s, (uint32_t)((it / STAGES - 1) & 1), status, 63)) { failed = true; break; }
                const uint32_t at = base + (uint32_t)(s * C::STAGE) + C::WTILE;
                if (t < BN) sts_v4(at + (uint32_t)(t * 128 + ((b ^ (t & 7)) << 4)), make_uint4(out[0], out[1], out[2], out[3]));
                asm volatile("st.shared.u8 [%0], %1;" ::"r"(at + C::XTILE + C::SF + (uint32_t)(b / kTileBlocks * kTileBytes + scale_at(t, b % kTileBlocks))), "r"(byte)
                             : "memory");
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_full + 8 * s);
#pragma unroll
                for (int k = 0; k < 16; ++k) w[k] = next[k];
            }
        }
        // ------------------------------------------------------------------ epilogue: lane = row of W, columns = tokens
        if (!mbar_wait_warp(bar_acc, 0, status, 64)) failed = true;
        tc_fence_after_sync();
        const int ri = q * 32 + lane, i = row0 + ri;
        const uint32_t acc = tmem_base + ((uint32_t)(q * 32) << 16);
        if (split > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
#pragma unroll
        for (int c0 = 0; c0 < BN; c0 += 16) {
            if (c0 >= tokens) break;
            uint32_t v[16];
            tmem_ld_32x16(acc + (uint32_t)c0, v);
            tmem_wait_ld(v);
#pragma unroll
            for (int c = 0; c < 16; ++c) {
                const int t = c0 + c;
                if (t >= tokens) break;
                if (split == 1) {
                    if (i < p.m && !failed) store_out(p.y, p.y_f32, (size_t)(tok0 + t) * p.m + i, __uint_as_float(v[c]));
                    continue;
                }
                // partial sums lie by slot (token / cluster), rank and row
                const int to = t % split;
                const uint32_t where = recv + (uint32_t)((((t / split) * split + rank) * kRows + ri) * 4);
                if (to == rank) sts_u32(where, v[c]);
                else st_async_cluster_f32(map_to_rank(where, (uint32_t)to), __uint_as_float(v[c]), map_to_rank(bar_recv, (uint32_t)to));
            }
        }
        if (split > 1 && rank < tokens) {
            if (!__all_sync(0xffffffffu, mbar_wait_cluster(bar_recv, 0, status, 65))) failed = true;
            for (int t = rank; t < tokens && !failed; t += split) {
                float sum = 0.0f;
                for (int r = 0; r < split; ++r) sum += __uint_as_float(lds_u32(recv + (uint32_t)((((t / split) * split + r) * kRows + ri) * 4)));
                if (i < p.m) store_out(p.y, p.y_f32, (size_t)(tok0 + t) * p.m + i, sum);
            }
        }
    }
    if (split > 1 && warp < kConvWarp0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");

    if (failed) ptx::record_give_up(p.status, LORDS_ERR_TIMEOUT);
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 2) {
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, C::TMEM);
    }
}

template <int BN, bool QX> int launch_variant(StreamParams &k, int split, const State &st, cudaStream_t stream)
{
    static bool done[kMaxDevices] = {};
    const int dev = device_slot(st);
    if (!done[dev]) {
        LORDS_CUDA_TRY(cudaFuncSetAttribute(lords_mxfp4_stream_kernel<BN, QX>, cudaFuncAttributeMaxDynamicSharedMemorySize, SCfg<BN>::SMEM));
        done[dev] = true;
    }
    const int row_tiles = (k.m + kRows - 1) / kRows, tok_tiles = (k.M + BN - 1) / BN;
    if (tok_tiles > 65535 || (long long)row_tiles * split > 2147483647LL) return LORDS_ERR_SHAPE;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)split;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = cudaLaunchConfig_t{};
    cfg.gridDim = dim3((unsigned)(row_tiles * split), (unsigned)tok_tiles);
    cfg.blockDim = dim3(kSThreads);
    cfg.dynamicSmemBytes = SCfg<BN>::SMEM;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    LORDS_CUDA_TRY(cudaLaunchKernelEx(&cfg, lords_mxfp4_stream_kernel<BN, QX>, k));
    return LORDS_OK;
}

// CTAs that share a row tile's steps: as many as SMs allow, at most eight and four steps at least to each.
int choose_split(int tiles, int steps, int sms)
{
    int c = 1;
    while (c < 8 && tiles * c * 2 <= sms && steps >= 4 * c * 2) c *= 2;
    return c;
}

}  // namespace

int launch_mxfp4_stream(const MxProblem &p, State &st, cudaStream_t stream)
{
    StreamParams k;
    k.ws = p.ws; k.xs = p.xs; k.x = p.x;
    k.M = p.M; k.m = p.m; k.n = p.n;
    k.blocks = blocks_of(p.n);
    k.ktiles = scale_tiles_of(p.n);
    k.steps = (p.n + kStep - 1) / kStep;
    k.y = p.y; k.y_f32 = p.y_f32;
    k.status = st.status_word;
    const bool qx = p.x != nullptr;
    const int bn = p.M <= 16 ? 16 : p.M <= 32 ? 32 : p.M <= 64 ? 64 : 128;
    if (qx && bn > 16) return LORDS_ERR_UNSUPPORTED;
    const uint64_t pitch = (uint64_t)codes_pitch(p.n);
    if (!make_map_2d(&k.tm_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.w, pitch, (uint64_t)p.m, 128, kRows, CU_TENSOR_MAP_SWIZZLE_128B)) return LORDS_ERR_CUDA;
    if (qx) k.tm_x = k.tm_w;
    else if (!make_map_2d(&k.tm_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.xq, pitch, (uint64_t)p.M, 128, (uint32_t)bn, CU_TENSOR_MAP_SWIZZLE_128B)) return LORDS_ERR_CUDA;
    const int split = choose_split((p.m + kRows - 1) / kRows * ((p.M + bn - 1) / bn), k.steps, st.sm_count);
    int rc;
    if (qx) rc = launch_variant<16, true>(k, split, st, stream);
    else if (bn == 16) rc = launch_variant<16, false>(k, split, st, stream);
    else if (bn == 32) rc = launch_variant<32, false>(k, split, st, stream);
    else if (bn == 64) rc = launch_variant<64, false>(k, split, st, stream);
    else rc = launch_variant<128, false>(k, split, st, stream);
    if (rc != LORDS_OK) return rc;
    st.last_launches += 1;
    st.last_path = "mxfp4_stream";
    return LORDS_OK;
}

}  // namespace lords

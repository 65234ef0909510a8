// y = x W^T on microscaled 4-bit operands, for many tokens: tcgen05.mma kind::mxf4 on CTA pairs (cta_group::2).
//
// A pair computes 256 tokens x BN out-features; the tokens are the MMA's rows, so that a thread of the epilogue holds one token's
// neighbouring out-features: it puts 128 bytes of them into its row of a shared-memory tile, which leaves by TMA.  A step is 256 columns, 128 bytes of codes a row: each CTA loads its 128
// tokens and its half of the out-features by TMA, its tokens' scales and the scales of all BN out-features, which go on to TMEM
// (tcgen05.cp) ahead of the step's four MMAs.  Tiles are dealt out to as many pairs as are resident; with BN = 128 two accumulators take turns, so
// that a tile's stores run beside the next one's MMAs, with 256 the loads of the next tile do.
//
// Bound: 4-bit MMAs (four times the bf16 rate, 512 cycles a step at BN = 256) and what L2 gives, 128 (128 + BN / 2) bytes of codes a step and CTA: all SMs
// together read 13 to 14 TB/s with either BN (0.29 and 0.36 us a step), with L2's own units at 36 % and the clock at 1.64 GHz under the
// power limit.  2048 tokens: 4096 x 14336 44 us (5.5 PFLOP/s), 14336 x 4096 48, its weight gradient in 32 bits 63.  The copies of the
// scales cost 3 % of that (left out: 42.5); a step's copies ahead of the step before's MMAs, or between them, cost 17 to 30 % more.
// No scratch memory.  Every wait is bounded; on expiry the role records LORDS_ERR_TIMEOUT and leaves its loop.
#include <cuda.h>
#include <cuda_bf16.h>

#include "lords_internal.h"
#include "lords_mx.cuh"
#include "lords_pair.cuh"
#include "lords_ptx.cuh"
#include "lords_tc_common.cuh"

namespace lords {

namespace {

using namespace ptx;
using namespace mx;

constexpr int kPTokens = 256;                // tokens per CTA pair
constexpr int kPEpiWarp0 = 4;                // warps from 4 on: epilogue; 0: TMA, 1: MMA issuer, 2: TMEM

template <int BN> struct PCfg {
    static constexpr int EPI = 8;
    static constexpr int THREADS = (kPEpiWarp0 + EPI) * 32;
    static constexpr int XTILE = 128 * 128;                      // this CTA's tokens
    static constexpr int WTILE = BN / 2 * 128;                   // this CTA's half of the out-features
    static constexpr int XSF = 2 * kTileBytes;                   // scales of a step: two tiles of four blocks
    static constexpr int WSF = BN / kTileRows * 2 * kTileBytes;
    static constexpr int STAGE = XTILE + WTILE + XSF + WSF;
    static constexpr int OUT = EPI * 4096;                       // 32 tokens x 128 bytes of y a warp, on their way out
    static constexpr int STAGES = (232448 - 1024 - 256 - OUT) / STAGE;
    static constexpr int SMEM = 1024 + STAGES * STAGE + OUT + 256;
    static constexpr int ACCS = BN <= 128 ? 2 : 1;
    static constexpr uint32_t SF_COL = ACCS * BN;                // behind the accumulators: two sets of scales of a step
    static constexpr uint32_t SF_COLS = 8 + BN / kTileRows * 8;
    static_assert(STAGE % 1024 == 0 && SMEM <= 232448 && SF_COL + 2 * SF_COLS <= 512, "shared memory and TMEM");
};

struct alignas(64) PairParams {
    CUtensorMap tm_x;        // bytes [M][pitch], box {128, 128}, 128-byte swizzle (zeros behind the last row and byte)
    CUtensorMap tm_w;        // bytes [m][pitch], box {128, BN / 2}
    CUtensorMap tm_xs;       // scale tiles as words [row tiles][128 ktiles], box {256, 1}
    CUtensorMap tm_ws;       // the same, box {256, BN / 128}
    CUtensorMap tm_y;        // y, box {128 bytes, 32 rows}, 128-byte swizzle; used if rows of y are 16-byte multiples
    int y_by_tma;
    int M, m;
    int tok_tiles, w_tiles, tiles, steps, blocks;
    int pairs;
    void *y;
    int y_f32;
    int *status;

    // Tiles go in bands of eight out-feature tiles, token tile after token tile.  (All token tiles of one out-feature tile first: weight gradients of 4096 x
    // 14336 and 2048 columns 67.5 us, of 14336 x 4096 and 512 columns 48.8; all out-feature tiles first 62.6 and 41.9, but 14336 x 4096 and 2048
    // columns 66.9; so 62.1, 45.3 and 63.5.  Results in bf16 are level.)
    __device__ __forceinline__ void place(int tile, int &wt, int &tt) const
    {
        constexpr int kBand = 8;
        if (tok_tiles == 1) {            // (a division is a tenth of a microsecond of a small call)
            tt = 0;
            wt = tile;
            return;
        }
        const int per = tok_tiles * kBand, band = tile < per ? 0 : tile / per, in = tile - band * per, wide = w_tiles - band * kBand;
        tt = wide >= kBand ? in / kBand : in / wide;
        wt = band * kBand + in - tt * (wide < kBand ? wide : kBand);
    }
};

__device__ __forceinline__ uint32_t pack_bf16(uint32_t lo, uint32_t hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(__uint_as_float(lo), __uint_as_float(hi));
    return *reinterpret_cast<const uint32_t *>(&v);
}
// A tile of shared memory to global memory, rows and columns outside the tensor left out; a group of its own.
__device__ __forceinline__ void tma_store_2d(const void *tmap, int x, int y, uint32_t src, uint64_t policy)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group.L2::cache_hint [%0, {%2, %3}], [%1], %4;" ::"l"(tmap), "r"(src), "r"(x), "r"(y), "l"(policy) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// The thread's stores have read their shared memory.
__device__ __forceinline__ void tma_store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }

template <int BN>
__global__ void __launch_bounds__(PCfg<BN>::THREADS, 1) lords_mxfp4_pair_kernel(const __grid_constant__ PairParams p)
{
    using C = PCfg<BN>;
    constexpr int STAGES = C::STAGES;
    extern __shared__ uint8_t p_smem[];
    const uint32_t base = (smem_u32(p_smem) + 1023u) & ~1023u;
    const uint32_t out_s = base + STAGES * C::STAGE, bars = out_s + C::OUT;
    const uint32_t bar_full = bars, bar_empty = bars + 8 * STAGES, bar_acc_full = bar_empty + 8 * STAGES, bar_acc_empty = bar_acc_full + 16;
    const uint32_t tmem_slot = bar_acc_empty + 16;
    static_assert(8 * (2 * STAGES + 4) + 4 <= 256, "barrier area");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster_ctarank(), pair = (int)(blockIdx.x >> 1);
    const int *status = p.status;
    bool failed = false;

    if (warp == 0) {
        if (lane < 2 * STAGES + 2) mbar_init(bars + 8 * lane, 1);
        if (lane >= 2 * STAGES + 2 && lane < 2 * STAGES + 4) mbar_init(bars + 8 * lane, 2 * C::EPI);       // read by both CTAs' epilogue
        fence_mbar_init();
        if (lane == 0) { tma_prefetch_desc(&p.tm_x); tma_prefetch_desc(&p.tm_w); tma_prefetch_desc(&p.tm_xs); tma_prefetch_desc(&p.tm_ws); }
    } else if (warp == 2) {
        tmem_alloc2(tmem_slot, 512);
    }
    tc_fence_before_sync();
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");       // both CTAs' barriers exist
    tc_fence_after_sync();
    uint32_t tmem_base;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem_base) : "r"(tmem_slot));
    griddep_launch_dependents();
    griddep_wait();

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA.  (The lane that elect.sync names: the compiler then knows that one
        // thread runs the branch.  Under lane == 0 the four loads of a step took longer than its MMAs: 2048 tokens, 4096 x 14336, 78.6 us with BN
        // = 128 and 45.3 with 256, 65.9 and 43.9 so; by the whole warp under a predicate 97.5 and 53.9.)
        if (elect_one()) {
            const uint32_t full0 = map_to_rank(bar_full, 0);
            int it = 0;
            for (int tile = pair; tile < p.tiles && !failed; tile += p.pairs) {
                int wt, tt;
                p.place(tile, wt, tt);
                for (int k = 0; k < p.steps; ++k, ++it) {
                    const int s = it % STAGES;
                    if (it >= STAGES && !mbar_wait(bar_empty + 8 * s, (uint32_t)((it / STAGES - 1) & 1), status, 71)) { failed = true; break; }
                    if (rank == 0) mbar_expect_tx(bar_full + 8 * s, 2u * C::STAGE);
                    const uint32_t dst = base + (uint32_t)(s * C::STAGE), bar = full0 + 8 * s;
                    tma_load_2d_pair(dst, &p.tm_x, k * 128, tt * kPTokens + rank * 128, bar);
                    tma_load_2d_pair(dst + C::XTILE, &p.tm_w, k * 128, wt * BN + rank * (BN / 2), bar);
                    tma_load_2d_pair(dst + C::XTILE + C::WTILE, &p.tm_xs, k * 256, tt * 2 + rank, bar);
                    tma_load_2d_pair(dst + C::XTILE + C::WTILE + C::XSF, &p.tm_ws, k * 256, wt * (BN / kTileRows), bar);
                }
            }
            // nothing of this CTA is in flight when it ends: the last round of stages has been read
            for (int k = it > STAGES ? it - STAGES : 0; k < it && !failed; ++k)
                if (!mbar_wait(bar_empty + 8 * (k % STAGES), (uint32_t)((k / STAGES) & 1), status, 72)) failed = true;
        }
        __syncwarp();
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------------------------ MMA issuer (the pair's even CTA)
        const uint32_t hi = (uint32_t)(umma_desc_sw128(0, 1024, 16) >> 32), lo0 = (uint32_t)umma_desc_sw128(0, 1024, 16);
        const uint32_t tmem_u = warp_uniform(tmem_base), leader = elect_one();
        int it = 0, n = 0;
        for (int tile = pair; tile < p.tiles && !failed; tile += p.pairs, ++n) {
            const int a = n % C::ACCS;
            if (n >= C::ACCS && !mbar_wait_warp(bar_acc_empty + 8 * a, (uint32_t)((n / C::ACCS - 1) & 1), status, 73)) { failed = true; break; }
            tc_fence_after_sync();
            for (int k = 0; k < p.steps; ++k, ++it) {
                const int s = it % STAGES;
                if (!mbar_wait_warp(bar_full + 8 * s, (uint32_t)((it / STAGES) & 1), status, 74)) { failed = true; break; }
                tc_fence_after_sync();
                const uint32_t at = base + (uint32_t)(s * C::STAGE), sx = at + C::XTILE + C::WTILE, sw = sx + C::XSF;
                const uint32_t a_lo = lo0 | ((at & 0x3FFFFu) >> 4), b_lo = lo0 | (((at + C::XTILE) & 0x3FFFFu) >> 4);
                const uint32_t cx = tmem_u + C::SF_COL + (uint32_t)((it & 1) * C::SF_COLS), cw = cx + 8;
                const int mmas = (p.blocks - 8 * k + 1) / 2 < 4 ? (p.blocks - 8 * k + 1) / 2 : 4;
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (2 * j < mmas) {
                        scales_to_tmem2(cx + 4 * j, scales_desc(sx + (uint32_t)(j * kTileBytes)), leader);
                        // (a row of tiles after the other in shared memory, the tiles of a K side by side in TMEM)
#pragma unroll
                        for (int r = 0; r < BN / kTileRows; ++r)
                            scales_to_tmem2(cw + (uint32_t)(j * (BN / 32) + 4 * r), scales_desc(sw + (uint32_t)((2 * r + j) * kTileBytes)), leader);
                    }
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    if (kk < mmas)
                        umma2_mxf4_ss(tmem_u + (uint32_t)(a * BN), umma_desc_pack(a_lo + 2 * kk, hi), umma_desc_pack(b_lo + 2 * kk, hi),
                                      umma_idesc_mxf4(kPTokens, BN, kk & 1), cx + 4 * (kk >> 1), cw + (BN / 32) * (kk >> 1), (k > 0 || kk > 0) ? 1u : 0u, leader);
                umma2_commit(bar_empty + 8 * s, leader);
                if (k == p.steps - 1) umma2_commit(bar_acc_full + 8 * a, leader);
            }
        }
    } else if (warp >= kPEpiWarp0) {
        // ------------------------------------------------------------------ epilogue: lane = token, columns = out-features
        const int q = warp & 3, ch = (warp - kPEpiWarp0) >> 2;                // quadrant of the tokens, share of the columns
        constexpr int CW = BN / (C::EPI / 4);
        const uint32_t empty0 = map_to_rank(bar_acc_empty, 0);
        const uint32_t acc = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(ch * CW);
        uint64_t policy;
        asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
        const uint32_t own = out_s + (uint32_t)((warp - kPEpiWarp0) * 4096), row = own + (uint32_t)(lane * 128);
        int n = 0;
        for (int tile = pair; tile < p.tiles; tile += p.pairs, ++n) {
            const int a = n % C::ACCS;
            int wt, tt;
            p.place(tile, wt, tt);
            if (!__all_sync(0xffffffffu, mbar_wait_cluster(bar_acc_full + 8 * a, (uint32_t)((n / C::ACCS) & 1), status, 75))) { failed = true; break; }
            tc_fence_after_sync();
            const int t0 = tt * kPTokens + rank * 128 + q * 32;
            auto put = [&](int c, const uint32_t *w) {        // 16 bytes of the thread's row, chunk c of 8
                sts_v4(row + (uint32_t)((c ^ (lane & 7)) << 4), make_uint4(w[0], w[1], w[2], w[3]));
            };
            auto leave = [&](int i) {                          // 128 bytes of 32 tokens, from out-feature i on
                if (p.y_by_tma) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0 && t0 < p.M && i < p.m) tma_store_2d(&p.tm_y, i, t0, own, policy);
                    return;
                }
                // rows of y that TMA cannot express: token after token, the warp's lanes side by side (2048 tokens, 4094 x 4096: 88 us when every lane
                // stored its own token's values)
                __syncwarp();
                const int count = p.M - t0 < 32 ? p.M - t0 : 32;
                for (int r = 0; r < count; ++r) {
                    auto at = [&](int byte) { return own + (uint32_t)(r * 128 + (((byte >> 4) ^ (r & 7)) << 4) + (byte & 15)); };
                    const size_t to = (size_t)(t0 + r) * p.m + i;
                    if (p.y_f32) {
                        if (i + lane < p.m) static_cast<uint32_t *>(p.y)[to + lane] = lds_u32(at(4 * lane));
                    } else if ((p.m & 1) == 0) {
                        if (i + 2 * lane < p.m) *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(p.y) + to + 2 * lane) = lds_u32(at(4 * lane));
                    } else {
                        const uint32_t two = lds_u32(at(4 * lane));
                        uint16_t *dst = static_cast<uint16_t *>(p.y) + to + 2 * lane;
                        if (i + 2 * lane < p.m) dst[0] = (uint16_t)two;
                        if (i + 2 * lane + 1 < p.m) dst[1] = (uint16_t)(two >> 16);
                    }
                }
                __syncwarp();
            };
            auto load = [&](int c0, uint32_t (&v)[32]) {
                tmem_ld_32x32(acc + (uint32_t)(a * BN + c0), v);
                tmem_wait_ld(v);
            };
            auto release = [&]() {                             // the accumulator has been read
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_pair(empty0 + 8 * a);
            };
            auto room = [&]() {                                // what left last has been read from the warp's tile
                if (p.y_by_tma && lane == 0) tma_store_wait_read();
                __syncwarp();
            };
            const int i0 = wt * BN + ch * CW;
            if (p.y_f32) {
                // all of it into registers first, so that the next tile's MMAs wait no longer than that takes
                uint32_t v[CW / 32][32];
#pragma unroll
                for (int c = 0; c < CW / 32; ++c) tmem_ld_32x32(acc + (uint32_t)(a * BN + 32 * c), v[c]);
#pragma unroll
                for (int c = 0; c < CW / 32; ++c) tmem_wait_ld(v[c]);
                release();
#pragma unroll
                for (int g = 0; g < CW / 32; ++g) {
                    room();
#pragma unroll
                    for (int c = 0; c < 8; ++c) put(c, v[g] + 4 * c);
                    leave(i0 + 32 * g);
                }
            } else {
                uint32_t w[CW / 2];
#pragma unroll
                for (int c0 = 0; c0 < CW; c0 += 32) {
                    uint32_t v[32];
                    load(c0, v);
#pragma unroll
                    for (int c = 0; c < 16; ++c) w[c0 / 2 + c] = pack_bf16(v[2 * c], v[2 * c + 1]);
                }
                release();
#pragma unroll
                for (int c0 = 0; c0 < CW; c0 += 64) {
                    room();
#pragma unroll
                    for (int c = 0; c < 8; ++c) put(c, w + c0 / 2 + 4 * c);
                    leave(i0 + c0);
                }
            }
        }
        if (lane == 0) tma_store_wait_read();
        __syncwarp();
    }

    if (failed) ptx::record_give_up(p.status, LORDS_ERR_TIMEOUT);
    tc_fence_before_sync();
    __syncthreads();
    // neither CTA leaves while the other may still signal its barriers or read its operands
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (warp == 2) {
        tc_fence_after_sync();
        tmem_dealloc2(tmem_base, 512);
    }
}

template <int BN> struct PairVariant {
    static void fill(cudaLaunchConfig_t &cfg, cudaLaunchAttribute *attr, int pairs, cudaStream_t stream)
    {
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg = cudaLaunchConfig_t{};
        cfg.gridDim = dim3((unsigned)(2 * pairs));
        cfg.blockDim = dim3(PCfg<BN>::THREADS);
        cfg.dynamicSmemBytes = PCfg<BN>::SMEM;
        cfg.stream = stream;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
    }
    // CTA pairs that can be resident at once
    static int resident(const State &st)
    {
        static int cache[kMaxDevices] = {};
        const int dev = device_slot(st);
        if (cache[dev] == 0) {
            if (cudaFuncSetAttribute(lords_mxfp4_pair_kernel<BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, PCfg<BN>::SMEM) != cudaSuccess) return 0;
            cudaLaunchConfig_t cfg;
            cudaLaunchAttribute attr[2];
            fill(cfg, attr, 1, nullptr);
            int n = 0;
            if (cudaOccupancyMaxActiveClusters(&n, lords_mxfp4_pair_kernel<BN>, &cfg) != cudaSuccess) (void)cudaGetLastError();
            cache[dev] = n >= 1 ? n : -1;
        }
        return cache[dev] > 0 ? cache[dev] : 0;
    }
};

template <int BN> int run_pair(const MxProblem &p, State &st, cudaStream_t stream)
{
    const int resident = PairVariant<BN>::resident(st);
    if (resident < 1) return LORDS_ERR_UNSUPPORTED;
    PairParams k;
    const uint64_t pitch = (uint64_t)codes_pitch(p.n), words = (uint64_t)scale_tiles_of(p.n) * (kTileBytes / 4);
    const uint64_t xt = (uint64_t)((p.M + kTileRows - 1) / kTileRows), wt = (uint64_t)((p.m + kTileRows - 1) / kTileRows);
    if (!make_map_2d(&k.tm_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.xq, pitch, (uint64_t)p.M, 128, 128, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_map_2d(&k.tm_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.w, pitch, (uint64_t)p.m, 128, BN / 2, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_map_2d(&k.tm_xs, CU_TENSOR_MAP_DATA_TYPE_INT32, 4, p.xs, words, xt, 256, 1, CU_TENSOR_MAP_SWIZZLE_NONE) ||
        !make_map_2d(&k.tm_ws, CU_TENSOR_MAP_DATA_TYPE_INT32, 4, p.ws, words, wt, 256, BN / kTileRows, CU_TENSOR_MAP_SWIZZLE_NONE))
        return LORDS_ERR_CUDA;
    k.y_by_tma = ((size_t)p.m * (p.y_f32 ? 4 : 2)) % 16 == 0;
    k.tm_y = k.tm_x;
    if (k.y_by_tma && !make_map_2d(&k.tm_y, p.y_f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, p.y_f32 ? 4 : 2, p.y, (uint64_t)p.m,
                                   (uint64_t)p.M, p.y_f32 ? 32 : 64, 32, CU_TENSOR_MAP_SWIZZLE_128B))
        return LORDS_ERR_CUDA;
    k.M = p.M; k.m = p.m;
    k.tok_tiles = (p.M + kPTokens - 1) / kPTokens;
    k.w_tiles = (p.m + BN - 1) / BN;
    const long long tiles = (long long)k.tok_tiles * k.w_tiles;
    if (tiles > 2147483647LL - 65536) return LORDS_ERR_SHAPE;
    k.tiles = (int)tiles;
    k.steps = (p.n + 255) / 256;
    k.blocks = blocks_of(p.n);
    k.pairs = k.tiles < resident ? k.tiles : resident;
    k.y = p.y; k.y_f32 = p.y_f32;
    k.status = st.status_word;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    PairVariant<BN>::fill(cfg, attr, k.pairs, stream);
    LORDS_CUDA_TRY(cudaLaunchKernelEx(&cfg, lords_mxfp4_pair_kernel<BN>, k));
    st.last_launches += 1;
    st.last_path = "mxfp4_pair";
    return LORDS_OK;
}

}  // namespace

// Microseconds of a launch with W from memory: its fixed part, and waves of tiles with a step's and a tile's own (2048 tokens, 14336 x 4096, 4096 x
// 14336, 4096 x 4096, the weight gradients of 512 and 2048 tokens; y in 32 bits leaves more slowly than the next tile's MMAs take; fewer tiles than
// pairs: 64 tokens, 1024 x 1024 4.1, 4096 x 4096 7.4).
static double pair_us(const MxProblem &p, int bn, int pairs)
{
    const double steps = (p.n + 255) / 256;
    const long long tiles = (long long)((p.M + kPTokens - 1) / kPTokens) * ((p.m + bn - 1) / bn);
    const double waves = (double)((tiles + pairs - 1) / pairs);
    if (bn == 256) return 4.7 + waves * (0.36 * steps + (p.y_f32 ? 2.0 : 0.7));
    return 2.6 + 1.4 * (double)(tiles < pairs ? tiles : pairs) / pairs + waves * (0.29 * steps + (p.y_f32 ? 0.6 : 0.42));
}

double mxfp4_pair_us(const MxProblem &p, const State &st)
{
    const int pairs = PairVariant<256>::resident(st);
    const double a = pair_us(p, 256, pairs > 0 ? pairs : 1), b = pair_us(p, 128, pairs > 0 ? pairs : 1);
    return a < b ? a : b;
}

int launch_mxfp4_pair(const MxProblem &p, State &st, cudaStream_t stream)
{
    if (p.x) return LORDS_ERR_UNSUPPORTED;
    if (st.forced_bn == 128 || st.forced_bn == 256) return st.forced_bn == 128 ? run_pair<128>(p, st, stream) : run_pair<256>(p, st, stream);
    // 256 out-features a tile read a quarter less for the same work, 128 fill the pairs better: 512 tokens, 14336 x 4096: 18.1 and 25.7 us;
    // 1024 tokens, 1024 x 4096: 9.3 and 8.4.
    const int pairs = PairVariant<256>::resident(st);
    if (pairs < 1) return LORDS_ERR_UNSUPPORTED;
    return pair_us(p, 256, pairs) <= pair_us(p, 128, pairs) ? run_pair<256>(p, st, stream) : run_pair<128>(p, st, stream);
}

}  // namespace lords

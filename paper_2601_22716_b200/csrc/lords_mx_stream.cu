// y = x W^T on microscaled 4-bit operands, for few tokens.
//
// The tensor cores take e2m1 codes and their scales as they are stored (tcgen05.mma kind::mxf4, fp32 sums), so nothing is decoded: a
// CTA streams 128 rows of W through shared memory by TMA, 256 columns a step, as the MMA's 128-row operand; the tokens are its N = BN columns.
// The scales of a step follow their codes through shared memory and from there into TMEM (tcgen05.cp), where the MMA reads them.
//
//   QX:    x arrives in bf16; warps bring it to 4 bits on the way: four of them, eight steps' slices at a time, for calls of up to four tokens;
//          sixteen, all at once, for calls of more tokens but few steps a CTA.
//   QX 0:  x arrives as codes and scales, by TMA like W.
//
// A cluster of CTAs divides a tile's steps where the row tiles alone leave SMs idle; tokens are added up four at a time, group g by CTA g mod cluster in
// distributed shared memory, in the order of the ranks, so results do not depend on timing.  No scratch memory: calls on different streams
// do not touch each other.
//
// Bound: the stream of codes and scales, 17/32 bytes a weight, behind some 2.4 us of launch, set-up and epilogue: 14336 x 4096, one token, codes given
// 7.9 us, of which the loads alone 7.5 (31 MB in 5.1 us, 6.1 TB/s); with x in bf16 8.5.  4096 x 4096: 3.4 and 4.4.  Everything is read in the
// stream's order.  (Asking L2 for the first tiles of W ahead of the previous launch's end: 8.3 -> 8.0 us, but 4.0 -> 4.15 for the smaller layer and
// 9.8 with all tiles; CTAs small enough for two on an SM 9.0: both against the kernel before its last steps.  Reading W while the launch before
// converts x, which then has to hold this one back until all before it has ended: 8 tokens 9.5 -> 10.5, 32 tokens of 4096 x 4096 5.8 -> 6.3.)
//
// Every wait is bounded; on expiry the role records LORDS_ERR_TIMEOUT and leaves its loop.
#include <cuda.h>
#include <cuda_bf16.h>

#include <atomic>

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
constexpr int kConvWarp0 = 4;                // warps from 4 on: x to 4 bits, then (the first four) the epilogue; 0: TMA, 1: MMA issuer, 2: TMEM
constexpr int kSplitMax = 8;                 // CTAs that share a tile's steps
constexpr int kStagesMax = 12;

// QX: warps that bring x to 4 bits; 0: x arrives as codes.
template <int BN, int QX> struct SCfg {
    static constexpr int CONV = QX > 4 ? QX : 4;                    // converter and epilogue warps
    static constexpr int THREADS = (kConvWarp0 + CONV) * 32;
    // most tokens x steps of a batch (four warps two blocks a thread, sixteen one); steps whose slice of x is converted together, and such batches in shared
    // memory; sixteen warps: one, of the steps that the fewest tokens of this tile may have
    static constexpr int WORK = QX == 16 ? 64 : QX * 8;
    static constexpr int BATCH = QX == 16 ? WORK / (BN == 16 ? 5 : BN / 2 + 1) : 8;
    static constexpr int BATCHES = QX == 16 ? 1 : 2;
    static constexpr int WTILE = kRows * 128;
    static constexpr int XTILE = BN * 128;
    static constexpr int SF = 2 * kTileBytes;                       // scales of a step: two tiles of four blocks
    static constexpr int XSTEP = XTILE + SF;                        // x of a step with its scales
    static constexpr int STAGE = WTILE + SF + (QX ? 0 : XSTEP);
    static constexpr int XRING = QX ? BATCHES * BATCH * XSTEP : 0;
    static constexpr int BARS = 16 * kStagesMax + 16 + 16 * BATCHES + 8;
    static constexpr int FIXED = 1024 + XRING + (BARS + 255) / 256 * 256;      // shared memory apart from stages and partial sums
    static constexpr int SMEM = 232448, SMEM_SM = 233472;
    static constexpr uint32_t ACC = BN < 32 ? 32 : BN;              // accumulator columns; behind them two sets of scales
    static constexpr uint32_t TMEM = ACC + 32 <= 64 ? 64 : ACC + 32 <= 128 ? 128 : 256;
    static_assert(STAGE % 1024 == 0 && XSTEP % 1024 == 0, "tiles begin at 1024 bytes");
};

// Tokens that are added up together, and the shared memory of a cluster's partial sums: ceil(groups / split) * split places of a group x 128 rows.
__host__ __device__ constexpr int group_of(int tokens) { return tokens > 2 ? 4 : tokens; }
__host__ __device__ constexpr int sums_bytes(int tokens, int split)
{
    const int gw = group_of(tokens), groups = (tokens + gw - 1) / gw;
    return split > 1 ? (groups + split - 1) / split * split * kRows * 4 * gw : 0;
}

struct alignas(64) StreamParams {
    CUtensorMap tm_w;        // bytes [m][pitch], box {128, 128}, 128-byte swizzle (zeros behind the last row and byte)
    CUtensorMap tm_x;        // bytes [M][pitch], box {128, BN}; not used with QX
    const uint8_t *ws;       // scale tiles of W
    const uint8_t *xs;       // scale tiles of x; not used with QX
    const uint16_t *x;       // bf16 [M][n]; QX only
    int M, m, n;
    int steps, blocks, ktiles;       // of a row: steps of 256 columns, blocks, scale tiles
    int stages;              // of the ring: what the partial sums leave room for, and no more than a CTA has steps
    void *y;
    int y_f32;
    int *status;
};

// One, two or four sums of a row, asynchronously to a CTA of the cluster; counted in bytes on its barrier.
template <int GW> __device__ __forceinline__ void send(uint32_t addr, const uint32_t *v, uint32_t bar)
{
    if constexpr (GW == 1)
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(addr), "r"(v[0]), "r"(bar) : "memory");
    else if constexpr (GW == 2)
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(bar) : "memory");
    else
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]),
                     "r"(v[3]), "r"(bar) : "memory");
}

__device__ __forceinline__ void put(float *at, float v) { *at = v; }
__device__ __forceinline__ void put(__nv_bfloat16 *at, float v) { *at = __float2bfloat16_rn(v); }

// The epilogue's four warps have taken the sums from TMEM, and the issuer has issued its last MMA: the warp that allocated TMEM may return it.  Returns
// whether any of them waited for the MMAs in vain, which may then still be at work.
__device__ __forceinline__ bool sums_read(bool in_vain)
{
    __syncwarp();
    tc_fence_before_sync();
    uint32_t any;
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.u32 p, %1, 0;\n"
        "bar.red.or.pred q, 1, 192, p;\n"
        "selp.u32 %0, 1, 0, q;\n"
        "}\n"
        : "=r"(any)
        : "r"((uint32_t)in_vain)
        : "memory");
    return any != 0u;
}

// The sums of a row (y: where its value of token 0 goes, `inside`: it is a row of W) as the one CTA of a tile has them.
template <class T> __device__ __forceinline__ void write_out(uint32_t acc, int tokens, T *y, int m, bool inside)
{
    const size_t pitch = (size_t)m;
#pragma unroll 1
    for (int c0 = 0; c0 < tokens; c0 += 16, y += 16 * pitch) {
        uint32_t v[16];
        tmem_ld_32x16(acc + (uint32_t)c0, v);
        tmem_wait_ld(v);
        const int left = inside ? tokens - c0 : 0;
        T *at = y;
#pragma unroll
        for (int c = 0; c < 16; ++c, at += pitch)
            if (c < left) put(at, __uint_as_float(v[c]));
    }
}

// The cluster's sums: tokens in groups of GW, group g to rank g mod cluster; a received value's place is (group / cluster, rank, row).
// (64 tokens of 1024 x 1024 on two CTAs 4.1 us, 3.3 on one.  Level or slower: the tokens on eight warps, all ranks' values loaded at once; by copies in bulk from
// shared memory, with a wait for them at the end, 4.45.)
template <int GW, class T>
__device__ __forceinline__ bool add_up(uint32_t acc, uint32_t recv, uint32_t bar_recv, int rank, int split, int tokens, T *y, int m, bool inside, int ri,
                                       const int *status, bool failed)
{
    constexpr uint32_t PLACE = kRows * 4 * GW;
    const int groups = (tokens + GW - 1) / GW;
    const uint32_t row_at = recv + (uint32_t)(ri * 4 * GW);
    int to = 0;
    uint32_t where = row_at + (uint32_t)rank * PLACE;
#pragma unroll 1
    for (int c0 = 0; c0 < tokens; c0 += 16) {
        uint32_t v[16];
        if (!failed) {
            tmem_ld_32x16(acc + (uint32_t)c0, v);
            tmem_wait_ld(v);
        } else {                       // MMAs may still write them: the others get zeros, so that their waits end
#pragma unroll
            for (int c = 0; c < 16; ++c) v[c] = 0u;
        }
#pragma unroll
        for (int c = 0; c < 16 && (GW == 4 || c == 0); c += GW) {
            if (c0 + c >= tokens) break;
            if (to == rank) {
                if constexpr (GW == 4) {
                    sts_v4(where, make_uint4(v[c], v[c + 1], v[c + 2], v[c + 3]));
                } else {
#pragma unroll
                    for (int k = 0; k < GW; ++k) sts_u32(where + 4 * k, v[c + k]);
                }
            } else {
                send<GW>(map_to_rank(where, (uint32_t)to), v + c, map_to_rank(bar_recv, (uint32_t)to));
            }
            if (++to == split) { to = 0; where += (uint32_t)split * PLACE; }
        }
    }
    sums_read(failed);
    if (rank >= groups) return true;
    if (!__all_sync(0xffffffffu, mbar_wait_cluster(bar_recv, 0, status, 65))) return false;
    if (failed) return true;
    const size_t pitch = (size_t)m;
    uint32_t from = row_at;
    y += (size_t)(rank * GW) * pitch;
    for (int g = rank; g < groups; g += split, y += (size_t)(split * GW) * pitch) {
        float sum[GW];
#pragma unroll
        for (int k = 0; k < GW; ++k) sum[k] = 0.0f;
#pragma unroll 4
        for (int r = 0; r < split; ++r, from += PLACE) {
            if constexpr (GW == 4) {
                const uint4 u = lds_v4(from);
                sum[0] += __uint_as_float(u.x); sum[1] += __uint_as_float(u.y); sum[2] += __uint_as_float(u.z); sum[3] += __uint_as_float(u.w);
            } else {
#pragma unroll
                for (int k = 0; k < GW; ++k) sum[k] += __uint_as_float(lds_u32(from + 4 * k));
            }
        }
        const int left = inside ? tokens - g * GW : 0;
        T *at = y;
#pragma unroll
        for (int k = 0; k < GW; ++k, at += pitch)
            if (k < left) put(at, sum[k]);
    }
    return true;
}

template <int BN, int QX>
__global__ void __launch_bounds__(SCfg<BN, QX>::THREADS, 1) lords_mxfp4_stream_kernel(const __grid_constant__ StreamParams p)
{
    using C = SCfg<BN, QX>;
    constexpr int kBatch = C::BATCH, kBatches = C::BATCHES;
    const int stages = p.stages;
    extern __shared__ uint8_t s_smem[];
    const uint32_t base = (smem_u32(s_smem) + 1023u) & ~1023u;
    const uint32_t xring = base + (uint32_t)(stages * C::STAGE), bars = xring + C::XRING, recv = bars + (C::BARS + 255) / 256 * 256;
    const uint32_t bar_full = bars, bar_empty = bar_full + 8 * kStagesMax, bar_acc = bar_empty + 8 * kStagesMax, bar_recv = bar_acc + 8;
    const uint32_t bar_x = bar_recv + 8, bar_x_free = bar_x + 8 * kBatches, tmem_slot = bar_x_free + 8 * kBatches;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster_ctarank(), split = (int)cluster_nctarank();
    const int rt = (int)(blockIdx.x / split), row0 = rt * kRows, tok0 = (int)blockIdx.y * BN;
    const int s_a = (int)((long long)p.steps * rank / split), s_b = (int)((long long)p.steps * (rank + 1) / split);
    const int tokens = p.M - tok0 < BN ? p.M - tok0 : BN;
    const int gw = group_of(tokens);
    const int *status = p.status;
    bool failed = false, alone = false;

    if (warp == 0) {
        if (lane == 0) {
            for (int s = 0; s < stages; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
            mbar_init(bar_acc, 1);
            mbar_init(bar_recv, 1);
            for (int s = 0; s < kBatches; ++s) { mbar_init(bar_x + 8 * s, C::CONV); mbar_init(bar_x_free + 8 * s, 1); }
            fence_mbar_init();
            const int groups = (tokens + gw - 1) / gw, own = groups > rank ? (groups - rank + split - 1) / split : 0;
            if (split > 1) mbar_expect_tx(bar_recv, (uint32_t)((split - 1) * own * kRows * 4 * gw));
            tma_prefetch_desc(&p.tm_w);
            if (!QX) tma_prefetch_desc(&p.tm_x);
        }
        __syncwarp();
    }
    // No CTA waits for another of its cluster while it holds TMEM: beside clusters of another stream that do the same each could hold what the other waits
    // for.  So it says that its barriers exist before it asks for TMEM, and returns that before it waits for the others' sums.
    if (split > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // waited for before the first store to another CTA
    if (warp == 2) {
        tmem_alloc(tmem_slot, C::TMEM);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    uint32_t tmem_base;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem_base) : "r"(tmem_slot));
    griddep_launch_dependents();
    griddep_wait();

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA: codes and scales of W, and of x.  (Under lane == 0; under elect.sync, which
        // the kernel on pairs gains by, 14336 x 4096 with the codes given took 8.3 us in place of 8.0.)
        if (lane == 0) {
            int s = 0;
            uint32_t phase = 1;                // of the empties: the first time around nothing is waited for
            for (int st = s_a; st < s_b; ++st, s = s + 1 == stages ? 0 : s + 1) {
                if (s == 0) phase ^= 1u;
                if (st - s_a >= stages && !mbar_wait(bar_empty + 8 * s, phase ^ 1u, status, 61)) { failed = true; break; }
                const uint32_t dst = base + (uint32_t)(s * C::STAGE), bar = bar_full + 8 * s;
                const int kt = p.ktiles - 2 * st < 2 ? 1 : 2;
                mbar_expect_tx(bar, (uint32_t)(C::WTILE + kt * kTileBytes + (QX ? 0 : C::XTILE + kt * kTileBytes)));
                tma_load_2d(dst, &p.tm_w, st * 128, row0, bar);
                load_words(dst + C::WTILE, p.ws + ((size_t)rt * p.ktiles + 2 * st) * kTileBytes, (uint32_t)(kt * kTileBytes), bar);
                if (!QX) {
                    tma_load_2d(dst + C::WTILE + C::SF, &p.tm_x, st * 128, tok0, bar);
                    load_words(dst + C::WTILE + C::SF + C::XTILE, p.xs + ((size_t)(tok0 / kTileRows) * p.ktiles + 2 * st) * kTileBytes, (uint32_t)(kt * kTileBytes), bar);
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        const uint32_t hi = (uint32_t)(umma_desc_sw128(0, 1024, 16) >> 32), lo0 = (uint32_t)umma_desc_sw128(0, 1024, 16);
        const uint32_t tmem_u = warp_uniform(tmem_base), leader = elect_one();
        int it = 0, s = 0;
        uint32_t phase = 1;
        for (int st = s_a; st < s_b; ++st, ++it, s = s + 1 == stages ? 0 : s + 1) {
            if (s == 0) phase ^= 1u;
            const int batch = it / kBatch;
            if (QX && it % kBatch == 0 && !mbar_wait_warp(bar_x + 8 * (batch % kBatches), (uint32_t)((batch / kBatches) & 1), status, 66)) { failed = true; break; }
            if (!mbar_wait_warp(bar_full + 8 * s, phase, status, 62)) { failed = true; break; }
            tc_fence_after_sync();
            const uint32_t at = base + (uint32_t)(s * C::STAGE), sw = at + C::WTILE;
            const uint32_t xt = QX ? xring + (uint32_t)(it % (kBatch * kBatches) * C::XSTEP) : sw + C::SF, sx = xt + C::XTILE;
            const uint32_t a_lo = lo0 | ((at & 0x3FFFFu) >> 4), b_lo = lo0 | ((xt & 0x3FFFFu) >> 4);
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
                                 cx + 4 * (k >> 1), (it > 0 || k > 0) ? 1u : 0u, leader);
            umma_commit(bar_empty + 8 * s, leader);
            if (QX && it % kBatch == kBatch - 1) umma_commit(bar_x_free + 8 * (batch % kBatches), leader);
        }
        umma_commit(bar_acc, leader);
        sums_read(false);
    } else if (warp >= kConvWarp0) {
        if constexpr (QX > 0) {
            // -------------------------------------------------------------- x to 4 bits, a block at a time, a batch of steps after the other.  (Tokens
            // from M on are columns of the product that nobody reads: whatever their shared memory holds.)
            // A batch is at most WORK tokens x steps of eight blocks, two blocks a thread (a quarter of a block: one token 5.8 us at 4096 x 4096 and 9.1 at
            // 14336 x 4096, 4.5 and 8.9 so): block e is block e % (8 count) of token e / (8 count).  The next batch's
            // loads are on their way while this one is converted.
            constexpr int PER = C::WORK * 8 / (C::CONV * 32);
            const int steps = s_b - s_a, id = tid - kConvWarp0 * 32;
            auto place = [&](int first, int h, int &t, int &kb) {
                const int count = steps - first < kBatch ? steps - first : kBatch, e = id + h * C::CONV * 32;
                t = count == kBatch ? e / (8 * kBatch) : e / (8 * count);
                kb = e - t * 8 * count;
                return t < p.M;
            };
            auto load_batch = [&](int first, uint32_t (&w)[PER][16]) {
#pragma unroll
                for (int h = 0; h < PER; ++h) {
                    int t, kb;
#pragma unroll
                    for (int k = 0; k < 16; ++k) w[h][k] = 0u;
                    if (first >= steps || !place(first, h, t, kb)) continue;
                    const int c = (s_a + first) * kStep + kb * kBlock;
                    if (c < p.n) load_values<16>(p.x + (size_t)t * p.n, p.n, c, p.x + (size_t)p.M * p.n, w[h]);
                }
            };
            uint32_t w[PER][16], next[PER][16];
            load_batch(0, w);
            for (int first = 0; first < steps && !failed; first += kBatch) {
                const int batch = first / kBatch;
                if constexpr (kBatches > 1) load_batch(first + kBatch, next);
                if (batch >= kBatches && !mbar_wait_warp(bar_x_free + 8 * (batch % kBatches), (uint32_t)((batch / kBatches - 1) & 1), status, 63)) { failed = true; break; }
                const uint32_t to = xring + (uint32_t)((batch % kBatches) * kBatch * C::XSTEP);
#pragma unroll
                for (int h = 0; h < PER; ++h) {
                    int t, kb;
                    if (!place(first, h, t, kb)) break;
                    uint32_t top = magnitudes(w[h][0]), out[4];
#pragma unroll
                    for (int k = 1; k < 15; k += 2) top = larger(top, magnitudes(w[h][k]), magnitudes(w[h][k + 1]));
                    top = larger(top, magnitudes(w[h][15]));
                    const uint32_t byte = scale_byte<2>(larger_half(top));
#pragma unroll
                    for (int g = 0; g < 4; ++g) out[g] = to_codes4(w[h] + 4 * g, byte);
                    const int b = kb & 7;
                    const uint32_t at = to + (uint32_t)((kb >> 3) * C::XSTEP);
                    sts_v4(at + (uint32_t)(t * 128 + ((b ^ (t & 7)) << 4)), make_uint4(out[0], out[1], out[2], out[3]));
                    asm volatile("st.shared.u8 [%0], %1;" ::"r"(at + C::XTILE + (uint32_t)(b / kTileBlocks * kTileBytes + scale_at(t, b % kTileBlocks))), "r"(byte)
                                 : "memory");
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_x + 8 * (batch % kBatches));
#pragma unroll
                for (int h = 0; h < PER; ++h)
#pragma unroll
                    for (int k = 0; k < 16; ++k) w[h][k] = next[h][k];
            }
        }
        // ------------------------------------------------------------------ epilogue: lane = row of W, columns = tokens
        if (split > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        const int q = warp & 3;
        if (warp < kConvWarp0 + 4) {
            if (!mbar_wait_warp(bar_acc, 0, status, 64)) failed = true;
            tc_fence_after_sync();
            const int ri = q * 32 + lane, i = row0 + ri;
            const uint32_t acc = tmem_base + ((uint32_t)(q * 32) << 16);
            auto out = [&](auto *base) {
                auto *y = base + (size_t)tok0 * p.m + i;
                if (split <= 1) {
                    if (!failed) write_out(acc, tokens, y, p.m, i < p.m);
                    sums_read(failed);
                    return;
                }
                const bool ok = gw == 4   ? add_up<4>(acc, recv, bar_recv, rank, split, tokens, y, p.m, i < p.m, ri, status, failed)
                                : gw == 2 ? add_up<2>(acc, recv, bar_recv, rank, split, tokens, y, p.m, i < p.m, ri, status, failed)
                                          : add_up<1>(acc, recv, bar_recv, rank, split, tokens, y, p.m, i < p.m, ri, status, failed);
                alone = !ok;
                failed = failed || alone;
            };
            if (p.y_f32) out(static_cast<float *>(p.y));
            else out(static_cast<__nv_bfloat16 *>(p.y));
        }
    }
    if (warp == 2) {
        // (After a wait in vain the MMAs end soon after the last one has been issued.  A wait in every call: 256 x 256, four tokens 0.1 us more.)
        if (sums_read(false) && !mbar_wait_warp(bar_acc, 0, status, 67)) failed = true;
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, C::TMEM);
    }
    if (split > 1 && warp < kConvWarp0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (failed) {
        ptx::record_give_up(p.status, LORDS_ERR_TIMEOUT);
        // A CTA whose wait for the others' sums gave up holds its shared memory until they have stored theirs, or have left: a thread that has exited counts
        // as arrived, and the waits of the others are bounded.
        if (alone) {
            asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        }
    }
}

template <int BN, int QX> struct StreamVariant {
    using C = SCfg<BN, QX>;
    static void fill(cudaLaunchConfig_t &cfg, cudaLaunchAttribute *attr, int row_tiles, int tok_tiles, int split, cudaStream_t stream)
    {
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)split;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg = cudaLaunchConfig_t{};
        cfg.gridDim = dim3((unsigned)(row_tiles * split), (unsigned)tok_tiles);
        cfg.blockDim = dim3(SCfg<BN, QX>::THREADS);
        cfg.dynamicSmemBytes = C::SMEM;
        cfg.stream = stream;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
    }
    // The kernel may use its shared memory, once per device.
    static cudaError_t allow(const State &st)
    {
        static std::atomic<bool> done[kMaxDevices];
        std::atomic<bool> &d = done[device_slot(st)];
        if (d.load(std::memory_order_acquire)) return cudaSuccess;
        const cudaError_t e = cudaFuncSetAttribute(lords_mxfp4_stream_kernel<BN, QX>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
        if (e == cudaSuccess) d.store(true, std::memory_order_release);
        return e;
    }
    // Clusters of `split` CTAs that can be resident at once.  (Host threads may ask at the same time: each stores the answer, and nothing before it.)
    static int resident(int split, const State &st)
    {
        static std::atomic<int> cache[kMaxDevices][kSplitMax + 1];      // 0: not asked yet, -1: none
        std::atomic<int> &c = cache[device_slot(st)][split];
        int known = c.load(std::memory_order_relaxed);
        if (known == 0) {
            cudaLaunchConfig_t cfg;
            cudaLaunchAttribute attr[2];
            fill(cfg, attr, 1, 1, split, nullptr);
            int n = 0;
            if (allow(st) != cudaSuccess || cudaOccupancyMaxActiveClusters(&n, lords_mxfp4_stream_kernel<BN, QX>, &cfg) != cudaSuccess) {
                (void)cudaGetLastError();
                return 0;
            }
            known = n >= 1 ? n : -1;
            c.store(known, std::memory_order_relaxed);
        }
        return known > 0 ? known : 0;
    }
    // CTAs that share a tile's steps: the least waves x (steps of a CTA + a fixed part worth four + what joining the sums takes, a step and a twentieth for
    // every token).  64 tokens, 1024 x 1024: 3.3 us on one CTA, 4.1 on two; 1024 x 2048 4.4 and on four 3.9; 128 tokens, 4096 x 1024 4.1 and on two
    // 5.9.  Up to 32 tokens without that last part, so that more layers have few enough steps a CTA to take x in bf16: 32 tokens, 4096 x 1024 4.44 us,
    // 4.61 with it.  With the codes given it changes nothing: forty products of 1 to 32 tokens, 1024 x 1024 to 14336 x 4096, within 2 % either way.
    static int choose_split(int tiles, int steps, int tokens, const State &st)
    {
        const int joining = tokens > 32 ? 20 + tokens : 0;
        int best = 0;
        long long least = 0;
        for (int c = 1; c <= kSplitMax && (c == 1 || 2 * c <= steps); ++c) {
            const int n = resident(c, st);
            if (n < 1) continue;
            const long long t = (long long)((tiles + n - 1) / n) * (20 * ((steps + c - 1) / c + 4) + (c > 1 ? joining : 0));
            if (best == 0 || t < least) { best = c; least = t; }
        }
        return best;
    }
    static int launch(StreamParams &k, const State &st, cudaStream_t stream)
    {
        const int row_tiles = (k.m + kRows - 1) / kRows, tok_tiles = (k.M + BN - 1) / BN;
        // (the same for every kind of x: sums are in the same order then)
        const int split = StreamVariant<BN, 0>::choose_split(row_tiles * tok_tiles, k.steps, k.M < BN ? k.M : BN, st);
        if (split < 1) return LORDS_ERR_UNSUPPORTED;
        if (tok_tiles > 65535) return LORDS_ERR_SHAPE;
        const int own = (k.steps + split - 1) / split;
        const int sums = sums_bytes(k.M < BN ? k.M : BN, split), room = (C::SMEM - C::FIXED - sums) / C::STAGE;
        k.stages = room < own ? room : own;
        // (with x in bf16, more loads of W in flight hold up those of x: 14336 x 4096, one token 9.1 us with five to seven stages, 9.7 with twelve, 9.5 with four)
        constexpr int most = QX > 0 ? 6 : kStagesMax;
        if (k.stages > most) k.stages = most;
        // More tiles than are resident: two CTAs to an SM, so that one's set-up and epilogue run beside the other's loads (28672 x 4096, one token 16.2 us
        // on one, 13.3 so; 65536 x 4096 33.8 and 26.7; 32000 x 1024, 128 tokens 9.0 and 5.9).
        if (row_tiles * tok_tiles > StreamVariant<BN, 0>::resident(split, st)) {
            const int two = (C::SMEM_SM / 2 - 1024 - C::FIXED - sums) / C::STAGE;
            if (two >= 2 && k.stages > two) k.stages = two;
        }
        if (QX > 0 && k.M * (QX == 4 && own > C::BATCH ? C::BATCH : own) > C::WORK) return LORDS_ERR_UNSUPPORTED;
        cudaLaunchConfig_t cfg;
        cudaLaunchAttribute attr[2];
        fill(cfg, attr, row_tiles, tok_tiles, split, stream);
        cfg.dynamicSmemBytes = (size_t)(C::FIXED + sums + k.stages * C::STAGE);
        LORDS_CUDA_TRY(allow(st));
        LORDS_CUDA_TRY(cudaLaunchKernelEx(&cfg, lords_mxfp4_stream_kernel<BN, QX>, k));
        return LORDS_OK;
    }
};

template <int BN> double stream_us(const MxProblem &p, const State &st)
{
    const int steps = (p.n + kStep - 1) / kStep, tiles = (p.m + kRows - 1) / kRows * ((p.M + BN - 1) / BN);
    const int tokens = p.M < BN ? p.M : BN, split = StreamVariant<BN, 0>::choose_split(tiles, steps, tokens, st);
    const int n = split > 0 ? StreamVariant<BN, 0>::resident(split, st) : 0;
    if (n < 1) return 1e30;
    // W from memory at 5.4 TB/s or the busiest SM's MMAs; set-up and epilogue of each round (two CTAs an SM if one is not enough), more of it with sums to be
    // joined; the launch
    const double waves = (double)((tiles + n - 1) / n), rounds = tiles > n ? (double)((tiles + 2 * n - 1) / (2 * n)) : 1.0;
    const double load = 0.0032 * steps * ((p.m + kRows - 1) / kRows), mma = waves * ((steps + split - 1) / split) * (BN <= 64 ? 0.29 : 0.33);
    return (load > mma ? load : mma) + rounds * (split > 1 ? 2.7 + 0.021 * tokens : 2.5 + 0.007 * tokens) - 0.75;
}

int tile_for(int M) { return M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : 128; }

}  // namespace

// Estimate in microseconds with x in 4 bits, fitted to some twenty layers at 4 to 512 tokens (within 10 % on nearly all, 15 % at worst).
double mxfp4_stream_us(const MxProblem &p, const State &st)
{
    switch (tile_for(p.M)) {
        case 16: return stream_us<16>(p, st);
        case 32: return stream_us<32>(p, st);
        case 64: return stream_us<64>(p, st);
        default: return stream_us<128>(p, st);
    }
}

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
    const int bn = tile_for(p.M);
    if (qx && bn > 64) return LORDS_ERR_UNSUPPORTED;
    const uint64_t pitch = (uint64_t)codes_pitch(p.n);
    if (!make_map_2d(&k.tm_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.w, pitch, (uint64_t)p.m, 128, kRows, CU_TENSOR_MAP_SWIZZLE_128B)) return LORDS_ERR_CUDA;
    if (qx) k.tm_x = k.tm_w;
    else if (!make_map_2d(&k.tm_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.xq, pitch, (uint64_t)p.M, 128, (uint32_t)bn, CU_TENSOR_MAP_SWIZZLE_128B)) return LORDS_ERR_CUDA;
    int rc;
    // x in bf16: up to four tokens four converter warps.  Up to 64 tokens sixteen warps, where a CTA has few steps (64 tokens x steps, a block a thread): every
    // row tile converts x again and reads it in 16 bits.  4096 x 4096, 16 tokens of four steps: 5.7 us, with eight warps 5.8, with two launches
    // 5.6; 1024 x 4096, 32 tokens of two steps 4.9, with two launches 5.4.  With twice as many blocks a thread, 4096 x 4096, 32 tokens of
    // four steps takes 7.5 us, 6.3 with two launches.  A call from the host takes 2 us more for two launches (5.7 and 7.9).
    if (qx && p.M <= 4) rc = StreamVariant<16, 4>::launch(k, st, stream);
    else if (qx && bn == 16) rc = StreamVariant<16, 16>::launch(k, st, stream);
    else if (qx && bn == 32) rc = StreamVariant<32, 16>::launch(k, st, stream);
    else if (qx) rc = StreamVariant<64, 16>::launch(k, st, stream);
    else if (bn == 16) rc = StreamVariant<16, 0>::launch(k, st, stream);
    else if (bn == 32) rc = StreamVariant<32, 0>::launch(k, st, stream);
    else if (bn == 64) rc = StreamVariant<64, 0>::launch(k, st, stream);
    else rc = StreamVariant<128, 0>::launch(k, st, stream);
    if (rc != LORDS_OK) return rc;
    st.last_launches += 1;
    st.last_path = "mxfp4_stream";
    return LORDS_OK;
}

}  // namespace lords

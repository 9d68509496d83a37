// Matrix products of the layer operators on the fifth-generation tensor cores (tcgen05).
#include "ssd_layers.cuh"
#include "ssd_tile.cuh"

#include <cmath>

namespace ssd_layers {

struct Maps {
    CUtensorMap a, b[2];
};

namespace {

// The contraction of a tile is a list of 64-wide steps, segment after segment.  The tensor cores add to a float32 accumulator
// without rounding to nearest: every addition cuts towards zero, a bias of up to half a unit in the last place each that all terms share (measured:
// 6.7e-6 of the result after 2816 x 2 products).  A bfloat16 result does not see that.  For a float32 result
// (DRAIN) the leading terms are therefore summed in runs of kRunSteps steps, each from zero in one of two accumulators, and
// the epilogue's warps add the runs in registers, rounded to nearest, while the next run is on its way.

// End of the run that starts at step `it`: all smaller segments make one run.
template <bool DRAIN> __device__ __forceinline__ int run_end(int it, int small, int end)
{
    if (!DRAIN) return end;
    const int e = it < small ? small : it + kRunSteps;
    return e < end ? e : end;
}

// ---------------------------------------------------------------------------------------------------------
// tile_kernel: one 128 x BN tile of the result per cluster of `split` blocks, which share its contraction.
//
// In every block one thread streams 64-wide slices of both operands into a ring of shared-memory stages by TMA, one thread issues
// tcgen05.mma into float32 accumulators in tensor memory, and four warps take the result out.  The blocks of a cluster put their partial
// tiles into shared memory and each adds up its share of the rows over the cluster, in rank order, so the bits do not depend
// on timing and no partial sum goes through HBM.
// What bounds it is the way into shared memory: 24 KB a step where the products take 256 cycles, and few tiles to hide a start behind.  It is
// for products too small for pair_kernel: 128 x 4096 x 4096 12.0 us (W comes in at 2.8 TB/s),
// 16 x 1024 x 1024 5.8, 64 x 4096 x 25088 41 (5 TB/s).
// Rows of the tile beyond the operands hold whatever was in shared memory: they are never stored.
template <int BN, int STAGES> struct TileShape {
    static constexpr int a_bytes = kBlockM * kBlockK * 2, b_bytes = BN * kBlockK * 2;
    static constexpr int stage_bytes = a_bytes + b_bytes;
    static constexpr int ring_bytes = STAGES * stage_bytes;
    static constexpr int tile_bytes = kBlockM * kTilePitch<BN> * 4;
    static constexpr int body = ring_bytes > tile_bytes ? ring_bytes : tile_bytes;
    static constexpr int bytes = body + 1024;                          // room to align the ring to 1024
};

constexpr int kTileThreads = 192;

template <int BN, int STAGES, bool AMN, bool BMN, bool GATED, bool DRAIN>
__global__ void __launch_bounds__(kTileThreads) tile_kernel(const __grid_constant__ Product p, const __grid_constant__ Maps maps, int split, int a_rows)
{
    using S = TileShape<BN, STAGES>;
    constexpr int kBuffers = DRAIN ? 2 : 1;
    extern __shared__ unsigned char raw[];
    __shared__ uint64_t full[STAGES], empty[STAGES], sum_full[kBuffers], sum_empty[kBuffers];
    __shared__ uint32_t tmem_at;
    const uint32_t ring = (s32(raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = split > 1 ? int(cluster_rank()) : 0;
    constexpr int kOutCols = GATED ? BN / 2 : BN;                      // columns of the result in a tile
    const int tiles_n = (p.n + kOutCols - 1) / kOutCols, at_tile = int(blockIdx.x / split);
    const int n0 = at_tile % tiles_n * kOutCols, m0 = at_tile / tiles_n * kBlockM, group = blockIdx.y;
    const int kblocks = (p.k + kBlockK - 1) / kBlockK;
    const int total = kblocks * p.nseg, small = total - kblocks * p.nmain;
    const int it0 = int(int64_t(total) * rank / split), it1 = int(int64_t(total) * (rank + 1) / split);

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            bar_init(&full[s], 1);
            bar_init(&empty[s], 1);
        }
        for (int s = 0; s < kBuffers; ++s) {
            bar_init(&sum_full[s], 1);
            bar_init(&sum_empty[s], 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<1, kBuffers * BN>(&tmem_at);
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    dependents_may_start();
    wait_for_previous();
    const uint32_t tmem = tmem_at;

    if (warp == 0 && elected()) {
        const uint32_t bytes = (AMN ? S::a_bytes : a_rows * kBlockK * 2) + S::b_bytes;
        int seg = it0 / kblocks, kb = it0 % kblocks, i = 0;
        bool ok = true;
        for (Ring<STAGES> at; ok && i < it1 - it0; ++seg, kb = 0) {
            const Segment sg = p.seg[seg];
            const int az = sg.az + group, bz = sg.bz;
            const CUtensorMap *mb = &maps.b[sg.b];
            const int left = it1 - it0 - i, end = left < kblocks - kb ? kb + left : kblocks;
            for (; kb < end; ++kb, ++i, at.next()) {
                if (i >= STAGES && !(ok = bar_wait(&empty[at.stage], at.phase ^ 1))) break;
                uint64_t *bar = &full[at.stage];
                bar_expect(bar, bytes);
                const uint32_t a = ring + at.stage * S::stage_bytes, b = a + S::a_bytes;
                const int k = kb * kBlockK;
                if (AMN) {
                    for (int j = 0; j < kBlockM / 64; ++j) tma_load(a + j * 8192, &maps.a, m0 + 64 * j, k, az, bar);
                } else {
                    tma_load(a, &maps.a, k, m0, az, bar);
                }
                if (BMN) {
                    for (int j = 0; j < BN / 64; ++j) tma_load(b + j * 8192, mb, n0 + 64 * j, k, bz, bar);
                } else if (GATED) {
                    tma_load(b, &maps.b[0], k, n0, bz, bar);
                    tma_load(b + S::b_bytes / 2, &maps.b[1], k, n0, bz, bar);
                } else {
                    tma_load(b, mb, k, n0, bz, bar);
                }
            }
        }
        // nothing may still be on its way into this block's memory when it ends
        for (int j = i > STAGES ? i - STAGES : 0; j < i; ++j)
            if (!bar_wait(&full[j % STAGES], (j / STAGES) & 1)) break;
    } else if (warp == 1 && elected()) {
        constexpr uint32_t kind = mma_kind(kBlockM, BN, AMN, BMN);
        const uint64_t a0 = smem_operand(ring, AMN ? 8192 : 16, 1024), b0 = smem_operand(ring + S::a_bytes, BMN ? 8192 : 16, 1024);
        bool ok = true;
        Ring<STAGES> at;
        int run = 0;
        for (int it = it0; ok && it < it1; ++run) {
            const int buf = run % kBuffers, end = run_end<DRAIN>(it, small, it1);
            if (run >= kBuffers && !(ok = bar_wait(&sum_empty[buf], (run / kBuffers - 1) & 1))) break;
            tmem_after_sync();
            const uint32_t d = tmem + buf * BN;
            for (bool add = false; it < end; ++it, at.next()) {
                if (!(ok = bar_wait(&full[at.stage], at.phase))) break;
                tmem_after_sync();
                const uint64_t da = a0 + at.stage * (S::stage_bytes / 16), db = b0 + at.stage * (S::stage_bytes / 16);
#pragma unroll
                for (int k = 0; k < kBlockK / 16; ++k) {    // 16 of the contraction: 32 bytes along a row, or 16 rows of 128 bytes
                    mma_bf16<1>(d, da + k * (AMN ? 2048 / 16 : 2), db + k * (BMN ? 2048 / 16 : 2), kind, add);
                    add = true;
                }
                mma_commit<1>(&empty[at.stage]);
            }
            mma_commit<1>(&sum_full[buf]);
        }
    }
    __syncwarp();
    if (warp >= 2) {
        const int quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t at = tmem + (uint32_t(quarter * 32) << 16);
        if (DRAIN) {
            float acc[BN];
#pragma unroll
            for (int j = 0; j < BN; ++j) acc[j] = 0.0f;
            int run = 0;
            for (int it = it0; it < it1; ++run) {
                const int buf = run % kBuffers;
                const bool ok = bar_wait(&sum_full[buf], (run / kBuffers) & 1);
                __syncwarp();
                if (!ok) break;
                tmem_after_sync();
#pragma unroll
                for (int c = 0; c < BN; c += 32) {
                    float v[32];
                    tmem_load32(at + buf * BN + c, v);
#pragma unroll
                    for (int j = 0; j < 32; ++j) acc[c + j] += v[j];
                }
                tmem_before_sync();
                __syncwarp();
                if (lane == 0) bar_arrive(&sum_empty[buf]);
                it = run_end<DRAIN>(it, small, it1);
            }
            // the ring is free: the last run's products are done
#pragma unroll
            for (int c = 0; c < BN; c += 32) {
                float v[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = acc[c + j];
                put_row<BN>(ring, row, c, v);
            }
        } else {
            bar_wait(&sum_full[0], 0);
            __syncwarp();
            tmem_after_sync();
#pragma unroll 1
            for (int c = 0; c < BN; c += 32) {
                float v[32];
                tmem_load32(at + c, v);
                put_row<BN>(ring, row, c, v);
            }
        }
    }
    tmem_before_sync();
    if (split > 1) {
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }
    tmem_after_sync();
    if (warp == 1) tmem_free<1, kBuffers * BN>(tmem);

    if (p.e.vec) join_rows<GATED, DRAIN, BN, kTileThreads / 32, true>(p, group, m0, n0, ring, split, rank);
    else join_rows<GATED, DRAIN, BN, kTileThreads / 32, false>(p, group, m0, n0, ring, split, rank);
    if (split > 1) {      // the others may still be reading this block's part
        cluster_arrive();
        cluster_wait();
    }
}

// ---------------------------------------------------------------------------------------------------------
// pair_kernel: 256 x BN tiles by pairs of blocks, BN = 256 or 128.
//
// The two blocks of a pair (one SM each) hold 128 rows of A and BN / 2 of B a stage, and the even block issues
// tcgen05.mma over both: each SM's share of a 256 x 256 x 64 step reads 32 KB where a block alone would read 48 KB for 128 x 256.
// split == 1: a pair works through its tiles without stopping; while the eight epilogue warps take a tile out of one
// accumulator, the products of the next one go to the other.  Tiles are walked in bands of kBand rows of tiles, so that the pairs at work
// share rows of A and B in L2.
// Inside a round the tensor pipe is the bound (72 % of the elapsed time at 4096^3, where 256 tiles make 3.46 rounds of 74): 4096^3 95 us, 1.45 PFLOP/s, in
// bursts; gated 8192 x 4096 x 8192 with gate and up kept 706 us, 1.56 PFLOP/s, in bursts and 850 when it runs for long under the power limit.
// split > 1, for few tiles with a long contraction: a pair's work is a slice of a tile's contraction, whose sums go to `partial`,
// and join_kernel adds the slices up in their order.  (Joining over clusters of pairs instead cost a fixed 10 us and left SMs idle: 33
// clusters of 4 such blocks fit, 15 of 8.)
constexpr int kPairThreads = 64 + 256;
constexpr int kPairM = 256, kBand = 8;

template <int BN, bool GATED> struct PairShape {
    static constexpr int a_bytes = 128 * kBlockK * 2, b_bytes = BN / 2 * kBlockK * 2;     // a block's rows of A and of B
    static constexpr int stage_bytes = a_bytes + b_bytes;
    static constexpr int pitch = 33;
    static constexpr int stage_words = 32 * pitch * (GATED ? 2 : 1);   // a warp's transposition buffer
    static constexpr int stages = BN == 256 ? (GATED ? 4 : 6) : (GATED ? 6 : 8);
    static constexpr int ring_bytes = stages * stage_bytes;
    static constexpr int bytes = ring_bytes + 8 * stage_words * 4 + 1024;
};

template <int BN, bool AMN, bool BMN, bool GATED, bool DRAIN>
__global__ void __launch_bounds__(kPairThreads, 1) pair_kernel(const __grid_constant__ Product p, const __grid_constant__ Maps maps, int split, float *partial)
{
    using S = PairShape<BN, GATED>;
    constexpr int STAGES = S::stages;
    constexpr int kBlocks = BN / 64;                                   // blocks of 32 columns that an epilogue warp takes out
    extern __shared__ unsigned char raw[];
    __shared__ uint64_t full[STAGES], empty[STAGES], sum_full[2], sum_empty[2];
    __shared__ uint32_t tmem_at;
    const uint32_t ring = (s32(raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = int(cluster_rank());
    constexpr int kOutCols = GATED ? BN / 2 : BN;
    const int tiles_m = (p.m + kPairM - 1) / kPairM, tiles_n = (p.n + kOutCols - 1) / kOutCols;
    const int group_tiles = tiles_m * tiles_n, tiles = group_tiles * p.groups;
    const int kblocks = (p.k + kBlockK - 1) / kBlockK, steps = kblocks * p.nseg, small = steps - kblocks * p.nmain;
    const int first = int(blockIdx.x >> 1), stride = int(gridDim.x >> 1), items = tiles * split;

    // the steps of a piece of work: slice t % split of tile t / split
    auto from = [&](int t) { return int(int64_t(steps) * (t % split) / split); };
    auto to = [&](int t) { return int(int64_t(steps) * (t % split + 1) / split); };
    // its tile: group, row and column of tiles
    auto locate = [&](int t, int &group, int &tm, int &tn) {
        t /= split;
        group = t / group_tiles;
        t -= group * group_tiles;
        const int band = t / (kBand * tiles_n), rest = t - band * kBand * tiles_n;
        const int height = tiles_m - band * kBand < kBand ? tiles_m - band * kBand : kBand;
        tm = band * kBand + rest % height;
        tn = rest / height;
    };

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            bar_init(&full[s], 1);
            bar_init(&empty[s], 1);
        }
        for (int s = 0; s < 2; ++s) {
            bar_init(&sum_full[s], 1);
            bar_init(&sum_empty[s], 16);       // the epilogue warps of both blocks
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<2, 2 * BN>(&tmem_at);
    tmem_before_sync();
    __syncthreads();
    cluster_arrive();
    cluster_wait();                             // the other block's barriers are ready
    tmem_after_sync();
    dependents_may_start();
    wait_for_previous();
    const uint32_t tmem = tmem_at;

    if (warp == 0 && elected()) {
        // both blocks load their halves; the even block's barrier counts the bytes of both
        const uint32_t full_lead = peer_addr(s32(&full[0]), 0);
        int i = 0;
        bool ok = true;
        Ring<STAGES> at;
        for (int t = first; ok && t < items; t += stride) {
            const int it0 = from(t), it1 = to(t);
            int group, tm, tn;
            locate(t, group, tm, tn);
            const int m0 = tm * kPairM + rank * 128;
            const int n0 = tn * kOutCols + (GATED ? 0 : rank * (BN / 2));
            int seg = it0 / kblocks, kb = it0 - seg * kblocks;
            for (int left = it1 - it0; ok && left > 0; ++seg, kb = 0) {
                const Segment sg = p.seg[seg];
                const int az = sg.az + group, bz = sg.bz;
                const CUtensorMap *mb = GATED ? &maps.b[rank] : &maps.b[sg.b];
                const int end = left < kblocks - kb ? kb + left : kblocks;
                left -= end - kb;
                for (; kb < end; ++kb, ++i, at.next()) {
                    if (i >= STAGES && !(ok = bar_wait(&empty[at.stage], at.phase ^ 1))) break;
                    if (rank == 0) bar_expect(&full[at.stage], 2 * S::stage_bytes);
                    const uint32_t bar = full_lead + at.stage * 8;
                    const uint32_t a = ring + at.stage * S::stage_bytes, b = a + S::a_bytes;
                    const int k = kb * kBlockK;
                    if (AMN) {
                        tma_load_pair(a, &maps.a, m0, k, az, bar);
                        tma_load_pair(a + 8192, &maps.a, m0 + 64, k, az, bar);
                    } else {
                        tma_load_pair(a, &maps.a, k, m0, az, bar);
                    }
                    if (BMN) {
                        for (int j = 0; j < BN / 128; ++j) tma_load_pair(b + j * 8192, mb, n0 + 64 * j, k, bz, bar);
                    } else {
                        tma_load_pair(b, mb, k, n0, bz, bar);
                    }
                }
            }
        }
        // nothing may still be on its way into this block's memory when it ends: the products have read it all
        for (int j = i > STAGES ? i - STAGES : 0; j < i; ++j)
            if (!bar_wait(&empty[j % STAGES], (j / STAGES) & 1)) break;
    } else if (warp == 1 && rank == 0 && elected()) {
        constexpr uint32_t kind = mma_kind(kPairM, BN, AMN, BMN);
        const uint16_t both = 3;
        const uint64_t a0 = smem_operand(ring, AMN ? 8192 : 16, 1024), b0 = smem_operand(ring + S::a_bytes, BMN ? 8192 : 16, 1024);
        int run = 0;
        bool ok = true;
        Ring<STAGES> at;
        for (int t = first; ok && t < items; t += stride) {
            const int it0 = from(t), it1 = to(t);
            for (int it = it0; ok && it < it1; ++run) {
                const int buf = run & 1, end = run_end<DRAIN>(it, small, it1);
                if (run >= 2 && !(ok = bar_wait(&sum_empty[buf], (run / 2 - 1) & 1))) break;
                tmem_after_sync();
                const uint32_t d = tmem + buf * BN;
                for (bool add = false; it < end; ++it, at.next()) {
                    if (!(ok = bar_wait(&full[at.stage], at.phase))) break;
                    tmem_after_sync();
                    const uint64_t da = a0 + at.stage * (S::stage_bytes / 16), db = b0 + at.stage * (S::stage_bytes / 16);
#pragma unroll
                    for (int k = 0; k < kBlockK / 16; ++k) {
                        mma_bf16<2>(d, da + k * (AMN ? 2048 / 16 : 2), db + k * (BMN ? 2048 / 16 : 2), kind, add);
                        add = true;
                    }
                    mma_commit<2>(&empty[at.stage], both);
                }
                mma_commit<2>(&sum_full[buf], both);
            }
        }
    } else if (warp >= 2) {
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const uint32_t at = tmem + (uint32_t(quarter * 32) << 16);
        float *stage = reinterpret_cast<float *>(raw + (ring - s32(raw)) + S::ring_bytes) + (warp - 2) * S::stage_words;
        const Epilogue &e = p.e;
        // the warp's blocks of 32 accumulator columns; gated, half of them of the gate and the others of up that belong to them
        auto column = [&](int j) { return GATED ? half * (BN / 4) + (j % (kBlocks / 2)) * 32 + j / (kBlocks / 2) * (BN / 2) : half * (BN / 2) + j * 32; };
        constexpr int kOuts = GATED ? kBlocks / 2 : kBlocks;
        int run = 0;
        bool ok = true;
        for (int t = first; ok && t < items; t += stride) {
            const int it0 = from(t), it1 = to(t);
            int group, tm, tn;
            locate(t, group, tm, tn);
            const int m0 = tm * kPairM + rank * 128 + quarter * 32, n0 = tn * kOutCols;
            const int rows = p.m - m0 < 32 ? p.m - m0 : 32;
            // 32 columns of the warp's rows, a row a lane: straight from the registers where the rows are aligned; otherwise through
            // `stage`, a row at a time and a lane a column
            auto take_out = [&](int c, float (&v)[32], float (&u)[32]) {
                if (e.vec && n0 + c + 32 <= p.n) {
                    finish_row<GATED, DRAIN>(e, group, lane < rows, m0 + lane, n0 + c, v, u);
                    return;
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    stage[lane * S::pitch + j] = v[j];
                    if (GATED) stage[(32 + lane) * S::pitch + j] = u[j];
                }
                __syncwarp();
                const int n = n0 + c + lane;
                if (n < p.n) {
                    const float b0 = e.bias[0] ? e.bias[0][n] : 0.0f, b1 = GATED && e.bias[1] ? e.bias[1][n] : 0.0f;
                    constexpr int kAtOnce = 8;
#pragma unroll 1
                    for (int r = 0; r < rows; r += kAtOnce) {
                        float x[kAtOnce], y[kAtOnce], add[kAtOnce];
#pragma unroll
                        for (int q = 0; q < kAtOnce; ++q) {
                            x[q] = stage[(r + q) * S::pitch + lane] + b0;
                            y[q] = GATED ? stage[(32 + r + q) * S::pitch + lane] + b1 : 0.0f;
                            add[q] = r + q < rows ? residual_at(e, m0 + r + q, n) : 0.0f;
                        }
#pragma unroll
                        for (int q = 0; q < kAtOnce; ++q)
                            if (r + q < rows) finish<GATED>(e, group, m0 + r + q, n, x[q], y[q], add[q]);
                    }
                }
                __syncwarp();
            };
            // a slice's sums, a row a lane
            auto put_partial = [&](int c, const float (&v)[32]) {
                const int64_t row = (int64_t(t % split) * tiles + t / split) * kPairM + rank * 128 + quarter * 32 + lane;
                if (lane < rows) store_row<true>(partial, row * BN + c, v, 32);
            };
            if (DRAIN) {
                float acc[kBlocks][32];
#pragma unroll
                for (int j = 0; j < kBlocks; ++j)
#pragma unroll
                    for (int q = 0; q < 32; ++q) acc[j][q] = 0.0f;
                for (int it = it0; it < it1; ++run) {
                    const int buf = run & 1;
                    ok = bar_wait(&sum_full[buf], (run / 2) & 1);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tmem_after_sync();
#pragma unroll
                    for (int j = 0; j < kBlocks; ++j)
#pragma unroll
                        for (int h = 0; h < 32; h += 16) {
                            float v[16];
                            tmem_load16(at + buf * BN + column(j) + h, v);
#pragma unroll
                            for (int q = 0; q < 16; ++q) acc[j][h + q] += v[q];
                        }
                    tmem_before_sync();
                    __syncwarp();
                    if (lane == 0) peer_arrive(peer_addr(s32(&sum_empty[buf]), 0));
                    it = run_end<DRAIN>(it, small, it1);
                }
                if (!ok) break;
                if (split > 1) {
#pragma unroll
                    for (int j = 0; j < kBlocks; ++j) put_partial(column(j), acc[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < kOuts; ++j) take_out(column(j), acc[j], acc[(j + kOuts) % kBlocks]);
                }
            } else {
                const int buf = run & 1;
                ok = bar_wait(&sum_full[buf], (run / 2) & 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tmem_after_sync();
                if (split > 1) {
#pragma unroll 1
                    for (int j = 0; j < kBlocks; ++j) {
                        float v[32];
                        tmem_load32(at + buf * BN + column(j), v);
                        put_partial(column(j), v);
                    }
                    tmem_before_sync();
                    __syncwarp();
                    if (lane == 0) peer_arrive(peer_addr(s32(&sum_empty[buf]), 0));
                } else {
#pragma unroll 1
                    for (int j = 0; j < kOuts; ++j) {
                        float v[32], u[32];
                        tmem_load32(at + buf * BN + column(j), v);
                        if (GATED) tmem_load32(at + buf * BN + column(j + kOuts), u);
                        if (j == kOuts - 1) {        // the accumulator is free as soon as it has been read
                            tmem_before_sync();
                            __syncwarp();
                            if (lane == 0) peer_arrive(peer_addr(s32(&sum_empty[buf]), 0));
                        }
                        take_out(column(j), v, u);
                    }
                }
                ++run;
            }
        }
    }
    __syncwarp();
    tmem_before_sync();
    cluster_arrive();
    cluster_wait();                             // neither block ends while the other may still reach it
    tmem_after_sync();
    if (warp == 1) tmem_free<2, 2 * BN>(tmem);
}

// Adds up the slices of a split product and finishes it, four columns a thread.
template <bool GATED, bool F32> __global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ Product p, const float *partial, int split, int bn)
{
    dependents_may_start();
    wait_for_previous();
    const int cols = GATED ? bn / 2 : bn, fours = (p.n + 3) / 4;
    const int tiles_m = (p.m + kPairM - 1) / kPairM, tiles_n = (p.n + cols - 1) / cols, group_tiles = tiles_m * tiles_n, tiles = group_tiles * p.groups;
    const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x, per_group = int64_t(p.m) * fours;
    if (at >= per_group * p.groups) return;
    const int group = int(at / per_group);
    const int64_t in_group = at - group * per_group;
    const int m = int(in_group / fours), n = int(in_group - int64_t(m) * fours) * 4;
    // the tile's number, as pair_kernel walks them
    const int tm = m / kPairM, tn = n / cols, band = tm / kBand, height = tiles_m - band * kBand < kBand ? tiles_m - band * kBand : kBand;
    const int tile = group * group_tiles + band * kBand * tiles_n + tn * height + tm - band * kBand;
    const float *from = partial + (int64_t(tile) * kPairM + m % kPairM) * bn + n % cols;
    const int64_t stride = int64_t(tiles) * kPairM * bn;
    float v[1][4] = {}, u[1][4] = {};
#pragma unroll 4
    for (int s = 0; s < split; ++s) {
        const float4 x = *reinterpret_cast<const float4 *>(from + s * stride);
        v[0][0] += x.x; v[0][1] += x.y; v[0][2] += x.z; v[0][3] += x.w;
        if (GATED) {
            const float4 y = *reinterpret_cast<const float4 *>(from + s * stride + bn / 2);
            u[0][0] += y.x; u[0][1] += y.y; u[0][2] += y.z; u[0][3] += y.w;
        }
    }
    finish_fours<GATED, F32, 1, 1>(p.e, group, m, 1, 1, n, p.n, v, u);
}

// ---------------------------------------------------------------------------------------------------------
// Host side.

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_entry()
{
    static const EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

// Boxes of 64 columns by `box_rows` rows of one plane; what lies outside the matrix reads as zero.
bool make_map(CUtensorMap *map, const Planes &m, int box_rows)
{
    const EncodeTiled encode = encode_entry();
    if (!encode) return false;
    const uint64_t pitch = uint64_t(m.ld) * 2, plane = m.nz > 1 ? uint64_t(m.zstride) * 2 : pitch;
    const cuuint64_t dims[3] = {cuuint64_t(m.cols), cuuint64_t(m.rows), cuuint64_t(m.nz)}, strides[2] = {pitch, plane};
    const cuuint32_t box[3] = {64, cuuint32_t(box_rows), 1}, step[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<__nv_bfloat16 *>(m.p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Lets the kernel have that much shared memory on the current device, once for each device.
template <typename Kernel> cudaError_t allow_shared(Kernel kernel, int bytes, std::atomic<uint64_t> &devices)
{
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    const uint64_t bit = uint64_t(1) << (device & 63);
    if (e != cudaSuccess || (devices & bit)) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) devices |= bit;
    return e;
}

// Tiles of a pair with bn accumulator columns.
int64_t pair_tiles(const Product &p, int bn)
{
    const int cols = p.gated ? bn / 2 : bn;
    return (int64_t(p.n) + cols - 1) / cols * ((int64_t(p.m) + kPairM - 1) / kPairM) * p.groups;
}

template <int BN, int STAGES, bool AMN, bool BMN, bool GATED, bool DRAIN> cudaError_t launch_tile(const Product &p, int split, cudaStream_t stream)
{
    using S = TileShape<BN, STAGES>;
    auto kernel = tile_kernel<BN, STAGES, AMN, BMN, GATED, DRAIN>;
    static std::atomic<uint64_t> devices{0};
    cudaError_t e = allow_shared(kernel, S::bytes, devices);
    if (e != cudaSuccess) return e;
    Maps maps;
    const int a_rows = p.m < kBlockM ? (p.m + 7) / 8 * 8 : kBlockM, b_rows = BMN ? 64 : (GATED ? BN / 2 : BN);
    if (!make_map(&maps.a, p.a, AMN ? 64 : a_rows) || !make_map(&maps.b[0], p.b[0], b_rows) || (p.b[1].p && !make_map(&maps.b[1], p.b[1], b_rows)))
        return cudaErrorUnknown;
    constexpr int cols = GATED ? BN / 2 : BN;
    const int64_t blocks = int64_t((p.n + cols - 1) / cols) * ((p.m + kBlockM - 1) / kBlockM) * split;
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    count_launches(1);
    return launch(kernel, dim3(unsigned(blocks), unsigned(p.groups)), kTileThreads, S::bytes, split, stream, p, maps, split, a_rows);
}

template <int BN, bool AMN, bool BMN, bool GATED, bool DRAIN> cudaError_t launch_pair(const Product &p, int split, float *partial, cudaStream_t stream)
{
    using S = PairShape<BN, GATED>;
    auto kernel = pair_kernel<BN, AMN, BMN, GATED, DRAIN>;
    static std::atomic<uint64_t> devices{0};
    cudaError_t e = allow_shared(kernel, S::bytes, devices);
    if (e != cudaSuccess) return e;
    Maps maps;
    const int b_rows = BMN ? 64 : BN / 2;
    if (!make_map(&maps.a, p.a, AMN ? 64 : 128) || !make_map(&maps.b[0], p.b[0], b_rows) || (p.b[1].p && !make_map(&maps.b[1], p.b[1], b_rows)))
        return cudaErrorUnknown;
    const int64_t items = pair_tiles(p, BN) * split;
    if (items > INT32_MAX / 2) return cudaErrorInvalidConfiguration;
    const int pairs = items < kSms / 2 ? int(items) : kSms / 2;
    e = launch(kernel, dim3(unsigned(2 * pairs)), kPairThreads, S::bytes, 2, stream, p, maps, split, partial);
    count_launches(1);
    if (e != cudaSuccess || split == 1) return e;
    const int64_t blocks = (int64_t(p.m) * ((p.n + 3) / 4) * p.groups + 255) / 256;
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    count_launches(1);
    return launch(join_kernel<GATED, DRAIN>, dim3(unsigned(blocks)), 256, 0, 1, stream, p, static_cast<const float *>(partial), split, BN);
}

// Which kernel takes a product, and over how many blocks its contraction is split: the shortest by this estimate, in microseconds, of
// start + rounds x (steps x time of a step + end of a tile) + join.  The constants are measured on bfloat16 products of 1 to 8192 rows, widths of
// 256 to 25088 and contractions of 16 to 25088 (a step is 64 of the contraction; clocks as they come):
//   pair 256 x 256: 0.28 a step (0.35 with all pairs at work), pair 256 x 128: 0.215, tile 128 x 64: 0.12 + 0.16 at 128 rows, and
//   1.4 times that with two blocks on an SM.  4096^3: 93 us / 110 / 185; 1024^3: 12.8 / 8.6 / 12.0 (split 2); 256 x 1000 x 4096:
//   24 / 17 / 10 (split 4); 16 x 4096 x 4096: 18.5 / 14.1 / 9.8 (split 4).
// A result whose rows allow no vectors goes out through shared memory, which ends a pair's tile 4 us later (190 x 88 x 1039: 14.6 us by pairs, 10.0 by tiles).
// A round is what fits the chip at a time: 74 pairs, and clusters as cudaOccupancyMaxActiveClusters gives them for tile_kernel's blocks.
struct Choice {
    int kind, split;       // kind: columns of a pair's tile, or 0 for tile_kernel
    double us;
};

Choice choose(const Product &p)
{
    const double steps = double((p.k + kBlockK - 1) / kBlockK) * p.nseg;
    Choice best{256, 1, 1e30};
    auto consider = [&](int kind, int split, double us) {
        if (us < best.us) best = Choice{kind, split, us};
    };
    for (int bn = 128; bn <= 256; bn += 128) {
        const double t = double(pair_tiles(p, bn)), start = bn == 256 ? 6.0 : 4.5, end = (bn == 256 ? 2.5 : 1.9) + (p.e.vec ? 0.0 : bn / 128 * 4.0);
        for (int split = 1; split <= 8 && (split == 1 || (steps >= 8 * split && t * (split - 1) < kSms / 2)); ++split) {
            const double step = bn == 256 ? (t * split > kSms / 4 ? 0.33 : 0.28) : 0.215;
            const double join = split == 1 ? 0.0 : 3.5 + t * kPairM * bn * 4 * (split + 1) / 5e6;
            consider(bn, split, start + ceil(t * split / (kSms / 2)) * (ceil(steps / split) * step + end) + join);
        }
    }
    const double t = double((int64_t(p.m) + kBlockM - 1) / kBlockM) * double(((p.gated ? 2 : 1) * int64_t(p.n) + 63) / 64) * p.groups;
    const double rows = p.m < kBlockM ? p.m / double(kBlockM) : 1.0;
    static const int clusters[4] = {2 * kSms, kSms, 71, 33};
    static const double join[4] = {0.0, 1.0, 1.5, 4.0};
    for (int q = 0; q < 4 && (q == 0 || steps >= (2 << q)); ++q) {
        const int split = 1 << q;
        const double step = (0.12 + 0.16 * (rows * 2 + 1) / 3) * (t * split > kSms ? 1.4 : 1.0);
        consider(0, split, 1.0 + ceil(t / clusters[q]) * (ceil(steps / split) * step + 3.0 + join[q] + rows * 3.0 / split));
    }
    return best;
}

template <bool AMN, bool BMN, bool GATED, bool DRAIN> cudaError_t launch_form(const Product &p, float *partial, cudaStream_t stream)
{
    Choice c = choose(p);
    if (c.kind == 256) return launch_pair<256, AMN, BMN, GATED, DRAIN>(p, c.split, partial, stream);
    if (c.kind == 128) return launch_pair<128, AMN, BMN, GATED, DRAIN>(p, c.split, partial, stream);
    return launch_tile<64, 4, AMN, BMN, GATED, DRAIN>(p, c.split, stream);
}

}  // namespace

int64_t product_partial_floats(const Product &p)
{
    const Choice c = choose(p);
    return c.kind == 0 || c.split == 1 ? 0 : pair_tiles(p, c.kind) * c.split * kPairM * c.kind;
}

double product_us(const Product &p) { return choose(p).us; }

cudaError_t launch_product(const Product &p, float *partial, cudaStream_t stream)
{
    if (p.gated) return p.e.f32 ? launch_form<false, false, true, true>(p, partial, stream) : launch_form<false, false, true, false>(p, partial, stream);
    if (p.a_mn) return p.e.f32 ? launch_form<true, true, false, true>(p, partial, stream) : launch_form<true, true, false, false>(p, partial, stream);
    if (p.b_mn) return p.e.f32 ? launch_form<false, true, false, true>(p, partial, stream) : launch_form<false, true, false, false>(p, partial, stream);
    return p.e.f32 ? launch_form<false, false, false, true>(p, partial, stream) : launch_form<false, false, false, false>(p, partial, stream);
}

cudaError_t read_product_error(int *flag) { return cudaMemcpyFromSymbol(flag, g_layer_error, sizeof *flag); }

}  // namespace ssd_layers

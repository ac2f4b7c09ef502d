// All steps of rcd_orthogonalize in one launch, for matrices whose products take less time than the launches between them.
//
// One CTA per SM, resident together (a cooperative launch).  A step is three phases: A = X X^T, B = b A + c A A, X = a X + B X (or their mirrored forms for a
// tall X); a barrier over the grid lies between two phases.  Within a phase a CTA takes tiles of 128 x 64: operands by TMA in boxes of 64 x 64, which serve either order and either side;
// one thread issues tcgen05.mma; eight warps finish a tile from tensor memory, a lane a row of 32 columns.  Where a phase has fewer tiles than SMs and a long k axis, several CTAs
// share a tile: each leaves its sums in fp32, waits for the others' (a counter per tile), and finishes its share of the rows, adding in the order of the pieces.
// 512 x 2048: DESCRIBE
//
// Every wait is bounded; whoever waits in vain notes it, and all leave at the end of the phase.
#include "rcd_orthogonal.h"
#include "rcd_tc.cuh"
#include "rcd_walk.h"

#ifndef FUSED_RULE
#define FUSED_RULE true
#endif
namespace rcd {

namespace {

constexpr int kRows = 128, kCols = 64, kBoxBytes = 64 * 128, kStage = 3 * kBoxBytes, kStages = 8, kThreads = 384, kFirstFinisher = 4, kFinishers = 8;
constexpr uint32_t kWaitTurns = 1u << 16, kPolls = 1u << 22;           // about a second either

struct __align__(8) FusedShared {
    uint64_t full[kStages], empty[kStages], accFull[2], accEmpty[2];
    uint32_t tmemBase;
    int32_t abort, leave;
};
constexpr int kSharedBytes = kStages * kStage + (int)sizeof(FusedShared);

__device__ __forceinline__ bool wait_for(uint64_t *bar, uint32_t parity, FusedShared *sh)
{
    for (uint32_t turn = 0; turn < kWaitTurns; ++turn) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(smem_addr(bar)), "r"(parity), "r"(20000) : "memory");
        if (ok) return true;
        if (*(volatile int32_t *)&sh->abort) return false;
    }
    atomicExch(&sh->abort, 1);
    return false;
}
__device__ __forceinline__ bool warp_wait_for(uint64_t *bar, uint32_t parity, FusedShared *sh) { return __all_sync(0xffffffffu, wait_for(bar, parity, sh)); }
__device__ __forceinline__ bool elect_one()
{
    uint32_t mine;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(mine));
    return mine != 0;
}
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async;" ::: "memory"); }
__device__ __forceinline__ uint32_t load_acquire(const uint32_t *p)
{
    uint32_t v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// Adds one to a counter that others wait for, and waits until it has reached `target` (one thread; what its CTA wrote before is visible to whoever sees it).
__device__ __forceinline__ void meet_at(uint32_t *counter, uint32_t target, FusedShared *sh)
{
    __threadfence();
    atomicAdd(counter, 1u);
    for (uint32_t poll = 0; poll < kPolls; ++poll)
        if ((int32_t)(load_acquire(counter) - target) >= 0) return;
    atomicExch(&sh->abort, 1);
}

// The same descriptor as make_smem_desc for an operand whose k elements lie next to each other; for the other order boxes of 64 x 64 follow one another.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool across)
{
    const uint64_t d = make_smem_desc(addr);
    return across ? (d & ~((uint64_t)0x3fff << 16)) | (uint64_t)(kBoxBytes >> 4) << 16 : d;
}

struct Phase {
    int32_t M, N, slabs, splits, per;      // per: slabs of a piece
    bool acrossA, acrossB, symmetric, residual, last;
    int32_t stepA, stepB, stepOut;         // rows from matrix to matrix
    int32_t tilesN, tiles;
    float alpha, beta;
    int32_t power;                         // of the matrix's factor, on alpha (and beta)
    int kind;
};
__device__ __forceinline__ Phase phase_of(const FusedParams &p, int ph)
{
    Phase f{};
    const int i = ph / 3, kind = ph - 3 * i;
    const float down = 1.0f / (1 << kUp), *c = p.coefficients + 3 * i;
    f.kind = kind;
    f.splits = p.splits[kind];
    f.symmetric = kind < 2;
    f.residual = kind > 0;
    f.last = ph == 3 * p.steps - 1;
    if (kind == 0) {
        f.M = f.N = p.side;
        f.slabs = (p.tall ? p.rows : p.cols) / 64;
        f.acrossA = f.acrossB = p.tall;
        f.stepA = f.stepB = p.rows;
        f.stepOut = p.side;
        f.alpha = down;
        f.power = i == 0 ? 2 : 0;
    } else if (kind == 1) {
        f.M = f.N = p.side;
        f.slabs = p.side / 64;
        f.stepA = f.stepB = f.stepOut = p.side;
        f.alpha = c[2] * down;
        f.beta = c[1];
    } else {
        f.M = p.rows;
        f.N = p.cols;
        f.slabs = p.side / 64;
        f.acrossB = !p.tall;
        f.stepA = p.tall ? p.rows : p.side;
        f.stepB = p.tall ? p.side : p.rows;
        f.stepOut = p.rows;
        f.alpha = f.last ? down * down : down;
        f.beta = f.last ? c[0] * down : c[0];
        f.power = i == 0 ? 1 : 0;
    }
    const int32_t tilesM = (f.M + kRows - 1) / kRows;
    f.tilesN = f.N / kCols;
    f.tiles = f.symmetric ? tilesM * (tilesM + 1) : tilesM * f.tilesN;
    f.per = (f.slabs + f.splits - 1) / f.splits;
    return f;
}
__device__ __forceinline__ Unit tile_of(const Phase &f, int32_t u)
{
    const Walk w{0, f.tilesN, f.tiles, f.tilesN, f.splits, f.symmetric ? 1 : 0, f.symmetric ? 2 : 0};
    if (f.symmetric) return unit_of(w, u);
    Unit t{};
    const int32_t piece = u / f.tiles, r = u - piece * f.tiles;
    t.batch = piece / f.splits;
    t.split = piece - t.batch * f.splits;
    t.m = r / f.tilesN;
    t.n = r - t.m * f.tilesN;
    return t;
}

__global__ void __launch_bounds__(kThreads, 1) newton_schulz_kernel(const __grid_constant__ CUtensorMap mapX0, const __grid_constant__ CUtensorMap mapX1, const __grid_constant__ CUtensorMap mapA,
                                                                     const __grid_constant__ CUtensorMap mapB, const __grid_constant__ FusedParams p)
{
    extern __shared__ __align__(1024) unsigned char smem[];
    FusedShared &sh = *reinterpret_cast<FusedShared *>(smem + kStages * kStage);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(&sh.full[s], 1); mbar_init(&sh.empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&sh.accFull[b], 1); mbar_init(&sh.accEmpty[b], kFinishers); }
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_addr(&sh.tmemBase)), "r"(2 * kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmemBase = sh.tmemBase;
    const int first = (int)blockIdx.x, step = (int)gridDim.x, phases = 3 * p.steps;

    int s = 0;                             // the ring's place and phase, the accumulators' turn: they go on from phase to phase
    uint32_t parity = warp == 0 ? 1 : 0, nt = 0;
    for (int ph = 0; ph < phases; ++ph) {
        const Phase f = phase_of(p, ph);
        const int i = ph / 3, units = f.tiles * f.splits * p.batch;
        const __half *const x = (i & 1) ? p.x1 : p.x0;
        if (warp == 0) {
            // ---------------- operands ----------------
            const CUtensorMap *const mapX = (i & 1) ? &mapX1 : &mapX0;
            const CUtensorMap *const a = f.kind == 0 ? mapX : f.kind == 1 ? &mapA : p.tall ? mapX : &mapB;
            const CUtensorMap *const b = f.kind == 0 ? mapX : f.kind == 1 ? &mapA : p.tall ? &mapB : mapX;
            const bool leader = elect_one();
            proxy_fence();
            bool ok = true;
            for (int u = first; u < units && ok; u += step) {
                const Unit t = tile_of(f, u);
                const int m0 = t.m * kRows, n0 = t.n * kCols, aRow = t.batch * f.stepA, bRow = t.batch * f.stepB, end = min(f.slabs, (t.split + 1) * f.per);
                for (int kb = t.split * f.per; kb < end; ++kb) {
                    if (!warp_wait_for(&sh.empty[s], parity, &sh)) { ok = false; break; }
                    if (leader) {
                        unsigned char *const to = smem + s * kStage;
                        mbar_expect_tx(&sh.full[s], kStage);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (f.acrossA) tma_load_2d(to + h * kBoxBytes, a, m0 + 64 * h, aRow + kb * 64, &sh.full[s]);
                            else tma_load_2d(to + h * kBoxBytes, a, kb * 64, aRow + m0 + 64 * h, &sh.full[s]);
                        }
                        if (f.acrossB) tma_load_2d(to + 2 * kBoxBytes, b, n0, bRow + kb * 64, &sh.full[s]);
                        else tma_load_2d(to + 2 * kBoxBytes, b, kb * 64, bRow + n0, &sh.full[s]);
                    }
                    __syncwarp();
                    if (++s == kStages) { s = 0; parity ^= 1; }
                }
            }
        } else if (warp == 1) {
            // ---------------- products ----------------
            const uint32_t idesc = (1u << 4) | (f.acrossA ? 1u << 15 : 0u) | (f.acrossB ? 1u << 16 : 0u) | ((uint32_t)(kCols >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24);
            const bool leader = elect_one();
            const uint64_t stepA = f.acrossA ? 128 : 2, stepB = f.acrossB ? 128 : 2;
            bool ok = true;
            for (int u = first; u < units && ok; u += step, ++nt) {
                const Unit t = tile_of(f, u);
                const uint32_t buf = nt & 1;
                if (!warp_wait_for(&sh.accEmpty[buf], ((nt >> 1) & 1) ^ 1, &sh)) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const int begin = t.split * f.per, end = min(f.slabs, begin + f.per);
                for (int kb = begin; kb < end; ++kb) {
                    if (!warp_wait_for(&sh.full[s], parity, &sh)) { ok = false; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t at = smem_addr(smem + s * kStage);
                    const uint64_t descA = operand_desc(at, f.acrossA), descB = operand_desc(at + 2 * kBoxBytes, f.acrossB);
                    if (leader) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) mma_issue<false>(tmemBase + buf * kCols, descA + stepA * k, descB + stepB * k, idesc, kb > begin || k > 0 ? 1u : 0u);
                        mma_commit(&sh.empty[s]);
                    }
                    __syncwarp();
                    if (++s == kStages) { s = 0; parity ^= 1; }
                }
                if (leader) mma_commit(&sh.accFull[buf]);
                __syncwarp();
            }
        } else if (warp >= kFirstFinisher) {
            // ---------------- finish: quarter q of the rows, half of the columns ----------------
            const int q = warp & 3, half = (warp - kFirstFinisher) >> 2;
            for (int u = first; u < units; u += step, ++nt) {
                const Unit t = tile_of(f, u);
                const uint32_t buf = nt & 1;
                const float factor = f.power ? p.factor[t.batch] : 1.0f;
                const float alpha = f.alpha * (f.power == 2 ? factor * factor : factor), beta = f.beta * factor;
                const int row0 = t.m * kRows, col0 = t.n * kCols;
                const __half *const from = f.kind == 1 ? p.a + (int64_t)t.batch * p.side * p.side : x + (int64_t)t.batch * p.rows * p.cols;       // residual: [M][N]
                __half *const to = f.kind == 0 ? p.a + (int64_t)t.batch * p.side * p.side
                                   : f.kind == 1 ? p.b + (int64_t)t.batch * p.side * p.side : ((i & 1) ? p.x0 : p.x1) + (int64_t)t.batch * p.rows * p.cols;
                // eight neighbours of a row, from fp32 sums on
                auto residual_of = [&](int row, int col) { return __ldcg(reinterpret_cast<const uint4 *>(from + (int64_t)row * f.N + col)); };
                auto put = [&](int row, int col, float (&z)[8], const uint4 &r) {
                    const int64_t at = (int64_t)row * f.N + col;
#pragma unroll
                    for (int j = 0; j < 8; ++j) z[j] *= alpha;
                    if (f.residual) {
                        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&w[j]));
                            z[2 * j] = fmaf(beta, v.x, z[2 * j]);
                            z[2 * j + 1] = fmaf(beta, v.y, z[2 * j + 1]);
                        }
                    }
                    if (f.last) {
                        __nv_bfloat16 *const o = p.o + t.batch * p.stepO + (int64_t)row * p.ldO + col;
                        if (row >= p.rowsO) return;
                        if (col + 8 <= p.colsO && ((uintptr_t)o) % 16 == 0) store_pack<8>(o, z);
                        else
                            for (int j = 0; j < 8 && col + j < p.colsO; ++j) o[j] = __float2bfloat16_rn(z[j]);
                        return;
                    }
                    store_pack<8>(to + at, z);
                    if (t.mirror) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) to[(int64_t)(col + j) * f.N + row] = __float2half_rn(z[j]);
                    }
                };
                const int row = row0 + q * 32 + lane;
                const bool inside = row < f.M && col0 < f.N;           // (a diagonal block's second tile may lie behind the last column)
                uint4 residual[4] = {};
                if (f.residual && f.splits == 1 && inside) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) residual[c] = residual_of(row, col0 + half * 32 + 8 * c);
                }
                const bool ok = warp_wait_for(&sh.accFull[buf], (nt >> 1) & 1, &sh);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                uint32_t v[32];
                if (ok) {
                    tmem_load_32cols(tmemBase + buf * kCols + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * 32), v);
                    tmem_load_wait();
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.accEmpty[buf]);
                if (f.splits == 1) {
                    if (ok && inside) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            float z[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) z[j] = __uint_as_float(v[8 * c + j]);
                            put(row, col0 + half * 32 + 8 * c, z, residual[c]);
                        }
                    }
                } else {
                    // (units are no more than CTAs here: whoever shares the tile is at work)
                    const int64_t tile = (int64_t)t.batch * f.tiles + (u % f.tiles), size = kRows * kCols;
                    float *const parts = p.parts + tile * f.splits * size;
                    if (ok) {
                        float4 *const mine = reinterpret_cast<float4 *>(parts + t.split * size + (q * 32 + lane) * kCols + half * 32);
#pragma unroll
                        for (int c = 0; c < 8; ++c) mine[c] = make_float4(__uint_as_float(v[4 * c]), __uint_as_float(v[4 * c + 1]), __uint_as_float(v[4 * c + 2]), __uint_as_float(v[4 * c + 3]));
                    }
                    asm volatile("bar.sync 1, %0;" :: "n"(32 * kFinishers) : "memory");
                    const int me = (int)threadIdx.x - 32 * kFirstFinisher;
                    if (me == 0) meet_at(p.counters + 1 + f.kind * kFusedTileCounters + tile, (uint32_t)((i + 1) * f.splits), &sh);
                    asm volatile("bar.sync 1, %0;" :: "n"(32 * kFinishers) : "memory");
                    if (!*(volatile int32_t *)&sh.abort) {
                        const int share = (kRows + f.splits - 1) / f.splits, r0 = t.split * share, r1 = min(kRows, r0 + share);
                        for (int e = me; e < (r1 - r0) * (kCols / 8); e += 32 * kFinishers) {
                            const int r = r0 + e / (kCols / 8), c = e % (kCols / 8) * 8;
                            if (row0 + r >= f.M || col0 >= f.N) continue;
                            const uint4 r0c = f.residual ? residual_of(row0 + r, col0 + c) : uint4{};
                            float z[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                            for (int k = 0; k < f.splits; ++k) {
                                const float4 *const at = reinterpret_cast<const float4 *>(parts + k * size + r * kCols + c);
                                const float4 lo = __ldcg(at), hi = __ldcg(at + 1);
                                z[0] += lo.x; z[1] += lo.y; z[2] += lo.z; z[3] += lo.w;
                                z[4] += hi.x; z[5] += hi.y; z[6] += hi.z; z[7] += hi.w;
                            }
                            put(row0 + r, col0 + c, z, r0c);
                        }
                    }
                }
            }
            proxy_fence();                                             // (the next phase reads by TMA what was written here)
        }
        if (ph == phases - 1) break;
        __syncthreads();
        if (threadIdx.x == 0) {
            meet_at(p.counters, (uint32_t)(ph + 1) * gridDim.x, &sh);
            sh.leave = *(volatile int32_t *)&sh.abort;
        }
        __syncthreads();
        if (*(volatile int32_t *)&sh.leave) break;
    }
    if (*(volatile int32_t *)&sh.abort) let_copies_land();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmemBase), "r"(2 * kCols) : "memory");
    }
    if (threadIdx.x == 0 && sh.abort) atomicOr(p.status, kDevTimeout);
}

}  // namespace

// Pieces: the least of slabs (a quarter of a microsecond each) and of what a tile in pieces takes besides.
FusedPlan fused_plan(const rcd_ctx *ctx, int64_t batch, int64_t rows, int64_t cols)
{
    FusedPlan f{};
    const int64_t side = std::min(rows, cols), tilesSide = (side + kRows - 1) / kRows;
    const int64_t tiles[3] = {batch * tilesSide * (tilesSide + 1), batch * tilesSide * (tilesSide + 1), batch * ((rows + kRows - 1) / kRows) * (cols / kCols)};
    const int64_t slabs[3] = {std::max(rows, cols) / 64, side / 64, side / 64};
    int64_t most = 0;
    for (int k = 0; k < 3; ++k) {
        double least = 1e300;
        for (int64_t s = 1; s <= slabs[k] && s <= 16; ++s) {
            if (s > 1 && (tiles[k] * s > ctx->smCount || tiles[k] > kFusedTileCounters)) break;
            if (s > 1 && (s - 1) * ((slabs[k] + s - 1) / s) >= slabs[k]) continue;       // (an empty piece)
            const double t = 0.25 * (double)((slabs[k] + s - 1) / s) + (s > 1 ? 1.8 : 0.0);
            if (t < least) {
                least = t;
                f.splits[k] = (int32_t)s;
            }
        }
        most = std::max(most, tiles[k] * f.splits[k]);
        if (f.splits[k] > 1) f.parts = std::max(f.parts, (size_t)(tiles[k] * f.splits[k]) * kFusedTile);
    }
    f.grid = (int32_t)std::min<int64_t>(most, ctx->smCount);
    f.use = ctx->cooperative && FUSED_RULE;
    return f;
}

rcd_status launch_fused(rcd_ctx *ctx, const FusedParams &p, const FusedPlan &plan, cudaStream_t st)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return fail(ctx, RCD_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
    CUtensorMap maps[4];
    __half *const base[4] = {p.x0, p.x1, p.a, p.b};
    for (int k = 0; k < 4; ++k) {
        const int64_t rows = k < 2 ? p.rows : p.side, cols = k < 2 ? p.cols : p.side;
        const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)(p.batch * rows)};
        const cuuint64_t strides[1] = {(cuuint64_t)cols * 2};
        const cuuint32_t box[2] = {64, 64}, estr[2] = {1, 1};
        const CUresult cr = fn(&maps[k], CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, base[k], dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
        if (cr != CUDA_SUCCESS) return fail(ctx, RCD_ERR_CUDA, "cuTensorMapEncodeTiled failed with %d", (int)cr);
    }
    if (!ctx->fusedReady) {
        RCD_CUDA(ctx, allow_shared(newton_schulz_kernel, kSharedBytes));
        ctx->fusedReady = true;
    }
    void *args[5] = {&maps[0], &maps[1], &maps[2], &maps[3], const_cast<FusedParams *>(&p)};
    ctx->kernelLaunches++;
    ctx->tcLaunches++;
    RCD_CUDA(ctx, cudaLaunchCooperativeKernel((const void *)newton_schulz_kernel, dim3((unsigned)plan.grid), dim3(kThreads), args, kSharedBytes, st));
    return RCD_OK;
}

}  // namespace rcd
